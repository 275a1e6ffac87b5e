"""The bounds of the accuracy tests against the orders of sums that they are derived from: what the kernels do is within them, the
ways that lose more are not."""
from __future__ import annotations

import numpy as np
import pytest

from tests import score_bounds as sb


@pytest.mark.parametrize("K", [4096, 8192])
def test_chains_of_products(K):
    size, V = 40.0, 96
    h, w = sb.one_sign(3, V, K, size, K)
    exact = h @ w.T
    assert 0.5 * size < exact[:, 1:].min() and exact.max() < 2 * size
    top = float(exact.max())
    far = lambda chain, between=24: np.abs(sb.log_p(sb.chained(h, w, chain, between)) - sb.log_p(exact)).max()
    for chain in (256, 512):
        limit = sb.product_bound(K, chain, top) + sb.softmax_bound(V, top + 5)
        assert far(chain) < 0.5 * limit
        assert far(K) > 1.5 * limit                              # one chain
        assert far(chain, 18) > 1.5 * limit                      # six bits lost between the chains


@pytest.mark.parametrize("lanes", [32, 128])
def test_sums_of_long_rows(lanes):
    V, off = 151936, {True: [], False: []}
    limit = sb.typical_bound(V, 32, 2.0)
    for seed in range(6):
        x = sb.standing_out(V, seed)
        d = x.astype(np.float64) - float(x.max())
        exact = np.exp(d).sum()
        assert np.log(exact) < 2
        for by_groups in off:
            off[by_groups].append(np.log(sb.lane_sums(x, lanes, by_groups)) - np.log(exact))
    rms = {n: float(np.sqrt(np.mean(np.square(v)))) for n, v in off.items()}
    assert rms[True] < 0.5 * limit
    if lanes == 32:
        assert rms[False] > 2 * limit, (rms, limit)              # straight into the running sums
