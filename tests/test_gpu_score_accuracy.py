"""The accuracy of log-probabilities where sums are not exact: both products of a head, whose accumulator cuts off, and long rows of
logits.  The bounds are derived in score_bounds.py and shown there to tell these sums from those that lose more."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import score_bounds as sb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("K", [4096, 8192])
@pytest.mark.parametrize("T", [1, 7, 90, 128, 129, 300])
def test_products_of_one_sign_through_a_head(T, K):
    """Chains of 256 products with up to 128 rows, of 512 with more."""
    V, size = 640, 40.0
    h, w = sb.one_sign(T, V, K, size, K + T)
    exact = h @ w.T
    want = sb.log_p(exact)
    tok = np.stack([np.zeros(T, np.int64), np.arange(T) % (V - 1) + 1, np.full(T, V - 1)], 1)
    put = lambda x, t: torch.from_numpy(x).to(t).to(DEV)
    s = sx.LogProbs(put(w, torch.bfloat16))
    torch.cuda.synchronize()
    got = s.sx_head_logprobs(put(h, torch.bfloat16), put(tok, torch.int32))["logp"].double().cpu().numpy()
    s.check_status()
    top = float(exact.max())
    limit = sb.product_bound(K, 256 if T <= 128 else 512, top) + sb.softmax_bound(V, top + 7)
    off = np.abs(got - np.take_along_axis(want, tok, 1))
    assert off.max() <= limit, (off.max(), off.mean(0), limit)


@pytest.mark.parametrize("T", [1, 16, 300, 1184, 2400])
def test_long_rows_of_logits(T):
    """Rows of 151936 in bf16, with fewer lanes the more rows there are (one warp each at 2400), a few tokens above the rest: the root
    mean square of the error of the largest one's log p."""
    V, lanes = 151936, 32
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.empty(T, V, dtype=torch.bfloat16, device=DEV)
    for i in range(0, T, 300):
        part = torch.randn(min(300, T - i), V, device=DEV, generator=g) * 2
        part[:, :12] = 4 + 12 * torch.rand(part.shape[0], 12, device=DEV, generator=g)
        part[:, 0] = 16
        x[i:i + 300] = part.to(torch.bfloat16)
    x = x.roll(V // 3, 1)
    tok = torch.full((T, 1), V // 3, dtype=torch.int32, device=DEV)
    s = sx.LogProbs()
    got = s.sx_logprobs(x, tok)["logp"][:, 0].double()
    s.check_status()
    want = torch.cat([-torch.log(torch.exp(x[i:i + 100].double() - 16).sum(1)) for i in range(0, T, 100)])
    assert float(want.min()) > -2
    rms = float((got - want).square().mean().sqrt())
    assert rms <= sb.typical_bound(V, lanes, 2.0), rms
