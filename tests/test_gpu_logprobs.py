"""Log-probabilities of given tokens, entropy and alternatives of rows of logits, against 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import score_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def make(T, V, dtype, seed, stride=None, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((T, stride or V), 1e4, dtype=dtype)               # what lies between the rows is larger than any logit
    buf[:, :V] = (torch.randn(T, V, generator=g) * spread).to(dtype)
    return buf.to(DEV)[:, :V]


def given(T, V, n, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-1, V, (T, n), generator=g).to(torch.int32).to(DEV)


def both(x, tok, top, temperature=1.0):
    s = sx.LogProbs()
    got = s.sx_logprobs(x, tok, top=top, temperature=temperature)
    s.check_status()
    ref.check(got, ref.scores(x, tok, top, temperature), x, temperature)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,stride", [
    (1, 1, 1), (2, 5, 5), (3, 15, 16), (3, 31, 33), (5, 32, 32), (4, 47, 49), (9, 1000, 1003), (7, 1023, 1024), (3, 4097, 4099), (2, 33000, 33001),
    (1, 151936, 151936), (3, 151937, 151939), (1, 262145, 262145), (600, 515, 515), (1300, 64, 65)])
def test_shapes(dtype, T, V, stride):
    both(make(T, V, dtype, T + V, stride), given(T, V, 3, 1), min(20, 32))


@pytest.mark.parametrize("top", [0, 1, 2, 31, 32])
@pytest.mark.parametrize("n", [0, 1, 64])
def test_numbers_of_alternatives_and_tokens(top, n):
    x = make(4, 5003, torch.bfloat16, 2)
    got = both(x, given(4, 5003, n, 3) if n else None, top)
    assert ("top_tok" in got) == (top > 0)


@pytest.mark.parametrize("temperature", [0.05, 0.7, 1.0, 3.0, 1e4])
def test_temperature(temperature):
    both(make(3, 2000, torch.float32, 4), given(3, 2000, 2, 5), 8, temperature)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [7, 640, 40000])
def test_ties_and_orders(dtype, V):
    """Rows of one value, ascending, descending and in steps (every value many times), both zeros, one value that stands alone."""
    i = torch.arange(V, dtype=torch.float32)
    rows = [torch.zeros(V), torch.full((V,), -3.5), i / V * 8, -i / V * 8, (i * 7919 % 5), (i // 100) % 3, -(i // 100) % 3,
            torch.where(i % 2 == 0, torch.tensor(-0.0), torch.tensor(0.0)), torch.where(i == V - 1, 9.0, -9.0), torch.where(i == 0, 9.0, -9.0)]
    x = torch.stack(rows).to(dtype).to(DEV)
    both(x, given(len(rows), V, 2, 6), min(V, 32))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [50, 3000, 100001])
def test_masked_rows(dtype, V):
    """Masks of -inf and of the type's lowest value: some tokens left, one, none; NaN and +inf at the ends and in masked rows."""
    x = make(14, V, dtype, 8).clone()
    low, inf, nan = torch.finfo(dtype).min, float("inf"), float("nan")
    x[0, :] = -inf
    x[1, :] = -inf
    x[1, V - 1] = 2.0
    x[2, :V - 3] = -inf
    x[3, ::2] = -inf
    x[4, :] = low
    x[5, :] = low
    x[5, V // 2] = 1.0
    x[6, 1:] = low
    x[7, 0] = nan
    x[8, V - 1] = nan
    x[9, V // 2] = inf
    x[10, :] = nan
    x[11, :] = -inf
    x[11, 3] = nan
    x[12, :] = inf
    x[13, : V // 2] = -inf
    both(x, given(14, V, 4, 9), 20)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("temperature", [0.1, 0.7, 4.0])
def test_lowest_values_at_other_temperatures(dtype, temperature):
    """Masks of the type's lowest value whose log p leaves fp32's range, or not; rows of nothing else."""
    x = make(6, 2001, dtype, 22).clone()
    x[:3, 5:1900] = torch.finfo(dtype).min
    x[3] = torch.finfo(dtype).min
    x[4, 1:] = torch.finfo(dtype).min
    both(x, given(6, 2001, 8, 23), 20, temperature)


def test_masked_rows_of_a_cluster_where_one_part_has_everything():
    """One long row per case, over several CTAs: all parts but one masked or spoilt."""
    V = 200003
    for at in (0, 70000, 199990):
        for value in (1.0, float("nan"), float("inf"), float("-inf")):
            x = torch.full((1, V), float("-inf"), dtype=torch.float32, device=DEV)
            x[0, at:at + 9] = torch.arange(9.0, device=DEV)
            x[0, at + 4] = value
            both(x, torch.tensor([[at, at + 4, 5]], dtype=torch.int32, device=DEV), 12)


def test_large_and_small_values():
    """Logits of the order 1e4, differences far beyond the range of an exponential, subnormal ones."""
    x = make(4, 3000, torch.float32, 10)
    x = torch.cat([x * 3000, x * 1e-40, x * 100 + 5e4, -x.abs() * 1e6])
    both(x, given(16, 3000, 3, 11), 32)


def test_peaked_rows():
    """Entropies down to 1e-9: the bound is absolute."""
    for gap in (5.0, 15.0, 30.0, 80.0):
        x = make(2, 5000, torch.float32, 12, spread=1.0).clone()
        x[:, 77] = 10 + gap
        both(x, torch.full((2, 1), 77, dtype=torch.int32, device=DEV), 3)


def test_a_token_outside_the_vocabulary_is_reported():
    x = make(3, 100, torch.bfloat16, 13)
    for bad in (100, -2, 2 ** 31 - 1):
        s = sx.LogProbs()
        tok = torch.tensor([[3], [bad], [-1]], dtype=torch.int32, device=DEV)
        got = s.sx_logprobs(x, tok, top=2)
        with pytest.raises(sx.SxError):
            s.check_status()
        ref.check(got, ref.scores(x, tok, 2), x)
        s.check_status()


def test_same_bits_every_time_streams_graphs_and_out():
    x, tok = make(40, 32001, torch.bfloat16, 14, 32003), given(40, 32001, 2, 15)
    s = sx.LogProbs()
    want = s.sx_logprobs(x, tok, top=20)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = s.sx_logprobs(x, tok, top=20)
    side.synchronize()
    assert all(torch.equal(want[n], other[n]) for n in want)
    out = {n: torch.zeros_like(t) for n, t in want.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert s.sx_logprobs(x, tok, top=20, out=out) is out
    for seed in (14, 16):
        x.copy_(make(40, 32001, torch.bfloat16, seed))
        graph.replay()
        torch.cuda.synchronize()
        ref.check(out, ref.scores(x, tok, 20), x)
        if seed == 14:
            assert all(torch.equal(want[n], out[n]) for n in want)
    s.check_status()


def test_rows_past_32_bits():
    """The last rows of a matrix of more than 2^32 elements."""
    V, T = 262144, 16500
    x = torch.zeros(T, V, dtype=torch.float16, device=DEV)
    x[-3:] = make(3, V, torch.float16, 17)
    tok = given(T, V, 1, 18)
    s = sx.LogProbs()
    got = s.sx_logprobs(x, tok, top=5)
    s.check_status()
    ref.check({n: t[-3:] for n, t in got.items()}, ref.scores(x[-3:], tok[-3:], 5), x[-3:])
    assert got["top_tok"][:-3].eq(torch.arange(5, device=DEV)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_slices_on_any_boundary(dtype):
    """Rows that begin at an element of any place: the first logits of a wider matrix cut off."""
    x = make(5, 3000, dtype, 21, 3001)
    for cut in (1, 2, 3, 5, 8, 15, 16, 17, 31):
        both(x[:, cut:], given(5, 3000 - cut, 2, cut), 9)


def test_python_side_refusals():
    s = sx.LogProbs()
    x = make(3, 100, torch.bfloat16, 19)
    tok = given(3, 100, 1, 20)
    for args in ((x.double(), tok), (x[0], tok), (x.t(), tok), (x.cpu(), tok), (x, tok.long()), (x, tok[:2]), (x, tok.cpu()), (x, tok[:, 0][:, None, None])):
        with pytest.raises(sx.SxError):
            s.sx_logprobs(*args)
    for kw in (dict(top=-1), dict(top=33), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf"))):
        with pytest.raises((sx.SxError, RuntimeError)):
            s.sx_logprobs(x, tok, **kw)
    with pytest.raises(sx.SxError, match="out"):
        s.sx_logprobs(x, tok, top=3, out=s.sx_logprobs(x, tok, top=2))
    assert s.sx_logprobs(x[:0], tok[:0], top=3)["top_tok"].shape == (0, 3)
