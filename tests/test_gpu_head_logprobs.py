"""Log-probabilities through a head, against 64 bits.  Hidden states and weights are small multiples of 1/16, so every product and
every partial sum is exact in fp32 and the logits are known to the bit: ids have to be equal, ties included."""
from __future__ import annotations

import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import score_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(T, V, H, seed, extra=0):
    """|h| <= 4/16, |w| <= 3/16, one in eight of the hidden elements not zero at most: |logit| < H / 8 * 12 / 256 * 8."""
    g = torch.Generator().manual_seed(seed)
    h = torch.randint(-4, 5, (T, H), generator=g) * (torch.rand(T, H, generator=g) < max(0.125, 8 / H))
    w = torch.randint(-3, 4, (V + extra, H), generator=g)
    h, w = (h / 16).to(torch.bfloat16), (w / 16).to(torch.bfloat16)
    w[V:] = float("nan")                                         # rows behind the vocabulary are not looked at
    tok = torch.randint(-1, V, (T, 2), generator=g).to(torch.int32)
    return h.to(DEV), w.to(DEV), tok.to(DEV)


def logits(h, w, V):
    return h.double().cpu() @ w[:V].double().cpu().T


def both(h, w, tok, V, top, temperature=1.0, scores=None):
    s = scores or sx.LogProbs(w, vocab=V)
    got = s.sx_head_logprobs(h, tok, top=top, temperature=temperature)
    s.check_status()
    x = logits(h, w, V)
    ref.check(got, ref.scores(x, tok, top, temperature), x, temperature)
    return got


@pytest.mark.parametrize("T,V,H,extra", [
    (1, 1, 8, 0), (3, 5, 16, 0), (7, 127, 64, 3), (17, 128, 72, 3), (16, 129, 128, 0), (33, 1000, 256, 3), (64, 2049, 136, 0), (65, 3000, 64, 1),
    (128, 640, 1024, 0), (255, 1300, 64, 3), (256, 257, 64, 0), (257, 700, 64, 3), (513, 300, 40, 0), (700, 515, 264, 3), (2, 40000, 512, 3),
    (1, 151936, 64, 3), (250, 20011, 128, 0), (300, 1, 8, 0), (129, 383, 1032, 3), (1025, 300, 40, 0), (2100, 130, 64, 3), (5, 200, 16384, 0),
    (140, 260, 8200, 0)])
def test_shapes(T, V, H, extra):
    both(*make(T, V, H, T + V, extra), V, min(20, 32))


@pytest.mark.parametrize("top", [0, 1, 31, 32])
@pytest.mark.parametrize("temperature", [0.3, 1.0, 2.5])
def test_alternatives_and_temperature(top, temperature):
    h, w, tok = make(40, 3001, 128, 3)
    both(h, w, tok, 3001, top, temperature)
    both(h, w, None, 3001, top, temperature)


def test_equal_tokens_everywhere():
    """Every row of the head the same, and a head that repeats: the lowest ids of the largest logits."""
    h, w, tok = make(5, 1024, 64, 4)
    both(h, w[:1].expand(1024, -1).contiguous(), tok, 1024, 32)
    both(h, w[:100].repeat(11, 1)[:1024].contiguous(), tok, 1024, 32)


@pytest.mark.parametrize("T", [70, 300])
@pytest.mark.parametrize("V,H,extra", [(300, 72, 0), (1000, 200, 3), (2048, 64, 3), (130, 640, 0)])
def test_repacked_head(V, H, extra, T):
    """The layout of sx_tile_weight, rows behind the vocabulary included, gives the same bits."""
    h, w, tok = make(T, V, H, 5, extra)
    want = both(h, w, tok, V, 8)
    got = sx.LogProbs(sx.sx_tile_weight(w), vocab=V, hidden=H).sx_head_logprobs(h, tok, top=8)
    assert all(torch.equal(want[n], got[n]) for n in want)


def test_logits_are_those_of_the_other_form():
    """Arbitrary values: the same scores as from the matrix of logits, up to what sums of H products in fp32 may be off by."""
    g = torch.Generator().manual_seed(6)
    T, V, H = 90, 5000, 1024
    h, w = torch.randn(T, H, generator=g).to(torch.bfloat16).to(DEV), (0.05 * torch.randn(V, H, generator=g)).to(torch.bfloat16).to(DEV)
    tok = torch.randint(0, V, (T, 3), generator=g).to(torch.int32).to(DEV)
    x = logits(h, w, V)
    got = sx.LogProbs(w).sx_head_logprobs(h, tok)
    more = H * 2.0 ** -23 * float((h.double().abs() @ w.double().abs().T).max())
    ref.check(got, ref.scores(x, tok, 0), x, more=more)


@pytest.mark.parametrize("T", [12, 270])
def test_rows_that_are_not_finite_stay_alone(T):
    h, w, tok = make(T, 900, 64, 7)
    h[2, 5] = float("nan")
    h[T - 5, :] = float("inf")                                   # inf times a zero or signs that differ: NaN
    got = sx.LogProbs(w).sx_head_logprobs(h, tok, top=4)
    x = logits(h, w, 900)
    ref.check(got, ref.scores(x, tok, 4), x)


def test_calls_in_a_row_and_beside_one_another():
    """Calls of both kinds and several sizes without a wait between them, then on two streams at once, each with an object of its
    own: what single calls give."""
    V, H = 3000, 512
    sizes = (7, 300, 1, 129, 128, 600, 33)
    made = [make(T, V, H, 40 + T) for T in sizes]
    w = made[0][1]
    want = []
    for h, _, tok in made:
        want.append(sx.LogProbs(w).sx_head_logprobs(h, tok, top=6))
        torch.cuda.synchronize()
    one = sx.LogProbs(w)
    got = [[one.sx_head_logprobs(h, tok, top=6) for h, _, tok in made] for _ in range(5)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    mine = [sx.LogProbs(w) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o in zip(streams, mine):
            with torch.cuda.stream(s):
                got.append([o.sx_head_logprobs(h, tok, top=6) for h, _, tok in made])
    torch.cuda.synchronize()
    for run in got:
        for a, b in zip(run, want):
            assert all(torch.equal(a[n], b[n]) for n in b)
    for o in (one, *mine):
        o.check_status()


def test_large_part_of_the_vocabulary_without_weight():
    """Logits far below the others, down to -3e38, and one row of them only."""
    h, w, tok = make(3, 700, 64, 8)
    w[5:] = 0
    w[5:, 0] = -2.0 ** 120
    h[:, 0] = 1.0
    h[2] = 0
    h[2, 0] = 128.0
    w[:5, 0] = -2.0 ** 120
    both(h, w, tok, 700, 12)


def test_a_token_outside_the_vocabulary_is_reported():
    h, w, tok = make(3, 200, 64, 9, 3)
    tok[1, 0] = 200                                              # a row of the head, but not of the vocabulary
    s = sx.LogProbs(w, vocab=200)
    got = s.sx_head_logprobs(h, tok, top=2)
    with pytest.raises(sx.SxError):
        s.check_status()
    x = logits(h, w, 200)
    ref.check(got, ref.scores(x, tok, 2), x)


@pytest.mark.parametrize("T", [30, 200])
def test_streams_graphs_and_growing_workspaces(T):
    """The same bits on another stream, from a captured call with new rows, and after a larger call has grown the workspace."""
    h, w, tok = make(T, 3000, 128, 10)
    big, _, many = make(500, 3000, 128, 11)
    s = sx.LogProbs(w)
    want = s.sx_head_logprobs(h, tok, top=5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = s.sx_head_logprobs(h, tok, top=5)
    side.synchronize()
    assert all(torch.equal(want[n], other[n]) for n in want)
    out = {n: torch.zeros_like(t) for n, t in want.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.sx_head_logprobs(h, tok, top=5, out=out)
    both(big, w, many, 3000, 5, scores=s)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(want[n], out[n]) for n in want)
    h.copy_(make(T, 3000, 128, 12)[0])
    graph.replay()
    torch.cuda.synchronize()
    x = logits(h, w, 3000)
    ref.check(out, ref.scores(x, tok, 5), x)
    s.check_status()


def test_python_side_refusals():
    h, w, tok = make(3, 200, 64, 13)
    for bad in (dict(head=w.float()), dict(head=w.t()), dict(head=w, vocab=201), dict(head=w, vocab=0), dict(head=w, hidden=72),
                dict(head=sx.sx_tile_weight(w)), dict(head=sx.sx_tile_weight(w), vocab=300, hidden=64)):
        with pytest.raises(sx.SxError):
            sx.LogProbs(**bad)
    with pytest.raises(sx.SxError, match="without a head"):
        sx.LogProbs().sx_head_logprobs(h, tok)
    s = sx.LogProbs(w)
    for args in ((h.float(), tok), (h[:, :56], tok), (h.cpu(), tok), (h, tok.long()), (h, tok[:2])):
        with pytest.raises(sx.SxError):
            s.sx_head_logprobs(*args)
    with pytest.raises(sx.SxError):
        s.sx_head_logprobs(h, tok, top=33)
    with pytest.raises(sx.SxError):
        sx.LogProbs(w[:, :60].contiguous()).sx_head_logprobs(h[:, :60].contiguous(), tok)
    assert s.sx_head_logprobs(h[:0], tok[:0], top=3)["top_tok"].shape == (0, 3)
