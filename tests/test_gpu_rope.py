"""Rotation of queries and keys, and rows turned on their way into a paged cache, against extended precision and against
the unfused calls."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import rope_ref as ref
from tests.test_rope_cpu import HOW

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LAYOUT = {"half": sx.ROPE_HALF, "interleaved": sx.ROPE_INTERLEAVED}


def rows(shape, dtype, seed, spare=0):
    """Rows of heads; with `spare` elements between them."""
    g = torch.Generator().manual_seed(seed)
    T, n, d = shape
    x = torch.randn(T, n * d + spare, generator=g) * torch.exp(torch.randn(T, 1, generator=g))
    return x.to(dtype).to(DEV)[:, :n * d].unflatten(1, (n, d))


def far_positions(T, seed):
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(0, 10 ** 6, (T,), generator=g)
    edge = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 131071, -70000])[:T]
    pos[:len(edge)] = edge
    return pos.to(torch.int32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("layout", list(LAYOUT))
@pytest.mark.parametrize("T,nq,nk,d,start,rot", [
    (1, 1, 0, 64, 0, 64), (1, 32, 8, 128, 0, 128), (9, 4, 2, 128, 64, 64), (7, 3, 1, 96, 0, 96), (33, 2, 2, 80, 16, 64), (5, 5, 3, 192, 128, 64),
    (8, 2, 1, 256, 0, 256), (6, 3, 2, 64, 4, 50), (4, 1, 1, 8, 0, 8), (3, 2, 2, 16, 2, 2), (11, 1, 2, 24, 0, 22), (700, 16, 4, 128, 0, 128),
    (300, 40, 0, 32, 0, 16)])
def test_rotation(dtype, layout, T, nq, nk, d, start, rot):
    rope = sx.Rope(d, 1e6, rot_dim=rot, rot_start=start, layout=LAYOUT[layout], magnitude=1.139)
    pos = far_positions(T, T)
    q, k = rows((T, nq, d), dtype, 1, 16), rows((T, nk, d), dtype, 2) if nk else None
    f = ref.frequencies(rot, 1e6)
    for transpose in (False, True):
        got = rope.sx_rope(pos.to(DEV), q, k, transpose=transpose)
        for x, y in zip((q, k), got):
            if x is not None:
                ref.close(y, *ref.turned(x, pos, f, layout, start, 1.139, transpose))


@pytest.mark.parametrize("scaling", list(HOW))
def test_scalings(scaling):
    T, d = 40, 128
    kw = dict(factor=1.0 if scaling == "none" else 6.5, low=1.0, high=32.0, original_len=8192)
    div = [1.0 + 0.1 * i for i in range(d // 2)] if scaling == "list" else None
    rope = sx.Rope(d, 5e5, scaling=HOW[scaling], divisors=div, **kw)
    pos = far_positions(T, 3)
    q = rows((T, 2, d), torch.float32, 4)
    ref.close(rope.sx_rope(pos.to(DEV), q)[0], *ref.turned(q, pos, ref.frequencies(d, 5e5, scaling, divisors=div, **kw), "half", 0))


@pytest.mark.parametrize("layout,start,rot", [("half", 0, 64), ("half", 2, 38), ("interleaved", 6, 50)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_place_into_slices_and_beside_them(layout, start, rot, dtype):
    """In place and into a buffer with other strides are the same bits, and nothing else is written."""
    T, nq, nk, d = 77, 6, 2, 64
    rope, pos = sx.Rope(d, 1e4, rot_dim=rot, rot_start=start, layout=LAYOUT[layout]), far_positions(T, 5).to(DEV)
    qkv = rows((T, nq + 2 * nk, d), dtype, 6, 8)
    q, k = qkv[:, :nq], qkv[:, nq:nq + nk]
    want = rope.sx_rope(pos, q, k)
    wide = torch.full((T, nq + nk + 1, d), -3.0, dtype=dtype, device=DEV)
    rope.sx_rope(pos, q, k, q_out=wide[:, :nq], k_out=wide[:, nq:nq + nk])
    assert torch.equal(wide[:, :nq], want[0]) and torch.equal(wide[:, nq:nq + nk], want[1]) and (wide[:, -1] == -3.0).all()
    before = qkv.clone()
    rope.sx_rope(pos, q, k, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, nq + nk:], before[:, nq + nk:])


def test_gradient_and_way_back():
    """The transposed rotation against the formula (<g, R x> = <R^T g, x>), against differences of the rotation, which is
    linear, and with magnitude 1 against its inverse.  fp32: sums of n = 2 * 64 products of values of order e, each off by
    2^-21 (|u| + |v|) at most."""
    T, d = 5, 64
    pos = far_positions(T, 7).to(DEV)
    rope = sx.Rope(d, 1e4, rot_dim=48, rot_start=8, layout=sx.ROPE_INTERLEAVED, magnitude=1.3)
    x, g = rows((T, 1, d), torch.float32, 8), rows((T, 1, d), torch.float32, 9)
    back = rope.sx_rope(pos, g, transpose=True)[0].double()
    bound = 4 * 1.3 * d * 2.0 ** -21 * float(x.abs().max()) * float(g.abs().max())
    assert ((rope.sx_rope(pos, x)[0].double() * g.double()).sum((1, 2)) - (back * x.double()).sum((1, 2))).abs().max() <= bound
    zero = torch.zeros_like(x)
    for e in range(0, d, 7):
        one = zero.clone()
        one[..., e] = 1.0
        slope = (rope.sx_rope(pos, one)[0].double() * g.double()).sum((1, 2))             # R (x + 1 e) - R x, linear: R e
        assert (slope - back[:, 0, e]).abs().max() <= bound
    plain = sx.Rope(d, 1e4)
    y = plain.sx_rope(pos, x)[0]
    again = plain.sx_rope(pos, y, transpose=True)[0]
    assert (again - x).abs().max() <= 6 * 2.0 ** -21 * float(x.abs().max())


def test_far_positions_turn_as_their_remainder():
    """A frequency that divides the turn: positions that differ by whole turns give the same bits."""
    rope = sx.Rope(8, 1e4, rot_dim=2, scaling=sx.ROPE_LIST, divisors=[4096 / (2 * np.pi)])
    x = rows((1, 4, 8), torch.float32, 10).expand(3, -1, -1).contiguous()
    # the step is 2^52 of 2^64 up to the rounding of the divisor (2^-53 of it): over 2^30 positions 2^-35 turns at most, below
    # the 2^-32 turns that an angle is held to, so the results agree to a rounding or two
    a, b, c = rope.sx_rope(torch.tensor([77, 77 + 4096 * 1000, 77 + 4096 * 250000], dtype=torch.int32, device=DEV), x)[0]
    assert (a - b).abs().max() <= 2.0 ** -21 * x.abs().max() and (a - c).abs().max() <= 2.0 ** -21 * x.abs().max()


def test_values_outside_the_part_keep_their_bits():
    """NaN payloads, infinities and -0 outside the rotated part arrive as they are, also where the partner of a pair is not finite."""
    d, rope = 64, sx.Rope(64, 1e4, rot_dim=32, rot_start=16)
    x = rows((3, 2, d), torch.bfloat16, 11)
    x[:, :, :16] = torch.tensor([0x7fc1, -1, -32768, 0x7f80], dtype=torch.int16).view(torch.bfloat16).to(DEV).repeat(4)
    x[:, :, 50] = float("-inf")
    x[1, 0, 20] = float("nan")
    y = rope.sx_rope(torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV), x)[0]
    keep = [*range(16), *range(48, 64)]
    assert torch.equal(x[..., keep].view(torch.int16), y[..., keep].view(torch.int16))
    bad = torch.isnan(y.float())[..., 16:48].nonzero().tolist()
    assert bad == [[1, 0, 4], [1, 0, 20]]


# ---- rows into a cache -----------------------------------------------------------------------------------------------
def cache(B, n_kv, d, page, M, kind, seed=0, spare=2):
    g = torch.Generator().manual_seed(seed)
    num = B * M + spare
    kv = dict(page_table=torch.randperm(num, generator=g)[:B * M].to(torch.int32).view(B, M).to(DEV),
              cache_len=torch.zeros(B, dtype=torch.int32, device=DEV))
    for n in "kv":
        fill = torch.randint(0, 120, (num, n_kv, page, d), generator=g)
        kv[n + "_pages"] = (fill.to(torch.uint8) if kind == "e4m3" else (fill / 8).to(torch.bfloat16)).to(DEV)
        if kind == "e4m3":
            kv[n + "_scale"] = torch.randint(100, 140, (num, n_kv, page), generator=g).to(torch.uint8).to(DEV)
    return kv


def rope_ref_rows(k, pos, rot, layout, start, n):
    """The first n rows turned in extended precision and rounded to bf16 (the others as they are)."""
    y = k.clone()
    y[:n] = ref.to_bf16(ref.turned(k[:n], pos[:n], ref.frequencies(rot, 1e4), layout, start)[0]).to(DEV)
    return y


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("kind,page", [("bf16", 16), ("bf16", 1), ("bf16", 7), ("e4m3", 16), ("e4m3", 48)])
@pytest.mark.parametrize("layout,start,frac", [("half", 0, 1.0), ("half", 0, 0.5), ("interleaved", 4, 0.5), ("half", 2, 0.75)])
@pytest.mark.parametrize("d,nq,nkv", [(128, 8, 2), (64, 3, 1), (32, 4, 4), (16, 2, 1)])
def test_append_is_rotation_then_placement(kind, page, layout, start, frac, d, nq, nkv):
    """The same bits as sx_rope on queries and keys and then the plain placement; codes are those of the exact rotation rounded
    to bf16 (sx_kv_append on it).  Every other slot, and rows behind the last sequence, as they were."""
    rot = int(d * frac) // 2 * 2
    start = min(start, d - rot)
    rope = sx.Rope(d, 1e4, rot_dim=rot, rot_start=start, layout=LAYOUT[layout])
    lens, at = [5, 0, 1, 40, 3], [0, 9, 100, 3, 30]
    B, T = len(lens), sum(lens) + 4
    M = -(-max(a + n for a, n in zip(at, lens)) // page)
    kv, two = (cache(B, nkv, d, page, M, kind) for _ in range(2))
    start_ = np.concatenate([[0], np.cumsum(lens)])
    qkv = rows((T, nq + 2 * nkv, d), torch.bfloat16, 12)
    q, k, v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
    pos = torch.zeros(T, dtype=torch.int32)
    for b in range(B):
        pos[start_[b]:start_[b + 1]] = torch.arange(at[b], at[b] + lens[b])
    c = sx.KVPages(kv)
    q_out = torch.full((T, nq, d), -5.0, dtype=torch.bfloat16, device=DEV)
    c.sx_kv_append_rope(rope, k, v, i32(start_), i32(at), q=q, q_out=q_out)
    c.check_status()
    wq, wk = rope.sx_rope(pos.to(DEV), q, k)
    n = sum(lens)
    assert torch.equal(q_out[:n], wq[:n]) and (q_out[n:] == -5.0).all()
    if kind == "e4m3":
        e = sx.KV8(two)
        exact = rope_ref_rows(k, pos, rot, layout, start, n)
        e.sx_kv_append(exact, v, i32(start_), i32(at))
        e.check_status()
    else:
        for b in range(B):
            for i in range(lens[b]):
                s = at[b] + i
                pp = int(two["page_table"][b, s // page])
                two["k_pages"][pp, :, s % page] = wk[start_[b] + i]
                two["v_pages"][pp, :, s % page] = v[start_[b] + i]
    for name in kv:
        assert torch.equal(kv[name], two[name]), name


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_append_without_plan_positions_of_its_own_and_in_place(kind):
    B, nq, nkv, d, page = 3, 4, 2, 64, 16
    kv, two, three = (cache(B, nkv, d, page, 4, kind, 3) for _ in range(3))
    qkv = rows((7, nq + 2 * nkv, d), torch.bfloat16, 13)
    q, k, v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
    kv["cache_len"].copy_(i32([10, 0, 30]))
    start = i32([0, 2, 2, 7])
    rope, pos = sx.Rope(d, 1e4), far_positions(7, 14).to(DEV)
    wq, wk = rope.sx_rope(pos, q, k)
    # behind cache_len, turned to positions of their own; then the turned rows without a plan
    c = sx.KVPages(kv)
    c.sx_kv_append_rope(rope, k, v, start, rot_pos=pos)
    e = sx.KVPages(two)
    e.sx_kv_append_rope(None, rope_ref_rows(k, pos.cpu(), d, "half", 0, 7) if kind == "e4m3" else wk, v, start, i32([10, 0, 30]))
    for name in ("k_pages", "v_pages", *(("k_scale", "v_scale") if kind == "e4m3" else ())):
        assert torch.equal(kv[name], two[name]), name
    assert kv["cache_len"].tolist() == [10, 0, 30]
    f = sx.KVPages(three)
    same = f.sx_kv_append_rope(rope, k, v, start, i32([10, 0, 30]), rot_pos=pos, q=q, q_out=q)
    assert same is q and torch.equal(q, wq) and torch.equal(three["k_pages"], kv["k_pages"])
    for x in (c, e, f):
        x.check_status()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_rows_without_a_place_are_reported_and_the_others_written(kind):
    B, d, page = 4, 32, 16
    kv, two = (cache(B, 1, d, page, 2, kind, 5) for _ in range(2))
    for t in (kv, two):
        t["page_table"][1, 1] = -1
        t["page_table"][2, 0] = 10 ** 6
    x = rows((8, 1, d), torch.bfloat16, 15)
    start, at = i32([0, 2, 4, 6, 8]), i32([3, 15, 0, 31])      # sequence 1's second, 2's both and 3's second row have no page
    c = sx.KVPages(kv)
    c.sx_kv_append_rope(None, x, x, start, at)
    with pytest.raises(sx.SxError):
        c.check_status()
    e = sx.KVPages(two)
    for t, b, s in ((0, 0, 3), (1, 0, 4), (2, 1, 15), (6, 3, 31)):
        e.sx_kv_append_rope(None, x[t:t + 1], x[t:t + 1], i32([0] * (b + 1) + [1] * (B - b)), i32([s] * B))
    e.check_status()
    for name in kv:
        assert torch.equal(kv[name], two[name]), name
    for bad in ([-1, 2, 4, 6, 8], [0, 4, 2, 6, 8], [0, 2, 4, 6, 9]):
        c.sx_kv_append_rope(None, x, x, i32(bad), i32([0] * B))
        with pytest.raises(sx.SxError):
            c.check_status()
    c.sx_kv_append_rope(sx.Rope(d, 1e4), x, x, start, i32([-1, 0, 0, -2 ** 31]))
    with pytest.raises(sx.SxError):
        c.check_status()


@pytest.mark.parametrize("B", [31, 32, 33, 1000, 1025, 3000])
def test_many_sequences(B):
    """Every row finds its sequence, empty ones between them."""
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 3, (B,), generator=g)
    start = torch.cat([torch.zeros(1, dtype=torch.long), lens.cumsum(0)])
    T = int(start[-1])
    kv = cache(B, 1, 16, 4, 1, "bf16", 6)
    x = rows((T, 1, 16), torch.bfloat16, 16)
    c = sx.KVPages(kv)
    c.sx_kv_append_rope(None, x, x, start.to(torch.int32).to(DEV), i32([1] * B))
    c.check_status()
    b = torch.repeat_interleave(torch.arange(B), lens)
    off = 1 + torch.arange(T) - start[b]
    pp = kv["page_table"][b.to(DEV), 0].long()
    assert torch.equal(kv["k_pages"][pp, 0, off.to(DEV)], x[:, 0]) and torch.equal(kv["v_pages"][pp, 0, off.to(DEV)], x[:, 0])


def test_pool_past_32_bits():
    """Pages whose offset passes 2^32 bytes and 2^31 elements."""
    d, page, num = 128, 64, 150000                              # 150000 * 2 * 64 * 128 * 2 bytes = 4.9 GB each
    kv = dict(k_pages=torch.zeros(num, 2, page, d, dtype=torch.bfloat16, device=DEV), cache_len=i32([0]),
              page_table=i32([[num - 1, 140001]]))
    kv["v_pages"] = torch.zeros_like(kv["k_pages"])
    x = rows((3, 2, d), torch.bfloat16, 17)
    rope = sx.Rope(d, 1e6)
    c = sx.KVPages(kv)
    c.sx_kv_append_rope(rope, x, x, i32([0, 3]), i32([62]))
    c.check_status()
    want = rope.sx_rope(i32([62, 63, 64]), x)[0]
    assert torch.equal(kv["k_pages"][num - 1, :, 62:].transpose(0, 1), want[:2]) and torch.equal(kv["k_pages"][140001, :, 0], want[2])
    assert torch.equal(kv["v_pages"][num - 1, :, 62:].transpose(0, 1), x[:2]) and int(kv["k_pages"].count_nonzero()) == int(want.count_nonzero())


def test_no_rows_is_no_work():
    kv = cache(2, 1, 64, 16, 1, "bf16", 7)
    x = torch.zeros(0, 1, 64, dtype=torch.bfloat16, device=DEV)
    c = sx.KVPages(kv)
    assert c.sx_kv_append_rope(sx.Rope(64, 1e4), x, x, i32([0, 0, 0]), q=x).shape == (0, 1, 64)
    assert sx.Rope(64, 1e4).sx_rope(i32([]), x)[0].shape == (0, 1, 64)


def test_other_streams_and_graphs():
    """On a side stream, and captured and replayed with new rows and positions."""
    T, nq, nkv, d = 9, 4, 2, 64
    rope, kv = sx.Rope(d, 1e4), cache(1, nkv, d, 16, 2, "bf16", 8)
    c = sx.KVPages(kv)
    qkv, pos, at = rows((T, nq + 2 * nkv, d), torch.bfloat16, 18), far_positions(T, 19).to(DEV), i32([3])
    q, k, v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
    start, q_out = i32([0, T]), torch.empty(T, nq, d, dtype=torch.bfloat16, device=DEV)
    turned = torch.empty_like(q_out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def step():
        c.sx_kv_append_rope(rope, k, v, start, at, rot_pos=pos, q=q, q_out=q_out)
        rope.sx_rope(pos, q, q_out=turned)

    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (20, 21):
        qkv.copy_(rows((T, nq + 2 * nkv, d), torch.bfloat16, seed))
        pos.copy_(far_positions(T, seed).to(DEV))
        at.fill_(seed - 10)
        graph.replay()
        torch.cuda.synchronize()
        wq, wk = rope.sx_rope(pos, q, k)
        assert torch.equal(q_out, wq) and torch.equal(turned, wq)
        pages = kv["k_pages"][kv["page_table"][0].long()].transpose(1, 2).reshape(32, nkv, d)
        assert torch.equal(pages[seed - 10:seed - 10 + T], wk)
    c.check_status()
