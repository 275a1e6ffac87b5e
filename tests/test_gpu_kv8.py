"""The operators of the 8-bit paged cache against the definitions in 64 bits: writing rows, reading them back, decode
attention with drafted slots and with shared prefixes."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import kv8_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def to_dev(kv):
    return {n: t.to(DEV) for n, t in kv.items()}


def empty_pool(B, n_kv, d, page, M, fill=0x7f):
    num = B * M + 2
    g = torch.Generator().manual_seed(B * 1000 + M)
    kv = {n: torch.full((num, n_kv, page, d), fill, dtype=torch.uint8) for n in ("k_pages", "v_pages")}
    kv |= {n: torch.full((num, n_kv, page), fill, dtype=torch.uint8) for n in ("k_scale", "v_scale")}
    kv["page_table"] = torch.randperm(num, generator=g)[:B * M].to(torch.int32).view(B, M)
    kv["cache_len"] = torch.zeros(B, dtype=torch.int32)
    return kv


# ---- writing and reading back ---------------------------------------------------------------------------------------
def rows_with_edges(T, n_kv, d, seed):
    """Rows of many magnitudes: ordinary ones, borders of the scale, ties of the code, zeros, huge and tiny ones, rows with
    values that are not finite."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, n_kv, d, generator=g) * torch.exp2(torch.randint(-12, 13, (T, n_kv, 1), generator=g).float())
    flat = x.view(-1, d)
    special = [torch.zeros(d), torch.full((d,), 448.0), torch.full((d,), 450.0), torch.full((d,), -447.0),
               torch.full((d,), 3.3e38), torch.full((d,), 1e-38), torch.full((d,), 2.0 ** -70), torch.full((d,), 2.0 ** -133),
               torch.arange(d).float() + 0.5, -torch.arange(d).float() * 1.0625, torch.linspace(-1, 1, d) * 2.0 ** -58]
    bad = torch.ones(d)
    bad[d - 1] = math.inf
    special.append(bad)
    bad = torch.zeros(d)
    bad[3] = math.nan
    special.append(bad)
    for i, v in enumerate(special[:len(flat)]):
        flat[(i * 7) % len(flat)] = v
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("n_kv,page,lens,at,pad", [
    (1, 16, [1], [0], 0), (2, 16, [5, 0, 17], [3, 9, 15], 4), (8, 64, [1] * 6, [63, 64, 0, 130, 1, 190], 0),
    (3, 48, [100, 1], [0, 77], 1), (8, 64, [700, 650], [0, 5], 3)])
def test_append_and_read(d, n_kv, page, lens, at, pad):
    B, T = len(lens), sum(lens)
    M = max(-(-(a + n) // page) for a, n in zip(at, lens))
    kv = empty_pool(B, n_kv, d, page, M)
    k, v = rows_with_edges(T + pad, n_kv, d, 1), rows_with_edges(T + pad, n_kv, d, 2)
    want = {n: t.clone() for n, t in kv.items()}
    codes = {"k": ref.quantise(k), "v": ref.quantise(v)}
    start = [0]
    for b in range(B):
        for i in range(lens[b]):
            pp, off = int(kv["page_table"][b, (at[b] + i) // page]), (at[b] + i) % page
            for n in "kv":
                want[n + "_pages"][pp, :, off] = codes[n][0][start[b] + i]
                want[n + "_scale"][pp, :, off] = codes[n][1][start[b] + i]
        start.append(start[-1] + lens[b])
    c = sx.KV8(to_dev(kv))
    rs, ps = (torch.tensor(t, dtype=torch.int32, device=DEV) for t in (start, at))
    both = torch.stack((k, v), 1).to(DEV)                      # strided rows, as a projection leaves them
    c.sx_kv_append(both[:, 0], both[:, 1], rs, ps)
    c.check_status()
    for n in ("k_pages", "v_pages", "k_scale", "v_scale"):
        assert torch.equal(c.kv[n].cpu(), want[n]), n         # everything else in the pool is as it was
    # back: exact, and rows behind the last sequence are left alone
    out = torch.full((T + pad, 2, n_kv, d), -7.0, dtype=torch.bfloat16, device=DEV)
    c.sx_kv_read(out[:, 0], out[:, 1], rs, ps)
    c.check_status()
    for i, n in enumerate("kv"):
        back = torch.from_numpy(ref.dequantise(*codes[n])).to(torch.bfloat16)
        back[T:] = -7.0
        assert torch.equal(torch.nan_to_num(out[:, i].cpu(), nan=12345.0), torch.nan_to_num(back, nan=12345.0)), n


def test_append_behind_the_cache_by_default():
    kv = empty_pool(3, 2, 64, 16, 3)
    kv["cache_len"] = torch.tensor([4, 0, 31], dtype=torch.int32)
    k, v = rows_with_edges(6, 2, 64, 3).to(DEV), rows_with_edges(6, 2, 64, 4).to(DEV)
    rs = torch.tensor([0, 2, 5, 6], dtype=torch.int32, device=DEV)
    a, b = sx.KV8(to_dev(kv)), sx.KV8(to_dev(kv))
    a.sx_kv_append(k, v, rs)
    b.sx_kv_append(k, v, rs, b.kv["cache_len"].clone())
    for n in ("k_pages", "v_pages", "k_scale", "v_scale"):
        assert torch.equal(a.kv[n], b.kv[n]) and not torch.equal(a.kv[n].cpu(), kv[n])
    assert a.kv["cache_len"].tolist() == [4, 0, 31]


@pytest.mark.parametrize("what", ["page out of range", "table too short", "negative position", "starts descend", "start past the rows"])
def test_rows_without_a_place_are_skipped_and_reported(what):
    kv = empty_pool(2, 1, 64, 16, 2)
    start, at = [0, 3, 6], [0, 0]
    if what == "page out of range":
        kv["page_table"][1, 0] = 99
    elif what == "table too short":
        at = [0, 30]
    elif what == "negative position":
        at = [0, -2]
    elif what == "starts descend":
        start = [0, 3, 1]
    else:
        start = [0, 3, 9]
    k = rows_with_edges(6, 1, 64, 5).to(DEV)
    c = sx.KV8(to_dev(kv))
    rs, ps = (torch.tensor(t, dtype=torch.int32, device=DEV) for t in (start, at))
    c.sx_kv_append(k, k, rs, ps)
    with pytest.raises(sx.SxError):
        c.check_status()
    # the first sequence's rows are written whatever the second's say
    codes, byte = ref.quantise(k[:3])
    pp = int(kv["page_table"][0, 0])
    if what not in ("starts descend",):
        assert torch.equal(c.kv["k_pages"][pp, :, :3].cpu(), codes.permute(1, 0, 2))
    out = torch.full((6, 1, 64), -7.0, dtype=torch.bfloat16, device=DEV)
    c.sx_kv_read(out, out.clone(), rs, ps)
    with pytest.raises(sx.SxError):
        c.check_status()


# ---- attention -----------------------------------------------------------------------------------------------------
def check(kv, q, drafted, mask, scale=None, kernel=sx.ATTN_AUTO, cache=None):
    if kernel == sx.ATTN_TC and q.shape[-1] != 128:
        with pytest.raises(sx.SxError):
            sx.KV8(to_dev(kv)).sx_attention(q.to(DEV), drafted, kernel=kernel)
        kernel = sx.ATTN_AUTO
    c = cache or sx.KV8(to_dev(kv))
    got = c.sx_attention(q.to(DEV), drafted, None if mask is None else mask.to(DEV), scale, kernel=kernel)
    c.check_status()
    want, bound = ref.attention(kv, q, drafted, mask, q.shape[-1] ** -0.5 if scale is None else scale,
                                2.0 ** -11 if kernel == sx.ATTN_SPLIT else 2.0 ** -8)
    got = got.double().cpu().numpy()
    far = np.abs(got - want) / bound
    worst = float(far.max())
    assert worst <= 1.0, f"{worst:.2f} x the bound at {np.unravel_index(far.argmax(), far.shape)}"
    return got


KERNELS = [sx.ATTN_SPLIT, sx.ATTN_TC]
LENS = [[1], [16], [15, 17, 1], [127, 128, 129, 0], [1000, 3, 260], [65, 2049]]


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_kv,G,page", [(1, 1, 16), (2, 4, 64), (1, 8, 32), (3, 2, 48), (2, 3, 128)])
@pytest.mark.parametrize("lens", LENS)
def test_attention_one_row(kernel, d, n_kv, G, page, lens):
    drafted = len(lens) % 3
    kv = ref.make_cache(len(lens), n_kv, d, page, lens, drafted, seed=d + n_kv + len(lens), fill=0x7f)
    check(kv, ref.make_q(len(lens), 1, n_kv * G, d, 5), drafted, None, kernel=kernel)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("rows,drafted,G", [(2, 2, 4), (3, 3, 8), (8, 41, 4), (5, 5, 8), (16, 16, 1), (7, 64, 3), (64, 64, 2), (4, 4, 2)])
def test_attention_rows_with_masks(kernel, rows, drafted, G):
    lens = [0, 1, 100, 515]
    kv = ref.make_cache(4, 2, 128, 64, lens, drafted, seed=rows, fill=0xff)
    q = ref.make_q(4, rows, 2 * G, 128, 6)
    check(kv, q, drafted, ref.causal_masks(4, rows, drafted), kernel=kernel)
    # the first sequence has no cached slot and its last row sees none: zero
    mask = ref.random_masks(4, rows, drafted, 7, empty=[(0, rows - 1), (2, 0)])
    got = check(kv, q, drafted, mask, kernel=kernel)
    assert (got[0, rows - 1] == 0).all()


@pytest.mark.parametrize("kernel", KERNELS)
def test_attention_of_nothing(kernel):
    kv = ref.make_cache(2, 2, 128, 64, [0, 0], 0, seed=1)
    assert (check(kv, ref.make_q(2, 1, 4, 128, 8), 0, None, kernel=kernel) == 0).all()


PREFIX = [
    # groups, prefix, own lengths behind the prefix
    ([0, 2], [64], [0, 5]),
    ([0, 3], [100], [1, 0, 300]),
    ([0, 1, 4, 4, 6], [50, 333, 7, 128], [3, 0, 64, 65, 200, 1]),
    ([0, 5], [0], [7, 80, 0, 1, 33]),
    ([0, 12], [1025], [0, 1, 2, 15, 16, 17, 40, 63, 64, 65, 100, 129]),
]


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("d,G,rows,drafted,page", [(128, 4, 1, 2, 64), (128, 8, 3, 3, 32), (64, 2, 1, 0, 16), (128, 1, 8, 20, 64), (64, 4, 2, 2, 48), (128, 4, 8, 41, 128)])
@pytest.mark.parametrize("groups,prefix,mine", PREFIX)
@pytest.mark.parametrize("share", [True, False])
def test_attention_shared_prefix(kernel, d, G, rows, drafted, page, groups, prefix, mine, share):
    B = len(mine)
    of = [next(g for g in range(len(prefix)) if groups[g] <= b < groups[g + 1]) for b in range(B)]
    lens = [prefix[of[b]] + mine[b] for b in range(B)]
    kv = ref.make_cache(B, 2, d, page, lens, drafted, seed=B + rows, groups=groups, prefix=prefix, share_pages=share, fill=0x7f)
    q = ref.make_q(B, rows, 2 * G, d, 9)
    check(kv, q, drafted, ref.random_masks(B, rows, drafted, 3) if rows > 1 else None, kernel=kernel)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("groups", [None, [0, 3]])
def test_values_and_weights_of_many_magnitudes(kernel, groups):
    """A sink (large key, tiny value), value rows whose scales span 2^40, scores far from zero, a flat tail of thousands of
    slots that weighs as much as the sink."""
    kv = ref.make_cache(3, 1, 128, 64, [4000, 2600, 2000], 1, seed=3, groups=groups, prefix=[1777] if groups else None, share_pages=False)
    g = torch.Generator().manual_seed(1)
    kv["v_scale"] = (kv["v_scale"].int() + torch.randint(-20, 20, kv["v_scale"].shape, generator=g)).to(torch.uint8)
    if groups:                             # keep the members' copies of the prefix equal
        t = kv["page_table"]
        for s in range(1777):
            for b in (1, 2):
                kv["v_scale"][int(t[b, s // 64]), :, s % 64] = kv["v_scale"][int(t[0, s // 64]), :, s % 64]
    for b in range(3):
        pp = int(kv["page_table"][b, 0])
        kv["k_scale"][pp, :, 0] += 3
        kv["v_scale"][pp, :, 0] -= 12
    q = ref.make_q(3, 2, 4, 128, 10)
    check(kv, q, 1, None, kernel=kernel)
    check(kv, q, 1, None, scale=0.5, kernel=kernel)
    check(kv, q, 1, None, scale=-0.05, kernel=kernel)
    check(kv, q, 1, None, scale=0.0, kernel=kernel)
    check(kv, q * 2.0 ** -30, 1, None, scale=2.0 ** 28, kernel=kernel)
    check(kv, torch.zeros_like(q), 1, None, kernel=kernel)


@pytest.mark.parametrize("kernel", KERNELS)
def test_rows_that_are_not_finite_reach_those_who_see_them(kernel):
    lens, drafted, rows = [200, 130], 5, 3
    kv = ref.make_cache(2, 2, 128, 64, lens, drafted, seed=4)
    mask = torch.tensor([[0b00111, 0b01001, 0b11111], [0b00001, 0b00010, 0b10000]])
    q = ref.make_q(2, rows, 8, 128, 11)
    want, bound = ref.attention(kv, q, drafted, mask, 128 ** -0.5)
    # drafted slot 1 of sequence 0: a value row with the byte 255 and, where nobody sees it (slot 3 of sequence 1),
    # codes that are not numbers and the byte 255
    p0, o0 = int(kv["page_table"][0, 201 // 64]), 201 % 64
    kv["v_scale"][p0, 1, o0], kv["v_pages"][p0, 1, o0] = 255, 0
    p1, o1 = int(kv["page_table"][1, 133 // 64]), 133 % 64
    for n in ("k", "v"):
        kv[n + "_scale"][p1, :, o1] = 255
        kv[n + "_pages"][p1, :, o1] = 0x7f
    c = sx.KV8(to_dev(kv))
    got = c.sx_attention(q.to(DEV), drafted, mask.to(DEV), kernel=kernel).double().cpu().numpy()
    c.check_status()
    sees = np.zeros(got.shape, bool)
    sees[0, [0, 2], 4:] = True                                # KV head 1 = query heads 4..7
    assert np.isnan(got[sees]).all()
    assert np.isfinite(got[~sees]).all()
    assert (np.abs(got[~sees] - want[~sees]) <= bound[~sees]).all()


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("byte,code", [(254, 0x7e), (254, 0x7f), (255, 0xff), (0, 0x7f), (200, 0xfe)])
def test_slots_that_nobody_sees_can_hold_anything(kernel, byte, code):
    """Slots behind the last one, drafted slots outside every mask, and the slots in front of a sequence's own in a page that
    the prefix ends in: any code and exponent byte there changes nothing."""
    lens, drafted, rows = [200, 131, 150], 9, 2
    kv = ref.make_cache(3, 2, 128, 64, lens, drafted, seed=24, groups=[0, 3], prefix=[100], share_pages=False)
    mask = torch.tensor([[0b000000111, 0b010000001], [0b000000001, 0b000100000], [0, 1]])
    q = ref.make_q(3, rows, 8, 128, 25)
    before = sx.KV8(to_dev(kv)).sx_attention(q.to(DEV), drafted, mask.to(DEV), kernel=kernel)
    for b in range(3):
        dead = [lens[b] + i for i in range(drafted) if not any((int(m) >> i) & 1 for m in mask[b])]
        dead += list(range(lens[b] + drafted, int(kv["page_table"].shape[1]) * 64))
        if b:
            dead += list(range(100))                          # the first member's table stands for the prefix
        for s in dead:
            pp, off = int(kv["page_table"][b, s // 64]), s % 64
            for n in "kv":
                kv[n + "_scale"][pp, :, off] = byte
                kv[n + "_pages"][pp, :, off] = code
    c = sx.KV8(to_dev(kv))
    after = c.sx_attention(q.to(DEV), drafted, mask.to(DEV), kernel=kernel)
    c.check_status()
    assert torch.equal(before, after) and bool((after[2, 0] == 0).sum() == 0)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("groups", [None, [0, 2]])
@pytest.mark.parametrize("power", [10, 55, 64])
def test_scores_that_are_all_very_low(kernel, groups, power):
    """Every key the same, every score -2^(57 + power): whatever that is, the weights are equal and the output is the mean
    of the values (equal value scales: a power of two beside such a score is lost)."""
    kv = ref.make_cache(2, 1, 128, 64, [300, 200], 2, seed=5, groups=groups, prefix=[150] if groups else None)
    kv["k_pages"].fill_(0xb8)                                   # -1
    kv["k_scale"].fill_(127 + power)
    kv["v_scale"].fill_(127)
    got = check_mean(kv, torch.full((2, 3, 4, 128), 2.0 ** 50, dtype=torch.bfloat16), kernel)
    assert (got != 0).any()


def check_mean(kv, q, kernel):
    c = sx.KV8(to_dev(kv))
    got = c.sx_attention(q.to(DEV), 2, scale=1.0, kernel=kernel).double().cpu().numpy()
    c.check_status()
    for b in range(q.shape[0]):
        pos = np.arange(int(kv["cache_len"][b]) + 2)
        pp = kv["page_table"][b].numpy()[pos // 64].astype(np.int64)
        V = ref.dequantise(kv["v_pages"][pp, :, pos % 64], kv["v_scale"][pp, :, pos % 64])[:, 0]
        # fp32 sums of a few hundred terms, one division, a bf16 result
        far = len(pos) * 2.0 ** -23 * np.abs(V).mean(0)
        want = V.mean(0)
        assert (np.abs(got[b] - want) <= far + 2.0 ** -8 * (np.abs(want) + far)).all()
    return got


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("groups,mine", [([0, 9, 10, 11, 12], 12), ([0, 1, 1, 40], 40), ([0, 0, 0, 33], 33)])
def test_groups_that_are_not_alike(kernel, groups, mine):
    """One group with most of the sequences (more queries than the tile that an average group would need), empty groups."""
    prefix = [200] + [70] * (len(groups) - 2)
    of = [max(g for g in range(len(prefix)) if groups[g] <= b and groups[g + 1] > b) for b in range(mine)]
    lens = [prefix[g] + (b * 7) % 40 for b, g in enumerate(of)]
    kv = ref.make_cache(mine, 1, 128, 32, lens, 1, seed=mine, groups=groups, prefix=prefix, fill=0xff)
    check(kv, ref.make_q(mine, 1, 4, 128, 12), 1, None, kernel=kernel)
    check(kv, ref.make_q(mine, 1, 4, 128, 12), 1, None)


@pytest.mark.parametrize("kernel", KERNELS)
def test_a_query_that_is_not_finite_spoils_its_own_row_only(kernel):
    kv = ref.make_cache(2, 2, 128, 64, [300, 70], 3, seed=26, groups=[0, 2], prefix=[64])
    q = ref.make_q(2, 3, 8, 128, 27)
    want, bound = ref.attention(kv, q, 3, None, 128 ** -0.5)
    q[0, 1, 2, 5], q[1, 0, 7, 100] = math.nan, math.inf
    c = sx.KV8(to_dev(kv))
    got = c.sx_attention(q.to(DEV), 3, kernel=kernel).double().cpu().numpy()
    c.check_status()
    assert np.isnan(got[0, 1, 2]).all() and np.isnan(got[1, 0, 7]).all()
    got[0, 1, 2], got[1, 0, 7] = want[0, 1, 2], want[1, 0, 7]
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("B,groups", [(300, None), (300, 7), (700, 3), (511, 511), (1023, 1)])
def test_many_sequences(B, groups):
    """More sequences than the tensor-memory kernel plans for fall to the other one; every group a sequence; the limit."""
    g = torch.Generator().manual_seed(B)
    start = None if groups is None else [B * i // groups for i in range(groups + 1)]
    prefix = None if groups is None else [int(v) for v in torch.randint(0, 40, (groups,), generator=g)]
    own = torch.randint(0, 60, (B,), generator=g).tolist()
    of = None if groups is None else [next(i for i in range(groups) if b < start[i + 1]) for b in range(B)]
    lens = own if groups is None else [n + prefix[of[b]] for b, n in enumerate(own)]
    kv = ref.make_cache(B, 1, 128, 32, lens, 1, seed=B, groups=start, prefix=prefix)
    check(kv, ref.make_q(B, 1, 2, 128, 28), 1, None)


def test_a_graph_keeps_its_workspace():
    """A larger call after a capture gets a workspace of its own; the replay goes on using the one it was captured with."""
    kv = ref.make_cache(2, 2, 128, 64, [900, 400], 8, seed=29)
    c = sx.KV8(to_dev(kv))
    q1, q8 = ref.make_q(2, 1, 8, 128, 30), ref.make_q(2, 8, 64, 128, 31)
    d1, out = q1.to(DEV), torch.empty(2, 1, 8, 128, dtype=torch.bfloat16, device=DEV)
    want = c.sx_attention(d1, 8).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.sx_attention(d1, 8, out=out)
    for _ in range(3):
        c.sx_attention(q8.to(DEV), 8)
        fill = [torch.full((1 << 24,), 0x7f, dtype=torch.uint8, device=DEV) for _ in range(8)]
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)
        assert all(int(f.min()) == 0x7f and int(f.max()) == 0x7f for f in fill)
    c.check_status()


def test_page_and_group_faults_are_reported():
    kv = ref.make_cache(3, 2, 128, 64, [200, 100, 70], 1, seed=6)
    q = ref.make_q(3, 1, 8, 128, 12)
    for change in ("page", "length", "negative", "prefix", "order", "cover"):
        bad = {n: t.clone() for n, t in kv.items()}
        if change in ("prefix", "order", "cover"):
            bad["group_start"] = torch.tensor({"prefix": [0, 3], "order": [0, 4, 3], "cover": [0, 2]}[change], dtype=torch.int32)
            bad["prefix_len"] = torch.tensor({"prefix": [71], "order": [10, 10], "cover": [10]}[change], dtype=torch.int32)
        if change == "page":
            bad["page_table"][1, 0] = -1
        if change == "length":
            bad["cache_len"][2] = 256
        if change == "negative":
            bad["cache_len"][2] = -5
        c = sx.KV8(to_dev(bad))
        got = c.sx_attention(q.to(DEV), 1)
        with pytest.raises(sx.SxError):
            c.check_status()
        if change in ("prefix", "order", "cover"):           # every sequence has read its own table
            want, bound = ref.attention(kv, q, 1, None, 128 ** -0.5)
            assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("kernel", KERNELS)
def test_strided_queries_streams_and_graphs(kernel):
    kv = ref.make_cache(4, 2, 128, 64, [300, 280, 500, 257], 2, seed=8, groups=[0, 4], prefix=[256])
    proj = ref.make_q(4, 1, 8 + 4, 128, 13).to(DEV)            # query heads, then key and value heads, in one row
    q = proj[:, :, :8]
    want, bound = ref.attention(kv, q.cpu(), 2, None, 128 ** -0.5)
    c = sx.KV8(to_dev(kv))
    one = c.sx_attention(q, 2, kernel=kernel)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two = c.sx_attention(q, 2, kernel=kernel)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(one, two)
    assert (np.abs(one.double().cpu().numpy() - want) <= bound).all()
    # captured: the replay follows lengths, queries and pages as they are then
    q2 = q.contiguous().clone()
    out = torch.empty_like(q2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.sx_attention(q2, 2, out=out, kernel=kernel)
    q2.copy_(q * 0.5)
    c.kv["cache_len"].copy_(torch.tensor([290, 256, 400, 300], dtype=torch.int32))
    graph.replay()
    kv["cache_len"] = c.kv["cache_len"].cpu()
    want, bound = ref.attention(kv, q2.cpu(), 2, None, 128 ** -0.5)
    assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
    c.check_status()


def test_the_same_call_gives_the_same_bits():
    kv = ref.make_cache(5, 2, 128, 64, [900, 33, 700, 64, 2000], 4, seed=9, groups=[0, 3, 5], prefix=[33, 64], share_pages=False)
    q, m = ref.make_q(5, 4, 16, 128, 14).to(DEV), ref.causal_masks(5, 4, 4).to(DEV)
    c = sx.KV8(to_dev(kv))
    first = c.sx_attention(q, 4, m)
    for _ in range(5):
        assert torch.equal(c.sx_attention(q, 4, m), first)


def test_append_then_attend_then_read():
    """The operators as a decoder uses them: a prompt written once for four answers, tokens appended to each, attention
    after every step without anything in between."""
    B, n_kv, G, d, page, P = 4, 2, 4, 128, 64, 150
    g = torch.Generator().manual_seed(20)
    M, num = 4, 3 * B + 3
    table = torch.zeros(B, M, dtype=torch.int32)
    table[:, :2] = torch.tensor([5, 9])                       # two shared pages
    table[:, 2:] = (torch.randperm(B * 2, generator=g) + 10 - 10).view(B, 2).to(torch.int32)
    free = [p for p in range(num) if p not in (5, 9)][:B * 2]
    table[:, 2:] = torch.tensor(free, dtype=torch.int32).view(B, 2)
    kv = {n: torch.full((num, n_kv, page, d), 0x7f, dtype=torch.uint8) for n in ("k_pages", "v_pages")}
    kv |= {n: torch.full((num, n_kv, page), 0xff, dtype=torch.uint8) for n in ("k_scale", "v_scale")}
    kv |= {"page_table": table, "cache_len": torch.zeros(B, dtype=torch.int32),
           "group_start": torch.tensor([0, B], dtype=torch.int32), "prefix_len": torch.tensor([0], dtype=torch.int32)}
    c = sx.KV8(to_dev(kv))
    prompt = torch.randn(P, 2, n_kv, d, generator=g).to(torch.bfloat16)
    # the whole pages once (through member 0), the page that the prompt fills in part for every member
    whole = P // page * page
    rest = prompt[whole:].repeat(B, 1, 1, 1)
    rows = torch.cat((prompt[:whole], rest)).to(DEV)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    tail = P - whole
    c.sx_kv_append(rows[:whole, 0], rows[:whole, 1], i32([0, whole, whole, whole, whole]), i32([0] * B))
    c.sx_kv_append(rows[whole:, 0], rows[whole:, 1], i32([tail * b for b in range(B + 1)]), i32([whole] * B))
    c.kv["cache_len"].fill_(P)
    c.kv["prefix_len"].fill_(P)
    for step in range(3):
        new = torch.randn(B, 2, n_kv, d, generator=g).to(torch.bfloat16)
        q = torch.randn(B, 1, n_kv * G, d, generator=g).to(torch.bfloat16)
        c.sx_kv_append(new[:, 0].to(DEV), new[:, 1].to(DEV), i32(list(range(B + 1))))
        got = c.sx_attention(q.to(DEV), drafted=1)
        c.kv["cache_len"] += 1
        c.check_status()
        now = {n: t.cpu() for n, t in c.kv.items()}
        want, bound = ref.attention(now, q, 0, None, d ** -0.5)
        assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()
    out = torch.zeros(B * (P + 3), 2, n_kv, d, dtype=torch.bfloat16, device=DEV)
    c.sx_kv_read(out[:, 0], out[:, 1], i32([(P + 3) * b for b in range(B + 1)]), i32([0] * B))
    c.check_status()
    back = torch.from_numpy(ref.dequantise(*ref.quantise(prompt))).to(torch.bfloat16)
    for b in range(B):
        assert torch.equal(out[(P + 3) * b:(P + 3) * b + P].cpu(), back)


def test_offsets_past_32_bits():
    """Pages behind 4 GB of codes: the last pages of a large pool."""
    n_kv, page, d, num = 8, 128, 128, 36000                    # 4.7 GB of codes in each of K and V
    kv = {n: torch.zeros(num, n_kv, page, d, dtype=torch.uint8, device=DEV) for n in ("k_pages", "v_pages")}
    kv |= {n: torch.full((num, n_kv, page), 127, dtype=torch.uint8, device=DEV) for n in ("k_scale", "v_scale")}
    kv["page_table"] = torch.tensor([[num - 1, 0, num - 2]], dtype=torch.int32, device=DEV)
    kv["cache_len"] = torch.tensor([300], dtype=torch.int32, device=DEV)
    c = sx.KV8(kv)
    g = torch.Generator().manual_seed(2)
    rows = torch.randn(300, 2, n_kv, d, generator=g).to(torch.bfloat16)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    c.sx_kv_append(rows[:, 0].to(DEV), rows[:, 1].to(DEV), i32([0, 300]), i32([0]))
    out = torch.empty(300, 2, n_kv, d, dtype=torch.bfloat16, device=DEV)
    c.sx_kv_read(out[:, 0], out[:, 1], i32([0, 300]), i32([0]))
    q = ref.make_q(1, 1, 32, d, 3)
    got = c.sx_attention(q.to(DEV))
    many = c.sx_attention(q.expand(1, 8, 32, d).contiguous().to(DEV))
    c.check_status()
    kq, vq = ref.quantise(rows[:, 0]), ref.quantise(rows[:, 1])
    assert torch.equal(out[:, 0].cpu(), torch.from_numpy(ref.dequantise(*kq)).to(torch.bfloat16))
    assert torch.equal(out[:, 1].cpu(), torch.from_numpy(ref.dequantise(*vq)).to(torch.bfloat16))
    small = {"k_pages": torch.zeros(3, n_kv, page, d, dtype=torch.uint8), "v_pages": torch.zeros(3, n_kv, page, d, dtype=torch.uint8),
             "k_scale": torch.zeros(3, n_kv, page, dtype=torch.uint8), "v_scale": torch.zeros(3, n_kv, page, dtype=torch.uint8),
             "page_table": torch.tensor([[0, 1, 2]]), "cache_len": torch.tensor([300])}
    for s in range(300):
        small["k_pages"][s // page, :, s % page], small["k_scale"][s // page, :, s % page] = kq[0][s], kq[1][s]
        small["v_pages"][s // page, :, s % page], small["v_scale"][s // page, :, s % page] = vq[0][s], vq[1][s]
    want, bound = ref.attention(small, q, 0, None, d ** -0.5)
    assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()
    assert (np.abs(many.double().cpu().numpy() - want) <= bound).all()
