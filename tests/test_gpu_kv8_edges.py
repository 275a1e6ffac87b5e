"""Rows and calls at the edges of the 8-bit cache: value rows of zeros, queries with an outlier channel, values at both ends
of the format, pages that do not exist, members without slots of their own, calls from two threads."""
from __future__ import annotations

import sys
import threading

import numpy as np
import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import kv8_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KERNELS = [sx.ATTN_SPLIT, sx.ATTN_TC]
WEIGHT = {sx.ATTN_SPLIT: 2.0 ** -11, sx.ATTN_TC: 2.0 ** -8, sx.ATTN_AUTO: 2.0 ** -8}    # half a step of a weight's type


def to_dev(kv):
    return {n: t.to(DEV) for n, t in kv.items()}


def near(got, want, bound):
    far = np.abs(got - want) / bound                              # NaN where either is
    worst = np.nan_to_num(far, nan=np.inf)
    assert worst.max() <= 1.0, f"{worst.max():.3g} x the bound at {np.unravel_index(worst.argmax(), far.shape)}: {got.flat[worst.argmax()]}, {want.flat[worst.argmax()]}"


def one_sequence(k, v, page=64):
    """A cache of one sequence (batch 1) that holds the rows ``k`` / ``v`` [n, n_kv, d], page behind page."""
    n, n_kv, d = k.shape
    M = -(-n // page)
    kv = {"page_table": torch.arange(M, dtype=torch.int32).view(1, M), "cache_len": torch.tensor([n], dtype=torch.int32)}
    for name, t in (("k", k), ("v", v)):
        codes, byte = ref.quantise(t.to(torch.bfloat16))
        full = torch.zeros(M * page, n_kv, d, dtype=torch.uint8)
        full[:n] = codes
        fb = torch.full((M * page, n_kv), 127, dtype=torch.uint8)
        fb[:n] = byte
        kv[name + "_pages"] = full.view(M, page, n_kv, d).permute(0, 2, 1, 3).contiguous()
        kv[name + "_scale"] = fb.view(M, page, n_kv).permute(0, 2, 1).contiguous()
    return kv


def many(kv, B, group=None):
    """The same sequence B times, in the same pages; ``group``: its first slots as a shared prefix of all of them."""
    out = {n: t for n, t in kv.items() if n not in ("page_table", "cache_len")}
    out["page_table"], out["cache_len"] = kv["page_table"].expand(B, -1).contiguous(), kv["cache_len"].expand(B).contiguous()
    if group is not None:
        out["group_start"], out["prefix_len"] = torch.tensor([0, B], dtype=torch.int32), torch.tensor([group], dtype=torch.int32)
    return out


def attend_like_one(kv, B, q, kernel, group=None, drafted=0, mask=None, scale=None):
    """B equal sequences with equal queries ``q`` [1, rows, nq, d]: every one of them against the reference of one."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    c = sx.KV8(to_dev(many(kv, B, group)))
    got = c.sx_attention(q.expand(B, -1, -1, -1).contiguous().to(DEV), drafted,
                         None if mask is None else mask.expand(B, -1).contiguous().to(DEV), scale, kernel=kernel)
    c.check_status()
    want, bound = ref.attention(kv, q, drafted, mask, scale, WEIGHT[kernel])
    got = got.double().cpu().numpy()
    for b in range(B):
        near(got[b:b + 1], want, bound)
    return got


# ---- value rows of zeros ------------------------------------------------------------------------------------------
def with_gap(n, n_kv, G, d, at, gap, size, seed, zero=True):
    """Keys whose scores are small, but for slots ``at``, which lie ``gap`` nats higher and whose value rows are zeros (or
    not); values of magnitude ``size``."""
    g = torch.Generator().manual_seed(seed)
    q = torch.ones(1, 1, n_kv * G, d) * torch.where(torch.rand(d, generator=g) < 0.5, -1.0, 1.0)
    k = torch.randn(n, n_kv, d, generator=g) * 0.3
    v = torch.randn(n, n_kv, d, generator=g) * size
    for i, s in enumerate(at):
        k[s] = q[0, 0, 0] * (gap - i) / d ** 0.5                    # scale q . k = gap - i
        if zero:
            v[s] = 0.0
    return q.to(torch.bfloat16), k, v


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("n,B", [(256, 222), (4096, 40)])
@pytest.mark.parametrize("size", [0.02, 2.0 ** -18])
@pytest.mark.parametrize("gap", [0, 8, 10, 12, 30, 80])
def test_a_value_row_of_zeros(kernel, n, B, size, gap):
    """A sink whose value is zero takes weight and gives nothing; the others keep their precision (runs of hundreds of
    slots: as many equal sequences as that takes)."""
    q, k, v = with_gap(n, 8, 1, 128, [0], gap, size, n + gap)
    attend_like_one(one_sequence(k, v), B, q, kernel)


@pytest.mark.parametrize("kernel", [sx.ATTN_SPLIT])
@pytest.mark.parametrize("d,G,n_kv", [(64, 1, 2), (64, 8, 2), (128, 2, 4), (128, 16, 1)])
@pytest.mark.parametrize("at", [[0], [3, 19, 20, 70], [255], list(range(64)), list(range(16, 256))])
@pytest.mark.parametrize("gap", [6, 13, 60])
def test_several_value_rows_of_zeros(kernel, d, G, n_kv, at, gap):
    q, k, v = with_gap(256, n_kv, G, d, at, gap, 1.0, gap + len(at))
    v[:, :, ::2] *= -1.0                                            # zero rows hold both zeros
    attend_like_one(one_sequence(k, v), 97, q, kernel)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("prefix", [100, 256])
@pytest.mark.parametrize("gap", [11, 40])
def test_a_value_row_of_zeros_in_a_shared_prefix(kernel, prefix, gap):
    q, k, v = with_gap(300, 2, 4, 128, [0, 130, 299], gap, 0.02, 5)
    attend_like_one(one_sequence(k, v), 40, q, kernel, group=prefix)


@pytest.mark.parametrize("kernel", KERNELS)
def test_drafted_value_rows_of_zeros(kernel):
    """Some rows see the drafted slot whose value is zero and whose score is high, others do not."""
    q, k, v = with_gap(70, 2, 2, 128, [66, 69], 14, 0.02, 6)
    kv = one_sequence(k, v)
    kv["cache_len"] -= 5                                            # slots 65 .. 69 are drafted
    mask = torch.tensor([[0b00000, 0b00010, 0b10001, 0b11111]])
    attend_like_one(kv, 33, q.expand(1, 4, -1, -1), kernel, drafted=5, mask=mask)


@pytest.mark.parametrize("kernel", KERNELS)
def test_nothing_but_value_rows_of_zeros(kernel):
    q, k, v = with_gap(200, 2, 2, 128, list(range(200)), 100, 1.0, 7)
    got = attend_like_one(one_sequence(k, v), 19, q, kernel)
    assert (got == 0).all()


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("n", [5, 256])
@pytest.mark.parametrize("size,gap", [(1.0, 64), (1.0, 68), (16.0, 70), (2.0 ** 40, 84)])
def test_a_value_row_of_zeros_far_above_the_rest(kernel, n, size, gap):
    """Outputs down to 2^-98: every one of the other slots still counts.  (Its weight is a number of 32 bits, so the gap ends
    at 2^-126 = e^-87.)"""
    q, k, v = with_gap(n, 2, 4, 128, [0], gap, size, 11)
    attend_like_one(one_sequence(k, v), 33, q, kernel)


@pytest.mark.parametrize("size", [2.0 ** 60, 2.0 ** 100])
@pytest.mark.parametrize("gap", [0, 12, 40])
def test_a_value_row_of_zeros_beside_huge_ones(size, gap):
    q, k, v = with_gap(256, 2, 4, 128, [0, 200], gap, size, gap)
    attend_like_one(one_sequence(k, v), 97, q, sx.ATTN_SPLIT)


# ---- queries with an outlier channel --------------------------------------------------------------------------------
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [0, 9, 11, 13])
def test_a_query_channel_far_above_the_rest(kernel, d, power):
    """A channel 2^power times the others in which every key is zero: it decides nothing, and what decides keeps its bits.
    (The others lie in [1, 2) and the outlier is 1.5 x 2^power, so that the smallest is 2^-14 of it or more.)"""
    if kernel == sx.ATTN_TC and d != 128:
        kernel = sx.ATTN_AUTO
    g = torch.Generator().manual_seed(power)
    q = (1 + torch.rand(1, 3, 8, d, generator=g)) * torch.where(torch.rand(1, 3, 8, d, generator=g) < 0.5, -1.0, 1.0)
    k, v = torch.randn(500, 2, d, generator=g), torch.randn(500, 2, d, generator=g)
    q[..., 5] = 1.5 * 2.0 ** power
    k[..., 5] = 0.0
    attend_like_one(one_sequence(k, v), 3, q.to(torch.bfloat16), kernel, scale=2.0 * d ** -0.5)


# ---- values at both ends of the format --------------------------------------------------------------------------------
def rising(n, n_kv, G, d, seed):
    """Scores that rise by 18 nats behind the first 128 slots: weights of 2^26 relative to those of the first block."""
    g = torch.Generator().manual_seed(seed)
    q = torch.where(torch.rand(1, 1, n_kv * G, d, generator=g) < 0.5, -1.0, 1.0)
    q[:] = q[:, :, :1]
    k, v = torch.randn(n, n_kv, d, generator=g) * 0.3, torch.randn(n, n_kv, d, generator=g)
    k[128:] += q[0, 0, 0] * 18.0 / d ** 0.5
    return q, k, v


@pytest.mark.parametrize("kernel", [sx.ATTN_AUTO, *KERNELS])
@pytest.mark.parametrize("group", [None, 333])
@pytest.mark.parametrize("power", [-62, -40, 96, 110, 122])
@pytest.mark.parametrize("rows", [1, 8])
def test_values_of_all_magnitudes_of_the_format(kernel, group, power, rows):
    """The mean of finite values is finite, whatever weights they met on the way (enough equal sequences that a block whose
    scores are low and one whose scores are high fall into one run)."""
    q, k, v = rising(600, 1, 4, 128, 3)
    v = v * 2.0 ** power
    attend_like_one(one_sequence(k, v), 200, q.expand(1, rows, -1, -1).to(torch.bfloat16), kernel, group=group)


@pytest.mark.parametrize("kernel", KERNELS)
def test_many_values_at_the_top_of_the_format(kernel):
    """20000 slots of +-1.5 x 2^126 with weights that rise: sums of what the format allows."""
    q, k, v = rising(20000, 1, 4, 128, 4)
    v = torch.where(v < -0.8, -1.5, 1.5) * 2.0 ** 126
    attend_like_one(one_sequence(k, v), 1, q.expand(1, 8, -1, -1).to(torch.bfloat16), kernel)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("low,high", [(-62, -55), (-30, 30), (70, 120)])
def test_values_of_many_magnitudes_in_one_sequence(kernel, low, high):
    g = torch.Generator().manual_seed(high)
    k, v = torch.randn(700, 2, 128, generator=g), torch.randn(700, 2, 128, generator=g)
    v *= torch.exp2(torch.randint(low, high + 1, (700, 2, 1), generator=g).float())
    q = ref.make_q(1, 6, 8, 128, 7)
    attend_like_one(one_sequence(k, v), 5, q, kernel)


# ---- pages that do not exist ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("page", [-1, 1 << 20])
@pytest.mark.parametrize("groups", [None, [0, 2, 4]])
def test_a_page_that_does_not_exist_holds_zeros_and_is_reported(kernel, page, groups):
    """Its slots count as rows of zeros; every other sequence, and every other group, is served as ever."""
    lens, drafted = [300, 280, 260, 301], 2
    kv = ref.make_cache(4, 2, 128, 64, lens, drafted, seed=41, groups=groups, prefix=[200, 140] if groups else None, share_pages=False, fill=0x7f)
    q = ref.make_q(4, 2, 8, 128, 42)
    bad = {n: t.clone() for n, t in kv.items()}
    bad["page_table"][0, 1] = page
    zero = {n: t.clone() for n, t in kv.items()}                   # the same with a page of zeros there
    for b in range(2 if groups else 1):                             # the first member's table stands for both members
        for n in ("k", "v"):
            zero[n + "_pages"][int(kv["page_table"][b, 1])] = 0
            zero[n + "_scale"][int(kv["page_table"][b, 1])] = 127
    c = sx.KV8(to_dev(bad))
    for _ in range(3):
        got = c.sx_attention(q.to(DEV), drafted, kernel=kernel).double().cpu().numpy()
        with pytest.raises(sx.SxError):
            c.check_status()
        near(got, *ref.attention(zero, q, drafted, None, 128 ** -0.5, WEIGHT[kernel]))


@pytest.mark.parametrize("kernel", KERNELS)
def test_a_page_that_does_not_exist_takes_nothing_from_the_sequences_before(kernel):
    """Sequences whose rows are not finite and sequences without a page in turn, several of them in a run: NaN and zero."""
    B = 200
    kv = ref.make_cache(1, 1, 128, 64, [384], 0, seed=43)
    for n in ("k_scale", "v_scale"):
        kv[n].fill_(255)
    kv = many(kv, B)
    kv["page_table"][1::2] = -1
    c = sx.KV8(to_dev(kv))
    got = c.sx_attention(ref.make_q(B, 2, 4, 128, 44).to(DEV), kernel=kernel)
    with pytest.raises(sx.SxError):
        c.check_status()
    assert bool(got[::2].isnan().all()) and bool((got[1::2] == 0).all())


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("what", ["length", "negative"])
def test_a_length_that_cannot_be_is_reported_and_the_others_are_served(kernel, what):
    kv = ref.make_cache(3, 2, 128, 64, [200, 100, 70], 1, seed=6)
    q = ref.make_q(3, 2, 8, 128, 12)
    bad = {n: t.clone() for n, t in kv.items()}
    bad["cache_len"][1] = 256 if what == "length" else -5
    c = sx.KV8(to_dev(bad))
    got = c.sx_attention(q.to(DEV), 1, kernel=kernel).double().cpu().numpy()
    with pytest.raises(sx.SxError):
        c.check_status()
    want, bound = ref.attention(kv, q, 1, None, 128 ** -0.5, WEIGHT[kernel])
    near(got[[0, 2]], want[[0, 2]], bound[[0, 2]])


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("drafted", [0, 1])
@pytest.mark.parametrize("prefix", [100, 128, 200])
def test_members_need_no_pages_for_the_prefix(kernel, drafted, prefix):
    """Only the first member's table is read for the prefix: the others' entries may be -1 there, also where a member has
    no slot of its own behind a prefix that ends inside a page."""
    lens = [prefix, prefix, prefix + 70, prefix]
    kv = ref.make_cache(4, 2, 128, 64, lens, drafted, seed=43, groups=[0, 4], prefix=[prefix], share_pages=False)
    q = ref.make_q(4, 2, 8, 128, 44)
    want, bound = ref.attention(kv, q, drafted, None, 128 ** -0.5, WEIGHT[kernel])
    for b in range(1, 4):
        own = lens[b] + drafted > prefix
        kv["page_table"][b, :prefix // 64 if own else None] = -1
    c = sx.KV8(to_dev(kv))
    got = c.sx_attention(q.to(DEV), drafted, kernel=kernel).double().cpu().numpy()
    c.check_status()
    near(got, want, bound)


# ---- callers ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kernel", KERNELS)
def test_threads_with_batches_of_different_sizes(kernel):
    """Each thread has a cache and a stream of its own; nothing of one call is state of another's."""
    jobs, wrong = [], []
    for B in (440, 440, 1, 1):
        kv = ref.make_cache(B, 1, 128, 16, [1] * B, 0, seed=B)
        c, q = sx.KV8(to_dev(kv)), ref.make_q(B, 1, 2, 128, B).to(DEV)
        jobs.append((c, q, c.sx_attention(q, kernel=kernel).clone()))
    torch.cuda.synchronize()
    gate, interval = threading.Barrier(len(jobs)), sys.getswitchinterval()
    sys.setswitchinterval(1e-6)

    def work(c, q, want):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                got = torch.empty_like(want)
                gate.wait()
                for i in range(20000):
                    c.sx_attention(q, kernel=kernel, out=got)
                    if i % 20 == 19:                                # short queues: the calls themselves meet
                        s.synchronize()
                if not torch.equal(got, want):
                    wrong.append("other bits")
        except Exception as e:
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    sys.setswitchinterval(interval)
    assert not wrong, wrong


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("power", [-50, 60, 110, 120])
def test_keys_of_all_magnitudes_of_the_format(kernel, power):
    """Huge keys under tiny queries, and the other way round: ordinary scores."""
    g = torch.Generator().manual_seed(9)
    k, v = torch.randn(400, 2, 128, generator=g), torch.randn(400, 2, 128, generator=g)
    q = ref.make_q(1, 3, 8, 128, 10) * 2.0 ** -power
    attend_like_one(one_sequence(k * 2.0 ** power, v), 4, q, kernel)
