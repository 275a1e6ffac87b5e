"""The draft step, the iteration and the commit on an 8-bit cache: parity with the oracle, whose cache then holds every
row as the codes read back.  The comparison is the one of tests/parity.py; only the caches differ."""
from __future__ import annotations

import dataclasses

import pytest
import torch

from oracle import specexit_oracle as orc
from paper_2509_24248_b200 import binding, synth
from tests import harness, kv8_ref as ref, parity

pytestmark = pytest.mark.gpu
SHAPE = synth.ModelShape(H=256, n_q=4, n_kv=2, d=64, F=688, V=4096)
SHAPE128 = synth.ModelShape(H=256, n_q=8, n_kv=2, d=128, F=512, V=3001, page=32)


class CodesKV(orc.PagedKV):
    """The oracle's cache with every written row rounded to codes and back."""

    def write(self, b, slot, k, v):
        super().write(b, slot, *(torch.from_numpy(ref.dequantise(*ref.quantise(t))).to(torch.bfloat16) for t in (k, v)))


def as_codes(kv):
    """A bf16 cache's pages as codes; what belongs to nobody (it is poisoned with NaN) becomes codes that are not numbers."""
    got = {n: kv[n] for n in ("page_table", "cache_len")}
    for n in "kv":
        pages = kv[n + "_pages"]
        codes, byte = ref.quantise(pages)
        dead = torch.isnan(pages.float()).any(-1)
        codes[dead] = 0x7f
        got[n + "_pages"], got[n + "_scale"] = codes, byte
    return got


def back(kv):
    """bf16 pages of a cache of codes (rows that are not numbers: NaN)."""
    return {n: torch.from_numpy(ref.dequantise(kv[n + "_pages"].cpu(), kv[n + "_scale"].cpu())).to(torch.bfloat16) for n in "kv"}


def on_codes(monkeypatch, groups=None, prefix=None):
    """Points the parity harness at 8-bit caches."""
    def make_gpu(case, act=(0, 0, 0), sample_drafts=False):
        wl = case.wl
        sx = binding.SpecExit(wl.shape, case.weights, wl.B, wl.mode, wl.K, wl.topk if wl.mode == synth.TREE else 1, wl.max_nodes,
                              act=act, sample_drafts=sample_drafts, tiled=parity.TILED, kv_dtype=binding.KV_E4M3)
        kv = as_codes(case.kv)
        if groups is not None:
            kv["group_start"] = torch.tensor(groups, dtype=torch.int32)
            kv["prefix_len"] = torch.tensor(prefix, dtype=torch.int32)
        sx.set_kv(kv)
        if parity.ATTN is not None:
            sx.sx_set_attention(parity.ATTN)
        return sx

    def oracle_kv(case):
        p = back(as_codes(case.kv))
        return CodesKV(p["k"], p["v"], case.kv["page_table"], case.kv["cache_len"])

    def replay(sx, case):
        p = back(sx.kv)
        table, lens, page = case.kv["page_table"], case.kv["cache_len"], case.wl.shape.page

        def f(kv, rows):
            for b in range(case.wl.B):
                for i in rows:
                    slot = int(lens[b]) + i
                    pp = int(table[b, slot // page])
                    orc.PagedKV.write(kv, b, slot, p["k"][pp, :, slot % page], p["v"][pp, :, slot % page])
        return f

    monkeypatch.setattr(parity, "make_gpu", make_gpu)
    monkeypatch.setattr(parity, "_kv_replay", replay)
    monkeypatch.setattr(harness, "oracle_kv", oracle_kv)


def share(case, groups, prefix):
    """Makes the members of a group hold the same first slots (whole pages shared, the rest copied)."""
    page, t, kv = case.wl.shape.page, case.kv["page_table"], case.kv
    for g, n in enumerate(prefix):
        for b in range(groups[g] + 1, groups[g + 1]):
            for lp in range(-(-n // page)):
                a0, b0 = int(t[groups[g], lp]), int(t[b, lp])
                if (lp + 1) * page <= n:
                    t[b, lp] = a0
                else:
                    for name in ("k_pages", "v_pages"):
                        kv[name][b0, :, :n - lp * page] = kv[name][a0, :, :n - lp * page]


CHAIN = dict(name="kv8", mode=synth.CHAIN, K=4, len_lo=100, len_hi=300, seed=31)
TREE = dict(name="kv8t", mode=synth.TREE, K=4, topk=4, max_nodes=20, len_lo=90, len_hi=260, seed=32)


@pytest.mark.parametrize("shape,kw,B,kernel", [
    (SHAPE, CHAIN, 1, None), (SHAPE, TREE, 2, None), (SHAPE, TREE, 3, binding.ATTN_SPLIT),
    *[(SHAPE128, kw, B, k) for kw, B in ((CHAIN, 3), (TREE, 2)) for k in (None, binding.ATTN_SPLIT, binding.ATTN_TC)]])
def test_iteration_parity(monkeypatch, shape, kw, B, kernel):
    monkeypatch.setattr(parity, "ATTN", kernel)
    on_codes(monkeypatch)
    case = harness.build_case(synth.Workload(shape=shape, B=B, **kw))
    (parity.run_chain if kw["mode"] == synth.CHAIN else parity.run_tree)(case)


@pytest.mark.parametrize("kernel", [None, binding.ATTN_SPLIT, binding.ATTN_TC])
@pytest.mark.parametrize("kw", [CHAIN, TREE])
def test_iteration_parity_with_shared_prefixes(monkeypatch, kw, kernel):
    monkeypatch.setattr(parity, "ATTN", kernel)
    groups, prefix = [0, 3, 4, 6], [85, 40, 64]
    on_codes(monkeypatch, groups, prefix)
    case = harness.build_case(synth.Workload(shape=SHAPE128, B=6, **kw))
    share(case, groups, prefix)
    (parity.run_chain if kw["mode"] == synth.CHAIN else parity.run_tree)(case)


def test_commit_writes_codes():
    """A committed iteration leaves in the cache what the same commit leaves in a bf16 cache, rounded to codes."""
    wl = synth.Workload(shape=SHAPE128, B=2, **CHAIN)
    case = harness.build_case(wl, poison_tail=False)
    P = wl.K + 1
    th = torch.randn(wl.B, P, SHAPE128.H, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    cand = torch.randint(0, SHAPE128.V, (wl.B, P), generator=torch.Generator().manual_seed(6), dtype=torch.int32)
    path = torch.tensor([[0, 1, 2, -1, -1], [0, 1, 2, 3, 4]], dtype=torch.int32)
    L, rec = torch.tensor([2, 4], dtype=torch.int32), torch.tensor([3, 5], dtype=torch.int32)
    got = {}
    for dtype in (binding.KV_BF16, binding.KV_E4M3):
        sx = binding.SpecExit(SHAPE128, case.weights, wl.B, wl.mode, wl.K, kv_dtype=dtype)
        sx.set_kv(as_codes(case.kv) if dtype else case.kv)
        feat, tok = sx.sx_commit(*(t.to(sx.dev) for t in (th, cand, path, L, rec)))
        sx.check_status()
        got[dtype] = (sx.kv, feat, tok)
    (a, fa, ta), (b, fb, tb) = got[binding.KV_BF16], got[binding.KV_E4M3]
    assert torch.equal(fa, fb) and torch.equal(ta, tb) and torch.equal(a["cache_len"], b["cache_len"])
    want = as_codes({n: t.cpu() for n, t in a.items()})
    for n in ("k_pages", "v_pages", "k_scale", "v_scale"):
        assert torch.equal(b[n].cpu(), want[n]), n


def test_prompt_iteration_commit_in_a_row():
    """Prompt into the cache with sx_kv_append, then iterations with commits, two answers of one prompt in a group: the
    prefix changes nothing but who reads it (same tokens and hidden states within the rounding of other sums)."""
    wl = synth.Workload(shape=SHAPE128, B=4, **CHAIN)
    case = harness.build_case(wl, poison_tail=False)
    n, page = 96, SHAPE128.page
    g = torch.Generator().manual_seed(8)
    rows = torch.randn(4 * n, 2, SHAPE128.n_kv, SHAPE128.d, generator=g).to(torch.bfloat16)
    rows[n:2 * n], rows[3 * n:] = rows[:n], rows[2 * n:3 * n]
    outs = []
    for groups in (None, [0, 2, 4]):
        kv = as_codes(case.kv)
        kv["cache_len"] = torch.zeros(4, dtype=torch.int32)
        if groups:
            kv["group_start"], kv["prefix_len"] = torch.tensor(groups, dtype=torch.int32), torch.tensor([n, n - 5], dtype=torch.int32)
        sx = binding.SpecExit(SHAPE128, case.weights, 4, wl.mode, wl.K, kv_dtype=binding.KV_E4M3)
        sx.set_kv(kv)
        c = binding.KV8(sx.kv)
        c.sx_kv_append(rows[:, 0].to(sx.dev), rows[:, 1].to(sx.dev), torch.arange(5, dtype=torch.int32, device=sx.dev) * n)
        sx.kv["cache_len"].fill_(n)
        st, out = sx.new_state(4), sx.new_outputs(4)
        feat, tok = case.f0.to(sx.dev), case.t0.to(sx.dev)
        th = torch.randn(4, wl.K + 1, SHAPE128.H, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).to(sx.dev)
        got = []
        for _ in range(2):
            sx.sx_spec_exit_iter(binding.ExitParams(), st, feat, tok, th, out)
            got.append((out["hidden_d"].clone(), out["cand_tok_d"].clone(), out["accept_len_out_d"].clone()))
            feat, tok = sx.sx_commit(th, out["cand_tok_d"], out["path_d"], out["accept_len_out_d"], out["recover_tok_out_d"])
        sx.check_status()
        c.check_status()
        outs.append(got)
    for (ha, ca, la), (hb, cb, lb) in zip(*outs):
        assert torch.equal(ca[:, :2], cb[:, :2]) and torch.equal(la, lb)
        assert float((ha[:, 0].double() - hb[:, 0].double()).norm() / ha[:, 0].double().norm()) < 2e-2


def test_refusals():
    wl = synth.Workload(shape=SHAPE128, B=2, **CHAIN)
    case = harness.build_case(wl, poison_tail=False)
    sx = binding.SpecExit(SHAPE128, case.weights, 2, wl.mode, wl.K)
    sx.set_kv(as_codes(case.kv))                                # a bf16 context
    with pytest.raises(binding.SxError):
        sx.sx_draft_step(1, case.f0.to(sx.dev), case.t0.to(sx.dev))
    sx = binding.SpecExit(SHAPE128, case.weights, 2, wl.mode, wl.K, kv_dtype=binding.KV_E4M3)
    sx.set_kv(case.kv)                                          # an 8-bit one
    with pytest.raises(binding.SxError):
        sx.sx_draft_step(1, case.f0.to(sx.dev), case.t0.to(sx.dev))
    for shape in (dataclasses.replace(SHAPE128, page=24), synth.ModelShape(H=64, n_q=4, n_kv=2, d=16, F=96, V=200, page=16)):
        with pytest.raises(binding.SxError):
            binding.SpecExit(shape, synth.make_weights(shape, 1), 2, wl.mode, wl.K, kv_dtype=binding.KV_E4M3)
