"""Draft calls on an 8-bit cache: what they refuse, and what they do not look at."""
from __future__ import annotations

import pytest
import torch

from paper_2509_24248_b200 import binding, synth
from tests import harness, kv8_ref as ref
from tests.test_gpu_kv8_draft import CHAIN, SHAPE, as_codes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv_dtype", [binding.KV_BF16, binding.KV_E4M3])
def test_a_forced_kernel_that_cannot_run_is_refused_before_anything_is_written(kv_dtype):
    wl = synth.Workload(shape=SHAPE, B=2, **CHAIN)                  # head dimension 64: no tensor-memory kernel
    case = harness.build_case(wl, poison_tail=False)
    sx = binding.SpecExit(SHAPE, case.weights, 2, wl.mode, wl.K, kv_dtype=kv_dtype)
    sx.set_kv(as_codes(case.kv) if kv_dtype == binding.KV_E4M3 else case.kv)
    before = {n: t.clone() for n, t in sx.kv.items()}
    sx.sx_set_attention(binding.ATTN_TC)
    with pytest.raises(binding.SxError):
        sx.sx_draft_step(1, case.f0.to(sx.dev), case.t0.to(sx.dev))
    out = sx.new_outputs(2)
    th = torch.zeros(2, wl.K + 1, SHAPE.H, dtype=torch.bfloat16, device=sx.dev)
    with pytest.raises(binding.SxError):
        sx.sx_spec_exit_iter(binding.ExitParams(), sx.new_state(2), case.f0.to(sx.dev), case.t0.to(sx.dev), th, out)
    torch.cuda.synchronize()
    assert all(torch.equal(before[n], sx.kv[n]) for n in before)
    sx.sx_set_attention(binding.ATTN_AUTO)
    sx.sx_draft_step(1, case.f0.to(sx.dev), case.t0.to(sx.dev))
    sx.check_status()


def test_a_bf16_cache_is_seven_fields():
    """What lies behind v_pages_d is not looked at in a context whose cache is bf16: a caller that knows only the first seven
    fields, or sets no others, is served as before."""
    wl = synth.Workload(shape=SHAPE, B=2, **CHAIN)
    case = harness.build_case(wl, poison_tail=False)
    got = []
    for junk in (False, True):
        sx = binding.SpecExit(SHAPE, case.weights, 2, wl.mode, wl.K)
        sx.set_kv(case.kv)
        if junk:
            k = sx._kv_struct
            k.dtype, k.n_groups, k.k_scale_d, k.v_scale_d, k.group_start_d, k.prefix_len_d = 0x5a5a5a5a, 77, 3, 5, 7, 9
        one = sx.sx_draft_step(1, case.f0.to(sx.dev), case.t0.to(sx.dev))
        out, st = sx.new_outputs(2), sx.new_state(2)
        th = torch.randn(2, wl.K + 1, SHAPE.H, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(sx.dev)
        sx.sx_spec_exit_iter(binding.ExitParams(), st, case.f0.to(sx.dev), case.t0.to(sx.dev), th, out)
        nxt = sx.sx_commit(th, out["cand_tok_d"], out["path_d"], out["accept_len_out_d"], out["recover_tok_out_d"])
        sx.check_status()
        got.append([*(t for t in one if t is not None), *(out[n] for n in sorted(out)), *nxt, *sx.kv.values()])
    for a, b in zip(*got):
        assert torch.equal(torch.nan_to_num(a.float(), nan=9.0), torch.nan_to_num(b.float(), nan=9.0))


@pytest.mark.parametrize("ctas", [2, 301])
def test_waits_that_sleep_give_up_too(ctas):
    """Odd CTAs of the self-test wait as the attention's kernels do: none may report success, all must return, and the
    attention must go on working."""
    lib = binding.load_library()
    status, reached = (torch.zeros(n, dtype=torch.int32, device="cuda:0") for n in (1, 2))
    assert lib.sx_selftest_bounded_wait(50, ctas, status.data_ptr(), reached.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert int(status.item()) == -6 and reached.tolist() == [0, ctas]
    kv = ref.make_cache(2, 2, 128, 64, [300, 200], 0, seed=1)
    q = ref.make_q(2, 3, 8, 128, 2)
    c = binding.KV8({n: t.to("cuda:0") for n, t in kv.items()})
    got = c.sx_attention(q.to("cuda:0"), kernel=binding.ATTN_TC).double().cpu().numpy()
    c.check_status()
    want, bound = ref.attention(kv, q, 0, None, 128 ** -0.5)
    assert (abs(got - want) <= bound).all()


def test_strides_of_single_heads_do_not_matter():
    """With one KV head (or one query head) the distance between heads is never used, whatever the view says."""
    kv = ref.make_cache(3, 1, 64, 16, [20, 7, 33], 1, seed=3)
    g = torch.Generator().manual_seed(4)
    rows = torch.randn(1, 3, 64, generator=g).to(torch.bfloat16).to("cuda:0").transpose(0, 1)      # strides 64, 192, 1
    q = torch.randn(1, 3, 2, 64, generator=g).to(torch.bfloat16).to("cuda:0").permute(1, 2, 0, 3)  # strides 128, 64, 384, 1
    assert rows.stride(1) != 64 and q.stride(2) != 64
    start = torch.arange(4, dtype=torch.int32, device="cuda:0")
    got = []
    for k, x in ((rows, q), (rows.clone(memory_format=torch.contiguous_format), q.clone(memory_format=torch.contiguous_format))):
        c = binding.KV8({n: t.to("cuda:0") for n, t in kv.items()})
        c.sx_kv_append(k, k, start)
        back = torch.empty_strided(k.shape, k.stride(), dtype=torch.bfloat16, device="cuda:0")
        c.sx_kv_read(back, back.clone(), start, c.kv["cache_len"].clone())
        got.append((c.sx_attention(x, 1), back, *c.kv.values()))
        c.check_status()
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_a_draft_step_behind_a_negative_length_writes_nothing():
    """Such a sequence's new row has no place: reported, its pages and everyone else's as they were."""
    wl = synth.Workload(shape=SHAPE, B=2, **CHAIN)
    case = harness.build_case(wl, poison_tail=False)
    sx = binding.SpecExit(SHAPE, case.weights, 2, wl.mode, wl.K, kv_dtype=binding.KV_E4M3)
    sx.set_kv(as_codes(case.kv))
    sx.kv["cache_len"][1] = -5
    before = {n: t.clone() for n, t in sx.kv.items()}
    hid, *_ = sx.sx_draft_step(1, case.f0.to(sx.dev), case.t0.to(sx.dev))
    with pytest.raises(binding.SxError):
        sx.check_status()
    n, page = int(before["cache_len"][0]), SHAPE.page
    pp, off = int(before["page_table"][0, n // page]), n % page
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        before[name][pp, :, off] = sx.kv[name][pp, :, off]          # the first sequence's new row
        assert torch.equal(before[name], sx.kv[name]), name
    ok = binding.SpecExit(SHAPE, case.weights, 2, wl.mode, wl.K, kv_dtype=binding.KV_E4M3)
    ok.set_kv(as_codes(case.kv))
    want, *_ = ok.sx_draft_step(1, case.f0.to(sx.dev), case.t0.to(sx.dev))
    ok.check_status()
    assert torch.equal(hid[0], want[0])
