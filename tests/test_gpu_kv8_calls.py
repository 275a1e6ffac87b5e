"""Draft calls on an 8-bit cache: what they refuse, and what they do not look at."""
from __future__ import annotations

import pytest
import torch

from paper_2509_24248_b200 import binding, synth
from tests import harness
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
