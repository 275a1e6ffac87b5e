"""The operators of the 8-bit paged cache without a GPU: what the entry points refuse (before any launch), the reference
that the GPU tests compare with, and the cases of perf/operators.py."""
from __future__ import annotations

import ctypes as C
import importlib.util
import math
import os
import random

import numpy as np
import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import kv8_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                   # an aligned address that no call gets far enough to read


def shape(**kw):
    return sx.KVShape(*[{"n_q_heads": 8, "n_kv_heads": 2, "head_dim": 128, "page_size": 64, **kw}[n]
                        for n in ("n_q_heads", "n_kv_heads", "head_dim", "page_size")])


def cache(**kw):
    f = dict(batch=2, cache_len_d=P, page_table_d=P, max_pages=4, num_pages=8, k_pages_d=P, v_pages_d=P, dtype=sx.KV_E4M3,
             n_groups=0, k_scale_d=P, v_scale_d=P, group_start_d=None, prefix_len_d=None)
    f.update(kw)
    return sx.KV(**f)


def append(sh=None, kv=None, T=4, rs=P, ps=P, k=P, ks=256, v=P, vs=256, status=P, fn="sx_kv_append"):
    return getattr(sx.load_library(), fn)(C.byref(sh or shape()), C.byref(kv or cache()), T, rs, ps, k, ks, v, vs, status, None)


@pytest.mark.parametrize("fn", ["sx_kv_append", "sx_kv_read"])
@pytest.mark.parametrize("kw,code", [
    (dict(kv=cache(dtype=sx.KV_BF16)), -2), (dict(sh=shape(page_size=24)), -2), (dict(sh=shape(head_dim=256)), -2),
    (dict(sh=shape(head_dim=40)), -2), (dict(sh=shape(n_kv_heads=0)), -1), (dict(kv=cache(batch=0)), -1),
    (dict(kv=cache(k_scale_d=None)), -1), (dict(kv=cache(v_scale_d=P + 8)), -1), (dict(kv=cache(k_pages_d=P + 4)), -1),
    (dict(kv=cache(cache_len_d=None)), -1), (dict(kv=cache(page_table_d=None)), -1), (dict(kv=cache(max_pages=1 << 26)), -2),
    (dict(T=-1), -1), (dict(rs=None), -1), (dict(k=None), -1), (dict(v=P + 2), -1), (dict(ks=255), -1), (dict(vs=260), -1),
    (dict(ks=128), -1), (dict(status=None), -1)])
def test_rows_calls_refuse(fn, kw, code):
    assert append(fn=fn, **kw) == code


def test_read_needs_positions_and_no_rows_is_no_work():
    assert append(fn="sx_kv_read", ps=None) == -1
    assert append(T=0) == 0 and append(T=0, fn="sx_kv_read") == 0


@pytest.mark.parametrize("kw,code", [
    (dict(kv=cache(dtype=sx.KV_BF16)), -2), (dict(sh=shape(head_dim=32)), -2), (dict(sh=shape(n_q_heads=7)), -2),
    (dict(sh=shape(page_size=8)), -2), (dict(rows=0), -1), (dict(rows=65), -1), (dict(drafted=-1), -1), (dict(drafted=65), -1),
    (dict(q=P + 8), -1), (dict(o=None), -1), (dict(stride=1000), -1), (dict(stride=1028), -1), (dict(status=None), -1),
    (dict(scale=math.nan), -1), (dict(scale=math.inf), -1), (dict(kernel=3), -1), (dict(kernel=-1), -1),
    (dict(kv=cache(n_groups=3, group_start_d=P, prefix_len_d=P)), -1), (dict(kv=cache(n_groups=1)), -1),
    (dict(kv=cache(n_groups=-1)), -1), (dict(kv=cache(batch=1025)), -2), (dict(kv=cache(batch=1024), rows=64), -2)])
def test_attention_refuses(kw, code):
    a = dict(sh=shape(), kv=cache(), rows=1, drafted=1, q=P, stride=1024, mask=None, scale=0.1, kernel=0, o=P, ws=P,
             nb=1 << 30, status=P)
    a.update(kw)
    got = sx.load_library().sx_attention(C.byref(a["sh"]), C.byref(a["kv"]), a["rows"], a["drafted"], a["q"], a["stride"],
                                         a["mask"], a["scale"], a["kernel"], a["o"], a["ws"], a["nb"], a["status"], None)
    assert got == code


def test_workspace_of_impossible_shapes_is_zero():
    lib = sx.load_library()
    for sh, args in ((shape(), (0, 1, 0)), (shape(), (1, 0, 0)), (shape(), (1, 1, -1)), (shape(n_q_heads=0), (1, 1, 0))):
        assert lib.sx_attention_ws_bytes(C.byref(sh), *args) == 0


def test_python_side_refuses_what_the_library_cannot_see():
    kv = ref.make_cache(2, 2, 64, 16, [5, 7], 0)
    with pytest.raises(sx.SxError):
        sx.KV8(kv)                                            # not on a device
    with pytest.raises(sx.SxError):
        sx.KV8({**kv, "k_pages": kv["k_pages"].to(torch.bfloat16)})


# ---- the reference of the GPU tests -----------------------------------------------------------------------------------
def test_codes_have_the_values_of_torch():
    mine = torch.from_numpy(ref.VALUES)
    theirs = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.nan_to_num(mine, nan=999.0), torch.nan_to_num(theirs, nan=999.0))


def test_quantise_by_hand():
    x = torch.tensor([[448.0, 1.0, -0.4375, 0.0], [449.0, 17.0, 18.0, 19.0], [0.0, 0.0, 0.0, -0.0], [2.0 ** -100, 0, 0, 0]],
                     dtype=torch.float64)
    codes, byte = ref.quantise(x)
    assert byte.tolist() == [127, 128, 127, 63]
    back = ref.dequantise(codes, byte)
    assert back[0].tolist() == [448.0, 1.0, -0.4375, 0.0]
    # scale 2: 224.5 -> 224, 8.5 -> 8 (tie to even), 9 exact, 9.5 -> 10 (tie to even)
    assert back[1].tolist() == [448.0, 16.0, 18.0, 20.0]
    assert back[2].tolist() == [0.0] * 4 and back[3].tolist() == [0.0] * 4
    assert ref.quantise(torch.tensor([[1.0, math.inf]]))[1].tolist() == [255]
    assert np.isnan(ref.dequantise(*ref.quantise(torch.tensor([[1.0, math.nan]])))).all()


def test_rounding_is_half_a_step_and_reading_back_is_exact_in_bf16():
    g = torch.Generator().manual_seed(0)
    x = (torch.randn(200, 64, generator=g) * torch.exp2(torch.randint(-30, 30, (200, 1), generator=g).float())).to(torch.bfloat16)
    codes, byte = ref.quantise(x)
    back = ref.dequantise(codes, byte)
    top = np.abs(x.double().numpy()).max(1, keepdims=True)
    # half a step of e4m3, 2^-4 relative, and 2^-10 of the scale below its normal range; the scale is at most top / 224
    assert (np.abs(back - x.double().numpy()) <= np.maximum(2.0 ** -4 * np.abs(x.double().numpy()), 2.0 ** -10 * top / 224)).all()
    assert torch.equal(torch.from_numpy(back).to(torch.bfloat16).double(), torch.from_numpy(back))
    again = ref.quantise(torch.from_numpy(back))
    assert np.array_equal(ref.dequantise(*again), back)


def test_attention_reference_against_torch():
    kv = ref.make_cache(2, 2, 64, 16, [19, 3], 2, seed=1)
    q = ref.make_q(2, 2, 4, 64, 2)
    mask = ref.causal_masks(2, 2, 2)
    want, _ = ref.attention(kv, q, 2, mask, 0.125)
    for b, n in enumerate([19, 3]):
        pos = torch.arange(n + 2)
        pp = kv["page_table"][b][pos // 16].long()
        k = torch.from_numpy(ref.dequantise(kv["k_pages"][pp, :, pos % 16], kv["k_scale"][pp, :, pos % 16])).repeat_interleave(2, 1)
        v = torch.from_numpy(ref.dequantise(kv["v_pages"][pp, :, pos % 16], kv["v_scale"][pp, :, pos % 16])).repeat_interleave(2, 1)
        vis = pos < n + 1 + torch.arange(2).unsqueeze(1)
        o = torch.nn.functional.scaled_dot_product_attention(q[b].double().transpose(0, 1), k.transpose(0, 1), v.transpose(0, 1),
                                                             attn_mask=vis, scale=0.125)
        assert np.allclose(o.transpose(0, 1).numpy(), want[b], rtol=1e-12, atol=1e-12)


# ---- perf/operators.py ----------------------------------------------------------------------------------------------
def test_cases_are_well_formed():
    spec = importlib.util.spec_from_file_location("operators", os.path.join(ROOT, "perf", "operators.py"))
    ops = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ops)
    listed = ops.listed()
    assert len({c["name"] for c in listed}) == len(listed)
    most = max(ops.work(c)["bytes"] for c in listed)
    for seed in range(200):
        c = ops.draw(random.Random(seed))
        w = ops.work(c)
        assert 0 <= w["flops"] and 0 < w["bytes"] <= most
