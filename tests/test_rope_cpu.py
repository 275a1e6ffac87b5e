"""The plan of a rotation against extended precision, and what the calls refuse before they look for a device."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import rope_ref as ref

HOW = {"none": sx.ROPE_NONE, "linear": sx.ROPE_LINEAR, "base": sx.ROPE_BASE, "bands": sx.ROPE_BANDS, "ramp": sx.ROPE_RAMP,
       "list": sx.ROPE_LIST}


@pytest.mark.parametrize("scaling", list(HOW))
@pytest.mark.parametrize("d,rot,theta", [(128, 128, 1e6), (64, 32, 1e4), (96, 70, 5e5), (256, 256, 1e4), (8, 4, 1e4)])
def test_steps_of_the_plan(scaling, d, rot, theta):
    """Within 2^-62 turns, a few roundings of the extended type, of the formula's frequency modulo one turn."""
    kw = dict(factor=1.0 if scaling == "none" else 3.7, low=1.0, high=20.0, original_len=4096)
    div = [1.0 + 0.3 * i for i in range(rot // 2)] if scaling == "list" else None
    plan = sx.Rope(d, theta, rot_dim=rot, scaling=HOW[scaling], divisors=div, **kw).plan
    f = ref.frequencies(rot, theta, scaling, divisors=div, **kw) / ref.TURN
    got = np.array([np.longdouble(int(v)) for v in plan.step[:rot // 2]]) / np.longdouble(2) ** 64
    off = np.abs(got - (f - np.floor(f)))
    assert (np.minimum(off, 1 - off) <= np.longdouble(2) ** -62).all()
    assert all(v == 0 for v in plan.step[rot // 2:])


@pytest.mark.parametrize("bad", [
    dict(head_dim=0), dict(head_dim=12), dict(head_dim=264), dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=66), dict(rot_dim=-2),
    dict(rot_start=1), dict(rot_start=-2), dict(rot_start=2), dict(layout=2), dict(layout=-1), dict(theta=0.0), dict(theta=-1.0),
    dict(theta=float("nan")), dict(theta=float("inf")), dict(magnitude=0.0), dict(magnitude=float("nan")), dict(magnitude=1e39),
    dict(scaling=6), dict(scaling=-1), dict(scaling=sx.ROPE_LINEAR, factor=0.0), dict(scaling=sx.ROPE_LINEAR, factor=float("inf")),
    dict(scaling=sx.ROPE_BASE, rot_dim=2, factor=2.0), dict(scaling=sx.ROPE_BANDS, factor=2.0),
    dict(scaling=sx.ROPE_BANDS, factor=2.0, original_len=4096, low=4.0, high=4.0),
    dict(scaling=sx.ROPE_RAMP, factor=2.0, original_len=4096, low=0.0), dict(scaling=sx.ROPE_RAMP, factor=2.0, original_len=0),
    dict(scaling=sx.ROPE_RAMP, factor=2.0, original_len=4096, theta=1.0),
    dict(scaling=sx.ROPE_LIST), dict(scaling=sx.ROPE_LIST, divisors=[1.0] * 31), dict(scaling=sx.ROPE_LIST, divisors=[0.0] * 32),
    dict(divisors=[1.0] * 32)])
def test_plans_that_cannot_be_are_refused(bad):
    with pytest.raises(sx.SxError):
        sx.Rope(**{**dict(head_dim=64, theta=1e4), **bad})


def test_calls_that_cannot_be_are_refused():
    lib, plan = sx.load_library(), sx.Rope(64, 1e4).plan_ref
    ok = [plan, 0, 0, 3, 256, 2, 256, 128, 512, 128, 1, 1024, 64, 2048, 64, None]
    INVALID, UNSUPPORTED = -1, -2

    def rope(**change):
        a = list(ok)
        for i, v in change.items():
            a[int(i[1:])] = v
        return lib.sx_rope(*a)

    blank = sx.Rotation()
    for change in (dict(_0=None), dict(_0=C.byref(blank)), dict(_1=3), dict(_1=-1), dict(_2=2), dict(_3=-1), dict(_4=None), dict(_5=-1),
                   dict(_6=None), dict(_6=8), dict(_7=127), dict(_7=120), dict(_7=132), dict(_8=None), dict(_8=24), dict(_9=100),
                   dict(_8=256, _9=136), dict(_10=-1), dict(_11=None), dict(_13=4), dict(_14=60)):
        assert rope(**change) == INVALID, change
    assert rope(_5=4097, _7=1 << 20, _9=1 << 20) == UNSUPPORTED
    assert rope(_3=0) == 0 and rope(_5=0, _10=0) == 0            # nothing to do: no device needed

    shape, kv = sx.KVShape(2, 1, 64, 5), sx.KV(2, 256, 256, 4, 8, 256, 256)
    ok[:] = [plan, C.byref(shape), C.byref(kv), 3, 256, None, None, 256, 64, 256, 64, 256, 128, 512, 128, 256, None]

    def append(**change):
        a = list(ok)
        for i, v in change.items():
            a[int(i[1:])] = v
        return lib.sx_kv_append_rope(*a)

    other = sx.Rope(128, 1e4)
    for change in (dict(_0=other.plan_ref), dict(_1=None), dict(_2=None), dict(_3=-1), dict(_4=None), dict(_7=None), dict(_7=8),
                   dict(_8=63), dict(_8=68), dict(_9=None), dict(_10=8), dict(_11=None), dict(_11=8), dict(_12=120), dict(_13=None),
                   dict(_14=127), dict(_13=256, _14=136), dict(_15=None)):
        assert append(**change) == INVALID, change
    assert append(_3=0) == 0 and append(_0=None, _3=0) == 0
    for field, value, code in (("batch", 0, INVALID), ("max_pages", 0, INVALID), ("num_pages", 0, INVALID), ("k_pages_d", None, INVALID),
                               ("v_pages_d", 8, INVALID), ("cache_len_d", None, INVALID), ("page_table_d", None, INVALID),
                               ("dtype", 2, UNSUPPORTED), ("dtype", 1, INVALID), ("max_pages", 1 << 30, UNSUPPORTED)):
        bad = sx.KV(2, 256, 256, 4, 8, 256, 256)
        setattr(bad, field, value)
        assert append(_2=C.byref(bad)) == code, field
    eight = sx.KV(2, 256, 256, 4, 8, 256, 256, 1, 0, 256, 256)
    assert append(_2=C.byref(eight)) == UNSUPPORTED              # codes need pages of a multiple of 16 slots
    for d in (8, 24, 256):
        assert append(_1=C.byref(sx.KVShape(2, 1, d, 5)), _0=None) == UNSUPPORTED
    assert append(_1=C.byref(sx.KVShape(2, 0, 64, 5))) == INVALID and append(_1=C.byref(sx.KVShape(0, 1, 64, 5))) == INVALID


def test_python_side_refusals():
    rope = sx.Rope(64, 1e4)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(sx.SxError, match="on a device"):
        rope.sx_rope(torch.zeros(3, dtype=torch.int32), x)
    with pytest.raises(sx.SxError, match="contiguous on"):
        sx.KVPages(dict(k_pages=torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16), v_pages=torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16),
                        page_table=torch.zeros(1, 4, dtype=torch.int32), cache_len=torch.zeros(1, dtype=torch.int32)))
    with pytest.raises(sx.SxError, match="num_pages"):
        sx.KVPages(dict(k_pages=torch.zeros(4, 16, 64, dtype=torch.bfloat16)))
