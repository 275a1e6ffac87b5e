"""The largest sizes that the calls take, asked of the C entries and of the binding without a device."""
from __future__ import annotations

import ctypes as C

import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests.test_calls_at_once_cpu import on_host  # noqa: F401

UNSUPPORTED = -2


@pytest.mark.parametrize("T", [0x7ffffff1, 0x7fffffff])
def test_rows_of_a_rotation_beyond_the_grid_are_refused(T):
    """Refused by their number alone, before anything is computed from it."""
    plan, lib = sx.Rope(8, 1e4).plan_ref, sx.load_library()
    assert lib.sx_rope(plan, 0, 0, T, 256, 1, 256, 8, 256, 8, 0, None, 0, None, 0, None) == UNSUPPORTED
    kv = sx.KV(2, 256, 256, 4, 8, 256, 256)
    assert lib.sx_kv_append_rope(None, C.byref(sx.KVShape(1, 1, 16, 16)), C.byref(kv), T, 256, None, None, 256, 16, 256, 16,
                                 None, 0, None, 0, 256, None) == UNSUPPORTED


MANY = 2 ** 32 + 3                                               # what 32 bits hold of it is 3


def test_sizes_that_do_not_fit_a_call_are_refused(on_host, monkeypatch):
    """Rows, heads, columns, tokens and alternatives beyond 32 bits: refused, not cut off to what their lower bits say."""
    none = lambda *_: pytest.fail("the call was made")
    s = sx.LogProbs(device="host")
    monkeypatch.setattr(s, "_logprobs", none)
    f = lambda *shape: torch.empty(shape, device="meta")         # no memory behind them, and an index of -1 as well
    i = lambda *shape: torch.empty(shape, dtype=torch.int32, device="meta")
    for x, kw in ((f(MANY, 1), {}), (f(1, MANY), {}), (f(1, 1), dict(tokens=i(1, MANY))), (f(1, 1), dict(tokens=i(1, 65))),
                  (f(1, 1), dict(top=MANY)), (f(1, 1), dict(top=33)), (f(1, 1), dict(top=-1))):
        with pytest.raises(sx.SxError):
            s.sx_logprobs(x, **kw)
    rope = sx.Rope(8, 1e4)
    monkeypatch.setattr(rope, "_call", none)
    for shape in ((MANY, 1, 8), (1, MANY, 8)):
        q = f(*shape)
        with pytest.raises(sx.SxError):
            rope.sx_rope(i(shape[0]), q, q_out=q)
