"""The largest sizes that the calls take, asked of the C entries without a device."""
from __future__ import annotations

import ctypes as C

import pytest

from paper_2509_24248_b200 import binding as sx

UNSUPPORTED = -2


@pytest.mark.parametrize("T", [0x7ffffff1, 0x7fffffff])
def test_rows_of_a_rotation_beyond_the_grid_are_refused(T):
    """Refused by their number alone, before anything is computed from it."""
    plan, lib = sx.Rope(8, 1e4).plan_ref, sx.load_library()
    assert lib.sx_rope(plan, 0, 0, T, 256, 1, 256, 8, 256, 8, 0, None, 0, None, 0, None) == UNSUPPORTED
    kv = sx.KV(2, 256, 256, 4, 8, 256, 256)
    assert lib.sx_kv_append_rope(None, C.byref(sx.KVShape(1, 1, 16, 16)), C.byref(kv), T, 256, None, None, 256, 16, 256, 16,
                                 None, 0, None, 0, 256, None) == UNSUPPORTED
