"""What the calls for log-probabilities refuse before they look for a device."""
from __future__ import annotations

import ctypes as C

import pytest
import torch

from paper_2509_24248_b200 import binding as sx

INVALID, UNSUPPORTED = -1, -2


def test_calls_that_cannot_be_are_refused():
    lib = sx.load_library()
    out = sx.LogProbOut(256, 256, 256, 256)
    ok = [0, 3, 100, 256, 100, 2, 256, 1.0, 4, C.byref(out), 256, None]

    def call(**change):
        a = list(ok)
        for i, v in change.items():
            a[int(i[1:])] = v
        return lib.sx_logprobs(*a)

    inf, nan = float("inf"), float("nan")
    for change in (dict(_0=3), dict(_0=-1), dict(_1=-1), dict(_2=0), dict(_3=None), dict(_3=257), dict(_0=2, _3=258), dict(_4=99), dict(_5=-1), dict(_6=None),
                   dict(_6=258), dict(_7=0.0), dict(_7=-1.0), dict(_7=inf), dict(_7=nan), dict(_7=1e-38), dict(_8=-1), dict(_9=None), dict(_10=None)):
        assert call(**change) == INVALID, change
    for change in (dict(_5=65), dict(_8=33), dict(_2=(1 << 24) + 1, _4=1 << 25)):
        assert call(**change) == UNSUPPORTED, change
    for fields, bad in (((None, 256, 256, 256), INVALID), ((256, 256, None, None), INVALID), ((256, 2, 256, 256), INVALID)):
        o = sx.LogProbOut(*fields)
        assert call(_9=C.byref(o)) == bad
    assert call(_1=0) == 0

    ok[:] = [256, 0, 100, 64, 3, 256, 2, 256, 1.0, 4, C.byref(out), 256, 1 << 30, 256, None]

    def head(**change):
        a = list(ok)
        for i, v in change.items():
            a[int(i[1:])] = v
        return lib.sx_head_logprobs(*a)

    for change in (dict(_0=None), dict(_0=8), dict(_1=2), dict(_2=0), dict(_4=-1), dict(_5=None), dict(_5=24), dict(_6=-1), dict(_7=None),
                   dict(_8=0.0), dict(_9=-1), dict(_10=None), dict(_13=None)):
        assert head(**change) == INVALID, change
    for change in (dict(_3=0), dict(_3=63), dict(_6=65), dict(_9=33)):
        assert head(**change) == UNSUPPORTED, change
    assert head(_4=0) == 0
    assert lib.sx_head_logprobs_ws_bytes(0, 100) == 0 and lib.sx_head_logprobs_ws_bytes(1, 0) == 0


def test_a_head_on_the_host_is_refused():
    with pytest.raises(sx.SxError, match="CUDA device"):
        sx.LogProbs(torch.zeros(8, 8, dtype=torch.bfloat16))
