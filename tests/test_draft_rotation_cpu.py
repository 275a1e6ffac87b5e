"""Prompts for a draft layer: its cache takes no rotation but the one that its own rounds turn by (nothing is launched)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests.test_calls_at_once_cpu import cache, on_host  # noqa: F401

THETA = 1e6
OTHERS = {
    "another theta": dict(theta=1e4),
    "part of the head": dict(rot_dim=32),
    "interleaved": dict(layout=sx.ROPE_INTERLEAVED),
    "a magnitude": dict(magnitude=1.1),
    "linear": dict(scaling=sx.ROPE_LINEAR, factor=2.0),
    "base": dict(scaling=sx.ROPE_BASE, factor=2.0),
    "bands": dict(scaling=sx.ROPE_BANDS, factor=8.0, original_len=8192),
    "ramp": dict(scaling=sx.ROPE_RAMP, factor=8.0, original_len=8192),
    "list": dict(scaling=sx.ROPE_LIST, divisors=[1.0] * 31 + [1.01]),
}
SAME = {
    "plain": {},
    "theta as the context holds it": dict(theta=float(np.float32(1e6))),
    "linear by 1": dict(scaling=sx.ROPE_LINEAR, factor=1.0),
    "base that makes it": dict(theta=1e6 / 4.0 ** (64 / 62), scaling=sx.ROPE_BASE, factor=4.0),
    "list of ones": dict(scaling=sx.ROPE_LIST, divisors=[1.0] * 32),
}


@pytest.mark.parametrize("how", [*OTHERS, *SAME, "none"])
@pytest.mark.parametrize("kind", [sx.KVPages, sx.KV8])
def test_rotations_of_a_draft_layers_cache(on_host, monkeypatch, kind, how):
    kw = {**OTHERS, **SAME}.get(how, {})
    rope = None if how == "none" else sx.Rope(64, kw.get("theta", THETA), **{n: v for n, v in kw.items() if n != "theta"})
    qkv, start, calls = torch.zeros(3, 10, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), []
    args = (rope, qkv[:, 6:8], qkv[:, 8:], start)
    for theta in (None, THETA):
        c = cache(monkeypatch, kind, theta=theta)
        monkeypatch.setattr(c, "_append_rope", lambda *a: calls.append(a) or 0)
        if theta and how in OTHERS:
            for _ in range(2):
                with pytest.raises(sx.SxError, match="draft"):
                    c.sx_kv_append_rope(*args)
        else:
            c.sx_kv_append_rope(*args)
            c.sx_kv_append_rope(*args)
    assert len(calls) == (2 if how in OTHERS else 4)


def test_a_theta_between_two_fp32_numbers():
    """A context holds theta in fp32: the rotation by it and by the number that was asked for are the same here."""
    theta = 1234567.0625
    assert float(np.float32(theta)) != theta
    rope = sx.Rope(64, theta)
    assert rope.turns_as(theta) and rope.turns_as(float(np.float32(theta))) and not rope.turns_as(theta * 1.0001)
