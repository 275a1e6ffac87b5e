"""Objects of the binding used from several threads: what the C entries are handed, with recorders in their place and tensors of
the host (nothing is launched)."""
from __future__ import annotations

import types

import pytest
import torch

from paper_2509_24248_b200 import binding as sx


class HostTorch:
    """torch with the host as its device: index -1, which is what get_device() says of a host tensor."""

    def __init__(self):
        self._C = types.SimpleNamespace(_cuda_getDevice=lambda: -1, _cuda_getCurrentRawStream=lambda index: 0)

    def __getattr__(self, name):
        return getattr(torch, name)

    @staticmethod
    def device(*_):
        return types.SimpleNamespace(type="cuda", index=-1)

    @staticmethod
    def zeros(*shape, device=None, **kw):
        return torch.zeros(*shape, **kw)

    @staticmethod
    def empty(*shape, device=None, **kw):
        return torch.empty(*shape, **kw)


@pytest.fixture
def on_host(monkeypatch):
    monkeypatch.setattr(sx, "torch", HostTorch())


def scores(monkeypatch, T):
    s = sx.LogProbs(device="host")
    return s, torch.zeros(T, 50), torch.zeros(T, 2, dtype=torch.int32)


def pointers(ref):
    o = ref._obj
    return [o.logp_d, o.entropy_d, o.top_tok_d, o.top_logp_d]


def test_a_call_keeps_its_own_results(on_host, monkeypatch):
    """A second call that comes in while the first is on its way into the library leaves the first one's results alone."""
    s, x, tok = scores(monkeypatch, 3)
    seen, other = [], []

    def entry(*args):
        if not other:
            other.append(None)                                   # the second call, from within the first
            other[0] = s.sx_logprobs(x[:1], tok[:1], top=4)
        seen.append(pointers(args[9]))
        return 0

    monkeypatch.setattr(s, "_logprobs", entry)
    mine = s.sx_logprobs(x, tok, top=4)
    for got, want in zip(seen, (other[0], mine)):
        assert got == [want[n].data_ptr() for n in ("logp", "entropy", "top_tok", "top_logp")]
