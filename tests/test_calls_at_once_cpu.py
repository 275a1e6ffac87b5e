"""Objects of the binding used from several threads: what the C entries are handed, with recorders in their place and tensors of
the host (nothing is launched)."""
from __future__ import annotations

import threading
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


def head_of(rows, H):
    head = torch.zeros(rows, H, dtype=torch.bfloat16)
    return types.SimpleNamespace(device=types.SimpleNamespace(type="cuda", index=-1), dtype=head.dtype, dim=head.dim, shape=head.shape,
                                 is_contiguous=head.is_contiguous, data_ptr=head.data_ptr, numel=head.numel, keep=head)


class Library:
    """The C library with recorders for the calls that own a workspace: an entry waits until another thread is in too, or a while."""

    def __init__(self, lib):
        self.lib, self.inside, self.most, self.calls, self.guard = lib, 0, 0, [], threading.Lock()
        self.second = threading.Event()

    def __getattr__(self, name):
        return getattr(self.lib, name)

    def enter(self, call):
        with self.guard:
            self.inside += 1
            self.most = max(self.most, self.inside)
            self.calls.append(call)
            if self.inside > 1:
                self.second.set()
        self.second.wait(0.3)
        with self.guard:
            self.inside -= 1
        return 0

    def sx_head_logprobs_ws_bytes(self, T, V):
        return 1000 * T

    def sx_head_logprobs(self, *args):
        return self.enter((args[4], pointers(args[10]), args[11], args[12]))


def run_all(calls):
    threads = [threading.Thread(target=c) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join(30)
    assert not any(t.is_alive() for t in threads)


def test_calls_through_a_head_come_one_after_the_other(on_host, monkeypatch):
    """Both kernels of a call are on the stream before those of another thread's, since they share the object's workspace; the
    workspace that a call is given has the size it is said to have."""
    lib = Library(sx.load_library())
    monkeypatch.setattr(sx, "load_library", lambda: lib)
    s = sx.LogProbs(head_of(50, 16))
    rows = {T: torch.zeros(T, 16, dtype=torch.bfloat16) for T in (3, 40, 7)}
    tok = {T: torch.zeros(T, 2, dtype=torch.int32) for T in rows}
    out = {}
    run_all([lambda T=T: out.__setitem__(T, s.sx_head_logprobs(rows[T], tok[T], top=4)) for T in rows])
    assert lib.most == 1 and sorted(c[0] for c in lib.calls) == sorted(rows)
    for T, where, at, size in lib.calls:
        assert where == [out[T][n].data_ptr() for n in ("logp", "entropy", "top_tok", "top_logp")]
        assert size >= 1000 * T and any(w.data_ptr() <= at and at + size <= w.data_ptr() + w.numel() for w in s._ws)


def cache(monkeypatch, kind, lib=None, theta=None):
    """A cache of 2 sequences with 2 heads of 64, its device block made without a device; theta: a draft layer's."""
    if lib is not None:
        monkeypatch.setattr(sx, "load_library", lambda: lib)
    monkeypatch.setattr(sx, "_kv_struct", lambda kv, *_: sx.KV(2, 256, 256, 4, 8, 256, 256))
    kv = dict(k_pages=torch.zeros(8, 2, 16, 64, dtype=torch.uint8), cache_len=torch.zeros(2, dtype=torch.int32))
    c = kind(kv if theta is None else sx.DraftCache(kv, theta))
    c._index = -1
    return c


def test_an_append_keeps_its_number_of_query_heads(on_host, monkeypatch):
    """An append without queries that comes in while one with queries is on its way into the library."""
    c = cache(monkeypatch, sx.KVPages)
    qkv, start = torch.zeros(3, 10, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    seen = []

    def entry(*args):
        if not seen:
            seen.append(None)
            c.sx_kv_append_rope(None, qkv[:, 6:8], qkv[:, 8:], start)
        seen.append((args[1]._obj.n_q_heads, args[11]))
        return 0

    monkeypatch.setattr(c, "_append_rope", entry)
    c.sx_kv_append_rope(None, qkv[:, 6:8], qkv[:, 8:], start, q=qkv[:, :6])
    assert seen[1:] == [(0, None), (6, qkv.data_ptr())]


class Attention(Library):
    def sx_attention_ws_bytes(self, shape, batch, rows, groups):
        return 1000 * rows * shape._obj.n_q_heads

    def sx_attention(self, *args):
        return self.enter((args[2], args[4], args[0]._obj.n_q_heads, args[10], args[11]))


def test_attention_calls_come_one_after_the_other(on_host, monkeypatch):
    """The launches of an attention over the object's workspace, and its number of query heads, beside other threads' calls."""
    lib = Attention(sx.load_library())
    c = cache(monkeypatch, sx.KV8, lib)
    monkeypatch.setattr(sx, "_raw_stream", lambda dev: 0)
    q = {n: torch.zeros(2, rows, n, 64, dtype=torch.bfloat16) for rows, n in ((1, 2), (8, 16), (3, 4))}
    run_all([lambda n=n: c.sx_attention(q[n], kernel=sx.ATTN_AUTO) for n in q])
    assert lib.most == 1 and len(lib.calls) == 3
    for rows, at, n, ws, size in lib.calls:
        assert at == q[n].data_ptr() and rows == q[n].shape[1] and size >= 1000 * rows * n
        assert any(w.data_ptr() <= ws and ws + size <= w.data_ptr() + w.numel() for w in c._ws)


def test_device_0_is_device_0(monkeypatch):
    """A device given by its number, 0 among them, is not the current one."""
    asked = []
    monkeypatch.setattr(sx, "torch", HostTorch())
    monkeypatch.setattr(HostTorch, "device", staticmethod(lambda *a: asked.append(a) or types.SimpleNamespace(type="cuda", index=-1)))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    sx.LogProbs(device=0)
    assert asked == [(0,)]
