"""The operators together, as a program uses them: prompts turned into a cache, attention over it, log-probabilities of what
comes out; a draft layer whose context was written that way; the scores of verified slots beside sx_verify's tokens."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2509_24248_b200 import binding as sx, synth
from tests import harness, kv8_ref, rope_ref, score_ref
from tests.test_gpu_kv8_draft import as_codes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Scorer:
    """One attention layer in front of a head: prompt rows into the cache, then given tokens one at a time, each row's
    queries, keys and values a projection of an embedding."""

    def __init__(self, lens, steps, nq=4, nkv=2, d=64, page=16, V=701, seed=3):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.steps, self.nq, self.nkv, self.d, self.V = lens, steps, nq, nkv, d, V
        self.B, H = len(lens), nq * d
        self.emb = torch.randn(V, (nq + 2 * nkv) * d, generator=g).to(torch.bfloat16).to(DEV)
        self.head = (torch.randn(V + 3, H, generator=g) * 0.3).to(torch.bfloat16).to(DEV)
        self.tokens = torch.randint(0, V, (self.B, max(lens) + steps + 1), generator=g).to(DEV)
        M = -(-(max(lens) + steps) // page)
        num = self.B * M + 2
        self.kv = dict(page_table=torch.randperm(num, generator=g)[:self.B * M].to(torch.int32).view(self.B, M).to(DEV),
                       cache_len=torch.zeros(self.B, dtype=torch.int32, device=DEV))
        for n in "kv":
            self.kv[n + "_pages"] = torch.zeros(num, nkv, page, d, dtype=torch.uint8, device=DEV)
            self.kv[n + "_scale"] = torch.full((num, nkv, page), 127, dtype=torch.uint8, device=DEV)
        self.cache, self.scores = sx.KV8(self.kv), sx.LogProbs(self.head, vocab=V)
        self.rope = sx.Rope(d, 1e4, rot_dim=d // 2, layout=sx.ROPE_INTERLEAVED, scaling=sx.ROPE_LINEAR, factor=2.0)
        self.start = i32([0, *np.cumsum(lens)])
        self.one = i32(list(range(self.B + 1)))
        self.rows = torch.cat([self.emb[self.tokens[b, :n]] for b, n in enumerate(lens)]).unflatten(1, (-1, d))
        self.at = torch.tensor(lens, device=DEV)
        self.next = torch.zeros(self.B, 1, dtype=torch.int32, device=DEV)
        self.x = torch.zeros(self.B, (nq + 2 * nkv) * d, dtype=torch.bfloat16, device=DEV)
        self.q = torch.zeros(self.B, nq, d, dtype=torch.bfloat16, device=DEV)
        self.o = torch.zeros(self.B, 1, nq, d, dtype=torch.bfloat16, device=DEV)
        self.out = None

    def split(self, x):
        return x[:, :self.nq], x[:, self.nq:self.nq + self.nkv], x[:, self.nq + self.nkv:]

    def prompt(self):
        _, k, v = self.split(self.rows)
        self.cache.sx_kv_append_rope(self.rope, k, v, self.start, i32([0] * self.B))
        self.kv["cache_len"].copy_(self.at.to(torch.int32))

    def step(self):
        """Row t of every sequence: into the cache, over the cache, and the log-probability of token t + 1."""
        i = self.kv["cache_len"].long().unsqueeze(1)
        self.x.copy_(self.emb[self.tokens.gather(1, i).squeeze(1)])
        self.next.copy_(self.tokens.gather(1, i + 1).to(torch.int32))
        q, k, v = self.split(self.x.unflatten(1, (-1, self.d)))
        self.cache.sx_kv_append_rope(self.rope, k, v, self.one, q=q, q_out=self.q)
        self.cache.sx_attention(self.q.unsqueeze(1), drafted=1, out=self.o)
        self.out = self.scores.sx_head_logprobs(self.o.view(self.B, -1), self.next, top=5, out=self.out)
        self.kv["cache_len"].add_(1)


def check_step(s: Scorer, lens):
    """Every stage against its formula on what the stage before it left: keys within half a step of their codes (2^-4 of the value,
    2^-10 of the row's largest) and of bf16, attention and log-probabilities within their own bounds."""
    kv = {n: t.cpu() for n, t in s.kv.items()}
    f = rope_ref.frequencies(s.d // 2, 1e4, "linear", factor=2.0)
    for b, n in enumerate(lens):
        rows = s.emb[s.tokens[b, :n]].unflatten(1, (-1, s.d))
        q, k, v = s.split(rows)
        y, far = rope_ref.turned(k, np.arange(n), f, "interleaved", 0)
        pp, off = kv["page_table"][b].long()[torch.arange(n) // 16], torch.arange(n) % 16
        for name, want, more in (("k", y, far), ("v", v.double().cpu().numpy(), 0.0)):
            got = kv8_ref.dequantise(kv[name + "_pages"][pp, :, off], kv[name + "_scale"][pp, :, off])
            want_off = 2.0 ** -8 * np.abs(want) + more
            bound = want_off + (2.0 ** -4 * (np.abs(want) + want_off) + 2.0 ** -10 * 1.01 * np.abs(want).max(-1, keepdims=True))
            assert (np.abs(got - want) <= bound).all()
        yq, farq = rope_ref.turned(q[-1:], [n - 1], f, "interleaved", 0)
        rope_ref.close(s.q[b:b + 1], yq, farq)
    seen = {**kv, "cache_len": torch.tensor(lens, dtype=torch.int32)}
    want, bound = kv8_ref.attention(seen, s.q.cpu().unsqueeze(1), 0, None, s.d ** -0.5)
    assert (np.abs(s.o.double().cpu().numpy() - want) <= bound).all()
    h, w = s.o.view(s.B, -1), s.head[:s.V]
    x = h.double().cpu() @ w.double().cpu().T
    more = h.shape[1] * 2.0 ** -23 * float((h.double().abs() @ w.double().abs().T).max())
    ref = score_ref.scores(x, s.next, 5)
    score_ref.check({n: s.out[n] for n in ("logp", "entropy", "top_logp")}, {n: ref[n] for n in ("logp", "entropy", "top_logp")}, x, more=more)


def test_a_prompt_and_given_tokens_after_it():
    lens = [37, 1, 16, 90]
    s = Scorer(lens, 3)
    s.prompt()
    for i in range(3):
        s.step()
        check_step(s, [n + i + 1 for n in lens])
    s.cache.check_status()
    s.scores.check_status()


def test_the_same_from_a_captured_step():
    """A step captured once and replayed gives what direct calls give, bit for bit."""
    lens, got = [20, 5, 64], []
    for captured in (False, True):
        s = Scorer(lens, 5)
        s.prompt()
        s.step()                                                 # warms up, and makes s.out
        if captured:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                s.step()
        seen = []
        for _ in range(3):
            graph.replay() if captured else s.step()
            seen += [t.clone() for t in s.out.values()]
        got.append(seen + list(s.kv.values()))
        s.cache.check_status()
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("kv_dtype", [sx.KV_BF16, sx.KV_E4M3])
def test_a_draft_step_on_a_prompt_written_by_append(kv_dtype):
    """A draft layer's context written through KVPages(spec.kv) serves a draft step as one placed by hand does."""
    sh = synth.ModelShape(H=256, n_q=4, n_kv=2, d=64, F=688, V=1000, page=32)
    wl = synth.Workload("prompt", sh, B=3, mode=synth.CHAIN, K=3, len_lo=5, len_hi=70, seed=21)
    case = harness.build_case(wl, poison_tail=False)
    lens = case.kv["cache_len"].tolist()
    g = torch.Generator().manual_seed(22)
    k, v = (torch.randn(sum(lens), 2, 64, generator=g).to(torch.bfloat16).to(DEV) for _ in "kv")
    start, zero = i32([0, *np.cumsum(lens)]), i32([0] * 3)
    rope = sx.Rope(64, sh.theta)
    got = []
    for fused in (True, False):
        spec = sx.SpecExit(sh, case.weights, 3, wl.mode, wl.K, kv_dtype=kv_dtype)
        spec.set_kv(as_codes(case.kv) if kv_dtype == sx.KV_E4M3 else case.kv)
        if fused:
            sx.KVPages(spec.kv).sx_kv_append_rope(rope, k, v, start, zero)
        else:
            pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).to(DEV)
            turned = rope.sx_rope(pos, k)[0]
            if kv_dtype == sx.KV_E4M3:                # codes are those of the exact rotation
                turned = rope_ref.to_bf16(rope_ref.turned(k, pos.cpu(), rope_ref.frequencies(64, sh.theta), "half", 0)[0]).to(DEV)
                sx.KV8(spec.kv).sx_kv_append(turned, v, start, zero)
            else:
                for b, n in enumerate(lens):
                    for i in range(n):
                        pp = int(spec.kv["page_table"][b, i // 32])
                        spec.kv["k_pages"][pp, :, i % 32], spec.kv["v_pages"][pp, :, i % 32] = turned[int(start[b]) + i], v[int(start[b]) + i]
        got.append([t for t in spec.sx_draft_step(1, case.f0.to(DEV), case.t0.to(DEV)) if t is not None])
        spec.check_status()
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("tiled", [False, True])
def test_scores_of_verified_slots(tiled):
    """A context's own target head, in the layout it keeps it in, scores the slots that sx_verify verified: the best alternative
    is the token that sx_verify returns.  Small multiples of 1/16, so the logits are exact on both sides."""
    sh = synth.ModelShape(H=256, n_q=4, n_kv=2, d=64, F=688, V=1000, page=32)
    wl = synth.Workload("slots", sh, B=2, mode=synth.CHAIN, K=4, len_lo=5, len_hi=70, seed=23)
    weights = synth.make_weights(sh, wl.seed)
    g = torch.Generator().manual_seed(24)
    weights["head"] = (torch.randint(-3, 4, (sh.V + sh.S, sh.H), generator=g) / 16).to(torch.bfloat16)
    spec = sx.SpecExit(sh, weights, 2, wl.mode, wl.K, tiled=tiled)
    th = (torch.randint(-4, 5, (2, 5, sh.H), generator=g) / 16).to(torch.bfloat16).to(DEV)
    cand = torch.randint(0, sh.V, (2, 5), generator=g).to(torch.int32).to(DEV)
    target, _, _, _ = spec.sx_verify(th, cand)
    scores = sx.LogProbs(spec.w["target_head"], vocab=sh.V, hidden=sh.H)
    out = scores.sx_head_logprobs(th.view(10, sh.H), cand.view(10, 1), top=3)
    assert torch.equal(out["top_tok"][:, 0].view(2, 5), target)
    x = th.view(10, -1).double().cpu() @ weights["head"][:sh.V].double().T
    score_ref.check(out, score_ref.scores(x, cand.view(10, 1), 3), x)
    spec.check_status()
    scores.check_status()
