"""Positions, the rows of a cache and the log-probabilities of an answer as cases to time and compare.

Four operators, as a program calls them that scores or continues text over a paged cache:

``rope``    rotary positions of queries and keys: both orders of the pairs, a part of the head, frequencies scaled for
            long contexts, and the transposed rotation
``append``  new tokens on their way into a paged cache: keys (and queries) turned to their positions, keys and values
            written to their pages, as bf16 or as e4m3 codes with a power-of-two scale per row
``logits``  from rows of logits: log-probabilities of given tokens, the entropy, the best alternatives
``head``    the same from hidden states and the head's weights, without a matrix of logits in the caller's hands

Rotation: pair i of a head's rotated part (r elements from rot_start on) is (x_i, x_(i + r/2)) in the half order and
(x_2i, x_(2i + 1)) in the interleaved one; it turns by position * f_i, times a magnitude.  f_i = theta^(-2i / r) without
scaling; the scalings are at ``_frequencies``.  A row of an 8-bit cache is the rotated row rounded to bf16, then quantised:
scale 2^e with e = ceil(log2(max|x| / 448)) held to [-64, 120] (0 for a row of zeros), stored as the byte e + 127.

Log-probabilities are those of softmax(logits / temperature).  Alternatives: the largest logits, best first, the lower id
first among equals; an alternative without probability has the id -1.
"""
import itertools
import math
import random

import torch

own = False          # set from outside: False runs the plain forms, True the package's entry points

_8B = dict(n_q=32, n_kv=8, d=128, page=64)       # 32 query heads, 8 KV heads
_32B = dict(n_q=64, n_kv=8, d=128, page=64)      # 64 query heads, 8 KV heads
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------
def _turn(shape, layout="half", rot_start=0, rot_dim=None, theta=1e6, scaling="none", factor=1.0, low=1.0, high=32.0,
          original=32768, magnitude=1.0):
    return dict(layout=layout, rot_start=rot_start, rot_dim=shape["d"] if rot_dim is None else rot_dim, theta=theta,
                scaling=scaling, factor=factor, low=low, high=high, original=original, magnitude=magnitude)


def _rope(name, shape, tokens, far, dtype="bf16", transpose=False, **turn):
    return dict(name=name, op="rope", tokens=tokens, far=far, dtype=dtype, transpose=transpose, **shape, **_turn(shape, **turn))


def _append(name, shape, batch, lo, hi, at_lo, at_hi, lens, cache="bf16", queries=True, pad=0, **turn):
    return dict(name=name, op="append", batch=batch, lo=lo, hi=hi, at_lo=at_lo, at_hi=at_hi, lens=lens, cache=cache,
                queries=queries, pad=pad, **shape, **_turn(shape, **turn))


def _logits(name, rows, vocab, dtype, given=1, top=5, temperature=1.0, masked=0.0, pad=0):
    return dict(name=name, op="logits", rows=rows, vocab=vocab, dtype=dtype, given=given, top=top, temperature=temperature,
                masked=masked, pad=pad)


def _head(name, rows, hidden, vocab, given=1, top=5, temperature=1.0, extra=3):
    return dict(name=name, op="head", rows=rows, hidden=hidden, vocab=vocab, given=given, top=top, temperature=temperature,
                extra=extra)


def listed():
    return [
        # queries and keys of one decoded token of 32 sequences, far into contexts four times the trained length
        _rope("rope step x32", _8B, 32, 131072, scaling="ramp", factor=4.0, magnitude=0.1 * math.log(4.0) + 1),
        # the queries and keys of one long prompt
        _rope("rope prompt", _8B, 8192, 8192),
        # a head of which a part turns, pairs side by side, in 32 bits, turned back
        _rope("rope part, back", dict(n_q=16, n_kv=16, d=192, page=64), 2001, 70000, "fp32", True, layout="interleaved",
              rot_start=128, rot_dim=64, theta=5e5, scaling="bands", factor=8.0, low=1.0, high=4.0, original=8192),
        # one decoded token of each of 32 sequences: the call of every layer and step
        _append("append step x32", _8B, 32, 1, 1, 2048, 8192, 1),
        # prompts of a batch, ragged, behind a padded end of the row buffer
        _append("append prompts", _8B, 8, 1000, 8192, 0, 100, 2, pad=37),
        # the step over an 8-bit cache, 64 query heads
        _append("append step x32, 8 bits", _32B, 32, 1, 1, 2048, 30000, 3, "e4m3", scaling="linear", factor=2.0),
        # one prompt into an 8-bit cache, keys alone (a draft layer's context)
        _append("append prompt, 8 bits", _8B, 1, 4096, 4096, 0, 0, 4, "e4m3", queries=False, layout="interleaved", rot_dim=64),
        # one answer's next token with its best alternatives: the smallest call
        _logits("logits one row", 1, 151936, "bf16", top=20),
        # the slots of four verified trees, an odd vocabulary of which a grammar allows half
        _logits("logits tree slots", 244, 32001, "fp32", given=3, top=8, temperature=0.7, masked=0.5),
        # every token of a batch of prompts
        _logits("logits prompts", 4096, 151936, "bf16"),
        # the verified slots of one chain draft
        _head("head chain", 7, 4096, 151936, top=20),
        # the tokens of a prompt
        _head("head prompt", 1000, 4096, 151936),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rope", "append", "logits", "head"))
    if op in ("rope", "append"):
        d = rng.choice((64, 128, 128) if op == "append" else (64, 80, 96, 128, 128, 192, 256))
        n_kv = rng.choice((1, 2, 4, 8))
        shape = dict(n_q=n_kv * rng.choice((1, 2, 4, 8)), n_kv=n_kv, d=d, page=rng.choice((16, 32, 64, 64, 128)))
        rot = rng.choice((d, d, d // 2, 2 * rng.randint(2, d // 2)))
        scaling = rng.choice(("none", "linear", "base", "bands", "ramp", "list"))
        turn = dict(layout=rng.choice(("half", "interleaved")), rot_dim=rot,
                    rot_start=rng.choice((0, 0, (d - rot) // 2 * 2)), theta=rng.choice((1e4, 5e5, 1e6)), scaling=scaling,
                    factor=1.0 if scaling == "none" else round(rng.uniform(1.5, 16.0), 2), low=1.0,
                    high=rng.choice((4.0, 32.0)), original=rng.choice((4096, 8192, 32768)),
                    magnitude=rng.choice((1.0, 1.0, 1.139)))
        if op == "rope":
            most = 8192 * 40 * 128 // ((shape["n_q"] + n_kv) * d)
            case = _rope("", shape, _log(rng, 1, min(8192, most)), _log(rng, 100, 10 ** 6),
                         rng.choice(("bf16", "bf16", "fp16", "fp32")), rng.choice((False, False, True)), **turn)
        else:
            batch = _log(rng, 1, 64)
            hi = _log(rng, 1, min(8192, 30000 * 48 * 128 // (batch * (shape["n_q"] + 2 * n_kv) * d)))
            at = _log(rng, 1, 4000)
            cache = rng.choice(("bf16", "bf16", "e4m3"))
            if cache == "e4m3":
                hi = min(hi, max(1, 4096 // batch))
            case = _append("", shape, batch, rng.randint(1, hi), hi, rng.randint(0, at), at, rng.randint(0, 10 ** 6), cache,
                           rng.choice((True, True, False)), rng.choice((0, 0, 1, 50)), **turn)
    elif op == "logits":
        vocab = _log(rng, 50, 200000)
        dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
        most = 4096 * 151936 // (vocab * (2 if dtype == "fp32" else 1))
        case = _logits("", _log(rng, 1, min(4096, most)), vocab, dtype, rng.choice((1, 1, 2, 8)), rng.choice((0, 1, 5, 8, 20, 32)),
                       rng.choice((1.0, 1.0, 0.6, 1.7)), rng.choice((0.0, 0.0, 0.5, 0.9)), rng.choice((0, 0, 1, 8)))
    else:
        hidden, vocab = 8 * rng.randint(128, 640), _log(rng, 1000, 151936)
        case = _head("", _log(rng, 1, 1000), hidden, vocab, rng.choice((1, 1, 2, 8)),
                     rng.choice((0, 1, 5, 8) if hidden < 2048 else (0, 1, 5, 8, 20)), rng.choice((1.0, 1.0, 0.6, 1.7)),
                     rng.choice((0, 3)))
        if case["rows"] * hidden * vocab > 1000 * 4096 * 151936:
            case["rows"] = 1000 * 4096 * 151936 // (hidden * vocab)
    del case["name"]
    return case


def _span(rng, lo, hi, n):
    """n lengths between lo and hi, spread over their logarithm; the ends are among them."""
    got = [int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1 for _ in range(n)]
    got = [min(hi, max(lo, v)) for v in got]
    got[rng.randrange(n)] = hi
    if n > 1:
        got[rng.randrange(n)] = lo
    return got


def _plan(case):
    """Lengths, first slots and page counts of an append (the same for every seed)."""
    rng = random.Random(case["lens"])
    n = _span(rng, case["lo"], case["hi"], case["batch"])
    at = _span(rng, case["at_lo"], case["at_hi"], case["batch"])
    return dict(n=n, at=at, start=[0, *itertools.accumulate(n)], pages=-(-max(a + v for a, v in zip(at, n)) // case["page"]))


def _frequencies(case):
    """f_i of a case, in radians per position.

    linear: f / factor.  base: theta becomes theta * factor^(r / (r - 2)).  list: f / divisor_i.  bands: with n = original *
    f / (2 pi) turns over the trained length, f above `high` turns, f / factor below `low`, and between them the mean with
    the weight (n - low) / (high - low) on f.  ramp: f * (1 - w_i + w_i / factor), w_i rising from 0 to 1 with i between
    floor(index(high)) and ceil(index(low)), held to [0, r - 1], where index(n) = r ln(original / (2 pi n)) / (2 ln theta)."""
    r, how, factor = case["rot_dim"], case["scaling"], case["factor"]
    theta = case["theta"] * factor ** (r / (r - 2)) if how == "base" else case["theta"]
    f = [theta ** (-2.0 * i / r) for i in range(r // 2)]
    if how == "linear":
        return [v / factor for v in f]
    if how == "list":
        return [v / w for v, w in zip(f, _divisors(case))]
    if how == "bands":
        w = [min(1.0, max(0.0, (case["original"] * v / (2 * math.pi) - case["low"]) / (case["high"] - case["low"]))) for v in f]
        return [v * (a + (1 - a) / factor) for v, a in zip(f, w)]
    if how == "ramp":
        index = [r * math.log(case["original"] / (2 * math.pi * n)) / (2 * math.log(theta)) for n in (case["high"], case["low"])]
        a, b = max(math.floor(index[0]), 0), min(math.ceil(index[1]), r - 1)
        w = [min(1.0, max(0.0, (i - a) / max(b - a, 1e-3))) for i in range(r // 2)]
        return [v * (1 - u + u / factor) for v, u in zip(f, w)]
    return f


def _divisors(case):
    n = case["rot_dim"] // 2
    return [1.0 + (case["factor"] - 1.0) * i / max(1, n - 1) for i in range(n)]


def work(case):
    if case["op"] == "rope":
        rows = case["tokens"] * (case["n_q"] + case["n_kv"])
        return {"bytes": 2 * rows * case["d"] * _TYPES[case["dtype"]].itemsize + 4 * case["tokens"], "flops": 3 * rows * case["rot_dim"]}
    if case["op"] == "append":
        tokens, kv, d = _plan(case)["start"][-1], case["n_kv"], case["d"]
        turned = kv + (case["n_q"] if case["queries"] else 0)
        row = kv * (4 * d if case["cache"] == "bf16" else 2 * d + 2)
        return {"bytes": tokens * (kv * 4 * d + row + (case["n_q"] * 4 * d if case["queries"] else 0)),
                "flops": 3 * tokens * turned * case["rot_dim"]}
    out = case["rows"] * (8 * case["given"] + 4 + 8 * case["top"])
    if case["op"] == "logits":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * _TYPES[case["dtype"]].itemsize + out, "flops": 5 * n}
    return {"bytes": 2 * case["hidden"] * (case["vocab"] + case["rows"]) + out,
            "flops": 2 * case["rows"] * case["hidden"] * case["vocab"]}


# ---------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------
def _rows_like(shape, dtype, dev, gen):
    """Queries, keys or values as a projection makes them: some channels and some tokens are much larger than others."""
    x = torch.randn(shape, device=dev, generator=gen)
    x *= torch.exp(0.5 * torch.randn(shape[-2:], device=dev, generator=gen))
    x *= torch.exp(0.3 * torch.randn(shape[:-1], device=dev, generator=gen)).unsqueeze(-1)
    return x.to(dtype)


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    s = dict(case=case)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    if case["op"] in ("rope", "append"):
        s["freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device=dev)
    if case["op"] == "rope":
        dt, T, d = _TYPES[case["dtype"]], case["tokens"], case["d"]
        s["pos"] = torch.randint(0, case["far"], (T,), device=dev, generator=gen).to(torch.int32)
        s["q"], s["k"] = (_rows_like((T, case["n_" + n], d), dt, dev, gen) for n in ("q", "kv"))
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        return s
    if case["op"] == "append":
        p = _plan(case)
        B, kv, d, page, T = case["batch"], case["n_kv"], case["d"], case["page"], p["start"][-1] + case["pad"]
        num = B * p["pages"] + 3                              # a pool in no order, larger than its use
        s["page_table"] = torch.randperm(num, device=dev, generator=gen)[:num - 3].to(torch.int32).view(B, -1)
        # the projection's output: queries, keys and values of a token lie in one row
        s["qkv"] = _rows_like((T, case["n_q"] + 2 * kv, d), torch.bfloat16, dev, gen)
        s["q_out"] = torch.full((T, case["n_q"], d), -7.0, dtype=torch.bfloat16, device=dev)
        pool = (num, kv, page, d)
        kind = torch.bfloat16 if case["cache"] == "bf16" else torch.uint8
        s["k_pages"], s["v_pages"] = (torch.zeros(pool, dtype=kind, device=dev) for _ in "kv")
        if case["cache"] == "e4m3":
            s["k_scale"], s["v_scale"] = (torch.full(pool[:3], 127, dtype=torch.uint8, device=dev) for _ in "kv")
        s["cache_len"], s["row_start"], s["pos_start"] = i32(p["at"]), i32(p["start"]), i32(p["at"])
        return s
    R, V = case["rows"], case["vocab"]
    s["tokens"] = torch.randint(0, V, (R, case["given"]), device=dev, generator=gen).to(torch.int32)
    if case["op"] == "logits":
        dt = _TYPES[case["dtype"]]
        x = torch.empty((R, V + case["pad"]), dtype=dt, device=dev)[:, :V]
        x.copy_(torch.randn((R, V), device=dev, generator=gen) * 2.0)
        # a few tokens of a row stand out of the rest
        at = (torch.randint(0, V, (R, 1), device=dev, generator=gen) + torch.arange(12, device=dev) * (V // 12)) % V
        x.scatter_(1, at, (torch.rand((R, 12), device=dev, generator=gen) * 12 + 4).to(dt))
        if case["masked"]:
            drop = torch.rand((R, V), device=dev, generator=gen) < case["masked"]
            drop.scatter_(1, at[:, :1], False)
            x.masked_fill_(drop, -math.inf)
        s["logits"] = x
        return s
    H = case["hidden"]
    s["head"] = torch.empty((V + case["extra"], H), dtype=torch.bfloat16, device=dev)
    s["head"].copy_(torch.randn((V + case["extra"], H), device=dev, generator=gen) * 0.02)
    # hidden states under which a few tokens stand out, as far from one another as the alternatives of a trained model:
    # h = noise + the smallest vector that gives these tokens their logits
    n = case["top"] + 4
    at = (torch.randint(0, V, (R, 1), device=dev, generator=gen) + torch.arange(n, device=dev) * (V // n)) % V
    want = 12.0 + 0.5 * (torch.arange(n, device=dev) + 0.6 * torch.rand((R, n), device=dev, generator=gen))
    want = torch.gather(want, 1, torch.rand((R, n), device=dev, generator=gen).argsort(1))
    h = 0.3 * torch.randn((R, H), device=dev, generator=gen)
    w = s["head"][at].float()                                                          # [R, n, H]
    gram = torch.bmm(w, w.transpose(1, 2))
    gap = want - torch.bmm(w, h.unsqueeze(2)).squeeze(2)
    h += torch.bmm(w.transpose(1, 2), torch.linalg.solve(gram, gap).unsqueeze(2)).squeeze(2)
    s["hidden"] = h.to(torch.bfloat16)
    s["tokens"][:, 0] = at[:, 0].to(torch.int32)
    return s


# ---------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------
def _angles(s, pos, wide):
    """cos and sin [T, 1, r / 2] of the pairs' angles, which far positions take beyond 32 bits."""
    a = pos.double().unsqueeze(1) * s["freq"]
    c, n = (torch.cos(a) * s["case"]["magnitude"]).unsqueeze(1), (torch.sin(a) * s["case"]["magnitude"]).unsqueeze(1)
    return (c, n) if wide else (c.float(), n.float())


def _turned(case, x, c, n):
    """x [T, heads, d] with its rotated part turned, in the type of c, rounded once."""
    a, r = case["rot_start"], case["rot_dim"]
    part = x[..., a:a + r].to(c.dtype)
    out = x.clone()
    if case["layout"] == "half":
        u, v = part[..., :r // 2], part[..., r // 2:]
        out[..., a:a + r // 2], out[..., a + r // 2:a + r] = (u * c - v * n).to(x.dtype), (v * c + u * n).to(x.dtype)
    else:
        u, v = part[..., 0::2], part[..., 1::2]
        out[..., a:a + r:2], out[..., a + 1:a + r:2] = (u * c - v * n).to(x.dtype), (v * c + u * n).to(x.dtype)
    return out


def _quantise(x):
    """Codes (uint8 holding e4m3) and exponent bytes of rows x [.., d]."""
    x = x.float()
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)
    e = (e - 9 + (m > 0.875)).clamp(-64, 120)
    e = torch.where(top == 0, torch.zeros_like(e), e)
    inv = ((127 - e).to(torch.int32) << 23).view(torch.float32)
    return (x * inv.unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _plain_append(s):
    case = s["case"]
    nq, kv, page = case["n_q"], case["n_kv"], case["page"]
    start = s["row_start"].long()
    t = torch.arange(s["qkv"].shape[0], device=start.device)
    t = t[t < start[-1]]
    b = torch.searchsorted(start, t, right=True) - 1
    pos = s["pos_start"].long()[b] + t - start[b]
    pp, off = s["page_table"].long()[b, pos // page], pos % page
    c, n = _angles(s, pos, case["cache"] == "e4m3")           # whole values next to a border take 64 bits
    k, v = _turned(case, s["qkv"][t, nq:nq + kv], c, n), s["qkv"][t, nq + kv:]
    if case["queries"]:
        s["q_out"][t] = _turned(case, s["qkv"][t, :nq], c, n)
    if case["cache"] == "bf16":
        s["k_pages"][pp, :, off], s["v_pages"][pp, :, off] = k, v
        return
    s["k_pages"][pp, :, off], s["k_scale"][pp, :, off] = _quantise(k)
    s["v_pages"][pp, :, off], s["v_scale"][pp, :, off] = _quantise(v)


def _plain_scores(case, raw, tokens):
    """raw [R, V] in 32 bits."""
    R, V = raw.shape
    x = raw / case["temperature"]
    d = x - x.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    lse = torch.log(total)
    got = {"logp": torch.gather(d, 1, tokens.long()) - lse,
           "entropy": (lse - (e * torch.where(e > 0, d, torch.zeros_like(d))).sum(1, keepdim=True) / total).squeeze(1)}
    if case["top"]:
        # larger first, then the lower id: one whole number that says both
        bits = raw.view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7fffffff), bits) * (1 << 20) + ((1 << 20) - 1 - torch.arange(V, device=raw.device))
        key, _ = torch.topk(key, min(case["top"], V), 1)
        at = (1 << 20) - 1 - (key & (1 << 20) - 1)
        logp = torch.gather(d, 1, at) - lse
        got["top_tok"], got["top_logp"] = torch.where(logp == -math.inf, -1, at).to(torch.int32), logp
    return got


def _plain(s):
    case = s["case"]
    if case["op"] == "rope":
        c, n = _angles(s, s["pos"], False)
        n = -n if case["transpose"] else n
        s["q_out"].copy_(_turned(case, s["q"], c, n))
        s["k_out"].copy_(_turned(case, s["k"], c, n))
        return None
    if case["op"] == "append":
        return _plain_append(s)
    if case["op"] == "logits":
        return _plain_scores(case, s["logits"].float(), s["tokens"])
    return _plain_scores(case, torch.matmul(s["hidden"].float(), s["head"][:case["vocab"]].float().T), s["tokens"])


def _call(s):
    from paper_2509_24248_b200 import binding as sx
    case = s["case"]
    if case["op"] in ("rope", "append") and "rope" not in s:
        s["rope"] = sx.Rope(case["d"], case["theta"], rot_dim=case["rot_dim"], rot_start=case["rot_start"],
                            layout={"half": sx.ROPE_HALF, "interleaved": sx.ROPE_INTERLEAVED}[case["layout"]],
                            scaling={"none": sx.ROPE_NONE, "linear": sx.ROPE_LINEAR, "base": sx.ROPE_BASE, "bands": sx.ROPE_BANDS,
                                     "ramp": sx.ROPE_RAMP, "list": sx.ROPE_LIST}[case["scaling"]],
                            factor=case["factor"], low=case["low"], high=case["high"], original_len=case["original"],
                            magnitude=case["magnitude"], divisors=_divisors(case) if case["scaling"] == "list" else None)
    if case["op"] == "rope":
        s["rope"].sx_rope(s["pos"], s["q"], s["k"], q_out=s["q_out"], k_out=s["k_out"], transpose=case["transpose"])
        return None
    if case["op"] == "append":
        if "cache" not in s:
            s["cache"] = sx.KVPages({n: s[n] for n in ("k_pages", "v_pages", "k_scale", "v_scale", "page_table", "cache_len") if n in s})
        nq, kv = case["n_q"], case["n_kv"]
        q = s["qkv"][:, :nq] if case["queries"] else None
        s["cache"].sx_kv_append_rope(s["rope"], s["qkv"][:, nq:nq + kv], s["qkv"][:, nq + kv:], s["row_start"], s["pos_start"],
                                     q=q, q_out=s["q_out"] if case["queries"] else None)
        return None
    if "scores" not in s:
        s["scores"] = sx.LogProbs(s["head"] if case["op"] == "head" else None, vocab=case["vocab"])
    if case["op"] == "logits":
        return s["scores"].sx_logprobs(s["logits"], s["tokens"], top=case["top"], temperature=case["temperature"])
    return s["scores"].sx_head_logprobs(s["hidden"], s["tokens"], top=case["top"], temperature=case["temperature"])


def run(state):
    got = _call(state) if own else _plain(state)
    case = state["case"]
    if case["op"] == "rope":
        return {"q": state["q_out"], "k": state["k_out"]}
    if case["op"] == "append":
        if case["cache"] == "bf16":
            return {"k": state["k_pages"], "v": state["v_pages"], "q": state["q_out"]}
        return {"k": state["k_pages"].view(torch.float8_e4m3fn), "v": state["v_pages"].view(torch.float8_e4m3fn),
                "k_scale": state["k_scale"], "v_scale": state["v_scale"], "q": state["q_out"]}
    return {n: got[n] for n in (("logp", "entropy", "top_tok", "top_logp") if case["top"] else ("logp", "entropy"))}


# ---------------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------
def _exact_turned(case, x, pos, back=False):
    """The rotated part as complex numbers, multiplied by magnitude * e^(i angle) (its conjugate when turned back)."""
    a, r = case["rot_start"], case["rot_dim"]
    x = x.double()
    part = x[..., a:a + r]
    pairs = part.unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else part.unflatten(-1, (r // 2, 2))
    angle = pos.double()[:, None, None] * torch.tensor(_frequencies(case), dtype=torch.float64, device=x.device)
    by = torch.polar(torch.full_like(angle, case["magnitude"]), -angle if back else angle)
    pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by)
    part = (pairs.transpose(-1, -2) if case["layout"] == "half" else pairs).flatten(-2)
    return torch.cat((x[..., :a], part, x[..., a + r:]), -1)


def _exact_codes(x):
    """Nearest code values and exponent bytes of finite rows, in 64 bits."""
    x = x.double()
    top = x.abs().amax(-1)
    e = torch.zeros_like(top)
    alive = top > 0
    # the smallest e with top <= 448 * 2^e, from a guess put right by comparing
    e[alive] = torch.round(torch.log2(top[alive] / 448.0))
    e = torch.where(alive & (top > 448.0 * torch.exp2(e)), e + 1, e)
    e = torch.where(alive & (top <= 448.0 * torch.exp2(e - 1)), e - 1, e)
    e = torch.where(alive, e.clamp(-64, 120), e)
    y = x / torch.exp2(e).unsqueeze(-1)
    a = y.abs()
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)        # distance of neighbouring codes
    r = a / step
    lo = torch.floor(r)
    up = (r - lo > 0.5) | ((r - lo == 0.5) & (lo % 2 == 1))
    return torch.copysign((lo + up) * step, y), (e + 127).to(torch.uint8)


def _to_bf16(x):
    """Values of x (64 bits) rounded to 8 significand bits, ties to even, in 64 bits."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 256.0), e - 8)


def _exact_append(case, s):
    p, nq, kv, page = _plan(case), case["n_q"], case["n_kv"], case["page"]
    out = {n: s[n + "_pages"].double() for n in "kv"}
    out["q"] = s["q_out"].double()
    scale = {n: s[n + "_scale"].clone() for n in "kv"} if case["cache"] == "e4m3" else None
    for b in range(case["batch"]):
        pos = p["at"][b] + torch.arange(p["n"][b], device="cuda")
        rows = s["qkv"][p["start"][b]:p["start"][b + 1]]
        at = (s["page_table"][b].long()[pos // page], slice(None), pos % page)
        new = {"k": _exact_turned(case, rows[:, nq:nq + kv], pos), "v": rows[:, nq + kv:].double()}
        if case["queries"]:
            out["q"][p["start"][b]:p["start"][b + 1]] = _exact_turned(case, rows[:, :nq], pos)
        for n in "kv":
            if scale is None:
                out[n][at] = new[n]
            else:
                out[n][at], scale[n][at] = _exact_codes(_to_bf16(new[n]))
    return out if scale is None else {**out, "k_scale": scale["k"], "v_scale": scale["v"]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return {n: _exact_turned(case, s[n], s["pos"], case["transpose"]) for n in "qk"}
    if case["op"] == "append":
        return _exact_append(case, s)
    V, got = case["vocab"], []
    for i in range(0, case["rows"], 128):
        if case["op"] == "logits":
            raw = s["logits"][i:i + 128].double()
        else:
            h = s["hidden"][i:i + 128].double()
            raw = torch.cat([h @ s["head"][j:min(V, j + 20000)].double().T for j in range(0, V, 20000)], 1)
        x = raw / case["temperature"]
        logp = x - torch.logsumexp(x, 1, keepdim=True)
        p = torch.exp(logp)
        one = {"logp": torch.gather(logp, 1, s["tokens"][i:i + 128].long()),
               "entropy": -torch.where(p > 0, p * logp, 0.0).sum(1)}
        if case["top"]:
            value, at = torch.sort(raw, dim=1, descending=True, stable=True)
            value, at = value[:, :case["top"]], at[:, :case["top"]]
            one["top_tok"] = torch.where(value == -math.inf, -1, at).to(torch.int32)
            one["top_logp"] = torch.gather(logp, 1, at)
        got.append(one)
    return {n: torch.cat([g[n] for g in got]) for n in got[0]}
