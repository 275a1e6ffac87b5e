"""The operators of the 8-bit paged KV cache as cases to time and compare.

Three operators, as a program calls them that decodes many answers over a quantised cache:

``append``     keys and values of new tokens (bf16) are written into the pages as e4m3 codes with one power-of-two
               scale per (token, KV head), the scale as a biased exponent byte
``read``       a range of slots of every sequence is read back to bf16
``attention``  decode attention over such a cache: one to a few query rows per sequence, drafted slots behind the
               cached ones with a visibility mask, and groups of sequences that share a prefix

Format: a row x[0..d) of one token and head has the scale 2^e with e = ceil(log2(max|x| / 448)) held to
[-64, 120] (0 for a row of zeros), stored as the byte e + 127, and the codes e4m3(x * 2^-e), round to nearest even.
A row with a value that is not finite has the byte 255 and codes of zero, and reads back as NaN.
"""
import itertools
import math
import random

import torch

own = False          # set from outside: False runs the plain forms, True the package's entry points

_8B = dict(n_kv=8, group=4, d=128, page=64)       # 32 query heads, 8 KV heads
_32B = dict(n_kv=8, group=8, d=128, page=64)      # 64 query heads, 8 KV heads
_TINY = dict(n_kv=2, group=2, d=64, page=64)      # 4 query heads, 2 KV heads


# ---------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------
def _rows(name, op, shape, batch, lo, hi, at_lo, at_hi, lens, pad=0):
    return dict(name=name, op=op, batch=batch, lo=lo, hi=hi, at_lo=at_lo, at_hi=at_hi, lens=lens, pad=pad, **shape)


def _attn(name, shape, batch, lo, hi, rows, drafted, lens, groups=0, prefix_lo=0, prefix_hi=0):
    return dict(name=name, op="attention", batch=batch, lo=lo, hi=hi, rows=rows, drafted=drafted, lens=lens,
                groups=groups, prefix_lo=prefix_lo, prefix_hi=prefix_hi, **shape)


def listed():
    return [
        # one decoded token of each of 32 sequences: the smallest call, made once per step
        _rows("append one token x32", "append", _8B, 32, 1, 1, 2048, 8192, 1),
        # prompts of a batch, ragged, behind a padded end of the row buffer
        _rows("append prompts", "append", _8B, 8, 1000, 8192, 0, 100, 2, pad=37),
        # one prompt moved to a bf16 cache
        _rows("read one prompt", "read", _8B, 1, 4096, 4096, 0, 0, 3),
        # the caches of a whole batch
        _rows("read batch 32", "read", _8B, 32, 2048, 8192, 0, 0, 4),
        # tiny shape: three short ragged sequences, latency alone
        _attn("attention tiny", _TINY, 3, 1, 129, 1, 1, 5),
        # chain draft of one sequence, second round
        _attn("attention chain 4k", _8B, 1, 4096, 4096, 1, 2, 6),
        # chain draft of a batch of ragged sequences
        _attn("attention chain x32", _8B, 32, 2048, 8192, 1, 3, 7),
        # the wide group of 64 query heads on long reasoning contexts
        _attn("attention chain 16k x8", _32B, 8, 16384, 16384, 1, 6, 8),
        # last round of a top-8 tree of depth 6 on long contexts
        _attn("attention tree 32k x4", _8B, 4, 32768, 32768, 8, 41, 9),
        # 32 sampled answers of one question with a long prompt
        _attn("attention prefix x32", _8B, 32, 64, 2048, 1, 3, 10, 1, 16384, 16384),
        # a tree over 8 answers of one long context
        _attn("attention prefix tree x8", _8B, 8, 500, 4096, 8, 41, 11, 1, 30001, 30001),
        # several questions with several answers each, wide group, verification rows
        _attn("attention prefix 4x8", _32B, 32, 100, 3000, 2, 5, 12, 4, 1000, 16000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    shape = dict(n_kv=rng.choice((1, 2, 4, 8)), group=rng.choice((1, 2, 4, 8)), d=rng.choice((64, 128, 128)),
                 page=rng.choice((16, 32, 64, 64, 128)))
    op = rng.choice(("append", "read", "attention", "attention", "attention"))
    batch = _log(rng, 1, 64)
    if op != "attention":
        hi = _log(rng, 1, min(16384, 130000 // batch))
        lo = rng.randint(min(hi, 1), hi)
        at = _log(rng, 1, 4000)
        case = _rows("", op, shape, batch, lo, hi, rng.randint(0, at), at, rng.randint(0, 10 ** 6),
                     rng.choice((0, 0, 1, 50)))
        del case["name"]
        return case
    groups = rng.choice((0, 0, 1, min(batch, 3), min(batch, 7)))
    hi = _log(rng, 1, min(32768, 130000 // batch))
    lo = rng.randint(0, hi)
    rows = rng.choice((1, 1, 1, 2, 3, 4, 5, 8))
    drafted = rows if rows > 1 else rng.choice((0, 1, 2, 6))
    drafted += rng.choice((0, 1, 9, 33)) if rows > 1 else 0
    p_hi = _log(rng, 1, min(32768, 130000 // batch)) if groups else 0
    case = _attn("", shape, batch, lo, hi, rows, drafted, rng.randint(0, 10 ** 6), groups,
                 rng.randint(0, p_hi) if groups else 0, p_hi)
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
    """Lengths, groups and page counts of a case (the same for every seed)."""
    rng = random.Random(case["lens"])
    B, page = case["batch"], case["page"]
    if case["op"] != "attention":
        n = _span(rng, case["lo"], case["hi"], B)
        at = _span(rng, case["at_lo"], case["at_hi"], B)
        return dict(n=n, at=at, start=[0, *itertools.accumulate(n)], pages=-(-max(a + v for a, v in zip(at, n)) // page))
    mine = _span(rng, case["lo"], case["hi"], B)
    g = case["groups"]
    start = [B * i // g for i in range(g + 1)] if g else []
    prefix = _span(rng, case["prefix_lo"], case["prefix_hi"], g) if g else []
    of = [next(i for i in range(g) if b < start[i + 1]) for b in range(B)] if g else []
    n = [m + (prefix[of[b]] if g else 0) for b, m in enumerate(mine)]
    return dict(n=n, mine=mine, start=start, prefix=prefix, of=of,
                pages=max(1, -(-(max(n) + case["drafted"]) // page)))


def work(case):
    p, kv, d = _plan(case), case["n_kv"], case["d"]
    row = kv * (2 * d + 2)                                   # codes and scale bytes of one token
    if case["op"] != "attention":
        tokens = p["start"][-1]
        return {"bytes": tokens * (kv * d * 4 + row), "flops": tokens * kv * d * 4}
    B, rows, q = case["batch"], case["rows"], case["n_kv"] * case["group"]
    cached = sum(p["mine"]) + sum(p["prefix"]) + B * case["drafted"]
    seen = sum(p["n"]) + B * case["drafted"]
    return {"bytes": cached * row + 2 * B * rows * q * d * 2 + 4 * B * (p["pages"] + 1) + 8 * B * rows,
            "flops": 4 * d * rows * q * seen}


# ---------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------
def _kv_like(shape, dev, gen):
    """Keys or values as a model makes them: some channels and some tokens are much larger than others."""
    x = torch.randn(shape, device=dev, generator=gen)
    x *= torch.exp(0.5 * torch.randn(shape[-2:], device=dev, generator=gen))
    x *= torch.exp(0.3 * torch.randn(shape[:-1], device=dev, generator=gen)).unsqueeze(-1)
    return x.to(torch.bfloat16)


def _scale_of(byte):
    """2^(byte - 127) in 32 bits, from the bits of the number; the byte 255 gives NaN."""
    f = (byte.to(torch.int32) << 23).view(torch.float32)
    return torch.where(byte == 255, torch.full_like(f, float("nan")), f)


def _quantise(x):
    """Codes (uint8 holding e4m3) and exponent bytes of rows x [.., d]."""
    x = x.float()
    top = x.abs().amax(-1)
    bad = ~torch.isfinite(top)
    m, e = torch.frexp(torch.where(bad, torch.ones_like(top), top))
    e = (e - 9 + (m > 0.875)).clamp(-64, 120)
    e = torch.where(top == 0, torch.zeros_like(e), e)
    inv = ((127 - e).to(torch.int32) << 23).view(torch.float32)
    x = torch.where(bad.unsqueeze(-1), torch.zeros_like(x), x * inv.unsqueeze(-1))
    byte = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return x.to(torch.float8_e4m3fn).view(torch.uint8), byte


def prepare(case, seed):
    dev = "cuda"
    p = _plan(case)
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device=dev).manual_seed(seed)
    B, kv, d, page = case["batch"], case["n_kv"], case["d"], case["page"]
    num = B * p["pages"] + 3                                  # a pool in no order, larger than its use
    table = torch.randperm(num, generator=cpu)[:num - 3].to(torch.int32).view(B, -1)
    for i, n in enumerate(p.get("prefix", ())):
        # the whole pages of a shared prefix are the same in its group
        a, b = p["start"][i], p["start"][i + 1]
        table[a:b, :n // page] = table[a, :n // page].clone()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    s = dict(case=case, page_table=table.to(dev), n_max=p["pages"] * page)
    pool = (num, kv, page, d)
    if case["op"] == "append":
        T = p["start"][-1] + case["pad"]
        # the projection's output: keys and values of a token lie in one row
        s["kv_rows"] = torch.stack((_kv_like((T, kv, d), dev, gen), _kv_like((T, kv, d), dev, gen)), 1)
        s["k_pages"], s["v_pages"] = (torch.zeros(pool, dtype=torch.uint8, device=dev) for _ in "kv")
        s["k_scale"], s["v_scale"] = (torch.full(pool[:3], 127, dtype=torch.uint8, device=dev) for _ in "kv")
        s["cache_len"] = i32([0] * B)
    else:
        s["k_pages"], s["k_scale"] = _quantise(_kv_like(pool, dev, gen))
        s["v_pages"], s["v_scale"] = _quantise(_kv_like(pool, dev, gen) * 0.5)
        s["cache_len"] = i32(p["n"] if case["op"] == "attention" else [a + v for a, v in zip(p["at"], p["n"])])
    if case["op"] != "attention":
        s["row_start"], s["pos_start"] = i32(p["start"]), i32(p["at"])
        if case["op"] == "read":
            T = p["start"][-1] + case["pad"]
            s["k_out"], s["v_out"] = (torch.full((T, kv, d), -7.0, dtype=torch.bfloat16, device=dev) for _ in "kv")
        return s
    for i, n in enumerate(p["prefix"]):
        # a page that the prefix fills in part is a copy of its own for every member
        a, b, cut, lp = p["start"][i], p["start"][i + 1], n % page, n // page
        if cut:
            src, dst = table[a, lp].item(), table[a + 1:b, lp].tolist()
            for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
                s[name][dst, :, :cut] = s[name][src, :, :cut]
    rows, E, q = case["rows"], case["drafted"], kv * case["group"]
    s["q"] = _kv_like((B, rows, q, d), dev, gen)
    s["out"] = torch.empty_like(s["q"])
    if p["prefix"]:
        s["group_start"], s["prefix_len"] = i32(p["start"]), i32(p["prefix"])
    if rows > 1:
        # the last `rows` drafted slots are these rows' own; each also sees slot 0 and some of the others before
        first = E - rows
        bits = [[1 | 1 << (first + j) | (random.Random(seed * 1000003 + b * 64 + j).getrandbits(64) & ((1 << first) - 1))
                 for j in range(rows)] for b in range(B)]
        s["row_mask"] = torch.tensor([[v - (1 << 64) if v >> 63 else v for v in r] for r in bits], device=dev)
    return s


# ---------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------
def _row_places(s):
    """(rows that exist, their flat slots page * page_size + offset) of an append or a read."""
    T = (s["kv_rows"] if "kv_rows" in s else s["k_out"]).shape[0]
    start, page = s["row_start"].long(), s["k_pages"].shape[2]
    t = torch.arange(T, device=start.device)
    t = t[t < start[-1]]
    b = torch.searchsorted(start, t, right=True) - 1
    pos = s["pos_start"].long()[b] + t - start[b]
    return t, s["page_table"].long()[b, pos // page], pos % page


def _plain(s):
    case = s["case"]
    if case["op"] == "append":
        t, pp, off = _row_places(s)
        for_k, k_byte = _quantise(s["kv_rows"][t, 0])
        for_v, v_byte = _quantise(s["kv_rows"][t, 1])
        s["k_pages"][pp, :, off], s["k_scale"][pp, :, off] = for_k, k_byte
        s["v_pages"][pp, :, off], s["v_scale"][pp, :, off] = for_v, v_byte
        return
    if case["op"] == "read":
        t, pp, off = _row_places(s)
        s["k_out"][t] = (s["k_pages"][pp, :, off].view(torch.float8_e4m3fn).float()
                         * _scale_of(s["k_scale"][pp, :, off]).unsqueeze(-1)).to(torch.bfloat16)
        s["v_out"][t] = (s["v_pages"][pp, :, off].view(torch.float8_e4m3fn).float()
                         * _scale_of(s["v_scale"][pp, :, off]).unsqueeze(-1)).to(torch.bfloat16)
        return
    q, E, page = s["q"], case["drafted"], case["page"]
    B, rows, nq, d = q.shape
    kv, G = case["n_kv"], case["group"]
    slot = torch.arange(s["n_max"], device=q.device)
    pp, off = s["page_table"].long()[:, slot // page], slot % page                  # [B, L]
    k = s["k_pages"][pp, :, off].view(torch.float8_e4m3fn).float() * _scale_of(s["k_scale"][pp, :, off]).unsqueeze(-1)
    v = s["v_pages"][pp, :, off].view(torch.float8_e4m3fn).float() * _scale_of(s["v_scale"][pp, :, off]).unsqueeze(-1)
    behind = slot - s["cache_len"].long().unsqueeze(1)                              # [B, L]: >= 0 is a drafted slot
    bit = behind.clamp(0, 63).unsqueeze(1)
    mask = s["row_mask"] if "row_mask" in s else torch.full((B, rows), (1 << min(E, 62)) - 1, device=q.device)
    seen = ((mask.unsqueeze(2) >> bit) & 1).bool() & (behind < E).unsqueeze(1)      # [B, rows, L]
    seen = seen | (behind < 0).unsqueeze(1)
    qh = q.float().view(B, rows, kv, G, d).permute(0, 2, 1, 3, 4).reshape(B, kv, rows * G, d)
    a = torch.matmul(qh, k.permute(0, 2, 3, 1)) / math.sqrt(d)                      # [B, kv, rows * G, L]
    a = a.view(B, kv, rows, G, -1).masked_fill(~seen.view(B, 1, rows, 1, -1), -math.inf).view(B, kv, rows * G, -1)
    top = a.amax(-1, keepdim=True)
    a = torch.exp(a - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = a.sum(-1, keepdim=True)
    o = torch.matmul(a, v.permute(0, 2, 1, 3)) / torch.where(total == 0, torch.ones_like(total), total)
    s["out"].copy_(o.view(B, kv, rows, G, d).permute(0, 2, 1, 3, 4).reshape(B, rows, nq, d))


def _call(s):
    from paper_2509_24248_b200 import binding as sx
    case = s["case"]
    if "cache" not in s:
        s["cache"] = sx.KV8({n: s[n] for n in ("k_pages", "v_pages", "k_scale", "v_scale", "page_table", "cache_len",
                                               "group_start", "prefix_len") if n in s})
    if case["op"] == "append":
        s["cache"].sx_kv_append(s["kv_rows"][:, 0], s["kv_rows"][:, 1], s["row_start"], s["pos_start"])
    elif case["op"] == "read":
        s["cache"].sx_kv_read(s["k_out"], s["v_out"], s["row_start"], s["pos_start"])
    else:
        s["cache"].sx_attention(s["q"], drafted=case["drafted"], row_mask=s.get("row_mask"), out=s["out"])


def run(state):
    if own:
        _call(state)
    else:
        _plain(state)
    if state["case"]["op"] == "append":
        return {"k": state["k_pages"].view(torch.float8_e4m3fn), "v": state["v_pages"].view(torch.float8_e4m3fn),
                "k_scale": state["k_scale"], "v_scale": state["v_scale"]}
    if state["case"]["op"] == "read":
        return {"k": state["k_out"], "v": state["v_out"]}
    return {"o": state["out"]}


# ---------------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------
def _e4m3_values(dev):
    """The value of each of the 256 codes: sign, 4 exponent bits with bias 7, 3 mantissa bits."""
    plus = [math.nan if c == 127 else (8 + c % 8) * 2.0 ** (c // 8 - 10) if c > 7 else c * 2.0 ** -9 for c in range(128)]
    return torch.tensor(plus + [-v for v in plus], dtype=torch.float64, device=dev)


def _exact_rows(x):
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


def exact(case, seed):
    s = prepare(case, seed)
    p = _plan(case)
    page, table = case["page"], s["page_table"].long()
    value = _e4m3_values("cuda")
    if case["op"] == "append":
        k, v = (torch.zeros(s["k_pages"].shape, dtype=torch.float64, device="cuda") for _ in "kv")
        ks, vs = s["k_scale"].clone(), s["v_scale"].clone()
        for b in range(case["batch"]):
            pos = p["at"][b] + torch.arange(p["n"][b], device="cuda")
            at = (table[b, pos // page], slice(None), pos % page)
            rows = s["kv_rows"][p["start"][b]:p["start"][b + 1]]
            k[at], ks[at] = _exact_rows(rows[:, 0])
            v[at], vs[at] = _exact_rows(rows[:, 1])
        return {"k": k, "v": v, "k_scale": ks, "v_scale": vs}

    def rows_of(name, b, pos):
        at = (table[b, pos // page], slice(None), pos % page)
        return value[s[name + "_pages"][at].long()] * torch.exp2(s[name + "_scale"][at].double() - 127).unsqueeze(-1)

    if case["op"] == "read":
        out = {n: s[n + "_out"].double() for n in "kv"}
        for b in range(case["batch"]):
            pos = p["at"][b] + torch.arange(p["n"][b], device="cuda")
            for n in "kv":
                out[n][p["start"][b]:p["start"][b + 1]] = rows_of(n, b, pos)
        return out
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    G, E = case["group"], case["drafted"]
    for b in range(case["batch"]):
        n = p["n"][b]
        if n + E == 0:
            continue
        pos = torch.arange(n + E, device="cuda")
        k, v = rows_of("k", b, pos), rows_of("v", b, pos)
        for j in range(case["rows"]):
            use = torch.ones(n + E, dtype=torch.bool, device="cuda")
            if "row_mask" in s:
                m = int(s["row_mask"][b, j].item()) & (1 << 64) - 1
                use[n:] = torch.tensor([bool(m >> i & 1) for i in range(E)], device="cuda")
            for h in range(case["n_kv"]):
                q = s["q"][b, j, h * G:(h + 1) * G].double()
                w = torch.softmax(q @ k[use, h].T / case["d"] ** 0.5, -1)
                o[b, j, h * G:(h + 1) * G] = w @ v[use, h]
    return {"o": o}
