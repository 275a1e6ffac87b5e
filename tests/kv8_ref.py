"""The 8-bit paged cache and the attention over it in 64 bits on the CPU, from the definitions: numpy, no code of the
product and none of the oracle."""
from __future__ import annotations

import math

import numpy as np
import torch


def e4m3_values() -> np.ndarray:
    """The value of each code: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are not numbers."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.nan if c & 127 == 127 else math.ldexp(8 + m, e - 10) if e else math.ldexp(m, -9)
        v[c] = -x if c & 128 else x
    return v


VALUES = e4m3_values()
_POS = VALUES[:127]                      # ascending, 0 .. 448


def quantise(x: torch.Tensor):
    """(codes uint8, exponent bytes uint8) of rows ``x [.., d]``: nearest code, ties to the even one."""
    a = x.detach().to(torch.float64).cpu().numpy()
    flat = a.reshape(-1, a.shape[-1])
    codes, byte = np.zeros(flat.shape, np.uint8), np.empty(len(flat), np.uint8)
    for i, row in enumerate(flat):
        if not np.isfinite(row).all():
            byte[i] = 255
            continue
        top = np.abs(row).max()
        e = 0
        if top > 0:
            e = math.frexp(top / 448.0)[1] - 1
            while top > math.ldexp(448.0, e):
                e += 1
            while top <= math.ldexp(448.0, e - 1):
                e -= 1
            e = min(120, max(-64, e))
        byte[i] = e + 127
        y = np.ldexp(np.abs(row), -e)
        hi = np.clip(np.searchsorted(_POS, y, side="left"), 1, 126)
        lo = hi - 1
        dl, dh = y - _POS[lo], _POS[hi] - y
        pick = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
        codes[i] = pick + np.where(np.signbit(row), 128, 0)
    return (torch.from_numpy(codes.reshape(a.shape)), torch.from_numpy(byte.reshape(a.shape[:-1])))


def dequantise(codes: torch.Tensor, byte: torch.Tensor) -> np.ndarray:
    s = np.where(byte.numpy() == 255, math.nan, np.ldexp(1.0, byte.numpy().astype(np.int64) - 127))
    return VALUES[codes.numpy()] * s[..., None]


def attention(kv, q: torch.Tensor, drafted: int, row_mask, scale: float, weight: float = 2.0 ** -8):
    """(output, bound) as float64 ``[B, rows, nq, d]``: the formula, and how far the kernels' fp32 sums, rounded weights
    (``weight``: half a step of their type, 2^-11 for fp16, 2^-8 for bf16) and bf16 result may be from it.

    With S the exact score of a slot and A = sum_s p_s |V_s|: a score is a sum of d products in fp32, so it is off by at
    most
        delta = scale * max_s d 2^-23 sum_i |q_i K_si| + 2^-20 (1 + max |S|)
    (the last term: the scaled score and the reference in fp32, and the exponential's own error of a few 2^-22).  Every
    weight is then off by a factor of e^delta at most, in the numerator and in the sum of the weights, and those of the
    numerator by their rounding: |error| <= (4 delta + weight) A, and half a bf16 step, 2^-8, of the result.  An fp16
    weight, which stands for p_s 2^(e_s), is held to 2^-25 of the largest one at worst (below its normal range), and a
    code is at most twice the largest of its row over 2^(e_s): n 2^-24 max_s(p_s max|V_s|) more."""
    B, rows, nq, d = q.shape
    page, n_kv = kv["k_pages"].shape[2], kv["k_pages"].shape[1]
    G = nq // n_kv
    out, bound = np.zeros(q.shape), np.full(q.shape, 1e-30)      # a row that sees nothing is exactly zero
    for b in range(B):
        n = int(kv["cache_len"][b])
        pos = np.arange(n + drafted)
        if len(pos) == 0:
            continue
        pp = kv["page_table"][b].numpy()[pos // page].astype(np.int64)
        K = dequantise(kv["k_pages"][pp, :, pos % page], kv["k_scale"][pp, :, pos % page])
        V = dequantise(kv["v_pages"][pp, :, pos % page], kv["v_scale"][pp, :, pos % page])
        for j in range(rows):
            m = int(row_mask[b, j]) & (2 ** 64 - 1) if row_mask is not None else 2 ** 64 - 1
            use = np.ones(n + drafted, bool)
            use[n:] = [(m >> i) & 1 for i in range(drafted)]
            if not use.any():
                continue
            for h in range(nq):
                x = q[b, j, h].to(torch.float64).numpy()
                Kh, Vh = K[use, h // G], V[use, h // G]
                S = Kh @ x * scale
                p = np.exp(S - S.max())
                p /= p.sum()
                out[b, j, h] = p @ Vh
                A = p @ np.abs(Vh)
                delta = abs(scale) * d * 2.0 ** -23 * (np.abs(Kh) @ np.abs(x)).max() + 2.0 ** -20 * (1 + np.abs(S).max())
                far = (4 * delta + weight) * A + len(S) * 2.0 ** -24 * (p * np.abs(Vh).max(1)).max()
                bound[b, j, h] = far + 2.0 ** -8 * (np.abs(out[b, j, h]) + far) + 1e-30
    return out, bound


def make_cache(B, n_kv, d, page, lens, drafted, seed=0, groups=None, prefix=None, share_pages=True, fill=None, spare=3):
    """A filled cache in CPU tensors: pages in shuffled order, larger pool than needed; members of a group hold the same
    rows in their first ``prefix[g]`` slots.  ``fill``: byte put into every code and exponent that no slot owns."""
    g = torch.Generator().manual_seed(seed)
    M = max(1, max(-(-(n + drafted) // page) for n in lens))
    num = B * M + spare
    table = torch.randperm(num, generator=g)[:B * M].to(torch.int32).view(B, M)
    x = torch.randn(num, n_kv, page, d, generator=g) * torch.exp(torch.randn(num, n_kv, page, 1, generator=g) * 0.5)
    y = torch.randn(num, n_kv, page, d, generator=g) * torch.exp(torch.randn(num, n_kv, page, 1, generator=g))
    kv = {}
    for name, t in (("k", x), ("v", y)):
        top = t.abs().amax(-1)
        byte = (torch.frexp(top / 448.0)[1]).clamp(-64, 120)           # a scale that fits, not always the smallest
        kv[name + "_pages"] = (t * torch.exp2(-byte.float()).unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8)
        kv[name + "_scale"] = (byte + 127).to(torch.uint8)
    kv["page_table"], kv["cache_len"] = table, torch.tensor(lens, dtype=torch.int32)
    if groups is not None:
        for i, n in enumerate(prefix):
            for b in range(groups[i] + 1, groups[i + 1]):
                for lp in range(-(-n // page)):
                    a0, b0 = int(table[groups[i], lp]), int(table[b, lp])
                    if share_pages and (lp + 1) * page <= n:
                        table[b, lp] = a0
                        continue
                    cut = min(page, n - lp * page)
                    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
                        kv[name][b0, :, :cut] = kv[name][a0, :, :cut]
        kv["group_start"] = torch.tensor(groups, dtype=torch.int32)
        kv["prefix_len"] = torch.tensor(prefix, dtype=torch.int32)
    if fill is not None:
        owned = torch.zeros(num, page, dtype=torch.bool)
        for b in range(B):
            for s in range(lens[b] + drafted):
                owned[int(table[b, s // page]), s % page] = True
        for name in ("k_pages", "v_pages"):
            kv[name].permute(0, 2, 1, 3)[~owned] = fill
        for name in ("k_scale", "v_scale"):
            kv[name].permute(0, 2, 1)[~owned] = fill
    return kv


def make_q(B, rows, nq, d, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(B, rows, nq, d, generator=g) * torch.exp(torch.randn(B, rows, nq, 1, generator=g) * 0.5)).to(torch.bfloat16)


def causal_masks(B, rows, drafted):
    """Row j sees the drafted slots up to its own, which is the (drafted - rows + j)-th."""
    m = [(2 << (drafted - rows + j)) - 1 for j in range(rows)]
    return torch.tensor([[v - 2 ** 64 if v >= 2 ** 63 else v for v in m]] * B, dtype=torch.int64)


def random_masks(B, rows, drafted, seed, empty=()):
    g = torch.Generator().manual_seed(seed)
    m = torch.randint(-2 ** 63, 2 ** 63 - 1, (B, rows), generator=g, dtype=torch.int64)
    for b, j in empty:
        m[b, j] = 0
    return m
