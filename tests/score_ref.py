"""Log-probabilities, entropy and alternatives of rows of logits in 64 bits on the CPU, from the definitions."""
from __future__ import annotations

import numpy as np
import torch


def scores(logits: torch.Tensor, tokens, top: int, temperature: float = 1.0):
    """dict of numpy arrays; what the header says of -inf, NaN, +inf, tokens of -1 and missing alternatives included."""
    x = logits.to(torch.float64).cpu().numpy()
    T, V = x.shape
    tok = np.zeros((T, 0), np.int64) if tokens is None else tokens.cpu().numpy().reshape(T, -1)
    out = dict(logp=np.zeros(tok.shape), entropy=np.zeros(T), top_tok=np.full((T, top), -1), top_logp=np.full((T, top), -np.inf))
    for r in range(T):
        y = x[r] / temperature
        if np.isnan(y).any() or (y == np.inf).any():
            out["entropy"][r], out["top_logp"][r] = np.nan, np.nan
            out["logp"][r] = np.where(tok[r] == -1, 0.0, np.nan)
            continue
        m = y.max()
        if m == -np.inf:
            out["logp"][r] = np.where(tok[r] == -1, 0.0, -np.inf)
            continue
        lp = (y - m) - np.log(np.exp(y - m).sum())             # the difference first: m may be a type's lowest value
        p = np.exp(lp)
        out["entropy"][r] = -(p[p > 0] * lp[p > 0]).sum()
        for i, t in enumerate(tok[r]):
            out["logp"][r, i] = 0.0 if t == -1 else lp[t] if 0 <= t < V else np.nan
        order = np.argsort(-x[r], kind="stable")[:top]
        order = order[x[r][order] > -np.inf]
        out["top_tok"][r, :len(order)], out["top_logp"][r, :len(order)] = order, lp[order]
    if top == 0:
        del out["top_tok"], out["top_logp"]
    return out


def check(got, want, logits, temperature: float = 1.0, more: float = 0.0):
    """Ids equal, values within the bound.

The difference of a logit and the row's largest is rounded once, its product with c = log2(e) / temperature twice (c itself is
    off by 2^-24): d is off by 3 2^-24 |d|, a power that counts (d > -40) by 2^-22 + 120 2^-24 of itself at most and a mean one
    by far less; a sum of n powers by n 2^-24 more at worst: a lane adds its groups' sums, of 32 at most each and n / 1024 of them at
    most, and some 20 joins follow.  ln s is then off by D = 2^-21 + (n / 1024 + 100) 2^-24, and so is t / s by D (2 + log2 n) + 20 D at most, t being
    a mean of |d| weighted by powers that sum to s (|d| above 40 does not count).  log p: D, the roundings of the difference, of its
    product and of the result, 2^-22 of their size.  `more`: what the logits themselves are off by."""
    x = logits.to(torch.float64).cpu().numpy() / temperature
    V = x.shape[1]
    D = 2.0 ** -21 + (V / 1024 + 100) * 2.0 ** -24
    for name in want:
        g = got[name].cpu().numpy()
        w = want[name]
        if name == "top_tok":
            assert (g == w).all(), np.argwhere(g != w)[:5]
            continue
        w = np.where(np.abs(w) > float(np.finfo(np.float32).max), np.copysign(np.inf, w), w)       # results are fp32
        assert (np.isnan(g) == np.isnan(w)).all() and (np.isinf(g) == np.isinf(w)).all(), name
        ok = np.isfinite(w)
        if name == "entropy":
            far = D * (22 + np.log2(V + 1)) + 2.0 ** -23 * np.abs(w) + 2 * more
        else:
            far = D + 2.0 ** -22 * (1 + np.abs(w)) + 2 * more
        off = np.abs(g[ok] - w[ok])
        assert (off <= np.broadcast_to(far, w.shape)[ok]).all(), (name, off.max())
