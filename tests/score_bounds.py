"""How far log-probabilities may be off where sums are not exact, derived from the order of the sums, and that order on the CPU."""
from __future__ import annotations

import numpy as np


def softmax_bound(V: int, size: float) -> float:
    """Worst case of log p beside its logits' own errors, |log p| and |ln s| up to `size`: the bound of score_ref.check."""
    return 2.0 ** -21 + (V / 1024 + 100) * 2.0 ** -24 + 2.0 ** -22 * (1 + size)


def product_bound(K: int, chain: int, size: float) -> float:
    """Of a logit of `size` whose K products have one sign, summed in chains of `chain` products whose sums are added rounding to
    nearest.  The tensor core takes 16 products at a time and cuts its sum off: less than an ulp, 2^-23 of the running sum, a step.
    The running sum of a chain of n = chain / 16 steps grows evenly to the chain's share of the whole: 2^-23 share (n + 1) / 2 in
    all, 2^-23 size (n + 1) / 2 over the chains.  The m = K / chain sums that are added: 2^-24 size (m + 1) / 2."""
    return size * (2.0 ** -23 * (chain / 16 + 1) / 2 + 2.0 ** -24 * (K / chain + 1) / 2)


def cut(x: np.ndarray, bits: int = 24) -> np.ndarray:
    """Towards zero to `bits` significant bits."""
    m, e = np.frexp(x)
    return np.ldexp(np.trunc(m * 2.0 ** bits), e - bits)


def chained(h: np.ndarray, w: np.ndarray, chain: int, between: int = 24) -> np.ndarray:
    """h . w^T as such an accumulator forms it; `between`: the bits that a sum of chains is held to."""
    K, total = h.shape[1], np.zeros((h.shape[0], w.shape[0]))
    for c in range(0, K, chain):
        acc = np.zeros_like(total)
        for k in range(c, min(K, c + chain), 16):
            acc = cut(acc + h[:, k:k + 16] @ w[:, k:k + 16].T)
        m, e = np.frexp(total + acc)
        total = np.ldexp(np.round(m * 2.0 ** between), e - between)
    return total


def one_sign(T: int, V: int, K: int, size: float, seed: int):
    """Hidden states and a head (values of bf16, as float64) whose logits are near `size` and sums of positive products of many
    orders, but for token 0, whose logit is 0: its log p shows what all the others lost."""
    g = np.random.default_rng(seed)
    h, w = bf16(np.exp(g.standard_normal((T, K)))), bf16(np.exp(g.standard_normal((V, K)) - 1) * (size / K))
    w[0] = 0
    return h, w


def bf16(x: np.ndarray) -> np.ndarray:
    m, e = np.frexp(x)
    return np.ldexp(np.round(m * 256.0), e - 8)


def log_p(x: np.ndarray) -> np.ndarray:
    d = x - x.max(-1, keepdims=True)
    return d - np.log(np.exp(d).sum(-1, keepdims=True))


def typical_bound(V: int, lanes: int, size: float) -> float:
    """Root mean square of log p's error over rows of V bf16 logits that `lanes` lanes share, |log p| and |ln s| up to `size`: roundings
    to nearest that know nothing of one another, 2^-24 / sqrt(3) of the running sum each at most.  A lane's n = V / 32 / lanes
    groups, a sum that grows evenly: 2^-24 sqrt(n / 9).  The powers 2^-22 (what the instruction promises, though they differ);
    ln s and the result half an ulp each, 2^-23 of themselves at most."""
    return 2.0 ** -24 * np.sqrt(V / 32 / lanes / 9) + 2.0 ** -22 + 2.0 ** -23 * size


def standing_out(V: int, seed: int) -> np.ndarray:
    """A row of logits as a model makes them, a few of them far above the rest, the largest first."""
    g = np.random.default_rng(seed)
    x = g.standard_normal(V) * 2
    x[:12] = 4 + 12 * g.random(12)
    x[0] = 16
    return bf16(x).astype(np.float32)


def lane_sums(x: np.ndarray, lanes: int, by_groups: bool) -> float:
    """Sum of 2^(c (x - max)) in fp32 as the lanes form it: groups of 32 in turn, summed by themselves before they meet the running
    sum, or straight into it (two of them, even and odd elements)."""
    f = np.float32
    d = (x.astype(np.float64) - float(x.max())) * 1.4426950408889634
    e = np.exp2(d).astype(f)
    e = np.concatenate([e, np.zeros(-len(e) % (32 * lanes), f)]).reshape(-1, lanes, 32)
    total, pair = np.zeros(lanes, f), np.zeros((2, lanes), f)
    for group in e:
        for i in range(0, 32, 2):
            pair = pair + group[:, i:i + 2].T
        if by_groups:
            total, pair = total + (pair[0] + pair[1]), np.zeros((2, lanes), f)
    return float((total + (pair[0] + pair[1])).astype(np.float64).sum())
