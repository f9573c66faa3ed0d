"""Float64 oracle of the prefix-cache operators: 4-bit blocks, attention with its
log-sum-exp and weights, and the eviction of tokens."""
from __future__ import annotations

import numpy as np

GROUP = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def block_exponents(x: np.ndarray) -> np.ndarray:
    """[..., hd] -> [..., hd / 32] int: least e with max|x| <= 7 2^e, clamped to
    [-125, 125]; 128 where the block holds a NaN or an infinity."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, GROUP)
    a = np.abs(g).max(-1)
    bad = ~np.isfinite(g).all(-1)
    m, e = np.frexp(np.where(bad | (a == 0), 1.0, a) / 7.0)     # a / 7 = m 2^e, 0.5 <= m < 1
    e = np.where(m == 0.5, e - 1, e)
    # a / 7 is rounded: settle the border with exact products
    e = np.where(np.where(bad, 0, a) > 7.0 * np.exp2(e.astype(float)), e + 1, e)
    e = np.where((a > 0) & (np.where(bad, 0, a) <= 7.0 * np.exp2(e - 1.0)), e - 1, e)
    e = np.clip(np.where(a == 0, -125, e), -125, 125)
    return np.where(bad, 128, e).astype(int)


def quantize(x: np.ndarray):
    """[..., hd] -> codes [..., hd / 2] uint8, scale bytes [..., hd / 32] uint8."""
    e = block_exponents(x)
    bad = e == 128
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, GROUP)
    y = np.abs(np.where(bad[..., None], 0.0, g)) / np.exp2(np.where(bad, 0, e).astype(float))[..., None]
    d = np.abs(y[..., None] - MAGNITUDES)
    best = d.min(-1, keepdims=True)
    hit = d == best                                             # one magnitude, or two neighbours on a tie
    even = np.where(hit & (np.arange(8) % 2 == 0), True, False)
    code = np.where(even.any(-1), even.argmax(-1), hit.argmax(-1))
    code = code + 8 * (np.signbit(g) & ~bad[..., None])
    code = code.reshape(*x.shape[:-1], -1).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), np.where(bad, 255, e + 127).astype(np.uint8)


def expand(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """Codes and scale bytes -> the values they stand for."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.where(c & 8, -1.0, 1.0) * MAGNITUDES[c & 7]
    s = np.where(scales == 255, np.nan, np.exp2(np.where(scales == 255, 0, scales.astype(float) - 127)))
    return v * np.repeat(s, GROUP, axis=-1)


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray):
    """q [H, nq, hd], k and v [n, nkv, hd] -> o [H, nq, hd], lse [H, nq], weights [H, nq, n]."""
    H, nq, hd = q.shape
    G = nq // k.shape[1]
    o, lse, w = np.empty(q.shape), np.empty((H, nq)), np.empty((H, nq, k.shape[0]))
    for g in range(nq):
        s = q[:, g] @ k[:, g // G].T / np.sqrt(hd)
        m = s.max(-1, keepdims=True)
        e = np.exp(s - m)
        l = e.sum(-1, keepdims=True)
        o[:, g], lse[:, g], w[:, g] = (e @ v[:, g // G]) / l, (m + np.log(l))[:, 0], e / l
    return o, lse, w


def masses(w: np.ndarray, nkv: int, P: int) -> np.ndarray:
    """Weights [H, nq, n] -> [nkv, P], summed over tokens and the head's queries."""
    H, nq, _ = w.shape
    return w[:, :, :P].reshape(H, nkv, nq // nkv, P).sum((0, 2))


def keep_tokens(mass: np.ndarray, keep: int, first: int, last: int) -> np.ndarray:
    """Indices kept of one row of masses [P], ascending."""
    P = len(mass)
    rest = range(first, P - last)
    key = {i: (-np.inf if np.isnan(mass[i]) else mass[i], not np.isnan(mass[i])) for i in rest}
    order = sorted(rest, key=lambda i: (-key[i][0], not key[i][1], i))
    return np.array(sorted([*range(first), *order[:keep - first - last], *range(P - last, P)]), np.int32)
