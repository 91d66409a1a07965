"""Rotary positions, 4-bit matrices and linear attention from their
definitions in plain NumPy: float64, or more where a comment says so."""
from __future__ import annotations

import numpy as np

LIMIT = 16384.0
NIBBLE = [(e >> 1) + 4 * (e & 1) for e in range(8)]  # nibble of a word's element e


# ------------------------------------------------------------------ rotary
def frequencies(dim, base=10000.0, scaling="none", factor=1.0, length=0.0, low=1.0, high=32.0):
    """Angles a token of the dim / 2 pairs, in numpy's longest float (64 bits of
    mantissa here: positions of 2^31 leave 2^-33 of an angle)."""
    f = np.longdouble
    base, factor = f(base), f(factor)
    if scaling == "base":
        base = base * factor ** (f(dim) / f(dim - 2))
    out = np.array([base ** (f(-2 * i) / f(dim)) for i in range(dim // 2)], np.longdouble)
    if scaling == "linear":
        out = out / factor
    if scaling == "ramp":
        turns = f(length) * out / (2 * PI)
        kept = np.clip((turns - f(low)) / (f(high) - f(low)), f(0), f(1))
        out = kept * out + (1 - kept) * out / factor
    return out


PI = np.longdouble("3.14159265358979323846264338327950288")


def rotate(x, positions, theta, interleaved=False, amplitude=1.0, inverse=False):
    """x [T, heads, head_dim] at positions [T]."""
    y = np.array(x, np.float64)
    d = 2 * len(theta)
    turn = np.outer(np.asarray(positions, np.int64).astype(np.longdouble), theta) / (2 * PI)
    angle = ((turn - np.rint(turn)) * (2 * PI)).astype(np.float64)[:, None] * (-1 if inverse else 1)
    c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
    a, b = (np.s_[..., 0:d:2], np.s_[..., 1:d:2]) if interleaved else (np.s_[..., :d // 2], np.s_[..., d // 2:d])
    x = np.asarray(x, np.float64)
    y[a], y[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return y


# ---------------------------------------------------------- 4-bit matrices
def quantise(w, group):
    """float32 [N, K] to levels [N, K] and s, b [N, ceil(K / group)] float16,
    each step rounded to float32 as the format says."""
    w = np.asarray(w, np.float32)
    N, K = w.shape
    n = np.zeros((N, K), np.int64)
    s, b = (np.zeros((N, -(-K // group)), np.float16) for _ in range(2))
    for g in range(s.shape[1]):
        x = w[:, g * group:(g + 1) * group]
        odd = ~np.isfinite(x).all(1)
        c = np.clip(np.where(odd[:, None], np.float32(0), x), np.float32(-LIMIT), np.float32(LIMIT))
        lo, hi = c.min(1), c.max(1)
        sg = ((hi - lo) / np.float32(15)).astype(np.float16)
        bg = (lo - np.float32(16) * sg.astype(np.float32)).astype(np.float16)
        s[:, g], b[:, g] = np.where(odd, np.float16(0), sg), np.where(odd, np.float16("nan"), bg)
        s32, b32 = s[:, g].astype(np.float32)[:, None], b[:, g].astype(np.float32)[:, None]
        with np.errstate(divide="ignore", invalid="ignore"):
            t = np.rint((c - b32) / s32) - 16
        n[:, g * group:(g + 1) * group] = np.where(s32 > 0, np.clip(t, 0, 15), 0)
    return n, s, b


def pack(n, s, b, group):
    """The format's bytes."""
    N, K = n.shape
    tiles, blocks = -(-N // 16), -(-K // 128)
    words = np.zeros((tiles, blocks, 64, 4), np.uint32)
    pairs = np.zeros((tiles, blocks, 16, 128 // group, 2), np.float16)
    for row in range(N):
        for ch in range(K):
            inside, e = ch % 128, ch % 8
            words[row // 16, ch // 128, 16 * ((inside % 32) // 8) + row % 16, inside // 32] |= np.uint32(
                int(n[row, ch]) << (4 * NIBBLE[e]))
        for g in range(s.shape[1]):
            at = g * group
            pairs[row // 16, at // 128, row % 16, at % 128 // group] = s[row, g], b[row, g]
    return np.concatenate([words.reshape(-1).view(np.uint8), pairs.reshape(-1).view(np.uint8)])


def values(n, s, b, group):
    """b + s (16 + n), exact in float64."""
    K = n.shape[1]
    s, b = (np.repeat(t.astype(np.float64), group, 1)[:, :K] for t in (s, b))
    return b + s * (16.0 + n)


def product(x, n, s, b, group):
    """x [M, K] times the matrix, and what bounds its rounding error: the sum of
    the sizes of what is added, (31 |s| + |b|) |x|."""
    x = np.asarray(x, np.float64)
    K = n.shape[1]
    size = np.repeat(31 * np.abs(s.astype(np.float64)) + np.abs(b.astype(np.float64)), group, 1)[:, :K]
    return x @ values(n, s, b, group).T, np.abs(x) @ size.T


# -------------------------------------------------------- linear attention
def linear_attention(q, k, v, g, state, scale):
    """q [T, group, D], k, v [T, D], g [T] of one kv head from state [D, D] on.
    Returns rows, the last state, and what bounds the rounding errors of both:
    the same sums of sizes."""
    T, G, D = q.shape
    S, M = np.array(state, np.float64), np.abs(np.array(state, np.float64))
    out, size = np.zeros((T, G, v.shape[1])), np.zeros((T, G, v.shape[1]))
    for t in range(T):
        keep = np.exp(max(float(g[t]), -200.0))
        S = keep * S + np.outer(k[t], v[t])
        M = keep * M + np.outer(np.abs(k[t]), np.abs(v[t]))
        out[t] = scale * (q[t] @ S)
        size[t] = abs(scale) * (np.abs(q[t]) @ M)
    return out, S, size, M
