"""Attention with windows and first tokens, and the 4-bit cache, from their
definitions in plain NumPy (float64 where nothing says otherwise)."""
from __future__ import annotations

import numpy as np

LIMIT = 16384.0
NIBBLE = [(e >> 1) + 4 * (e & 1) for e in range(8)]  # nibble of a word's element e


def quantise(x):
    """float32 [..., D] to (nibbles [..., D], s, b [..., D / 32] float16),
    each step rounded to float32 as the format says."""
    g = np.asarray(x, np.float32).reshape(*x.shape[:-1], -1, 32)
    odd = ~np.isfinite(g).all(-1)
    c = np.clip(np.where(odd[..., None], np.float32(0), g), np.float32(-LIMIT), np.float32(LIMIT))
    lo, hi = c.min(-1), c.max(-1)
    s = ((hi - lo) / np.float32(15)).astype(np.float16)
    s = np.where(odd, np.float16(0), s)
    b = (lo - np.float32(16) * s.astype(np.float32)).astype(np.float16)
    b = np.where(odd, np.float16("nan"), b)
    s32, b32 = s.astype(np.float32)[..., None], b.astype(np.float32)[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        t = np.rint((c - b32) / s32) - 16
    n = np.where(s32 > 0, np.clip(t, 0, 15), 0).astype(np.int64)
    return n.reshape(x.shape), s, b


def values(n, s, b):
    """What nibbles stand for: f16(b + s (16 + n)), rounded once (the sum is
    exact in float64), as float64."""
    s, b = (np.repeat(t.astype(np.float64), 32, -1) for t in (s, b))
    return (b + s * (16.0 + n)).astype(np.float16).astype(np.float64)


class Cache:
    """The pool as bytes, written and read one token at a time."""

    def __init__(self, pool, page_tokens, head_dim):
        self.pool, self.P, self.D, self.G = pool, page_tokens, head_dim, head_dim // 32
        P, D, G = self.P, self.D, self.G
        self.at = np.cumsum([0, P * D // 2, P * G * 4, P * D // 2])

    def _block(self, page, h):
        return self.pool[page, h]

    def write(self, page, h, slot, k, v):
        blk, P, D, G = self._block(page, h), self.P, self.D, self.G
        n, s, b = quantise(k)
        for j in range(G):
            for o in range(4):
                w = sum(int(n[32 * j + 8 * o + e]) << (4 * NIBBLE[e]) for e in range(8))
                i = self.at[0] + slot * (D // 2) + 4 * (o * G + j)
                blk[i:i + 4] = np.frombuffer(np.uint32(w).tobytes(), np.uint8)
            i = self.at[1] + 4 * (slot * G + j)
            blk[i:i + 4] = np.frombuffer(s[j].tobytes() + b[j].tobytes(), np.uint8)
        n, s, b = quantise(v)
        octet, e = divmod(slot, 8)
        for d in range(D):
            i = self.at[2] + 4 * (octet * D + d) + NIBBLE[e] // 2
            hi = NIBBLE[e] & 1
            blk[i] = (int(blk[i]) & (0x0F if hi else 0xF0)) | (int(n[d]) << (4 * hi))
        for j in range(G):
            for part, t in ((0, s), (1, b)):
                i = self.at[3] + 2 * ((octet * G + j) * 16 + 8 * part + e)
                blk[i:i + 2] = np.frombuffer(t[j].tobytes(), np.uint8)

    def read(self, page, h, slot):
        """(k, v) of one token, float64 [D]."""
        blk, D, G = self._block(page, h), self.D, self.G
        out = []
        n = np.zeros(D, np.int64)
        for d in range(D):
            j, o, e = d // 32, (d % 32) // 8, d % 8
            i = self.at[0] + slot * (D // 2) + 4 * (o * G + j) + NIBBLE[e] // 2
            n[d] = (int(blk[i]) >> (4 * (NIBBLE[e] & 1))) & 15
        pair = blk[self.at[1] + 4 * slot * G:self.at[1] + 4 * (slot + 1) * G].copy().view(np.float16).reshape(G, 2)
        out.append(values(n, pair[:, 0], pair[:, 1]))
        octet, e = divmod(slot, 8)
        for d in range(D):
            i = self.at[2] + 4 * (octet * D + d) + NIBBLE[e] // 2
            n[d] = (int(blk[i]) >> (4 * (NIBBLE[e] & 1))) & 15
        pair = blk[self.at[3] + 32 * octet * G:self.at[3] + 32 * (octet + 1) * G].copy().view(np.float16).reshape(G, 2, 8)
        out.append(values(n, pair[:, 0, e], pair[:, 1, e]))
        return out


def sees(p, j, n, causal, window, sinks):
    """Whether the query at position p sees token j of n."""
    if not 0 <= j < n or (causal and j > p):
        return False
    return window == 0 or abs(p - j) < window or j < sinks


def attention(q, k, v, scale, causal=True, window=0, sinks=0):
    """q [T, D] at the last T positions of k, v [N, D], one head.  Returns the
    rows, what bounds their rounding error (sum of p |v| per element) and the
    largest sum of |q k| scale a row sees."""
    T, N = len(q), len(k)
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    out, mass, size = np.zeros((T, v.shape[1])), np.zeros((T, v.shape[1])), np.zeros(T)
    j = np.arange(N)
    for i in range(T):
        p = N - T + i
        see = np.ones(N, bool)
        if causal:
            see &= j <= p
        if window:
            see &= (np.abs(p - j) < window) | (j < sinks)
        if not see.any():
            continue
        x = k[see] @ q[i] * scale
        with np.errstate(invalid="ignore"):
            e = np.exp(x - x.max())
        e /= e.sum()
        out[i] = e @ v[see]
        mass[i] = e @ np.abs(v[see])
        size[i] = (np.abs(k[see]) @ np.abs(q[i])).max() * scale
    return out, mass, size
