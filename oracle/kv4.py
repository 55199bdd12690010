"""Plain double-precision oracle of the paged 4-bit cache: the layout walked byte by byte, quantisation, attention
row by row, read-back and commit (numpy, test infrastructure only; shares nothing with the CUDA sources)."""
from __future__ import annotations

import numpy as np

_T = {"f16": np.float16, "f32": np.float32}


def block_bytes(R: int, d: int, dtype: str) -> int:
    return R * d + 4 * R * np.dtype(_T[dtype]).itemsize


class Pool:
    """One layer's pool on the host: uint8 [n_pages][heads][block], read and written row by row."""

    def __init__(self, n_pages, heads, R, d, dtype, data=None):
        self.heads, self.R, self.d, self.T = heads, R, d, _T[dtype]
        self.es = np.dtype(self.T).itemsize
        self.data = np.zeros((n_pages, heads, block_bytes(R, d, dtype)), np.uint8) if data is None else data.reshape(n_pages, heads, -1).copy()

    def _at(self, which, r):
        half = self.R * self.d // 2
        c = which * half + r * (self.d // 2)
        p = 2 * half + which * 2 * self.es * self.R + r * 2 * self.es
        return c, p

    def put(self, which, page, r, head, codes, scale, mn):
        c, p = self._at(which, r)
        self.data[page, head, c:c + self.d // 2] = codes[0::2] | (codes[1::2] << 4)
        self.data[page, head, p:p + 2 * self.es] = np.array([scale, mn], self.T).view(np.uint8)

    def params(self, which, page, r, head):
        _, p = self._at(which, r)
        return self.data[page, head, p:p + 2 * self.es].copy().view(self.T)

    def codes(self, which, page, r, head):
        c, _ = self._at(which, r)
        b = self.data[page, head, c:c + self.d // 2]
        out = np.empty(self.d, np.uint8)
        out[0::2], out[1::2] = b & 15, b >> 4
        return out

    def value(self, which, page, r, head):
        s, m = self.params(which, page, r, head).astype(np.float64)
        return m + s * self.codes(which, page, r, head).astype(np.float64)


def rotate(x, pos, theta):
    """x [heads][d] in float64 -> rotated (pairs t, t + d / 2)."""
    d = x.shape[-1]
    ang = float(pos) * theta ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(ang), np.sin(ang)
    a, b = x[..., : d // 2], x[..., d // 2:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def quantise(x, dtype):
    """float32 [d] -> (codes, scale, min); the quotient in float64."""
    T = _T[dtype]
    with np.errstate(all="ignore"):
        x = np.asarray(x, np.float32)
        lo, hi = np.min(x), np.max(x)                       # both keep a NaN
        mn, scale = T(lo), T(np.float32((np.float64(hi) - np.float64(lo)) / 15.0))
        if scale == 0:
            return np.zeros(x.size, np.uint8), scale, mn
        c = np.rint((x.astype(np.float64) - np.float64(mn)) / np.float64(scale))
        return np.clip(np.nan_to_num(c, nan=0.0, posinf=15, neginf=0), 0, 15).astype(np.uint8), scale, mn


def slots(table, R, s, t):
    return int(table[s][t // R]), t % R


def append(pool: Pool, table, kv_len, row_start, pos, q, k, v, theta):
    """q [n][H][d], k, v [n][heads][d] (storage type) -> rotated q in float64; the pool's rows are written."""
    q_out = np.zeros(q.shape, np.float64)
    dtype = "f16" if pool.T == np.float16 else "f32"
    for s in range(len(row_start) - 1):
        for i, r in enumerate(range(row_start[s], row_start[s + 1])):
            t = int(kv_len[s]) + i
            p = t if pos is None else int(pos[r])
            q_out[r] = rotate(q[r].astype(np.float64), p, theta)
            kr = rotate(k[r].astype(np.float64), p, theta).astype(np.float32)
            page, row = slots(table, pool.R, s, t)
            for h in range(pool.heads):
                pool.put(0, page, row, h, *quantise(kr[h], dtype))
                pool.put(1, page, row, h, *quantise(v[r][h], dtype))
    return q_out


def rows(pool: Pool, table, s, first, count):
    """-> K, V float64 [count][heads][d] of a sequence's cache rows."""
    out = np.zeros((2, count, pool.heads, pool.d))
    for i in range(count):
        page, row = slots(table, pool.R, s, first + i)
        for w in (0, 1):
            for h in range(pool.heads):
                out[w, i, h] = pool.value(w, page, row, h)
    return out[0], out[1]


def attention(pool: Pool, table, kv_len, row_start, visible, q):
    """q [n][H][d] (rotated); visible[s] bool [n_s][n_s] -> float64 [n][H][d]; a row that sees nothing gives zeros."""
    n, H, d = q.shape
    out = np.zeros((n, H, d))
    g = H // pool.heads
    for s in range(len(row_start) - 1):
        a, b = int(row_start[s]), int(row_start[s + 1])
        if a == b:
            continue
        K, V = rows(pool, table, s, 0, int(kv_len[s]) + b - a)
        for i in range(b - a):
            see = np.concatenate([np.ones(int(kv_len[s]), bool), np.asarray(visible[s])[i, :] & (np.arange(b - a) <= i)])
            if not see.any():
                continue
            for h in range(H):
                w = K[see, h // g] @ q[a + i, h].astype(np.float64) / np.sqrt(d)
                w = np.exp(w - w.max())
                out[a + i, h] = (w @ V[see, h // g]) / w.sum()
    return out


def commit(pools, table, kv_len, row_start, results):
    """results[s] = (n_matched, nodes) or None for 'keep all' -> new lengths; the pools' rows move."""
    new = []
    for s in range(len(row_start) - 1):
        n, L = int(row_start[s + 1] - row_start[s]), int(kv_len[s])
        if n == 0:
            new.append(L)
            continue
        if results is None:
            new.append(L + n)
            continue
        m, nodes = results[s]
        for pool in pools:
            for j in range(1, m + 1):
                pf, rf = slots(table, pool.R, s, L + int(nodes[j]))
                pt, rt = slots(table, pool.R, s, L + j)
                for w in (0, 1):
                    for h in range(pool.heads):
                        c, p = pool.codes(w, pf, rf, h), pool.params(w, pf, rf, h)
                        pool.put(w, pt, rt, h, c, p[0], p[1])
        new.append(L + m + 1)
    return new
