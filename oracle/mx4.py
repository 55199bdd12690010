"""Double-precision oracle of matrices in microscaled 4-bit floating point (host, numpy)."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def up(x):
    return -(-x // 128) * 128


def code_bytes(m, k):
    return up(m) * up(k) // 2


def scale_bytes(m, k):
    return up(m) * up(k) // 32


def code_place(m, k, r, c):
    """(byte, shift) of element (r, c)'s code."""
    tile = (r // 128) * (up(k) // 128) + c // 128
    return tile * 8192 + (r % 128) * 64 + (c % 128) // 2, 4 * (c % 2)


def scale_place(m, k, r, c):
    tile = (r // 128) * (up(k) // 128) + c // 128
    return tile * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + (c % 128) // 32


def quantise_block(x):
    """32 values -> (codes, scale byte)."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return np.zeros(len(x), np.uint8), 255
    top = np.abs(x).max()
    if top == 0:
        E = -127
    else:
        E = max(-127, int(np.frexp(top)[1]) - 1 - 2)
    y = np.abs(np.ldexp(x, -E))
    d = np.abs(y[:, None] - LEVELS[None, :])
    best = d.min(1, keepdims=True)
    codes = np.zeros(len(x), np.uint8)
    for i in range(len(x)):
        near = np.flatnonzero(d[i] == best[i])
        codes[i] = near[0] if len(near) == 1 else [c for c in near if c % 2 == 0][0]
    return codes | (np.signbit(x).astype(np.uint8) << 3), E + 127


def quantise(x):
    """[m][k] -> (codes uint8, scales uint8), flat, as the layout has them."""
    m, k = x.shape
    full = np.zeros((up(m), up(k)))
    full[:m, :k] = x
    codes = np.zeros(code_bytes(m, k), np.uint8)
    scales = np.zeros(scale_bytes(m, k), np.uint8)
    for r in range(m):
        for b in range(0, up(k), 32):
            c, s = quantise_block(full[r, b:b + 32])
            scales[scale_place(m, k, r, b)] = s
            for i in range(32):
                at, shift = code_place(m, k, r, b + i)
                codes[at] |= c[i] << shift
    return codes, scales


def values(codes, scales, m, k):
    """The matrix that codes and scales stand for, in 64 bits."""
    r, c = np.arange(m)[:, None], np.arange(k)[None, :]
    tile = (r // 128) * (up(k) // 128) + c // 128
    byte = codes.reshape(-1)[tile * 8192 + (r % 128) * 64 + (c % 128) // 2]
    code = np.where(c % 2 == 1, byte >> 4, byte & 15)
    s = scales.reshape(-1)[tile * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + (c % 128) // 32].astype(np.int64)
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    return np.where(s == 255, np.nan, np.ldexp(v, s - 127))


def product(x, codes, scales, m, k):
    return np.asarray(x, np.float64) @ values(codes, scales, m, k).T
