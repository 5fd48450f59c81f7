"""8-bit linear-layer operators and gradient clipping in fp64 (numpy), from their
definitions.

An 8-bit value with ``digits`` significant binary digits is a multiple of
2^(x - digits), where 2^(x-1) <= |v| < 2^x, and of the format's least step; E4M3
has 4 digits, least step 2^-9 and maximum 448, E5M2 3 digits, 2^-16 and 57344.
A block of 128 shares the scale 2^(s - 127), s in 0 .. 254 (255: not a number).
"""
from __future__ import annotations

import numpy as np

DIGITS = {"e4m3": 4, "e5m2": 3}
LEAST = {"e4m3": -9, "e5m2": -16}
MOST = {"e4m3": 448.0, "e5m2": 57344.0}


def round8(v, fmt):
    """Nearest 8-bit value (ties to even) of each |v| <= MOST."""
    v = np.asarray(v, dtype=np.float64)
    x = np.frexp(v)[1]
    step = np.ldexp(1.0, np.maximum(x - DIGITS[fmt], LEAST[fmt]))
    return np.rint(v / step) * step


def table8(fmt):
    """The value of each of the 256 bytes (sign, exponent, fraction)."""
    out = np.zeros(256)
    f = DIGITS[fmt] - 1
    for b in range(256):
        e, m = (b & 127) >> f, b & ((1 << f) - 1)
        v = np.ldexp(1 + m / (1 << f), e - (1 << (6 - f)) + 1) if e else np.ldexp(m, LEAST[fmt])
        if fmt == "e4m3" and (b & 127) == 127:
            v = np.nan
        if fmt == "e5m2" and e == 31:
            v = np.inf if m == 0 else np.nan
        out[b] = -v if b & 128 else v
    return out


def scale_bytes(amax, fmt):
    """Least s in 0 .. 254 with amax <= MOST 2^(s - 127); 255 where amax is not finite."""
    s = np.full(np.shape(amax), 255)
    for b in range(254, -1, -1):
        s = np.where(amax <= np.ldexp(MOST[fmt], b - 127), b, s)
    return np.where(np.isfinite(amax), s, 255)


def quantize8(y, fmt, tile=1):
    """(values q [R][K], exponent bytes [R][ceil(K/128)]) of y in blocks of
    ``tile`` rows x 128 columns; q of a block with a non-finite value is NaN."""
    R, K = y.shape
    nb, nr = -(-K // 128), -(-R // tile)
    q, s = np.empty((R, K)), np.empty((R, nb), dtype=np.int64)
    for i in range(nr):
        for j in range(nb):
            blk = y[i * tile:(i + 1) * tile, j * 128:(j + 1) * 128]
            finite = np.isfinite(blk).all()
            b = int(scale_bytes(np.abs(blk).max() if finite else np.inf, fmt))
            s[i * tile:(i + 1) * tile, j] = b
            q[i * tile:(i + 1) * tile, j * 128:(j + 1) * 128] = (
                round8(np.ldexp(blk, 127 - b), fmt) if finite else np.nan)
    return q, s


def values8(q, s):
    """What q and its exponents stand for."""
    w = np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    return q * np.repeat(w, 128, axis=1)[:, :q.shape[1]]


def rmsnorm(h, gain, eps):
    """(rstd, y) of rows h."""
    rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return rstd, h * rstd[:, None] * gain


def rmsnorm_grad(dy, h, gain, eps):
    """Gradients of sum(dy * y) to h and gain."""
    rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    a, n = dy * gain, h * rstd[:, None]
    return rstd[:, None] * (a - n * (a * n).mean(axis=1, keepdims=True)), (dy * n).sum(axis=0)


def grad_norm(tensors, ord=2):
    if ord == 2:
        return float(np.sqrt(sum(float((t * t).sum()) for t in tensors)))
    return float(max([np.abs(t).max() for t in tensors if t.size], default=0.0))


def clip_factor(norm, max_norm):
    return max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
