"""Plain 64-bit implementations of the operators of include/spec_ops.h, written from their definitions, for the tests."""
import numpy as np

BLOCK = 128
LEAST = np.float32(2.0 ** -96)


def blocks(n):
    return (n + BLOCK - 1) // BLOCK


def e4m3(v):
    """Nearest e4m3 value, ties to even, of float64 values; NaN stays NaN.  |v| up to 448 and half a step."""
    a = np.abs(v)
    _, e = np.frexp(np.where((a > 0) & np.isfinite(a), a, 1.0))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.round(v / step) * step


def e4m3_values():
    """The value of every e4m3 byte."""
    b = np.arange(256)
    s, e, f = np.where(b & 128, -1.0, 1.0), (b >> 3) & 15, b & 7
    v = s * np.where(e == 0, f * 2.0 ** -9, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    v[[127, 255]] = np.nan
    return v


def quantise(x):
    """x float32 [R][K] -> q float64 values [R][K], scale float32 [blocks][R]; every step rounded as the definition says."""
    R, K = x.shape
    q = np.zeros((R, K))
    scale = np.zeros((blocks(K), R), dtype=np.float32)
    with np.errstate(all="ignore"):
        for b in range(blocks(K)):
            part = x[:, b * BLOCK: (b + 1) * BLOCK].astype(np.float32)
            a = np.maximum(np.fmax.reduce(np.abs(part), axis=1), LEAST).astype(np.float32)
            a = np.where(np.isnan(a), LEAST, a).astype(np.float32)  # a block of NaN only
            f = (np.float32(448.0) / a).astype(np.float32)
            q[:, b * BLOCK: (b + 1) * BLOCK] = e4m3((part * f[:, None]).astype(np.float32).astype(np.float64))
            scale[b] = (a / np.float32(448.0)).astype(np.float32)
    return q, scale


def product(q, x_scale, w, w_scale):
    """(y, sum of magnitudes): q, w float64 values; x_scale [blocks of K][R], w_scale [blocks of N][blocks of K]."""
    R, K = q.shape
    N = w.shape[0]
    y, mag = np.zeros((R, N)), np.zeros((R, N))
    for b in range(blocks(K)):
        s = slice(b * BLOCK, (b + 1) * BLOCK)
        sc = x_scale[b].astype(np.float64)[:, None] * np.repeat(w_scale[:, b].astype(np.float64), BLOCK)[None, :N]
        y += (q[:, s] @ w[:, s].T) * sc
        mag += (np.abs(q[:, s]) @ np.abs(w[:, s]).T) * np.abs(sc)
    return y, mag


def norm_rope(h, g, eps, cos, sin):
    """(result, magnitude of its two terms): h float64 [R][heads][hd]; cos, sin [R][hd / 2]."""
    half = h.shape[2] // 2
    h = h / np.sqrt(np.mean(h * h, axis=2, keepdims=True) + eps) * g
    a, b = h[..., :half], h[..., half:]
    c, s = cos[:, None, :], sin[:, None, :]
    out = np.concatenate([a * c - b * s, b * c + a * s], axis=2)
    return out, np.concatenate([np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)], axis=2)
