"""Plain fp64 CPU oracle of the training operators: the 8-bit block format,
LayerNorm with its gradient, GELU's gradient, and the products of 8-bit tensors.
Written from the formulas; shares no code with the kernels."""
import math

import numpy as np

BLOCK = 128


def e4m3_decode(q):
    """Values of E4M3 bytes: sign, four exponent bits (bias 7), three of mantissa; 0x7F is NaN."""
    q = np.asarray(q, np.uint8).astype(np.int64)
    e, m = (q >> 3) & 15, (q & 7).astype(np.float64)
    v = np.where(e == 0, m * 2.0 ** -9, (1.0 + m / 8.0) * np.exp2(e - 7.0))
    v = np.where((q & 0x7F) == 0x7F, np.nan, v)
    return np.where(q >> 7, -v, v)


def e4m3_encode(x):
    """Nearest E4M3 bytes (ties to even) of values up to 448; NaN to 0x7F."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isnan(x), 0.0, np.abs(x))
    assert (a <= 448.0).all()
    _, ex = np.frexp(np.maximum(a, 2.0 ** -6))
    step = np.ldexp(1.0, ex - 4)
    r = np.rint(a / step) * step  # rint: ties to even
    _, ex = np.frexp(np.maximum(r, 2.0 ** -6))
    step = np.ldexp(1.0, ex - 4)
    mant = np.rint(r / step).astype(np.int64)  # 0..7 below 2^-6, 8..15 above
    q = np.where(r < 2.0 ** -6, mant, ((ex - 1 + 7) << 3) + (mant - 8))
    q = np.where(np.isnan(x), 0x7F, q)
    return (q | (np.signbit(x) & ~np.isnan(x)) << 7).astype(np.uint8)


def exponent(amax):
    """The smallest e >= -126 with amax <= 448 2^e."""
    m, ex = np.frexp(np.asarray(amax, np.float64))  # amax = m 2^ex, 448 = 0.875 2^9
    e = np.where(amax > 0, ex - 9 + (m > 0.875), -126)
    return np.maximum(e, -126).astype(np.int64)


def _finite_max(a, axis):
    return np.where(np.isfinite(a), np.abs(a), 0.0).max(axis=axis)


def pack(x):
    """x [rows, cols] -> (bytes [rows, cols], scale bytes [blocks, rows])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    q = np.zeros((rows, cols), np.uint8)
    scale = np.zeros((nb, rows), np.uint8)
    for b in range(nb):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        e = exponent(_finite_max(part, 1))
        scale[b] = e + 127
        part = np.where(np.isfinite(part), part, np.nan)
        q[:, b * BLOCK:(b + 1) * BLOCK] = e4m3_encode(part * np.exp2(-e.astype(np.float64))[:, None])
    return q, scale


def unpack(q, scale):
    cols = q.shape[1]
    s = np.exp2(scale.astype(np.float64) - 127.0)
    return e4m3_decode(q) * s[np.arange(cols) // BLOCK].T


def pack_weight(w):
    """w [N, K] -> (bytes [N, K], scale bytes [blocks of K, blocks of N])."""
    w = np.asarray(w, np.float64)
    N, K = w.shape
    q = np.zeros((N, K), np.uint8)
    scale = np.zeros((-(-K // BLOCK), -(-N // BLOCK)), np.uint8)
    for i in range(scale.shape[1]):
        for j in range(scale.shape[0]):
            at = np.s_[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK]
            e = exponent(_finite_max(w[at], (0, 1)))
            scale[j, i] = e + 127
            q[at] = e4m3_encode(np.where(np.isfinite(w[at]), w[at], np.nan) * 2.0 ** -float(e))
    return q, scale


def unpack_weight(q, scale):
    N, K = q.shape
    s = np.exp2(scale.astype(np.float64) - 127.0)
    return e4m3_decode(q) * s[np.arange(K) // BLOCK][:, np.arange(N) // BLOCK].T


def layernorm(x, g, b, eps):
    """(y, mean, rstd); g and b may be None."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if g is not None:
        y = y * g
    return (y if b is None else y + b), mean, rstd


def layernorm_grad(dy, x, mean, rstd, g):
    """(dx, dg, db) with the given statistics."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    xh = (x - mean[:, None]) * rstd[:, None]
    a = dy if g is None else dy * g
    dx = rstd[:, None] * (a - a.mean(1, keepdims=True) - xh * (a * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def _erfc(x):
    return np.vectorize(math.erfc, otypes=[np.float64])(x)


def gelu(x):
    x = np.asarray(x, np.float64)
    return 0.5 * x * _erfc(-x / math.sqrt(2.0))


def gelu_grad(x):
    x = np.asarray(x, np.float64)
    return 0.5 * _erfc(-x / math.sqrt(2.0)) + x * np.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)
