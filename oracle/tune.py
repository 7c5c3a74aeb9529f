"""fp64 forms of the layer norms, adapters and AdamW steps, from their definitions
(test infrastructure; shares no code with the library).

Arrays are numpy fp64 values (already rounded to the storage type), but for
``adamw_moments`` and ``e4m3_round``, which follow the definition in fp32 step by
step.
"""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ layer norm
def layer_norm(x, gain, bias, eps, r=None):
    """(H, Y)."""
    h = x if r is None else x + r
    c = h - h.mean(axis=1, keepdims=True)
    y = c / np.sqrt((c * c).mean(axis=1, keepdims=True) + eps)
    y = y if gain is None else y * gain
    return h, y if bias is None else y + bias


def layer_norm_backward(h, gain, dy, eps, dr=None):
    """(dX, dgain, dbias)."""
    c = h - h.mean(axis=1, keepdims=True)
    rho = 1.0 / np.sqrt((c * c).mean(axis=1, keepdims=True) + eps)
    hat = c * rho
    u = dy if gain is None else dy * gain
    dx = rho * (u - u.mean(axis=1, keepdims=True) - hat * (u * hat).mean(axis=1, keepdims=True))
    return (dx if dr is None else dx + dr), (dy * hat).sum(axis=0), dy.sum(axis=0)


# ------------------------------------------------------------------ adapters
def adapter_rows(ids, n):
    """(adapter, its rows) of every adapter that has some."""
    return [(a, np.flatnonzero(np.asarray(ids) == a)) for a in range(n) if (np.asarray(ids) == a).any()]


def adapter_forward(x, A, B, ids, scale=None, y0=None):
    y = np.zeros((x.shape[0], B.shape[1])) if y0 is None else np.array(y0)
    for a, rows in adapter_rows(ids, A.shape[0]):
        s = 1.0 if scale is None else scale[a]
        y[rows] += s * (x[rows] @ A[a].T) @ B[a].T
    return y


def adapter_backward(x, A, B, ids, dy, scale=None, dx0=None):
    """(dX, dA, dB)."""
    dx = np.zeros_like(x) if dx0 is None else np.array(dx0)
    dA, dB = np.zeros_like(A), np.zeros_like(B)
    for a, rows in adapter_rows(ids, A.shape[0]):
        s = 1.0 if scale is None else scale[a]
        u = s * dy[rows] @ B[a]
        dx[rows] += u @ A[a]
        dA[a] = u.T @ x[rows]
        dB[a] = s * dy[rows].T @ (x[rows] @ A[a].T)
    return dx, dA, dB


# ------------------------------------------------------------------ AdamW
def adamw(p, g, m, v, t, lr, b1, b2, eps, decay=0.0, grad_scale=1.0):
    """(p, m, v) after step t."""
    g = g * grad_scale
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p * (1 - lr * decay) - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps), m, v


def adamw_moments(g, m, v, b1, b2, grad_scale=None):
    """(m, v) in fp32, each operation rounded by itself."""
    f = np.float32
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        g = f(g) if grad_scale is None else f(g) * f(grad_scale)
        return f(m) * f(b1) + g * f(1 - b1), f(v) * f(b2) + (g * g) * f(1 - b2)


def mix(x):
    """The 32-bit hash."""
    x = np.asarray(x, np.uint64) & np.uint64(0xFFFFFFFF)
    low = np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667)) & low
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85)) & low
    return x ^ (x >> np.uint64(16))


def random_bits(seed, t, tensor, n):
    """(bits of m, bits of v) of a tensor's n values, 16 each."""
    i = np.arange(n, dtype=np.uint64)
    u = lambda k: np.uint64(int(k) & 0xFFFFFFFF)
    key = mix(mix(mix(mix(u(seed)) + u(t)) + u(tensor)) + (i >> np.uint64(12)))
    b = mix(key + (i & np.uint64(4095)))
    return (b >> np.uint64(16)).astype(np.int64), (b & np.uint64(0xFFFF)).astype(np.int64)


# magnitudes of the e4m3 codes 0 to 126, in units of the smallest
E4M3_UNITS = np.array([c if c < 8 else (8 + c % 8) << (c // 8 - 1) for c in range(127)], np.float64)


def e4m3_round(x, bits, smallest):
    """(codes, scale bytes) of fp32 values in groups of 32, rounded to a neighbour by
    their bits; `smallest`: the code that a value above zero has at least."""
    n = x.size
    pad = -n % 32
    x = np.concatenate([np.float32(x).ravel(), np.zeros(pad, np.float32)])
    bits = np.concatenate([bits, np.zeros(pad, np.int64)])
    g = np.abs(x).reshape(-1, 32).astype(np.float64)
    bad = ~np.isfinite(g).all(axis=1)
    top = np.where(bad, 0.0, np.where(np.isfinite(g), g, 0.0).max(axis=1))
    k = np.full(top.shape, -126)
    some = top > 0
    k[some] = np.maximum(-126, np.ceil(np.log2(top[some] / 448.0)).astype(int))
    k += (top > 448.0 * 2.0 ** k).astype(int)  # where the logarithm was rounded
    k -= ((k > -126) & (top <= 448.0 * 2.0 ** (k - 1))).astype(int)
    a = np.where(bad[:, None], 0.0, g * 2.0 ** (9.0 - k)[:, None]).ravel()  # exact: powers of two
    code = np.searchsorted(E4M3_UNITS, a, side="right") - 1
    low = E4M3_UNITS[code]
    step = np.where(code < 126, E4M3_UNITS[np.minimum(code + 1, 126)] - low, 32.0 * 512)
    rest = (a - low) / step
    code = code + (rest * 65536 + bits >= 65535.5)  # exact: 24 bits of rest, 16 of bits
    code = np.where(a > 0, np.maximum(code, smallest), code)
    code = code | np.where(x < 0, 128, 0)
    code = np.where(np.repeat(bad, 32), 127, code)
    return code[:n].astype(np.uint8), np.where(bad, 255, k + 127).astype(np.uint8)


def e4m3_values(codes, scales):
    """fp32 values of codes in groups of 32."""
    c = np.asarray(codes, np.int64)
    v = np.where(c & 127 == 127, np.nan, E4M3_UNITS[np.minimum(c & 127, 126)] / 512)
    s = np.asarray(scales, np.float64)
    s = np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return np.float32(np.where(c & 128, -v, v) * np.repeat(s, 32)[:c.size])
