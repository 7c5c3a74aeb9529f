"""fp64 forms of the norms and 4-bit layers, from their definitions (test
infrastructure; shares no code with the library).

Rows are numpy arrays of fp64 values (already rounded to the storage type).
"""
from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0
TINY = 2.0 ** -126
GROUP = 32
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rho(h, eps):
    """1 / the root mean square of each row (with eps under the root)."""
    return 1.0 / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)


def rms_norm(x, gain, eps, r=None):
    """(H, Y) of H = x + r, Y = H rho gain."""
    h = x if r is None else x + r
    y = h * rho(h, eps)
    return h, y if gain is None else y * gain


def rms_norm_backward(h, gain, dy, eps, dr=None):
    """(dX, dgain)."""
    p = rho(h, eps)
    u = dy if gain is None else dy * gain
    dx = p * u - p ** 3 * h * (u * h).mean(axis=1, keepdims=True)
    return (dx if dr is None else dx + dr), (dy * h * p).sum(axis=0)


def e4m3_scale(y):
    """The scale of each row held in 8 bits."""
    with np.errstate(invalid="ignore"):
        return np.maximum(np.abs(y).max(axis=1) / E4M3_MAX, TINY)


def e4m3_value(bits):
    """Values of e4m3 bytes."""
    b = np.asarray(bits, np.int64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b & 128, -v, v)


def mx_weights(codes, scales):
    """fp64 weights of packed codes (N x K / 2) and scales (N x K / 32)."""
    codes = np.asarray(codes)
    n = codes.shape[0]
    c = np.stack([codes & 15, codes >> 4], axis=2).reshape(n, -1)
    v = np.where(c & 8, -1.0, 1.0) * E2M1[c & 7]
    s = np.where(np.asarray(scales) == 255, np.nan, 2.0 ** (np.asarray(scales, np.float64) - 127))
    return v * np.repeat(s, GROUP, axis=1)


def mx_candidates(w):
    """The two quantizations of each group of 32 that a layer chooses from:
    lists of (scale bytes (N x K / 32), weights (N x K), squared errors (N x K /
    32)), and the index of the one to take.  Zero groups: scale 127."""
    n, k = w.shape
    g = w.reshape(n, k // GROUP, GROUP)
    amax = np.abs(g).max(axis=2)
    e = np.floor(np.log2(np.where(amax > 0, amax, 1.0)))
    out = []
    for c in range(2):
        s = np.clip(e - 2 + c, -127, 126)
        a = np.abs(g) / 2.0 ** s[:, :, None]
        # nearest, ties to the even code
        d = np.abs(a[..., None] - E2M1)
        near = d.min(axis=-1, keepdims=True)
        tie = d == near
        even = tie & (np.arange(8) % 2 == 0)
        code = np.where(even.any(axis=-1), even.argmax(axis=-1), tie.argmax(axis=-1))
        q = np.sign(g) * E2M1[code] * 2.0 ** s[:, :, None]
        out.append((np.where(amax > 0, s + 127, 127).astype(np.int64), q.reshape(n, k), ((g - q) ** 2).sum(axis=2)))
    return out, (out[1][2] < out[0][2]).astype(np.int64)
