"""Plain float64 CPU oracle of the operators next to the boundary: the residual
addition with its RMS norm (16- and 8-bit output) and its backward, AdamW with
states in 32 or 8 bits, and the gradient norm with its clip factor.

TEST INFRASTRUCTURE, NOT PART OF THE PRODUCT.  Only the test suite may import
this module.  It shares no code with the HIP path.

Where an op rounds a value that later steps build on (the stream h; the stored
8-bit states), the oracle takes the rounded value as its input or returns the
value before that rounding, so that a comparison counts one rounding only.
"""
from __future__ import annotations

import numpy as np

from .fusion_oracle import rms_norm

E4M3_MAX = 448.0
SCALE_FLOOR = 2.0 ** -126
TINY = 2.0 ** -9          # the smallest positive e4m3 value
BLOCK = 256


def f64(x):
    return np.asarray(x, dtype=np.float64)


def stream(x, res=None, b=None):
    """h = x + res + b I_{r x n}, unrounded."""
    h = f64(x).copy()
    if res is not None:
        h += f64(res)
    if b is not None:
        h[:, :b.shape[1]] += f64(b)
    return h


def rstd(h, eps):
    return 1.0 / np.sqrt(np.mean(f64(h) ** 2, axis=1) + eps)


def norm(h, gamma, eps):
    return rms_norm(f64(h), gamma, eps)


def norm_bwd(h, gamma, rs, g_y, g_h=None):
    """(g_x, dgamma) of y = h rstd(h) gamma, with rs the rows' rstd."""
    xh = f64(h) * f64(rs)[:, None]
    w = f64(g_y) * f64(gamma)[None, :]
    g = f64(rs)[:, None] * (w - xh * np.mean(w * xh, axis=1, keepdims=True))
    if g_h is not None:
        g = g + f64(g_h)
    return g, np.sum(f64(g_y) * xh, axis=0)


def e4m3(x):
    """Round to the nearest e4m3 value (ties to even), |x| at most 448 after rounding; NaN stays."""
    x = f64(x)
    out = np.full(x.shape, np.nan)
    ok = np.isfinite(x)
    a = np.abs(x[ok])
    _, E = np.frexp(a)
    step = np.ldexp(1.0, np.maximum(E - 1, -6) - 3)
    out[ok] = np.copysign(np.round(a / step) * step, x[ok])  # np.round: ties to even
    return out


def scales(x, axis=-1):
    """max(max|x| / 448, 2^-126) along an axis."""
    return np.maximum(np.max(np.abs(f64(x)), axis=axis) / E4M3_MAX, SCALE_FLOOR)


def adamw(p, g, m, v, lr, step, b1, b2, eps, wd, gs=1.0):
    """(p, m, v) after one step."""
    g = f64(g) * gs
    m = b1 * f64(m) + (1.0 - b1) * g
    v = b2 * f64(v) + (1.0 - b2) * g * g
    upd = (m / (1.0 - b1 ** step)) / (np.sqrt(v / (1.0 - b2 ** step)) + eps)
    return (1.0 - lr * wd) * f64(p) - lr * upd, m, v


def blocks(x):
    """A flat array as rows of 256, zeros behind its end."""
    x = f64(x).ravel()
    return np.pad(x, (0, -x.size % BLOCK)).reshape(-1, BLOCK)


def state8(x, root=False):
    """(values, scales) that an 8-bit state holds for x (root: for u = sqrt(x), whose non-zero values
    take the smallest code rather than zero); values are those before the multiplication by the scale."""
    rows = np.sqrt(blocks(x)) if root else blocks(x)
    s = scales(rows)
    t = rows / s[:, None]
    if root:
        t = np.where((rows > 0) & (t < TINY), TINY, t)
    return e4m3(t).ravel()[:np.size(x)], s


def grad_norm(grads, max_norm):
    """(norm, factor); the factor is NaN where the norm is not finite."""
    n = np.sqrt(sum(float(np.sum(f64(g) ** 2)) for g in grads))
    return n, min(1.0, max_norm / (n + 1e-6)) if np.isfinite(n) else np.nan
