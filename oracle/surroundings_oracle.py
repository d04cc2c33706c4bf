"""Definitions of the operators around the sparse layer, in numpy, independent of the package.

Norm, its gradient and the product: fp64.  The optimizer's states are part of a format (codes and scales have to come out the
same whatever computes them), so their arithmetic is written out in fp32, operation by operation; the update of the weights is
fp64.  8-bit values are OCP e4m3: sign, 4 bits of exponent (bias 7), 3 of mantissa, no infinity, 0x7F = NaN, largest 448.
"""
from __future__ import annotations

import numpy as np

F32 = np.float32
MAX, TINY, BLOCK = 448.0, 1e-30, 128


def e4m3_value(codes):
    c = np.asarray(codes, dtype=np.uint8).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(np.float64) - 10))
    v = np.where((c & 0x7F) == 0x7F, np.nan, v)
    return np.where(c & 0x80, -v, v)


_VALUES = e4m3_value(np.arange(0x7F))                          # the finite magnitudes, ascending


def e4m3_nearest(x):
    """Codes of the nearest values, ties to the even code; |x| <= 448."""
    a = np.minimum(np.abs(np.asarray(x, dtype=np.float64)), MAX)
    hi = np.clip(np.searchsorted(_VALUES, a), 0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    up, down = _VALUES[hi] - a, a - _VALUES[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def q8_scale(top):
    """(scale, reciprocal) in fp32 from the largest magnitudes."""
    top = np.asarray(top, dtype=F32)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        scale = np.where(top < F32(TINY), F32(0), top * F32(1.0 / MAX))
        inv = np.where(top < F32(TINY), F32(0), (F32(1) / top) * F32(MAX))
    return scale.astype(F32), inv.astype(F32)


def rmsnorm(h, w, eps):
    """(y, r) of the stored stream h."""
    h, w = np.asarray(h, np.float64), np.asarray(w, np.float64)
    r = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h * r[:, None] * w, r


def rmsnorm_grad(dy, h, w, r, dh=None):
    """(dx, dw); r is taken as it is given."""
    dy, h, w, r = (np.asarray(t, np.float64) for t in (dy, h, w, r))
    x = h * r[:, None]
    g = dy * w
    dx = r[:, None] * (g - x * (g * x).mean(1, keepdims=True))
    return (dx if dh is None else dx + np.asarray(dh, np.float64)), (dy * x).sum(0)


def product_q8(q, xs, wq, meta, ws, add=None):
    """q: codes [b, d_in]; wq: codes [d_out, d_in/2]; meta: u8[d_out, d_in/8].  (Y, the sum of its terms' magnitudes)."""
    d_out, half = wq.shape
    w = np.zeros((d_out, 2 * half))
    rows = np.arange(d_out)[:, None]
    for slot in range(4):
        col = 8 * np.arange(half // 4) + 4 * (slot // 2) + ((meta >> (2 * slot)) & 3)
        w[rows, col] = e4m3_value(wq[:, slot::4])
    x = e4m3_value(q)
    s = np.asarray(xs, np.float64)[:, None] * np.asarray(ws, np.float64)[None, :]
    y, terms = (x @ w.T) * s, (np.abs(x) @ np.abs(w).T) * s
    return (y if add is None else y + np.asarray(add, np.float64)), terms


def grad_norm(grads, inv_scale, max_norm):
    norm = inv_scale * np.sqrt(sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads))
    return norm, (inv_scale * min(1.0, max_norm / (norm + 1e-6)) if np.isfinite(norm) else 0.0)


def threshold(n, step, root):
    """u of each element: 20 bits, moved by the golden ratio each step; half a turn further for the roots."""
    h = (np.arange(n, dtype=np.uint64) * np.uint64(0x6A09E667) + np.uint64(step * 0x9E3779B9)) & np.uint64(0xFFFFFFFF)
    if root:
        h = h ^ np.uint64(0x80000000)
    return ((h >> np.uint64(12)).astype(np.float64) * 2.0 ** -20).astype(F32)


def dithered(a, u):
    """a in [0, 448] (fp32) to the code below, or the one above where the fraction between them plus u reaches 1."""
    a = np.asarray(a, F32)
    e = np.maximum(np.frexp(a)[1] - 1, -6).astype(np.float64)
    ulp = 2.0 ** (e - 3)
    return np.floor(a.astype(np.float64) / ulp + u) * ulp


def store_states(x, step, root):
    """fp32[n] -> (codes u8[n], scales fp32[blocks])."""
    n = x.size
    pad = np.zeros((n + BLOCK - 1) // BLOCK * BLOCK, F32)
    pad[:n] = x
    u = np.zeros_like(pad)
    u[:n] = threshold(n, step, root)
    a = np.abs(pad).reshape(-1, BLOCK)
    scale, inv = q8_scale(a.max(1))
    a = np.minimum(a * inv[:, None], F32(MAX)).astype(F32)
    q = dithered(a, u.reshape(-1, BLOCK))
    if root:
        q = np.where((a > 0) & (q == 0), 2.0 ** -9, q)
    codes = np.searchsorted(_VALUES, q.reshape(-1)[:n]).astype(np.uint8)
    assert (e4m3_value(codes) == q.reshape(-1)[:n]).all()
    return codes | np.where(np.signbit(x), 0x80, 0).astype(np.uint8), scale


def load_states(codes, scales):
    s = np.repeat(np.asarray(scales, F32), BLOCK)[: codes.size]
    return e4m3_value(codes).astype(F32) * s


def adamw(p, g, m, v, coef, lr, beta1, beta2, eps, decay, step):
    """(p, m, v) after a step: p in fp64, the moments in fp32 as the format says; v's root is np.sqrt of it in fp32."""
    m, v = np.asarray(m, F32), np.asarray(v, F32)
    x = np.asarray(g, F32) * F32(coef)
    m2 = m * F32(beta1) + x * F32(1.0 - beta1)
    v2 = v * F32(beta2) + (x * x) * F32(1.0 - beta2)
    m64, v64 = m2.astype(np.float64), v2.astype(np.float64)
    p = np.asarray(p, np.float64)
    p = p - lr * decay * p - lr * (m64 / (1 - beta1 ** step)) / (np.sqrt(v64 / (1 - beta2 ** step)) + eps)
    return p, m2, v2
