"""Float64 statement (numpy, CPU) of the recurrent-memory operators: norm, 8-bit quantisation and product, recurrence.

Written from the formulas, one step after the other; nothing here is shared with the CUDA library.
"""
from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0
AMAX_FLOOR = 2.0 ** -100
BLOCK = 128


def rms_norm(x, weight, eps, residual=None):
    """x [outer, C, inner] -> (y, s, rstd [outer, inner])."""
    s = np.asarray(x, np.float64)
    if residual is not None:
        s = s + np.asarray(residual, np.float64)
    rstd = 1.0 / np.sqrt((s * s).mean(axis=1) + eps)
    return s * rstd[:, None, :] * np.asarray(weight, np.float64)[None, :, None], s, rstd


def rms_norm_backward(grad_y, s, weight, rstd, grad_s=None):
    """(grad_x, grad_weight) of rms_norm; grad_x is the residual's gradient too."""
    gy, s = np.asarray(grad_y, np.float64), np.asarray(s, np.float64)
    rstd = np.asarray(rstd, np.float64)[:, None, :]
    n = s * rstd
    gn = gy * np.asarray(weight, np.float64)[None, :, None]
    gx = rstd * (gn - n * (gn * n).mean(axis=1, keepdims=True))
    if grad_s is not None:
        gx = gx + np.asarray(grad_s, np.float64)
    return gx, (gy * n).sum(axis=(0, 2))


def e4m3_values():
    """Every non-negative finite e4m3 value, ascending: 4 exponent bits (bias 7), 3 mantissa bits."""
    v = [m / 8 * 2.0 ** -6 for m in range(8)]
    v += [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]
    return np.array(v)


def to_e4m3(x):
    """The nearest e4m3 value (ties to the even mantissa, the largest finite value beyond the range)."""
    x = np.asarray(x, np.float64)
    vals = e4m3_values()
    a = np.minimum(np.abs(x), E4M3_MAX)
    hi = np.clip(np.searchsorted(vals, a), 1, len(vals) - 1)
    lo = hi - 1
    up, down = vals[hi] - a, a - vals[lo]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.copysign(vals[pick], x)


def quantize_rows(y):
    """y [rows, k] -> (values [rows, k], scale [ceil(k / 128), rows])."""
    y = np.asarray(y, np.float64)
    rows, k = y.shape
    scale = np.empty((-(-k // BLOCK), rows))
    q = np.empty_like(y)
    for j in range(scale.shape[0]):
        b = slice(j * BLOCK, (j + 1) * BLOCK)
        scale[j] = np.maximum(np.abs(y[:, b]).max(axis=1), AMAX_FLOOR) / E4M3_MAX
        q[:, b] = to_e4m3(y[:, b] / scale[j][:, None])
    return q, scale


def quantize_blocks(w):
    """w [n, k] -> (values [n, k], scale [ceil(n / 128), ceil(k / 128)])."""
    w = np.asarray(w, np.float64)
    n, k = w.shape
    scale, q = np.empty((-(-n // BLOCK), -(-k // BLOCK))), np.empty_like(w)
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            b = (slice(i * BLOCK, (i + 1) * BLOCK), slice(j * BLOCK, (j + 1) * BLOCK))
            scale[i, j] = max(np.abs(w[b]).max(), AMAX_FLOOR) / E4M3_MAX
            q[b] = to_e4m3(w[b] / scale[i, j])
    return q, scale


def matmul_fp8(x, x_scale, w, w_scale):
    """x [m, k], x_scale [kb, m], w [n, k], w_scale [nb, kb] -> [m, n]."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    col = np.arange(x.shape[1]) // BLOCK
    xs = x * np.asarray(x_scale, np.float64).T[:, col]
    ws = w * np.asarray(w_scale, np.float64)[np.arange(w.shape[0]) // BLOCK][:, col]
    return xs @ ws.T


def sigmoid(g):
    g = np.asarray(g, np.float64)
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1.0, e) / (1.0 + e)


def _ends(lengths, outer, n):
    if lengths is None:
        return np.full(outer, n)
    return np.clip(np.asarray(lengths), 0, n)


def gated_scan(v, g, h0=None, lengths=None, gate="sigmoid"):
    """v, g [outer, L, inner] -> (h, h_last [outer, inner], states in front of every step)."""
    v, g = np.asarray(v, np.float64), np.asarray(g, np.float64)
    outer, n, inner = v.shape
    s = np.zeros((outer, inner)) if h0 is None else np.array(h0, np.float64)
    h, before = np.zeros_like(v), np.zeros_like(v)
    end = _ends(lengths, outer, n)
    for t in range(n):
        for o in range(outer):
            before[o, t] = s[o]
            if t < end[o]:
                if gate == "sigmoid":
                    s[o] = sigmoid(g[o, t]) * s[o] + sigmoid(-g[o, t]) * v[o, t]
                else:
                    s[o] = g[o, t] * s[o] + v[o, t]
                h[o, t] = s[o]
    return h, s, before


def gated_scan_backward(grad_h, v, g, h0=None, lengths=None, grad_last=None, gate="sigmoid"):
    """(grad_v, grad_g, grad_h0) of gated_scan."""
    gh, v, g = (np.asarray(x, np.float64) for x in (grad_h, v, g))
    outer, n, inner = v.shape
    _, _, before = gated_scan(v, g, h0, lengths, gate)
    carry = np.zeros((outer, inner)) if grad_last is None else np.array(grad_last, np.float64)
    gv, gg = np.zeros_like(v), np.zeros_like(v)
    end = _ends(lengths, outer, n)
    for o in range(outer):
        for t in range(end[o] - 1, -1, -1):
            delta = gh[o, t] + carry[o]
            if gate == "sigmoid":
                a, b = sigmoid(g[o, t]), sigmoid(-g[o, t])
                gv[o, t], gg[o, t] = delta * b, delta * (before[o, t] - v[o, t]) * a * b
            else:
                a = g[o, t]
                gv[o, t], gg[o, t] = delta, delta * before[o, t]
            carry[o] = a * delta
    return gv, gg, carry


def rel_l2(a, b):
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    n = np.linalg.norm(b)
    return float(np.linalg.norm(a - b) / n) if n else float(np.linalg.norm(a - b))
