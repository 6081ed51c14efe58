"""Float64 statement (numpy, CPU) of the selective memory's operators: layer norm, causal convolution, selective scan, the
gradients' norm and clipping.

Written from the formulas, one step after the other; nothing here is shared with the CUDA library.
"""
from __future__ import annotations

import numpy as np


def f64(x):
    return np.asarray(x, np.float64)


def layer_norm(x, weight, bias, eps, residual=None):
    """x [outer, C, inner] -> (y, s, mean, rstd [outer, inner])."""
    s = f64(x) if residual is None else f64(x) + f64(residual)
    mean = s.mean(axis=1)
    d = s - mean[:, None, :]
    rstd = 1.0 / np.sqrt((d * d).mean(axis=1) + eps)
    y = d * rstd[:, None, :] * f64(weight)[None, :, None]
    return y if bias is None else y + f64(bias)[None, :, None], s, mean, rstd


def layer_norm_backward(grad_y, s, weight, mean, rstd, grad_s=None):
    """(grad_x, grad_weight, grad_bias)."""
    gy, r = f64(grad_y), f64(rstd)[:, None, :]
    n = (f64(s) - f64(mean)[:, None, :]) * r
    g = gy * f64(weight)[None, :, None]
    gx = r * (g - g.mean(axis=1, keepdims=True) - n * (g * n).mean(axis=1, keepdims=True))
    return gx if grad_s is None else gx + f64(grad_s), (gy * n).sum(axis=(0, 2)), gy.sum(axis=(0, 2))


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-f64(x)))


def _ends(lengths, B, T):
    return [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths]


def causal_conv(x, weight, bias, state=None, lengths=None, silu=True):
    """x [B, T, C] -> (y, new state [B, K - 1, C])."""
    x, w = f64(x), f64(weight)
    B, T, C = x.shape
    K = w.shape[1]
    y, last = np.zeros((B, T, C)), np.zeros((B, K - 1, C))
    for b, n in enumerate(_ends(lengths, B, T)):
        u = np.concatenate([np.zeros((K - 1, C)) if state is None else f64(state)[b], x[b, :n]])
        for t in range(n):
            p = (0.0 if bias is None else f64(bias)) + sum(w[:, k] * u[t + k] for k in range(K))
            y[b, t] = p * sigmoid(p) if silu else p
        last[b] = u[n:]
    return y, last


def causal_conv_backward(grad_y, x, weight, bias, state=None, lengths=None, grad_last=None, silu=True):
    """(grad_x, grad_weight, grad_bias, grad_state)."""
    x, w, gy = f64(x), f64(weight), f64(grad_y)
    B, T, C = x.shape
    K = w.shape[1]
    gx, gs, gw, gb = np.zeros_like(x), np.zeros((B, K - 1, C)), np.zeros_like(w), np.zeros(C)
    for b, n in enumerate(_ends(lengths, B, T)):
        u = np.concatenate([np.zeros((K - 1, C)) if state is None else f64(state)[b], x[b, :n]])
        gu = np.zeros_like(u)
        if grad_last is not None:
            gu[n:] += f64(grad_last)[b]
        for t in range(n):
            p = (0.0 if bias is None else f64(bias)) + sum(w[:, k] * u[t + k] for k in range(K))
            sg = sigmoid(p)
            g = gy[b, t] * (sg * (1 + p * (1 - sg)) if silu else 1.0)
            gb += g
            for k in range(K):
                gw[:, k] += g * u[t + k]
                gu[t + k] += w[:, k] * g
        gs[b], gx[b, :n] = gu[:K - 1], gu[K - 1:]
    return gx, gw, gb, gs


def _steps(dt, dt_bias, softplus):
    raw = f64(dt) if dt_bias is None else f64(dt) + f64(dt_bias)
    return raw, np.logaddexp(raw, 0.0) if softplus else raw


def _wide(m, C):
    """Maps [B, T, G, N] for every channel: [B, T, C, N]."""
    return np.repeat(f64(m), C // m.shape[2], axis=2)


def selective_scan(x, dt, A, B, C, D=None, z=None, dt_bias=None, h0=None, lengths=None, softplus=True, keep=False):
    """(y, h_last), and with `keep` the states [B, T + 1, channels, N] and what the output gate multiplies."""
    x = f64(x)
    nb, T, ch = x.shape
    _, d = _steps(dt, dt_bias, softplus)
    Bw, Cw, A = _wide(B, ch), _wide(C, ch), f64(A)
    y, core = np.zeros_like(x), np.zeros_like(x)
    h = np.zeros((nb, T + 1, ch, A.shape[1]))
    last = np.zeros((nb, ch, A.shape[1]))
    for b, n in enumerate(_ends(lengths, nb, T)):
        if h0 is not None:
            h[b, 0] = f64(h0)[b]
        for t in range(n):
            h[b, t + 1] = np.exp(d[b, t][:, None] * A) * h[b, t] + (d[b, t] * x[b, t])[:, None] * Bw[b, t]
            o = (Cw[b, t] * h[b, t + 1]).sum(axis=1)
            if D is not None:
                o = o + f64(D) * x[b, t]
            core[b, t] = o
            y[b, t] = o if z is None else o * f64(z)[b, t] * sigmoid(f64(z)[b, t])
        last[b] = h[b, n]
    return (y, last, h, core) if keep else (y, last)


def selective_scan_backward(grad_y, x, dt, A, B, C, D=None, z=None, dt_bias=None, h0=None, lengths=None, grad_last=None, softplus=True):
    """Gradients by name."""
    _, _, h, core = selective_scan(x, dt, A, B, C, D, z, dt_bias, h0, lengths, softplus, keep=True)
    x, gy, A = f64(x), f64(grad_y), f64(A)
    nb, T, ch = x.shape
    G = B.shape[2]
    raw, d = _steps(dt, dt_bias, softplus)
    slope = sigmoid(raw) if softplus else np.ones_like(raw)
    Bw, Cw = _wide(B, ch), _wide(C, ch)
    g = {k: np.zeros_like(x) for k in ("x", "dt", "z")}
    g["B"], g["C"] = np.zeros(B.shape), np.zeros(C.shape)
    g["A"], g["D"], g["dt_bias"], g["h0"] = np.zeros_like(A), np.zeros(ch), np.zeros(ch), np.zeros((nb,) + A.shape)
    group = lambda m: m.reshape(G, ch // G, -1).sum(axis=1)
    for b, n in enumerate(_ends(lengths, nb, T)):
        m = np.zeros_like(A) if grad_last is None else f64(grad_last)[b]
        for t in range(n - 1, -1, -1):
            gc = gy[b, t]
            if z is not None:
                zt = f64(z)[b, t]
                s = sigmoid(zt)
                g["z"][b, t] = gc * core[b, t] * s * (1 + zt * (1 - s))
                gc = gc * zt * s
            e = m + gc[:, None] * Cw[b, t]
            g["C"][b, t] = group(gc[:, None] * h[b, t + 1])
            g["B"][b, t] = group(e * (d[b, t] * x[b, t])[:, None])
            a = np.exp(d[b, t][:, None] * A)
            q = e * a * h[b, t]
            eb = (e * Bw[b, t]).sum(axis=1)
            g["x"][b, t] = d[b, t] * eb + (gc * f64(D) if D is not None else 0.0)
            g["dt"][b, t] = ((q * A).sum(axis=1) + x[b, t] * eb) * slope[b, t]
            g["A"] += q * d[b, t][:, None]
            g["D"] += gc * x[b, t]
            g["dt_bias"] += g["dt"][b, t]
            m = a * e
        g["h0"][b] = m
    if z is None:
        del g["z"]
    return g


def clip(grads, max_norm, eps=1e-6):
    """(norm, clipped gradients)."""
    norm = np.sqrt(sum((np.abs(g.astype(np.complex128 if np.iscomplexobj(g) else np.float64)) ** 2).sum() for g in grads))
    c = min(1.0, max_norm / (norm + eps))
    return norm, [g.astype(np.complex128 if np.iscomplexobj(g) else np.float64) * c for g in grads]
