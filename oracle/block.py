"""CPU oracle for the selective block -- TEST INFRASTRUCTURE ONLY.

Only ``tests/`` may import or run anything here.  The product path never calls it and
shares no code with it.  Plain float64 numpy, step by step, of layer norm, the short
causal convolution and the selective scan, and of their gradients:

    s = x + r,  y = (s - mean s) / sqrt(var s + eps) w + b
    o_t = bias + sum_k w[c, k] x_(t - K + 1 + k),  y_t = o_t or o_t sigmoid(o_t)
    delta = log(1 + e^(dt + dt_bias)),  x_t = e^(delta A) x_(t-1) + delta B_t u_t,
    y_t = (C_t . x_t + h0 u_t) z_t sigmoid(z_t)

Every function takes ``magnitude``: the same sums with every term's absolute value in
place of the term.  A float32 evaluation differs from the exact value by at most (its
roundings) x 2^-24 x that magnitude, which is what the tests' tolerances are made of.

Parity is pinned by ``tests/test_block_pins.py``.
"""
from __future__ import annotations

import numpy as np

__all__ = ["layer_norm", "layer_norm_grad", "short_conv", "short_conv_grad", "selective", "selective_grad"]


def _f(x):
    return None if x is None else np.asarray(x, np.float64)


def _mag(x, magnitude):
    return np.abs(x) if magnitude and x is not None else x


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def layer_norm(x, w, b, residual=None, eps=1e-5, magnitude=False):
    """``y, total, mean, rstd`` of the rows of ``x [rows, D]``."""
    s = _f(x) + (0 if residual is None else _f(residual))
    m = s.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((s - m) ** 2).mean(1, keepdims=True) + eps)
    w, b = _f(w), 0 if b is None else _f(b)
    if magnitude:
        top = np.abs(s).max(1, keepdims=True)
        return (np.abs(s) + top) * rstd * np.abs(w) + np.abs(b), np.abs(s), top[:, 0], rstd[:, 0]
    return (s - m) * rstd * w + b, s, m[:, 0], rstd[:, 0]


def layer_norm_grad(dy, x, w, mean, rstd, dtotal=None, magnitude=False):
    """``dx, dw, db``."""
    dy, x, w, mean, rstd = map(_f, (dy, x, w, mean, rstd))
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy * w
    t = 0 if dtotal is None else _f(dtotal)
    if magnitude:
        h = (np.abs(x) + np.abs(mean[:, None])) * rstd[:, None]
        g, dy = np.abs(g), np.abs(dy)
        dx = rstd[:, None] * (g + g.mean(1, keepdims=True) + h * (g * h).mean(1, keepdims=True)) + np.abs(t)
    else:
        dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True)) + t
    return dx, (dy * h).sum(0), dy.sum(0)


def _lengths(lengths, B, T):
    return np.full(B, T) if lengths is None else np.clip(np.asarray(lengths, np.int64), 0, T)


def short_conv(x, w, bias, silu, state=None, lengths=None, magnitude=False):
    """``y [B, T, D], state [B, K - 1, D]``; ``state=None`` starts from zeros."""
    x, w = _f(x), _mag(_f(w), magnitude)
    B, T, D = x.shape
    K = w.shape[1]
    bias = np.zeros(D) if bias is None else _mag(_f(bias), magnitude)
    y = np.zeros((B, T, D))
    out = np.zeros((B, K - 1, D))
    for b, n in enumerate(_lengths(lengths, B, T)):
        past = np.zeros((K - 1, D)) if state is None else _f(state)[b]
        xp = np.concatenate([past, x[b, :n]])
        xm = _mag(xp, magnitude)
        for t in range(n):
            o = bias.copy()
            for k in range(K):
                o += w[:, k] * xm[t + k]
            y[b, t] = o if not silu else o * (2.0 if magnitude else sigmoid(o))
        out[b] = xp[n:]
    return y, out


def short_conv_grad(dy, x, w, bias, silu, lengths=None, magnitude=False):
    """``dx, dw, dbias`` from zeros before the prompt."""
    dy, x, w = _f(dy), _f(x), _f(w)
    B, T, D = x.shape
    K = w.shape[1]
    bias = np.zeros(D) if bias is None else _f(bias)
    dx, dw, dbias = np.zeros_like(x), np.zeros_like(w), np.zeros(D)
    for b, n in enumerate(_lengths(lengths, B, T)):
        for t in range(n):
            g = dy[b, t].copy()
            if silu:
                o = bias.copy()
                for k in range(K):
                    if t - K + 1 + k >= 0:
                        o += w[:, k] * x[b, t - K + 1 + k]
                p = sigmoid(o)
                g *= p * (1 + o * (1 - p))
                if magnitude:
                    # the slope's own error: its steepness (<= 1/2) times that of o
                    om = np.abs(bias)
                    for k in range(K):
                        if t - K + 1 + k >= 0:
                            om = om + np.abs(w[:, k] * x[b, t - K + 1 + k])
                    g = np.abs(dy[b, t]) * (1.1 + om)
            g = _mag(g, magnitude)
            dbias += g
            for k in range(K):
                j = t - K + 1 + k
                if j >= 0:
                    dx[b, j] += _mag(w[:, k], magnitude) * g
                    dw[:, k] += g * _mag(x[b, j], magnitude)
    return dx, dw, dbias


def _selective_inputs(dt, Bm, Cm, u, h0, dt_bias, z, D, magnitude):
    pre = _f(dt) + (0 if dt_bias is None else _f(dt_bias))
    delta = np.logaddexp(0.0, pre)
    Bm, Cm, u = (_mag(_f(v), magnitude) for v in (Bm, Cm, u))
    G = Bm.shape[2]
    wide = lambda m: np.repeat(m, D // G, axis=2)  # noqa: E731  [B, T, G, N] -> [B, T, D, N]
    h0 = np.zeros(D) if h0 is None else _mag(_f(h0), magnitude)
    return pre, delta, wide(Bm), wide(Cm), u, h0, _f(z)


def selective(A, dt, Bm, Cm, u, h0=None, dt_bias=None, z=None, state=None, lengths=None, magnitude=False):
    """``y [B, T, D], state [B, D, N]``; ``state=None`` starts from zero."""
    A = _f(A)
    B, T, D = np.asarray(u).shape
    _, delta, Bw, Cw, u, h0, z = _selective_inputs(dt, Bm, Cm, u, h0, dt_bias, z, D, magnitude)
    y = np.zeros((B, T, D))
    x = np.zeros((B, D, A.shape[1])) if state is None else _mag(_f(state), magnitude).copy()
    for b, n in enumerate(_lengths(lengths, B, T)):
        for t in range(n):
            x[b] = np.exp(delta[b, t][:, None] * A) * x[b] + (delta[b, t] * u[b, t])[:, None] * Bw[b, t]
            o = (Cw[b, t] * x[b]).sum(1) + h0 * u[b, t]
            y[b, t] = o if z is None else o * _mag(z[b, t] * sigmoid(z[b, t]), magnitude)
    return y, x


def selective_grad(dy, A, dt, Bm, Cm, u, h0=None, dt_bias=None, z=None, lengths=None, magnitude=False):
    """Gradients from a zero state: dict of ``dA, ddt, dBm, dCm, du, dh0, ddt_bias, dz``."""
    A = _f(A)
    B, T, D = np.asarray(u).shape
    N, G = A.shape[1], np.asarray(Bm).shape[2]
    pre, delta, Bw, Cw, u, h0, z = _selective_inputs(dt, Bm, Cm, u, h0, dt_bias, z, D, magnitude)
    dy, Am = _mag(_f(dy), magnitude), _mag(A, magnitude)
    out = {k: np.zeros((B, T, D)) for k in ("ddt", "du", "dz")}
    out.update({k: np.zeros((B, T, G, N)) for k in ("dBm", "dCm")})
    out["dA"], out["dh0"], out["ddt_bias"] = np.zeros((D, N)), np.zeros(D), np.zeros(D)
    for b, n in enumerate(_lengths(lengths, B, T)):
        xs = np.zeros((n + 1, D, N))
        for t in range(n):
            xs[t + 1] = np.exp(delta[b, t][:, None] * A) * xs[t] + (delta[b, t] * u[b, t])[:, None] * Bw[b, t]
        g = np.zeros((D, N))  # of the state after step t
        for t in reversed(range(n)):
            d = dy[b, t]
            if z is not None:
                p = sigmoid(z[b, t])
                o = (Cw[b, t] * xs[t + 1]).sum(1) + h0 * u[b, t]
                out["dz"][b, t] = d * o * p * (1 + _mag(z[b, t], magnitude) * (1 - p))
                d = d * _mag(z[b, t] * p, magnitude)
            g = g + Cw[b, t] * d[:, None]
            step = (delta[b, t] * u[b, t])[:, None]
            out["dBm"][b, t] = (g * step).reshape(G, D // G, N).sum(1)
            out["dCm"][b, t] = (d[:, None] * xs[t + 1]).reshape(G, D // G, N).sum(1)
            ag = np.exp(delta[b, t][:, None] * A) * g
            gb = (g * Bw[b, t]).sum(1)
            ddt = ((Am * ag * xs[t]).sum(1) + u[b, t] * gb) * sigmoid(pre[b, t])
            out["ddt"][b, t] = ddt
            out["ddt_bias"] += ddt
            out["du"][b, t] = delta[b, t] * gb + h0 * d
            out["dh0"] += d * u[b, t]
            out["dA"] += delta[b, t][:, None] * ag * xs[t]
            g = ag
    if z is None:
        del out["dz"]
    return out
