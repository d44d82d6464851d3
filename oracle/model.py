"""CPU oracle for the gated recurrence and the two ends of a language model -- TEST
INFRASTRUCTURE ONLY.

Only ``tests/`` may import or run anything here.  The product path never calls it and
shares no code with it.  Plain float64 numpy, step by step:

    f = sigmoid(r + r_bias), p = sigmoid(i + i_bias), a = e^(-rate f)
    h_t = a h_(t-1) + sqrt(1 - a^2) p u_t, y_t = h_t (z sigmoid(z))
    y[k] = scale W[ids[k]], dW[v] = scale sum of dy[k] with ids[k] = v
    loss = scale tau^2 sum p (log p - log q), p and q softmaxes over tau
    verification of drafted tokens

``gated`` and ``gated_grad`` also return bounds of a float32 evaluation's error, in units of
2^-24, carried along with the values.  With X the largest |r + bias|, |i + bias| or |z| of the
inputs, the units of relative error are

    a sigmoid     G = 3 X + 8: its exponent has 3 roundings of X, exp, sum and rcp 2 each
    L = rate f    G + 3
    a = e^-L      (G + 3) L, and 3 of its own
    sqrt(1 - a^2) G + 20: half of (G + 3) + 26 (1 - a^2 >= 0.117 where it is a difference,
                  whose 3 roundings weigh 1 / 0.117), and 2 of its own
    v             2 G + 32

and a step rounds the state 3 times, so E_t = a E_(t-1) + a ((G + 3) L + 6) M_(t-1) + (2 G +
35) |v_t|, where M is the recurrence of the magnitudes.  The gradient's are built alike.

Parity is pinned by ``tests/test_model_pins.py``.
"""
from __future__ import annotations

import numpy as np

__all__ = ["gated", "gated_grad", "embed", "embed_grad", "distill_logits", "verify"]


def _f(x):
    return None if x is None else np.asarray(x, np.float64)


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def _lengths(lengths, B, T):
    return np.full(B, T) if lengths is None else np.clip(np.asarray(lengths, np.int64), 0, T)


class _Gates:
    def __init__(self, rate, r, i, u, r_bias, i_bias, z):
        self.rate = _f(rate)
        x = _f(r) + (0 if r_bias is None else _f(r_bias))
        y = _f(i) + (0 if i_bias is None else _f(i_bias))
        self.u, self.z = _f(u), _f(z)
        self.f, self.p = sigmoid(x), sigmoid(y)
        self.nf, self.np = sigmoid(-x), sigmoid(-y)
        self.L = self.rate * self.f
        self.a = np.exp(-self.L)
        self.q = -np.expm1(-2 * self.L)
        self.w = np.sqrt(self.q) * self.p
        self.v = self.w * self.u
        finite = lambda t: np.abs(t[np.isfinite(t)]).max(initial=0.0) if t is not None else 0.0  # noqa: E731
        self.G = 3 * max(finite(x), finite(y), finite(self.z)) + 8


def gated(rate, r, i, u, r_bias=None, i_bias=None, z=None, state=None, lengths=None):
    """``y [B, T, D], state [B, D], y's bound, state's bound, states before each token
    [B, T, D] and their bound``; ``state=None`` starts from zero."""
    g = _Gates(rate, r, i, u, r_bias, i_bias, z)
    B, T, D = g.u.shape
    y, ey, before, ebefore = (np.zeros((B, T, D)) for _ in range(4))
    h = np.zeros((B, D)) if state is None else _f(state).copy()
    E = np.zeros((B, D))
    for b, n in enumerate(_lengths(lengths, B, T)):
        M = np.abs(h[b])
        for t in range(n):
            before[b, t], ebefore[b, t] = h[b], E[b] + 3 * M
            a, v = g.a[b, t], g.v[b, t]
            E[b] = a * E[b] + a * ((g.G + 3) * g.L[b, t] + 6) * M + (2 * g.G + 35) * np.abs(v)
            h[b] = a * h[b] + v
            M = a * M + np.abs(v)
            y[b, t], ey[b, t] = h[b], E[b] + M
            if z is not None:
                s = g.z[b, t] * sigmoid(g.z[b, t])
                y[b, t] = h[b] * s
                ey[b, t] = np.abs(s) * (E[b] + (g.G + 4) * M)
    return y, h, ey, E, before, ebefore


def gated_grad(dy, rate, r, i, u, r_bias=None, i_bias=None, z=None, state=None, lengths=None, dlast=None):
    """Gradients: dict of ``drate, dr, di, du, dr_bias, di_bias, dz, dfirst``, and a dict of
    their bounds."""
    g = _Gates(rate, r, i, u, r_bias, i_bias, z)
    B, T, D = g.u.shape
    dy, G = _f(dy), g.G
    _, _, _, _, before, ebefore = gated(rate, r, i, u, r_bias, i_bias, z, state, lengths)
    out = {k: np.zeros((B, T, D)) for k in ("dr", "di", "du", "dz")}
    err = {k: np.zeros((B, T, D)) for k in out}
    for d in (out, err):
        d.update({k: np.zeros(D) for k in ("drate", "dr_bias", "di_bias")})
        d["dfirst"] = np.zeros((B, D)) if dlast is None else np.abs(_f(dlast)) * 0
    sums = {k: np.zeros(D) for k in ("drate", "dr_bias", "di_bias")}  # of magnitudes
    for b, n in enumerate(_lengths(lengths, B, T)):
        X = np.zeros(D) if dlast is None else _f(dlast)[b].copy()
        E, M = np.zeros(D), np.abs(X)
        for t in reversed(range(n)):
            a, L, w, v = g.a[b, t], g.L[b, t], g.w[b, t], g.v[b, t]
            q = dy[b, t]
            eq = np.abs(q)
            if z is not None:
                zz = g.z[b, t]
                s = sigmoid(zz)
                h = a * before[b, t] + v
                eh = a * ebefore[b, t] + a * ((G + 3) * L + 6) * np.abs(before[b, t]) + (2 * G + 35) * np.abs(v)
                slope = s * (1 + zz * (1 - s))
                out["dz"][b, t] = q * h * slope
                # the slope's terms: s, and s z (1 - s) with its difference's rounding
                terms = s * (1 + np.abs(zz))
                err["dz"][b, t] = np.abs(q) * (eh * np.abs(slope) + (2 * G + 12) * terms * (np.abs(h) + eh * 2.0 ** -24))
                q = q * zz * s
                eq = (G + 4) * np.abs(q)
            dh = q + X
            E, M = E + eq + 2 * (np.abs(q) + M), np.abs(q) + M  # (of dh)
            out["du"][b, t], err["du"][b, t] = dh * w, w * (E + (2 * G + 32) * M)
            di = dh * v * g.np[b, t]
            out["di"][b, t] = di
            err["di"][b, t] = np.abs(v) * g.np[b, t] * (E + (3 * G + 40) * M)
            with np.errstate(invalid="ignore", divide="ignore"):
                lq = np.where(L > 0, L / g.q[b, t], 0.5)
            one, two = v * a * a * lq, L * a * before[b, t]
            dl = one - two
            # L / (1 - a^2): 2 (G + 3) + 30, and the factors; the state's own bound
            edl = (5 * G + 80) * np.abs(one) + (2 * G + 12) * np.abs(two) + L * a * ebefore[b, t]
            ldl = dh * dl
            eldl = E * np.abs(dl) + M * edl + 2 * M * np.abs(dl)
            dr = ldl * g.nf[b, t]
            out["dr"][b, t] = dr
            err["dr"][b, t] = g.nf[b, t] * (eldl + (G + 2) * np.abs(ldl))
            with np.errstate(invalid="ignore", divide="ignore"):
                drate = np.where(g.rate > 0, ldl / g.rate, 0.0)
                edrate = np.where(g.rate > 0, eldl / g.rate, 0.0)
            for k, val, e in (("drate", drate, edrate), ("dr_bias", dr, err["dr"][b, t]), ("di_bias", di, err["di"][b, t])):
                out[k] += val
                err[k] += e
                sums[k] += np.abs(val) + e * 2.0 ** -24
            E = a * E + a * ((G + 3) * L + 6) * M
            X, M = a * dh, a * M
        out["dfirst"][b], err["dfirst"][b] = X, E + 3 * M
    for k in sums:  # additions over tokens, wavefronts, chunks and rows
        err[k] += (T + B + 64) * sums[k]
    if z is None:
        del out["dz"], err["dz"]
    return out, err


def embed(W, ids, scale=1.0):
    W, ids = _f(W), np.asarray(ids)
    y = np.zeros((*ids.shape, W.shape[1]))
    for k in np.ndindex(*ids.shape):
        if 0 <= ids[k] < len(W):
            y[k] = scale * W[ids[k]]
    return y


def embed_grad(dy, ids, V, scale=1.0, dW=None):
    """``dW`` and the bound of a float32 sum, in units of 2^-24: one rounding a token, one for
    the scale, one for what was there."""
    dy, ids = _f(dy), np.asarray(ids).reshape(-1)
    dy = dy.reshape(len(ids), -1)
    out, mag, count = np.zeros((V, dy.shape[1])), np.zeros((V, dy.shape[1])), np.zeros(V)
    for k, v in enumerate(ids):
        if 0 <= v < V:
            out[v] += dy[k]
            mag[v] += np.abs(dy[k])
            count[v] += 1
    out, bound = scale * out, abs(scale) * mag * (count + 1)[:, None]
    if dW is not None:
        bound += np.where(count[:, None] > 0, np.abs(_f(dW)) + abs(scale) * mag, 0.0)
        out = out + _f(dW)
    return out, bound


def distill_logits(logits, values, ids, scale=None, tau=1.0):
    """``loss [rows], dlogits [rows, V], lse [rows]`` and, for the tolerances, ``q + p``
    spread over the ids ``[rows, V]`` and the largest distance of an exponent from its row's
    largest ``[rows]``."""
    x, values, ids = _f(logits) / tau, _f(values) / tau, np.asarray(ids)
    rows, V = x.shape
    scale = np.ones(rows) if scale is None else _f(scale)
    loss, lse, far, grad, mag = np.zeros(rows), np.zeros(rows), np.zeros(rows), np.zeros((rows, V)), np.zeros((rows, V))
    for b in range(rows):
        slots = [k for k in range(ids.shape[1]) if 0 <= ids[b, k] < V and values[b, k] != -np.inf]
        if not slots or scale[b] == 0:
            continue
        t, at = values[b, slots], ids[b, slots]
        top = t.max()
        logp = t - top - np.log(np.exp(t - top).sum())
        p = np.exp(logp)
        most = x[b].max()
        if most == -np.inf:
            loss[b], lse[b], q = np.inf, -np.inf, np.zeros(V)
        else:
            lse[b] = most + np.log(np.exp(x[b] - most).sum())
            q = np.exp(x[b] - lse[b])
            loss[b] = scale[b] * tau ** 2 * sum(pk * (lp - (x[b, j] - lse[b])) for pk, lp, j in zip(p, logp, at) if pk > 0)
            d = np.concatenate([x[b], t - top + most]) - most
            far[b] = np.abs(d[np.isfinite(d)]).max()
        target = np.zeros(V)
        for pk, j in zip(p, at):
            target[j] += pk
        grad[b], mag[b] = scale[b] * tau * (q - target), q + target
    return loss, grad, lse, mag, far


def verify(drafted, target_p, u, u_last, draft_p=None, lengths=None):
    """``accepted [B], tokens [B, K + 1]``."""
    drafted, target_p, draft_p = np.asarray(drafted), _f(target_p), _f(draft_p)
    B, K = drafted.shape
    V = target_p.shape[2]
    accepted, tokens = np.zeros(B, np.int64), np.full((B, K + 1), -1, np.int64)
    for b, n in enumerate(_lengths(lengths, B, K)):
        m = 0
        while m < n:
            t = drafted[b, m]
            if not 0 <= t < V:
                break
            q = 1.0 if draft_p is None else draft_p[b, m, t]
            if not float(u[b][m]) * q < target_p[b, m, t]:
                break
            tokens[b, m] = t
            m += 1
        accepted[b] = m
        only = np.where(target_p[b, m] > 0, target_p[b, m], 0.0)
        w = only
        if m < n:
            q = np.zeros(V) if draft_p is None else draft_p[b, m]
            if draft_p is None and 0 <= drafted[b, m] < V:
                q[drafted[b, m]] = 1.0
            d = target_p[b, m] - q
            w = np.where(d > 0, d, 0.0)
            if not w.sum() > 0:
                w = only
        c = np.cumsum(w)
        past = np.flatnonzero((c > float(u_last[b]) * c[-1]) & (w > 0))
        some = np.flatnonzero(w > 0)
        tokens[b, m] = past[0] if len(past) else some[-1] if len(some) else -1
    return accepted, tokens
