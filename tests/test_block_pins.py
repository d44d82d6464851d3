"""Pins of the selective block's oracle (``oracle/block.py``): library routes, closed
forms, and gradients against differences of the forward functions."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.block as ob


def rng(seed=0):
    return np.random.default_rng(seed)


def test_layer_norm_against_torch():
    r = rng()
    x, res, w, b = r.normal(size=(5, 37)), r.normal(size=(5, 37)), r.normal(size=37), r.normal(size=37)
    y, total, mean, rstd = ob.layer_norm(x, w, b, res, eps=1e-3)
    ref = torch.nn.functional.layer_norm(torch.tensor(x + res), (37,), torch.tensor(w), torch.tensor(b), 1e-3)
    assert np.allclose(y, ref.numpy(), rtol=1e-12, atol=1e-12)
    assert np.allclose(total, x + res) and np.allclose(mean, (x + res).mean(1))
    assert np.allclose(rstd, 1 / np.sqrt((x + res).var(1) + 1e-3))


def test_short_conv_against_torch():
    r = rng(1)
    x, w, b = r.normal(size=(2, 11, 3)), r.normal(size=(3, 4)), r.normal(size=3)
    y, state = ob.short_conv(x, w, b, True)
    xt = torch.nn.functional.pad(torch.tensor(x).transpose(1, 2), (3, 0))
    o = torch.nn.functional.conv1d(xt, torch.tensor(w)[:, None], torch.tensor(b), groups=3)
    assert np.allclose(y, torch.nn.functional.silu(o).transpose(1, 2).numpy(), rtol=1e-12, atol=1e-12)
    assert np.array_equal(state, x[:, -3:])


def test_short_conv_in_two_parts_and_ragged():
    r = rng(2)
    x, w = r.normal(size=(2, 9, 3)), r.normal(size=(3, 4))
    y, state = ob.short_conv(x, w, None, False)
    y1, s1 = ob.short_conv(x[:, :2], w, None, False)
    y2, s2 = ob.short_conv(x[:, 2:], w, None, False, state=s1)
    assert np.allclose(np.concatenate([y1, y2], 1), y) and np.array_equal(s2, state)
    yr, sr = ob.short_conv(x, w, None, False, lengths=[9, 2])
    assert np.allclose(yr[1, :2], y[1, :2]) and not yr[1, 2:].any()
    assert np.array_equal(sr[1], np.concatenate([np.zeros((1, 3)), x[1, :2]]))


def test_selective_constant_input_is_a_geometric_series():
    # constant steps, inputs and outputs: x_t = delta B u (1 - a^t) / (1 - a)
    T, a_log, step = 40, -1.5, 0.3
    one = np.ones((1, T, 1))
    dt = np.full((1, T, 1), np.log(np.expm1(step)))
    y, x = ob.selective(np.array([[a_log]]), dt, 2.0 * one[..., None], 0.5 * one[..., None], 3.0 * one, h0=np.array([0.25]))
    a = np.exp(step * a_log)
    t = np.arange(1, T + 1)
    states = step * 2.0 * 3.0 * (1 - a ** t) / (1 - a)
    assert np.allclose(y[0, :, 0], 0.5 * states + 0.75, rtol=1e-12)
    assert np.allclose(x[0, 0, 0], states[-1], rtol=1e-12)


def test_selective_zero_decay_is_a_cumulative_sum():
    r = rng(3)
    B, T, D, N, G = 2, 13, 4, 3, 2
    dt, u = r.normal(size=(B, T, D)), r.normal(size=(B, T, D))
    Bm, Cm = r.normal(size=(B, T, G, N)), r.normal(size=(B, T, G, N))
    y, x = ob.selective(np.zeros((D, N)), dt, Bm, Cm, u)
    v = (np.log1p(np.exp(dt)) * u)[..., None] * np.repeat(Bm, 2, 2)
    states = np.cumsum(v, 1)
    assert np.allclose(x, states[:, -1]) and np.allclose(y, (states * np.repeat(Cm, 2, 2)).sum(-1))


def selective_case(seed=4, B=2, T=6, D=4, N=3, G=2):
    r = rng(seed)
    return dict(A=-np.exp(r.normal(size=(D, N))), dt=r.normal(size=(B, T, D)), Bm=r.normal(size=(B, T, G, N)),
                Cm=r.normal(size=(B, T, G, N)), u=r.normal(size=(B, T, D)), h0=r.normal(size=D),
                dt_bias=r.normal(size=D), z=r.normal(size=(B, T, D)))


def differences(f, x, eps=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        v = x[i]
        x[i] = v + eps
        hi = f()
        x[i] = v - eps
        lo = f()
        x[i] = v
        g[i] = (hi - lo) / (2 * eps)
    return g


@pytest.mark.parametrize("lengths", [None, [6, 2], [0, 5]])
def test_selective_gradient_against_differences(lengths):
    c = selective_case()
    dy = rng(5).normal(size=c["u"].shape)
    g = ob.selective_grad(dy, **c, lengths=lengths)
    f = lambda: (ob.selective(**c, lengths=lengths)[0] * dy).sum()  # noqa: E731
    for k in c:
        # central differences: truncation eps^2 and cancellation 1e-16 / eps, both below 1e-8
        assert np.allclose(g["d" + k], differences(f, c[k]), rtol=1e-6, atol=1e-7), k


def test_selective_gradient_in_a_case_by_hand():
    # one channel, one state, one step: y = C delta B u + h0 u
    one = lambda v: np.array([[[v]]])  # noqa: E731
    step = np.log1p(np.exp(0.2))
    g = ob.selective_grad(one(1.0), np.array([[-1.0]]), one(0.2), one(3.0)[..., None], one(5.0)[..., None], one(7.0),
                          h0=np.array([0.5]))
    assert np.isclose(g["du"][0, 0, 0], step * 15 + 0.5)
    assert np.isclose(g["dBm"][0, 0, 0, 0], 5 * step * 7) and np.isclose(g["dCm"][0, 0, 0, 0], step * 21)
    assert np.isclose(g["ddt"][0, 0, 0], 5 * 3 * 7 / (1 + np.exp(-0.2))) and g["dA"][0, 0] == 0


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("lengths", [None, [5, 0]])
def test_short_conv_gradient_against_differences(silu, lengths):
    r = rng(6)
    c = dict(x=r.normal(size=(2, 5, 3)), w=r.normal(size=(3, 4)), bias=r.normal(size=3))
    dy = r.normal(size=(2, 5, 3))
    g = ob.short_conv_grad(dy, **c, silu=silu, lengths=lengths)
    f = lambda: (ob.short_conv(**c, silu=silu, lengths=lengths)[0] * dy).sum()  # noqa: E731
    for k, v in zip(("x", "w", "bias"), g):
        assert np.allclose(v, differences(f, c[k]), rtol=1e-6, atol=1e-7), k


def test_layer_norm_gradient_against_differences():
    r = rng(7)
    c = dict(x=r.normal(size=(3, 7)), w=r.normal(size=7), b=r.normal(size=7))
    dy = r.normal(size=(3, 7))
    _, _, mean, rstd = ob.layer_norm(**c)
    g = ob.layer_norm_grad(dy, c["x"], c["w"], mean, rstd)
    f = lambda: (ob.layer_norm(**c)[0] * dy).sum()  # noqa: E731
    for k, v in zip(("x", "w", "b"), g):
        assert np.allclose(v, differences(f, c[k]), rtol=1e-6, atol=1e-7), k
    d = r.normal(size=(3, 7))
    assert np.allclose(ob.layer_norm_grad(dy, c["x"], c["w"], mean, rstd, d)[0], g[0] + d)


def test_a_planted_mistake_is_caught(monkeypatch):
    # the decay of the step after, in place of the step's own
    c = selective_case()
    y, _ = ob.selective(**c)
    shifted = dict(c, dt=np.roll(c["dt"], -1, axis=1))
    assert not np.allclose(ob.selective(**shifted)[0], y, rtol=1e-3)
    # magnitudes bound the values
    ym, xm = ob.selective(**c, magnitude=True)
    assert (np.abs(y) <= ym + 1e-12).all()
    dy = rng(8).normal(size=c["u"].shape)
    g, gm = ob.selective_grad(dy, **c), ob.selective_grad(dy, **c, magnitude=True)
    for k in g:
        assert (np.abs(g[k]) <= gm[k] + 1e-12).all(), k
