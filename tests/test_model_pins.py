"""Pins of the oracle ``oracle.model``: closed forms, library routines, differences and
distributions."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.model as om


def gen(seed):
    return np.random.default_rng(seed)


def gated_case(B, T, D, seed=0, z=True):
    r = gen(seed)
    c = dict(rate=np.exp(r.uniform(-5, 1, D)), r_bias=r.normal(size=D), i_bias=r.normal(size=D))
    c.update({k: r.normal(size=(B, T, D)) for k in ("r", "i", "u")})
    if z:
        c["z"] = r.normal(size=(B, T, D))
    return c


def torch_gated(c, state, lengths):
    B, T, D = c["u"].shape
    h, ys = state, []
    for t in range(T):
        f = torch.sigmoid(c["r"][:, t] + c["r_bias"])
        p = torch.sigmoid(c["i"][:, t] + c["i_bias"])
        a = torch.exp(-c["rate"] * f)
        new = a * h + torch.sqrt(1 - a * a) * p * c["u"][:, t]
        live = torch.as_tensor(lengths)[:, None] > t
        h = torch.where(live, new, h)
        y = h * torch.nn.functional.silu(c["z"][:, t]) if "z" in c else h
        ys.append(torch.where(live, y, torch.zeros_like(y)))
    return torch.stack(ys, 1), h


@pytest.mark.parametrize("z", [False, True])
def test_gated_and_gradients_against_autograd(z):
    B, T, D = 3, 9, 4
    c = gated_case(B, T, D, 1, z)
    lengths = [9, 5, 0]
    state, dy, dlast = gen(2).normal(size=(B, D)), gen(3).normal(size=(B, T, D)), gen(4).normal(size=(B, D))
    t = {k: torch.tensor(v, requires_grad=True) for k, v in c.items()}
    s = torch.tensor(state, requires_grad=True)
    y, h = torch_gated(t, s, lengths)
    ((y * torch.tensor(dy)).sum() + (h * torch.tensor(dlast)).sum()).backward()
    oy, oh = om.gated(**c, state=state, lengths=lengths)[:2]
    assert np.allclose(oy, y.detach().numpy(), atol=1e-13) and np.allclose(oh, h.detach().numpy(), atol=1e-13)
    out, err = om.gated_grad(dy, **c, state=state, lengths=lengths, dlast=dlast)
    for k, name in (("drate", "rate"), ("dr", "r"), ("di", "i"), ("du", "u"), ("dr_bias", "r_bias"), ("di_bias", "i_bias"),
                    ("dz", "z")):
        if name in t:
            assert np.allclose(out[k], t[name].grad.numpy(), atol=1e-11), k
    assert np.allclose(out["dfirst"], s.grad.numpy(), atol=1e-12)
    assert set(out) == set(err)


def test_gated_gradients_against_differences():
    c = gated_case(1, 6, 2, 5)
    dy = gen(6).normal(size=(1, 6, 2))
    out, _ = om.gated_grad(dy, **c)
    eps = 1e-6
    for k in ("rate", "r", "u", "z"):
        for at in [tuple(gen(7).integers(0, s) for s in c[k].shape)]:
            lo, hi = ({**c, k: c[k].copy()} for _ in range(2))
            lo[k][at] -= eps
            hi[k][at] += eps
            num = ((om.gated(**hi)[0] - om.gated(**lo)[0]) * dy).sum() / (2 * eps)
            assert abs(num - out["d" + k][at]) < 1e-7 * (1 + abs(num))


def test_gated_closed_forms():
    # gates at 1/2, constant input: h_t = g p u (1 - a^t) / (1 - a)
    D, T = 3, 40
    rate = np.array([0.1, 1.0, 3.0])
    zero = np.zeros((1, T, D))
    y, h, *_ = om.gated(rate, zero, zero, zero + 2.0)
    a = np.exp(-rate / 2)
    for t in (0, 1, 7, T - 1):
        assert np.allclose(y[0, t], np.sqrt(1 - a * a) * 0.5 * 2.0 * (1 - a ** (t + 1)) / (1 - a), rtol=1e-12)
    # rate 0 holds its state and takes no input
    y, h, *_ = om.gated(np.zeros(D), zero, zero, zero + 2.0, state=np.full((1, D), 5.0))
    assert (y == 5.0).all() and (h == 5.0).all()
    # unit noise in, at most unit variance out
    r = gen(8)
    u = r.normal(size=(1, 4000, 64))
    y = om.gated(np.full(64, 0.2), np.zeros_like(u), np.full_like(u, 50.0), u)[0]
    assert abs(y[0, 500:].var() - 1.0) < 0.05


def test_gated_bounds_hold_for_a_float32_evaluation():
    c = {k: v.astype(np.float32) for k, v in gated_case(2, 50, 8, 9).items()}
    y, h, ey, eh, *_ = om.gated(**c)
    t = {k: torch.tensor(v) for k, v in c.items()}
    ty, th = torch_gated(t, torch.zeros(2, 8), [50, 50])
    assert (np.abs(ty.numpy() - y) <= ey * 2.0 ** -24).all() and (np.abs(th.numpy() - h) <= eh * 2.0 ** -24).all()


def test_embedding_against_the_library():
    r = gen(10)
    W, ids, dy = r.normal(size=(7, 5)), np.array([[3, 3, -1], [6, 0, 7]]), r.normal(size=(2, 3, 5))
    t = torch.tensor(W, requires_grad=True)
    inside = torch.tensor((ids >= 0) & (ids < 7))[..., None]
    y = 3.0 * torch.nn.functional.embedding(torch.tensor(ids).clamp(0, 6), t) * inside
    (y * torch.tensor(dy)).sum().backward()
    assert np.allclose(om.embed(W, ids, 3.0), y.detach().numpy())
    assert np.allclose(om.embed_grad(dy, ids, 7, 3.0)[0], t.grad.numpy())
    assert np.allclose(om.embed_grad(dy, ids, 7, 3.0, W)[0], W + t.grad.numpy())


@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distillation_against_the_library(tau):
    r = gen(11)
    rows, V, K = 4, 9, 3
    x = torch.tensor(r.normal(size=(rows, V)), requires_grad=True)
    values, scale = r.normal(size=(rows, K)), np.array([1.0, 0.5, 0.0, 2.0])
    ids = np.stack([r.permutation(V)[:K] for _ in range(rows)])
    ids[3, 1] = -1
    loss, grad, lse, *_ = om.distill_logits(x.detach().numpy(), values, ids, scale, tau)
    t = torch.tensor(values).masked_fill(torch.tensor(ids < 0), float("-inf")) / tau
    full = torch.full((rows, V), float("-inf"), dtype=torch.float64).scatter(1, torch.tensor(ids).clamp(min=0), t)
    full[3] = float("-inf")
    for k in (0, 2):
        full[3, ids[3, k]] = t[3, k]
    kl = torch.nn.functional.kl_div(torch.log_softmax(x / tau, -1), torch.log_softmax(full, -1), log_target=True,
                                    reduction="none")
    kl = torch.where(full > float("-inf"), kl, torch.zeros_like(kl)).sum(-1) * torch.tensor(scale) * tau ** 2
    assert np.allclose(loss, kl.detach().numpy())
    kl.sum().backward()
    assert np.allclose(grad, x.grad.numpy())
    assert np.allclose(lse, torch.logsumexp(x / tau, -1).detach().numpy() * (scale != 0))


def test_distillation_of_an_id_given_twice_and_of_empty_rows():
    x = np.zeros((3, 4))
    x[1] = -np.inf
    values = np.array([[0.0, 0.0], [0.0, -np.inf], [1.0, 1.0]])
    ids = np.array([[2, 2], [1, 0], [-1, 9]])
    loss, grad, *_ = om.distill_logits(x, values, ids)
    assert np.allclose(loss[0], np.log(0.5) + np.log(4)) and np.allclose(grad[0], [0.25, 0.25, -0.75, 0.25])
    assert loss[1] == np.inf and np.allclose(grad[1], [0, -1, 0, 0])
    assert loss[2] == 0 and not grad[2].any()


def test_verification_by_hand():
    p = np.array([[[0.5, 0.25, 0.25], [0.0, 1.0, 0.0], [0.25, 0.25, 0.5]]])
    q = np.array([[[0.25, 0.5, 0.25], [0.5, 0.5, 0.0]]])
    ok = lambda d, u, last, **kw: [v.tolist() for v in om.verify([d], p, [u], [last], q, **kw)]  # noqa: E731
    assert ok([0, 1], [0.99, 0.99], 0.0) == [[2], [[0, 1, 0]]]   # p >= q at both
    assert ok([0, 1], [0.99, 0.99], 0.6) == [[2], [[0, 1, 2]]]
    assert ok([1, 1], [0.5, 0.0], 0.9) == [[0], [[0, -1, -1]]]   # 1/2 q is not less than p; what is left is token 0
    assert ok([1, 1], [0.49, 0.0], 0.9) == [[2], [[1, 1, 2]]]
    assert ok([0, 0], [0.0, 0.0], 0.3) == [[1], [[0, 1, -1]]]    # p = 0 is never accepted
    assert ok([0, 5], [0.0, 0.0], 0.3) == [[1], [[0, 1, -1]]]
    assert ok([0, 1], [0.0, 0.0], 0.3, lengths=[0]) == [[0], [[0, -1, -1]]]
    assert ok([0, 1], [0.0, 0.0], 0.7, lengths=[1]) == [[1], [[0, 1, -1]]]
    # a certain draft: accepted with p, else another token
    a, t = om.verify([[0, 1]], p, [[0.6, 0.0]], [0.1])
    assert a.tolist() == [0] and t.tolist() == [[1, -1, -1]]


@pytest.mark.parametrize("certain", [False, True])
def test_verification_keeps_the_targets_distribution(certain):
    r = gen(12)
    V, N = 5, 40000
    p, q = r.dirichlet(np.ones(V)), r.dirichlet(np.ones(V))
    if certain:
        q = np.eye(V)[2]
    drafted = r.choice(V, size=(N, 1), p=q)
    tile = lambda x, k: np.broadcast_to(x, (N, k, V))  # noqa: E731
    _, tokens = om.verify(drafted, tile(p, 2), r.random((N, 1)), r.random(N), None if certain else tile(q, 1))
    freq = np.bincount(tokens[:, 0], minlength=V) / N
    # five standard deviations of a frequency
    assert np.abs(freq - p).max() < 5 * 0.5 / np.sqrt(N)
