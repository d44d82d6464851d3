"""The gradient of the distillation from ``lse`` where the logits lie far from zero, as exact as the
one-call form: a float32 ``lse`` holds no more than 2^-24 of its own size, which is an error of
that size in every exponent.

Tolerances as in ``test_distill_logits_gpu.py``, with R the largest distance of an exponent from its
row's largest: k = 8 R + V / 128 + 80 units of 2^-24 of q + p.  Only where |lse| is 16 or less, and
is taken as it is, do its own rounding and those of its product and of the logits' scale add
5 |lse|, 80 units at most."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.model as om
import paper_2310_18780_amd as lh

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
IO = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    lh.lib()
    yield


def gen(seed):
    return np.random.default_rng(seed)


def dev(a, io="f32"):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.float32))).to(IO[io]).cuda()


def np64(t):
    return t.detach().double().cpu().numpy()


def nan_like(shape, io="f32"):
    return torch.full(shape, float("nan"), dtype=IO[io], device="cuda")


def check_gradient(c, io, tau, up, in_place=False):
    rows, V = c["logits"].shape
    loss, lse = nan_like((rows,)), nan_like((rows,))
    lh.distill_logits(loss=loss, lse=lse, tau=tau, **c)
    _, grad, rlse, mag, far = om.distill_logits(np64(c["logits"]), np64(c["values"]), c["ids"].cpu().numpy(), None, tau)
    got = c["logits"] if in_place else nan_like((rows, V), io)
    lh.distill_logits_backward(dev(up), lse=lse, dlogits=got, tau=tau, **c)
    up = np64(dev(up))
    near = np.where(np.abs(rlse) <= 16 + 1e-3, np.abs(rlse), 0)
    k = 8 * far + V / 128 + 80 + 5 * near
    ref = grad * up[:, None]
    tol = (k * tau * np.abs(up))[:, None] * mag * U
    if io == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    bad = ~(np.abs(np64(got) - ref) <= tol + 1e-30)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[0], np64(got)[bad][0], ref[bad][0], tol[bad][0])


# (columns, slots): rows that a workgroup of 256 and of 1024 holds, of every count of pieces, and rows that none holds
SIZES = [(1, 1), (7, 3), (300, 5), (4099, 300), (9001, 40), (32003, 13), (50001, 64), (70003, 8), (200007, 33)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient_of_logits_far_from_zero(size, io):
    V, K = size
    r = gen(V + K)
    # (as bfloat16 the far rows are steps of up to 64: most of their values are equal)
    off = np.array([0.0, 17.0, -30.0, 100.0, -1e3, 1e4])
    x = 2 * r.normal(size=(len(off), V)) + off[:, None]
    ids = np.stack([r.permutation(V)[:K] for _ in off]).astype(np.int32)
    c = dict(logits=dev(x, io), values=dev(2 * r.normal(size=(len(off), K)) + off[:, None]), ids=torch.from_numpy(ids).cuda())
    for tau, in_place in ((1.0, False), (0.125, False), (2.5, True)):
        check_gradient({**c, "logits": c["logits"].clone()}, io, tau, r.normal(size=len(off)), in_place)


@pytest.mark.parametrize("V", [500, 5000, 150001])
def test_large_and_equal_logits(V):
    rows = [1e4, -1e4, 1e37, -1e37, 0.0]
    n = len(rows)
    c = dict(logits=dev([[x] * V for x in rows]), values=dev([[x, x] for x in rows]),
             ids=torch.tensor([[0, V - 1]] * n, dtype=torch.int32, device="cuda"))
    loss, lse, grad = nan_like((n,)), nan_like((n,)), nan_like((n, V))
    lh.distill_logits(loss=loss, lse=lse, **c)
    lh.distill_logits_backward(dev([1, 1, 1, 1, 1]), lse=lse, dlogits=grad, **c)
    units = V / 128 + 80 + np.array([0, 0, 0, 0, 5 * np.log(V)])[:, None]
    got = np64(grad)
    assert (np.abs(got[:, 1:-1] * V - 1) <= units * U).all(), np.abs(got[:, 1:-1] * V - 1).max(1)
    assert (np.abs(got[:, [0, -1]] - (1 / V - 0.5)) <= units * U * (1 / V + 0.5)).all()


def test_logits_without_a_finite_one_and_infinities():
    V = 3000
    c = dict(logits=dev(gen(1).normal(size=(4, V)) + 200), values=dev([[0, 1]] * 4),
             ids=torch.tensor([[5, 7]] * 4, dtype=torch.int32, device="cuda"))
    c["logits"][0] = float("-inf")
    c["logits"][1, 9:] = float("-inf")
    c["logits"][2, 100] = float("nan")
    loss, lse, grad = nan_like((4,)), nan_like((4,)), nan_like((4, V))
    lh.distill_logits(loss=loss, lse=lse, dlogits=grad, **c)
    apart = nan_like((4, V))
    lh.distill_logits_backward(dev([1, 1, 1, 1]), lse=lse, dlogits=apart, **c)
    for b in (0, 1, 3):  # the same steps as in the one-call form
        assert torch.equal(apart[b], grad[b])
    assert torch.isnan(apart[2]).all()
