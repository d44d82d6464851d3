"""GPU parity of the distillation from a teacher's top logits against the float64 oracle
``oracle.model``.

Tolerances, from the arithmetic, in units of 2^-24.  With R the largest distance of an exponent
from its row's largest (in nats), an exponential has 3 roundings of R, and 4 of its own; a sum
of V of them at most V / 256 + 20 additions deep; q and p, two exponentials and their sums:
k = 8 R + V / 128 + 80.  The gradient is off by k (q + p), the loss by k times 1 + 2 R (each
exponent enters it once more as it is).  From ``lse`` its own rounding is in every q: 4 |lse|
more.  A bfloat16 gradient adds its rounding, 2^-8 of the value."""
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


def nan_like(shape, io="f32"):
    return torch.full(shape, float("nan"), dtype=IO[io], device="cuda")


def np64(t):
    return t.detach().double().cpu().numpy()


def case(rows, V, K, io, seed=0, masked=True):
    r = gen(seed + rows + V + K)
    c = dict(logits=dev(3 * r.normal(size=(rows, V)) + 10, io), values=dev(2 * r.normal(size=(rows, K)) - 20),
             ids=torch.from_numpy(np.stack([r.permutation(max(V, K))[:K] for _ in range(rows)]).astype(np.int32)).cuda())
    if masked:
        scale = r.uniform(0.2, 2, rows)
        scale[r.random(rows) < 0.3] = 0
        c["scale"] = dev(scale)
        c["values"][torch.from_numpy(r.random((rows, K)) < 0.1).cuda()] = float("-inf")
        c["ids"][torch.from_numpy(r.random((rows, K)) < 0.1).cuda()] = -1
        c["ids"][rows // 2] = -7  # no entry at all
    return c


def reference(c, tau, up=None):
    scale = np64(c["scale"]) if "scale" in c else np.ones(len(c["logits"]))
    out = om.distill_logits(np64(c["logits"]), np64(c["values"]), c["ids"].cpu().numpy(), scale, tau)
    loss, grad, lse, mag, far = out
    k = 8 * far + c["logits"].shape[1] / 128 + 80
    size = scale * tau
    if up is not None:
        grad, size = grad * up[:, None], np.abs(size * up)
        k = k + 4 * np.where(np.isfinite(lse), np.abs(lse), 0)  # (minus infinity is not rounded)
    return loss, grad, lse, (scale * tau ** 2 * k * (1 + 2 * far)), (k * size)[:, None] * mag, k


def check(got, ref, units, io, name):
    got = np64(got)
    tol = units * U + (2.0 ** -8 * (np.abs(ref) + units * U) if io == "bf16" else 0) + 1e-30
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, bad.sum(), np.argwhere(bad)[0], got[bad][0], ref[bad][0], tol[bad][0])


# a value to a row, ragged pieces, every count of pieces that a workgroup of 256 and of 1024 holds, and rows that none holds
SIZES = [(1, 1, 1), (3, 7, 3), (5, 64, 64), (9, 300, 5), (4, 2047, 13), (4, 4099, 300), (3, 9001, 40), (2, 17003, 64), (3, 32003, 13),
         (2, 50001, 64), (2, 70003, 1024), (1, 131075, 8), (2, 200007, 33)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_loss_and_gradient(size, io):
    rows, V, K = size
    for tau, masked in ((1.0, rows > 1), (2.5, False)):
        c = case(rows, V, K, io, masked=masked)
        loss, lse, grad = nan_like((rows,)), nan_like((rows,)), nan_like((rows, V), io)
        lh.distill_logits(loss=loss, lse=lse, dlogits=grad, tau=tau, **c)
        rl, rg, rs, tl, tg, k = reference(c, tau)
        check(loss, rl, tl, "f32", "loss")
        check(lse, rs, k + 4 * np.abs(rs), "f32", "lse")
        check(grad, rg, tg, io, "dlogits")
        # the loss alone, and the gradient from lse
        again, up = nan_like((rows,)), gen(1).normal(size=rows)
        lse2 = nan_like((rows,))
        lh.distill_logits(loss=again, lse=lse2, tau=tau, **c)
        check(again, rl, tl, "f32", "loss alone")
        lh.distill_logits_backward(dev(up), lse=lse2, dlogits=grad.fill_(float("nan")), tau=tau, **c)
        _, rg, _, _, tg, _ = reference(c, tau, np64(dev(up)))
        check(grad, rg, tg, io, "dlogits from lse")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("V", [33, 5003, 140001])
def test_in_place_and_rows_that_lie_apart(V, io):
    rows, K = 5, 9
    c = case(rows, V, K, io, seed=3)
    want, loss = nan_like((rows, V), io), nan_like((rows,))
    lh.distill_logits(loss=loss, dlogits=want, **c)
    wide = nan_like((rows, V + 5), io)
    wide[:, 1:V + 1] = c["logits"]
    c["logits"] = wide[:, 1:V + 1]
    out, l2 = nan_like((rows, V + 3), io), nan_like((rows,))
    lh.distill_logits(loss=l2, dlogits=out[:, 2:V + 2], **c)
    assert torch.equal(out[:, 2:V + 2], want) and torch.equal(l2, loss)
    assert torch.isnan(out[:, :2]).all() and torch.isnan(out[:, V + 2:]).all()
    lse = nan_like((rows,))
    lh.distill_logits(loss=l2, lse=lse, **c)
    one = dev(np.ones(rows))
    apart = nan_like((rows, V), io)
    lh.distill_logits_backward(one, lse=lse, dlogits=apart, **c)
    kept = wide.clone()
    lh.distill_logits_backward(one, lse=lse, dlogits=c["logits"], **c)
    assert torch.equal(wide[:, 1:V + 1], apart)
    wide.copy_(kept)
    lh.distill_logits(loss=l2, dlogits=c["logits"], **c)
    assert torch.equal(wide[:, 1:V + 1], want)
    assert torch.isnan(wide[:, 0]).all() and torch.isnan(wide[:, V + 1:]).all()


def test_rows_that_take_no_part_are_not_read():
    rows, V, K = 6, 1000, 4
    c = case(rows, V, K, "f32", masked=False)
    c["scale"] = dev([1, 0, 1, 0, 1, 1])
    c["logits"][1] = float("nan")
    c["logits"][3] = float("inf")
    c["ids"][4] = V
    c["logits"][4] = float("nan")
    loss, lse, grad = nan_like((rows,)), nan_like((rows,)), nan_like((rows, V))
    lh.distill_logits(loss=loss, lse=lse, dlogits=grad, **c)
    for b in (1, 3, 4):
        assert loss[b] == 0 and lse[b] == 0 and not grad[b].any()
    assert torch.isfinite(loss).all() and torch.isfinite(grad).all() and loss[0] != 0
    lh.distill_logits_backward(dev(np.ones(rows)), lse=lse, dlogits=grad.fill_(7), **c)
    assert not grad[[1, 3, 4]].any() and torch.isfinite(grad).all()
    # no rows at all
    lh.distill_logits(c["logits"][:0], c["values"][:0], c["ids"][:0], loss[:0], dlogits=grad[:0])


@pytest.mark.parametrize("V", [40, 3001, 150001])
def test_ids_given_twice_and_logits_of_minus_infinity(V):
    c = dict(logits=dev(gen(1).normal(size=(5, V))), values=dev([[0, 1, 2, 3]] * 5),
             ids=torch.tensor([[5, 5, 5, 5], [V - 1, 2, V - 1, 2], [0, 1, 2, 3], [3, 2, 1, 0], [1, 1, 2, -1]], dtype=torch.int32, device="cuda"))
    c["logits"][2, 10:] = float("-inf")
    c["logits"][3] = float("-inf")  # nothing to answer with: the loss is infinite, q is 0
    c["values"][3, 0] = float("-inf")
    loss, lse, grad = nan_like((5,)), nan_like((5,)), nan_like((5, V))
    lh.distill_logits(loss=loss, lse=lse, dlogits=grad, **c)
    rl, rg, rs, tl, tg, k = reference(c, 1.0)
    ok = [0, 1, 2, 4]
    check(loss[ok], rl[ok], tl[ok], "f32", "loss")
    assert loss[3] == float("inf") and lse[3] == float("-inf")
    check(grad, rg, tg, "f32", "dlogits")
    lh.distill_logits_backward(dev(np.ones(5)), lse=lse, dlogits=grad.fill_(float("nan")), **c)
    _, rg, _, _, tg, _ = reference(c, 1.0, np.ones(5))
    check(grad, rg, tg, "f32", "dlogits from lse")
    # a logit of minus infinity that the teacher asks for
    c["logits"][0, 5] = float("-inf")
    lh.distill_logits(loss=loss, dlogits=grad, **c)
    # (the four slots' p are all: the same four numbers are added in two orders, three roundings each, and divided)
    assert loss[0] == float("inf") and abs(grad[0, 5].item() + 1) <= 8 * U
    # NaN, on either side, is its row's alone
    c["logits"][0, 5] = 0
    c["logits"][1, 7], c["values"][4, 1] = float("nan"), float("nan")
    lh.distill_logits(loss=loss, dlogits=grad, **c)
    assert torch.isnan(loss[[1, 4]]).all() and torch.isnan(grad[1]).all() and torch.isnan(grad[4]).any()
    assert torch.isfinite(loss[[0, 2]]).all() and torch.isfinite(grad[[0, 2]]).all()


def test_large_and_equal_logits():
    V = 5000
    c = dict(logits=dev([[1e4] * V, [-1e4] * V, [3e38] * V, [0.0] * V]), values=dev([[1e4, 1e4]] * 2 + [[-3e38, -3e38], [0, 0]]),
             ids=torch.tensor([[0, V - 1]] * 4, dtype=torch.int32, device="cuda"))
    c["logits"][2] = 1e37
    loss, grad = nan_like((4,)), nan_like((4, V))
    lh.distill_logits(loss=loss, dlogits=grad, **c)
    want = np.log(0.5) + np.log(V)
    assert np.allclose(np64(loss), want, rtol=0, atol=(V / 128 + 80 + 4 * want) * U)
    assert np.allclose(np64(grad[:, 1:-1]), 1 / V, rtol=(V / 128 + 80) * U)
    assert np.allclose(np64(grad[:, [0, -1]]), 1 / V - 0.5, rtol=(V / 128 + 80) * U)


def test_gradient_against_differences():
    rows, V, K = 3, 500, 20
    c = case(rows, V, K, "f32", seed=9, masked=False)
    c["logits"] -= 10  # (so that the steps below are exact in most places)
    loss, grad, d = nan_like((rows,)), nan_like((rows, V)), dev(gen(2).normal(size=(rows, V)))
    lh.distill_logits(loss=loss, dlogits=grad, tau=1.5, **c)
    base = dict(c)
    val = []
    for h in (2.0 ** -5, 2.0 ** -6):
        pair = []
        for s in (h, -h):
            lh.distill_logits(loss=loss, tau=1.5, **{**base, "logits": c["logits"] + s * d})
            pair.append(np64(loss))
        val.append((pair[0] - pair[1]) / (2 * h))
    slope = (np64(grad) * np64(d)).sum(1)
    best = (4 * val[1] - val[0]) / 3
    _, _, _, tl, _, _ = reference(c, 1.5)
    # each loss is off by its bound, divided by the step; what the two steps' extrapolation leaves is a sixteenth of their difference
    assert (np.abs(best - slope) <= 3 * tl * U / 2.0 ** -6 + np.abs(val[1] - val[0]) / 8 + 1e-6).all(), (best, slope)


def test_offsets_past_32_bits():
    rows, V = 17000, 131101
    c = dict(logits=torch.zeros((rows, V), dtype=torch.bfloat16, device="cuda"), values=torch.zeros((rows, 1), device="cuda"),
             ids=torch.full((rows, 1), V - 1, dtype=torch.int32, device="cuda"))
    assert rows * V > 1 << 31
    loss = nan_like((rows,))
    lh.distill_logits(loss=loss, dlogits=c["logits"], **c)
    want = np.log(V)
    assert abs(loss[-1].item() - want) <= (V / 128 + 80 + 4 * want) * U and torch.equal(loss, loss[:1].expand(rows))
    assert c["logits"][-1, -1].item() == torch.tensor(1 / V - 1).bfloat16().item()
    assert torch.equal(c["logits"][-1, :-1], torch.full((V - 1,), 1 / V, device="cuda").bfloat16())
