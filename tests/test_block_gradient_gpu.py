"""GPU parity of the selective scan's gradient where it can go wrong beside the shapes of
``test_block_gpu``: orders that leave wavefronts with empty slots, and inputs that are not
finite.  Tolerances are those derived there.  Values that are not finite are compared by
kind (+inf, -inf, NaN): the inputs of those tests are positive, so that no sum of the
definition meets infinities of both signs by rounding or order.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.block as ob
import paper_2310_18780_amd as lh
from test_block_gpu import device_lengths, dev, gen, host, nan_like, np64, poison, scan_case, U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    lh.lib()
    yield


def outputs(c, G, io):
    B, T, D = c["u"].shape
    N = c["A"].shape[1]
    out = dict(dA=nan_like((D, N)), ddt=nan_like((B, T, D), io), dBm=nan_like((B, T, G, N), io),
               dCm=nan_like((B, T, G, N), io), du=nan_like((B, T, D), io), dh0=nan_like((D,)), ddt_bias=nan_like((D,)))
    if "z" in c:
        out["dz"] = nan_like((B, T, D), io)
    return out


def gradient(c, dy, lengths=None, io="f32"):
    out = outputs(c, c["Bm"].shape[2], io)
    lh.selective_backward(dy=dy, lengths=device_lengths(lengths), **c, **out)
    return out


def roundings(c):
    B, T, D = c["u"].shape
    return 8 * B * T + D + c["A"].shape[1] + 128


def compare(out, ref, mag, k, io="f32"):
    """Finite values within k roundings of their magnitude, the others of the same kind."""
    for name, v in out.items():
        got, want = np64(v), ref[name]
        plain = np.isfinite(want)
        same = np.where(np.isnan(want), np.isnan(got), got == want)
        with np.errstate(invalid="ignore"):
            near = np.abs(got - want) <= k * U * mag[name] + (2.0 ** -8 * np.abs(want) if v.dtype is torch.bfloat16 else 0) + 1e-30
        bad = ~np.where(plain, near, same)
        assert not bad.any(), (name, int(bad.sum()), tuple(np.argwhere(bad)[0]), got[bad][0], want[bad][0])


def reference(c, dy, lengths=None):
    with np.errstate(all="ignore"):
        args = dict(host(c), dy=np64(dy), lengths=lengths)
        return ob.selective_grad(**args), ob.selective_grad(**args, magnitude=True)


# orders whose last wavefronts hold some states or none
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("N", [3, 5, 10, 12, 20, 24, 40, 72])
def test_orders_that_leave_slots_empty(N, gate, io):
    c = scan_case((2, 150, 70, N, 1, None), io, gate, seed=9)
    dy = dev(gen(N).normal(size=(2, 150, 70)), io)
    ref, mag = reference(c, dy)
    out = gradient(c, dy, io=io)
    compare(out, ref, mag, roundings(c), io)
    again = gradient(c, dy, io=io)
    assert all(torch.equal(out[k], again[k]) for k in out)


def positive_case(B, T, D, N, seed, G=1):
    c = scan_case((B, T, D, N, G, None), "f32", seed=seed, strided=False)
    for k in ("Bm", "Cm", "u", "z"):
        c[k] = c[k].abs() + 0.1
    return c, dev(np.abs(gen(seed).normal(size=(B, T, D))) + 0.1)


@pytest.mark.parametrize("where", ["u", "dy"])
@pytest.mark.parametrize("N", [10, 16, 20])
def test_an_infinite_input_with_empty_slots(N, where):
    c, dy = positive_case(2, 128, 70, N, seed=N)
    clean = gradient(c, dy)
    (dy if where == "dy" else c["u"])[1, 70, 5] = float("inf")
    ref, mag = reference(c, dy)
    out = gradient(c, dy)
    compare(out, ref, mag, roundings(c))
    # the other channels and batch row are what they were
    for k in ("ddt", "du", "dz"):
        out[k][1, :, 5] = clean[k][1, :, 5]
        assert torch.equal(out[k], clean[k]), k
    assert torch.equal(out["dBm"][0], clean["dBm"][0]) and torch.equal(out["dCm"][0], clean["dCm"][0])


@pytest.mark.parametrize("at", [37, 69])
@pytest.mark.parametrize("N", [10, 16, 64])
def test_an_infinite_input_leaves_padded_tokens_zero(N, at):
    """Past a row's tokens every gradient is zero, whatever state the row ends in, and an
    input of the last token does not reach dA, which holds states before a token only."""
    lengths = [150, 70, 0]
    c, dy = positive_case(3, 150, 70, N, seed=N)
    c["u"][1, at, 5] = float("inf")
    ref, mag = reference(c, dy, lengths)
    assert np.isfinite(ref["dA"]).all() == (at == 69)
    poison(dict(c, dy=dy), lengths, ["dt", "Bm", "Cm", "u", "z", "dy"])
    out = gradient(c, dy, lengths)
    compare(out, ref, mag, roundings(c))
    for k in ("ddt", "du", "dz", "dBm", "dCm"):
        assert not out[k][1, 70:].any() and not out[k][2].any(), k


@pytest.mark.parametrize("lengths", [None, [200, 70]])
@pytest.mark.parametrize("N", [10, 16])
def test_poles_at_minus_infinity(N, lengths):
    """A state without memory: e^(delta A) = 0.  Only ddt (A times that zero) and its sum
    over tokens are NaN, in that channel."""
    c, dy = positive_case(2, 200, 70, N, seed=N + 1)
    c["A"][7, 3] = -float("inf")
    ref, mag = reference(c, dy, lengths)
    assert all(np.isfinite(ref[k]).all() for k in ("dA", "dBm", "dCm", "du", "dz", "dh0"))
    out = gradient(c, dy, lengths)
    compare(out, ref, mag, roundings(c))


@pytest.mark.parametrize("where", ["u", "dy", "Bm", "Cm"])
@pytest.mark.parametrize("D,G", [(70, 1), (6, 2), (64, 1)])
def test_an_infinite_input_in_a_narrow_tile(D, G, where):
    """Lanes past a group's channels repeat its last channel and add nothing to dBm and dCm,
    also where that channel's state or gradient, or a row of B or C, is infinite."""
    c, dy = positive_case(2, 128, D, 16, seed=D, G=G)
    at = (1, 20, G - 1, 3) if where in ("Bm", "Cm") else (1, 20, D - 1)
    (dy if where == "dy" else c[where])[at] = float("inf")
    ref, mag = reference(c, dy)
    assert not np.isnan(ref["dBm"]).any() and not np.isnan(ref["dCm"]).any()
    compare(gradient(c, dy), ref, mag, roundings(c))


# more chunks than the carry takes at a time (8), and than twice that: 18 of 64 steps, 33 and
# 41 of 32, with states that last over many chunks
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("case", [(1, 1100, 10, 8, 1, None), (2, 1030, 6, 33, 3, [1030, 333]), (1, 1312, 70, 64, 1, None),
                                  (2, 640, 65, 16, 5, [600, 640])], ids=str)
def test_many_chunks_and_slow_poles(case, io):
    B, T, D, N, G, lengths = case
    c = scan_case(case, io, seed=17)
    c["A"] = dev(-np.exp(gen(T).normal(size=(D, N)) - 5))
    dy = dev(gen(T + 2).normal(size=(B, T, D)), io)
    ref, mag = reference(c, dy, lengths)
    if lengths is not None:
        poison(dict(c, dy=dy), lengths, ["dt", "Bm", "Cm", "u", "z", "dy"])
    compare(gradient(c, dy, lengths, io), ref, mag, roundings(c), io)
