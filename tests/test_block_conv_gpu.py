"""GPU tests of the short convolution beside ``test_block_gpu``, whose tolerances they take."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.block as ob
import paper_2310_18780_amd as lh
from test_block_gpu import check, dev, device_lengths, gen, nan_like, np64, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    lh.lib()
    yield


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_one_tap_needs_no_state(io):
    B, T, D = 2, 9, 37
    r = gen(60)
    x, w, bias = dev(r.normal(size=(B, T, D)), io), dev(r.normal(size=(D, 1))), dev(r.normal(size=D))
    ref, _ = ob.short_conv(np64(x), np64(w), np64(bias), True)
    mag, _ = ob.short_conv(np64(x), np64(w), np64(bias), True, magnitude=True)
    y = nan_like((B, T, D), io)
    lh.short_conv_prefill(x, w, bias, None, y)
    check(y, ref, mag, 17, io, "y")
    y_t = nan_like((B, D), io)
    lh.short_conv_step(x[:, 4], w, bias, None, y_t)
    check(y_t, ref[:, 4], mag[:, 4], 17, io, "y_t")
    two = dev(r.normal(size=(D, 2)))
    for call in (lambda: lh.short_conv_prefill(x, two, bias, None, y), lambda: lh.short_conv_step(x[:, 4], two, bias, None, y_t)):
        with pytest.raises(TypeError, match="state"):
            call()


# Time steps are walked in runs of 4 to 64, longer ones where there are more threads.  With
# float32 these walk 16, 32, 64 and, with 6 taps, 64 steps (gradients too); bfloat16 holds
# twice the channels to a thread: 4, 8, 64 and 64 steps (gradients 4, 8, 32 and 32).  The last
# run of a row is shorter each time.
RUNS = [(16, 70, 3279, 4), (32, 70, 2731, 4), (192, 66, 2045, 4), (100, 66, 2045, 6)]


def ragged(B, T):
    n = np.random.default_rng(B).integers(0, T + 1, size=B)
    n[0], n[1], n[B // 2] = T, 0, 1
    return n.tolist()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("case", RUNS, ids=str)
def test_runs_of_every_length(case, io):
    B, T, D, K = case
    r = gen(B + D)
    lengths = ragged(B, T) if K == 4 else None
    f = lambda *s: r.standard_normal(size=s, dtype=np.float32)  # noqa: E731
    x, w, bias, state = rows(f(B, T, D), io), dev(f(D, K)), dev(f(D)), dev(f(B, K - 1, D), io)
    args = dict(x=np64(x), w=np64(w), bias=np64(bias), silu=True, state=np64(state), lengths=lengths)
    ref, sref = ob.short_conv(**args)
    mag, _ = ob.short_conv(**args, magnitude=True)
    n = device_lengths(lengths)
    y = nan_like((B, T, D), io)
    lh.short_conv_prefill(x, w, bias, state, y, lengths=n, resume=True)
    check(y, ref, mag, K + 16, io, "y")
    assert np.array_equal(np64(state), sref)
    dy = dev(f(B, T, D), io)
    args = dict(dy=np64(dy), x=args["x"], w=args["w"], bias=args["bias"], silu=True, lengths=lengths)
    ref, mag = ob.short_conv_grad(**args), ob.short_conv_grad(**args, magnitude=True)
    dx, dw, db = nan_like((B, T, D), io), nan_like((D, K)), nan_like((D,))
    lh.short_conv_backward(dy, x, w, bias, dx, dw, db, lengths=n)
    k = 3 * K + 24
    check(dx, ref[0], mag[0], k, io, "dx")
    check(dw, ref[1], mag[1], k + B * T, name="dw")
    check(db, ref[2], mag[2], k + B * T, name="dbias")
