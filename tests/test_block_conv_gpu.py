"""GPU tests of the short convolution beside ``test_block_gpu``, whose tolerances they take."""
from __future__ import annotations

import pytest
import torch

import oracle.block as ob
import paper_2310_18780_amd as lh
from test_block_gpu import check, dev, gen, nan_like, np64

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
