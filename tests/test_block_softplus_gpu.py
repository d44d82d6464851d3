"""The step of the selective scan, log(1 + e^x), against float64: a call with no decay, no
state and ones elsewhere returns it.  Its relative error is at most (7 + 1.25 max(-x, 0))
2^-24: the exponent -|x| log2 e carries its rounding and that of the constant (1.22 of 2^-24),
which are relative errors of e^-|x| in proportion to |x|; the exponential, the logarithm (an
ulp each) and three sums and products add seven."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2310_18780_amd as lh

pytestmark = pytest.mark.gpu


def test_steps_from_far_below_to_far_above_zero():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    n = 1 << 20
    x = np.concatenate([np.linspace(-60, 60, n // 2), np.random.default_rng(1).normal(size=n // 2) * 3]).astype(np.float32)
    dt = torch.from_numpy(x).cuda().view(n // 64, 64)
    one = torch.ones((n // 64, 1, 1), device="cuda")
    u, y, state = torch.ones_like(dt), torch.empty_like(dt), torch.zeros((n // 64, 64, 1), device="cuda")
    lh.selective_step(torch.zeros((64, 1), device="cuda"), dt, one, one.clone(), u, state, y)
    ref = np.logaddexp(0.0, x.astype(np.float64))
    got = y.double().cpu().numpy().ravel()
    assert (np.abs(got - ref) <= (7 + 1.25 * np.maximum(-x, 0)) * 2.0 ** -24 * ref).all()
    assert torch.equal(state.view_as(y), y)
