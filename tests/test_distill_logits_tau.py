"""Temperatures of the distillation: where their square, or their reciprocal, is no float32, a call is
refused on the host (no GPU needed); at the ends of the range the loss and its gradient are right."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.model as om
import paper_2310_18780_amd as lh

A = 0x7F0000000000
MB = 1 << 20
U = 2.0 ** -24
INVALID = 1


@pytest.mark.parametrize("tau", [1e-45, 1e-30, 2.0 ** -61, 2.0 ** 61, 1e30, 3e38])
def test_refusals(tau):
    L = lh.lib()
    assert L.lh_distill_logits(A, 32, A + 10 * MB, A + 11 * MB, None, 4, 32, 3, 0, tau, A + 12 * MB, None, None, 0, None, 0,
                               None) == INVALID
    assert "tau" in L.lh_last_error().decode()
    assert L.lh_distill_logits_backward(A + 14 * MB, A, 32, A + 10 * MB, A + 11 * MB, None, A + 15 * MB, 4, 32, 3, 0, tau,
                                        A + 16 * MB, 32, None) == INVALID
    assert "tau" in L.lh_last_error().decode()


@pytest.mark.gpu
@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 60])
def test_ends_of_the_range(size):
    """Logits that are as large as the temperature: p and q are those of temperature 1, and so are, times a
    power of 2, which is exact, the loss and its gradient."""
    r = np.random.default_rng(1)
    V, K = 300, 5
    x, v = 2 * r.normal(size=(3, V)).astype(np.float32), 2 * r.normal(size=(3, K)).astype(np.float32)
    ids = torch.from_numpy(np.stack([r.permutation(V)[:K] for _ in x]).astype(np.int32)).cuda()
    got = []
    for tau in (1.0, size):
        logits, values = (torch.from_numpy(a * np.float32(tau)).cuda() for a in (x, v))
        loss, lse, grad = torch.empty(3, device="cuda"), torch.empty(3, device="cuda"), torch.empty((3, V), device="cuda")
        lh.distill_logits(logits, values, ids, loss, dlogits=grad, lse=lse, tau=tau)
        apart = torch.empty_like(grad)
        lh.distill_logits_backward(torch.ones(3, device="cuda"), logits, values, ids, lse, apart, tau=tau)
        got.append((loss.double() / tau ** 2, grad.double() / tau, apart.double() / tau, lse.double()))
    rl, rg, rs, mag, far = om.distill_logits(x, v, ids.cpu().numpy())
    # (k as in test_distill_logits_gpu.py; log2 e / tau is rounded, and tau's product of the loss is not)
    k = (8 * far + V / 128 + 80 + 5 * np.abs(rs))[:, None]
    for loss, grad, apart, lse in got:
        assert (np.abs(loss.cpu().numpy() - rl) <= (k[:, 0] * (1 + 2 * far)) * U).all()
        assert (np.abs(lse.cpu().numpy() - rs) <= k[:, 0] * U).all()
        for g in (grad, apart):
            assert (np.abs(g.cpu().numpy() - rg) <= k * mag * U).all()
