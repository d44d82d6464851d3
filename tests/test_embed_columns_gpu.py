"""The gradient of the embedding's table with more than one block of 1024 columns, whose runs cross
windows of sorted tokens: written and added to what is there (tolerance as in ``test_embed_gpu.py``)."""
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


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("add", [False, True], ids=["written", "added"])
# up to 8192 tokens windows are of 16, above of 64; 1024 columns to a workgroup, the last block of 1, 1022 or 1024 of them
@pytest.mark.parametrize("n,V,D", [(300, 5, 1025), (300, 3, 2046), (900, 40, 2048), (9000, 30, 1025), (8500, 7, 2046)])
def test_runs_that_cross_windows(n, V, D, add, io):
    r = np.random.default_rng(n + D)
    ids = np.minimum((V * r.random(n) ** 3).astype(np.int32), V - 1)  # runs of several windows, and short ones between
    ids[r.random(n) < 0.05] = -1
    ids[ids == 1] = 0  # a row without a token
    # multiples of 1/4 up to 2: every partial sum is exact in float32, and so is half of it
    dy = np.clip(np.round(4 * r.normal(size=(n, D))), -8, 8) / 4
    there = np.round(8 * r.normal(size=(V, D))) / 8
    t = torch.from_numpy(dy.astype(np.float32)).to(IO[io]).cuda()
    dW = torch.from_numpy(there.astype(np.float32)).cuda() if add else torch.full((V, D), float("nan"), device="cuda")
    lh.embed_backward(t, torch.from_numpy(ids).cuda(), dW, scale=0.5, accumulate=add)
    ref, _ = om.embed_grad(dy, ids, V, 0.5, there if add else None)
    got = dW.double().cpu().numpy()
    assert (got == ref).all(), (np.argwhere(got != ref)[0], (got != ref).sum())
    # and values whose sums are rounded
    dy = r.normal(size=(n, D))
    t = torch.from_numpy(dy.astype(np.float32)).to(IO[io]).cuda()
    dW = torch.from_numpy(there.astype(np.float32)).cuda() if add else torch.full((V, D), float("nan"), device="cuda")
    lh.embed_backward(t, torch.from_numpy(ids).cuda(), dW, scale=0.3, accumulate=add)
    ref, bound = om.embed_grad(t.double().cpu().numpy(), ids, V, 0.3, there if add else None)
    # (0.3 is rounded as a float32: one unit of the sum more)
    mag, _ = om.embed_grad(t.double().abs().cpu().numpy(), ids, V, 0.3)
    assert (np.abs(dW.double().cpu().numpy() - ref) <= (bound + mag) * U + 1e-30).all()
