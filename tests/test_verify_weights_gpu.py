"""Verification of drafted tokens where the border falls to a rounding of the sums: the next token has
weight, and is -1 only where nothing has any."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2310_18780_amd as lh

pytestmark = pytest.mark.gpu

TILE = 2048  # tokens of a tile


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    lh.lib()
    yield


def verify(p, u, u_last, draft_p=None):
    B, K = u.shape
    accepted, tokens = torch.full((B,), -9, dtype=torch.int32, device="cuda"), torch.full((B, K + 1), -9, dtype=torch.int32, device="cuda")
    lh.verify_draft(torch.zeros((B, K), dtype=torch.int32, device="cuda"), p, u, u_last, accepted, tokens, draft_p=draft_p)
    return accepted.tolist(), tokens.tolist()


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("weights,last", [
    # tiles of 1/2, 2^-54, 0, 2^-54, 0, 1/2: sums of the first five tiles are 1/2 or 1/2 + 2^-53, by their order
    ({0: 0.5, 1: 2.0 ** -54, 3: 2.0 ** -54, 5: 0.5}, 5),
    # the same with more that is empty, up to the next 64 tiles
    ({0: 0.5, 1: 2.0 ** -54, 3: 2.0 ** -54, 70: 0.5}, 70),
    ({0: 0.5, 1: 2.0 ** -54, 3: 2.0 ** -54, 5: 0.25, 63: 0.25}, 5)], ids=["next", "far", "both"])
def test_a_tile_without_weight_is_not_picked(weights, last, io):
    V = 80 * TILE
    p = torch.zeros((1, 2, V), dtype=io, device="cuda")
    for tile, w in weights.items():
        p[:, :, tile * TILE + 77] = w
    # token 0 has no probability: refused; the draft's is elsewhere, so all of p is left
    q = torch.zeros((1, 1, V), dtype=io, device="cuda")
    q[..., 0] = 1
    a, t = verify(p, torch.full((1, 1), 0.5, device="cuda"), torch.full((1,), 0.5, device="cuda"), q)
    # the sum is 1, or 1 + 2^-53 before its rounding, and the border 1/2: the first tile's sum is not past it.  Of the
    # others any with weight is within the sums' rounding.
    allowed = [k * TILE + 77 for k in weights if 0 < k <= last]
    assert a == [0] and t[0][0] in allowed and t[0][1] == -1, t


@pytest.mark.parametrize("seed", range(6))
def test_borders_at_every_partial_sum(seed):
    """Few tokens of weights far apart in size, among tiles without any; the border at each sum in turn.
    Whatever the sums' rounding, the token has weight and lies next to the border."""
    r = np.random.default_rng(seed)
    tiles, B = 61, 64
    V = tiles * TILE - 5
    at = np.sort(1 + r.choice(V - 1, 24, replace=False))
    w = (2.0 ** -r.integers(0, 60, 24)).astype(np.float32)
    w[r.integers(0, 24)] = 1
    p = torch.zeros((B, 2, V), device="cuda")
    p[:, :, torch.from_numpy(at).cuda()] = torch.from_numpy(w).cuda()
    c = np.cumsum(w.astype(np.float64))
    u_last = np.minimum(np.r_[c / c[-1], r.random(B - 24)].astype(np.float32), 1 - 2.0 ** -24).astype(np.float32)
    q = torch.zeros((B, 1, V), device="cuda")
    q[..., 0] = 1
    a, t = verify(p, torch.full((B, 1), 0.5, device="cuda"), torch.from_numpy(u_last).cuda(), q)
    slack = 100 * 2.0 ** -53 * c[-1]  # more additions than the sum of 24 tokens goes through
    for b in range(B):
        k = int(np.searchsorted(at, t[b][0]))
        assert a[b] == 0 and k < 24 and at[k] == t[b][0], (b, t[b])
        border = float(u_last[b]) * c[-1]
        assert c[k] > border - slack and (k == 0 or c[k - 1] <= border + slack), (b, k)
