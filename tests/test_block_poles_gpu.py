"""The selective scan with states that have no memory (a pole at minus infinity, whose
decay is exactly 0): prompts whose last tile, or whose last chunks, hold steps past the
row's tokens leave the state alone.  And chunked prompts of bfloat16 rows.  Tolerances are
those derived in ``test_block_gpu``."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.block as ob
import paper_2310_18780_amd as lh
from test_block_gpu import LONG, check, dev, device_lengths, gen, host, nan_like, np64, poison, scan_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    lh.lib()
    yield


CASES = [  # B, T, D, N, G, lengths
    (1, 16, 70, 16, 1, None), (1, 17, 70, 16, 1, None), (2, 33, 20, 5, 2, [33, 7]), (2, 40, 20, 33, 1, [40, 0]),
    (1, 560, 70, 4, 2, None),               # chunks that carry by themselves
    (2, 1100, 10, 8, 1, [1100, 530]),       # chunks with a launch for the carry, some without tokens
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("resume", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_poles_at_minus_infinity(case, resume, io):
    B, T, D, N, G, lengths = case
    c = scan_case(case, io, seed=31)
    c["A"][3, N - 1] = c["A"][D - 1, 0] = -float("inf")
    state = dev(gen(T).normal(size=(B, D, N))) if resume else nan_like((B, D, N))
    args = dict(host(c), state=np64(state) if resume else None, lengths=lengths)
    ref, xref = ob.selective(**args)
    mag, xmag = ob.selective(**args, magnitude=True)
    assert np.isfinite(ref).all() and np.isfinite(xref).all()
    y = nan_like((B, T, D), io)
    lh.selective_prefill(state=state, y=y, lengths=device_lengths(lengths), resume=resume, **c)
    check(y, ref, mag, 3 * T + N + 64, io, "y")
    check(state, xref, xmag, 3 * T + N + 64, name="state")


@pytest.mark.parametrize("resume", [False, True])
@pytest.mark.parametrize("case", LONG, ids=str)
def test_prompts_in_chunks_with_bfloat16_rows(case, resume):
    B, T, D, N, G, lengths = case
    assert lh.selective_workspace_bytes(B, T, D, N, G) > 0
    c = scan_case(case, "bf16", seed=5)
    state = dev(gen(T).normal(size=(B, D, N))) if resume else nan_like((B, D, N))
    args = dict(host(c), state=np64(state) if resume else None, lengths=lengths)
    ref, xref = ob.selective(**args)
    mag, xmag = ob.selective(**args, magnitude=True)
    if lengths is not None:
        poison(c, lengths, ("dt", "Bm", "Cm", "u", "z"))
    y = nan_like((B, T, D), "bf16")
    lh.selective_prefill(state=state, y=y, lengths=device_lengths(lengths), resume=resume, **c)
    check(y, ref, mag, 3 * T + N + 64, "bf16", "y")
    check(state, xref, xmag, 3 * T + N + 64, name="state")
