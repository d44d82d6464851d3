"""Long prompts of the gated recurrence, whose blocks of 128 steps several workgroups take in turn,
against the float64 oracle with its own bounds: several groups of 16 blocks, more blocks than
workgroups to a tile, channels slow enough that the first block reaches the last state."""
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


def check(got, ref, bound, io, name):
    got = np64(got)
    tol = bound * U + (2.0 ** -8 * (np.abs(ref) + bound * U) if io == "bf16" else 0) + 1e-30
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, bad.sum(), np.argwhere(bad)[0], got[bad][0], ref[bad][0], tol[bad][0])


def case(B, T, D, io, gate):
    r = gen(B + T + D)
    # rates of 1e-5 to 1, the slowest first
    c = dict(rate=dev(np.geomspace(1e-5, 1.0, D)), r_bias=dev(0.3 * r.normal(size=D)), i_bias=dev(0.3 * r.normal(size=D)))
    c.update({k: dev(r.normal(size=(B, T, D)), io) for k in ("r", "i", "u") + (("z",) if gate else ())})
    return c, dev(3 + r.normal(size=(B, D)))


def ref_args(c):
    return {k: v.cpu().numpy() if k == "lengths" else np64(v) for k, v in c.items()}


# 40 blocks (two borders of groups), 70 (four), 33 of two tiles (a last group of one block); then 64 tiles of 11 blocks,
# which 8 workgroups share, and 130 of 7, which 4 do
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 5000, 3), (1, 8900, 2), (1, 4097, 70), (64, 1300, 4), (130, 800, 3)], ids=str)
def test_prompt(shape, io):
    B, T, D = shape
    c, start = case(B, T, D, io, gate=B > 1)
    if B > 1:  # rows that end in every block, some without a token
        c["lengths"] = torch.from_numpy(gen(1).integers(0, T + 1, B).astype(np.int32)).cuda()
        c["lengths"][0], c["lengths"][1] = T, 0
    args = ref_args(c)
    ry, rh, ey, eh, before, eb = om.gated(state=np64(start), **args)
    for _ in range(2):
        y, state = torch.full(shape, float("nan"), dtype=IO[io], device="cuda"), start.clone()
        marks = torch.zeros((B, -(-T // lh.GATED_MARK), D), device="cuda")
        lh.gated_prefill(state=state, y=y, resume=True, marks=marks, **c)
        check(y, ry, ey, io, "y")
        check(state, rh, eh, "f32", "state")
        check(marks, before[:, ::lh.GATED_MARK], eb[:, ::lh.GATED_MARK], "f32", "marks")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 5000, 3), (1, 8900, 2), (3, 1500, 5)], ids=str)
def test_gradients(shape, io):
    B, T, D = shape
    c, start = case(B, T, D, io, gate=B > 1)
    dy, dlast = dev(gen(2).normal(size=shape), io), dev(3 + gen(3).normal(size=(B, D)))
    marks = torch.full((B, -(-T // lh.GATED_MARK), D), float("nan"), device="cuda")
    lh.gated_prefill(state=start.clone(), y=torch.empty(shape, dtype=IO[io], device="cuda"), resume=True, marks=marks, **c)
    g = {k: torch.full(shape, float("nan"), dtype=IO[io], device="cuda") for k in ("dr", "di", "du") + (("dz",) if "z" in c else ())}
    g.update({k: torch.full((D,), float("nan"), device="cuda") for k in ("drate", "dr_bias", "di_bias")})
    g.update(dfirst=torch.full((B, D), float("nan"), device="cuda"))
    lh.gated_backward(dy, marks=marks, dlast=dlast, **c, **g)
    out, err = om.gated_grad(np64(dy), state=np64(start), dlast=np64(dlast), **ref_args(c))
    for k, t in g.items():
        check(t, out[k], err[k], io if t.dtype == torch.bfloat16 else "f32", k)
