"""The gated recurrence's gates where a sigmoid is about the smallest normal float32, with rates so large
that such a gate counts; and what lies beside the outputs."""
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


def check(got, ref, bound, name):
    got, tol = np64(got), bound * U + 1e-30
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, bad.sum(), np.argwhere(bad)[0], got[bad][0], ref[bad][0], tol[bad][0])


def test_gates_near_the_smallest_float():
    """e^87 lies between 2^125 and 2^126: a gate of 2^-125.5, and 1 less it is 1."""
    B, T = 1, 40
    x = np.array([-80.0, -86.0, -86.7, -87.0, -87.2, -87.3])
    D = len(x)
    r = gen(1)
    rate = (0.3 * np.exp(-x)).clip(max=1e38)
    c = dict(rate=dev(rate), r=dev(np.broadcast_to(x, (B, T, D))), i=dev(r.normal(size=(B, T, D))), u=dev(r.normal(size=(B, T, D))))
    y, state, marks = (torch.full(s, float("nan"), device="cuda") for s in ((B, T, D), (B, D), (B, -(-T // lh.GATED_MARK), D)))
    lh.gated_prefill(state=state, y=y, marks=marks, **c)
    args = {k: np64(v) for k, v in c.items()}
    ry, rh, ey, eh, *_ = om.gated(**args)
    check(y, ry, ey, "y")
    check(state, rh, eh, "state")
    g = {k: torch.full((B, T, D), float("nan"), device="cuda") for k in ("dr", "di", "du")}
    g.update(drate=torch.full((D,), float("nan"), device="cuda"))
    dy = dev(r.normal(size=(B, T, D)))
    lh.gated_backward(dy, marks=marks, **c, **g)
    out, err = om.gated_grad(np64(dy), **args)
    for k, t in g.items():
        check(t, out[k], err[k], k)


def guarded(shape, io, before=37, after=1000):
    """A tensor inside a buffer of 7 (what a row of stores could reach past the last), and a check that
    nothing around it was written."""
    n = int(np.prod(shape))
    store = torch.full((before + n + after,), 7.0, dtype=IO[io], device="cuda")
    return store[before:before + n].view(shape), lambda: bool((store[:before] == 7).all() and (store[before + n:] == 7).all())


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 65), (1, 3, 64), (2, 9, 130), (1, 127, 70), (3, 129, 1), (1, 390, 66), (1, 1001, 100)], ids=str)
def test_what_lies_around_the_outputs_is_left_alone(shape, io):
    B, T, D = shape
    r = gen(T)
    after = 8 * D + 64  # a run of rows past the last, and a tile
    c = dict(rate=dev(np.exp(r.uniform(-4, 1, D))), z=dev(r.normal(size=shape), io), r_bias=dev(r.normal(size=D)), i_bias=dev(r.normal(size=D)),
             lengths=torch.tensor([T, T // 2, 0][:B], dtype=torch.int32, device="cuda"))
    c.update({k: dev(r.normal(size=shape), io) for k in ("r", "i", "u")})
    M = -(-T // lh.GATED_MARK)
    spec = dict(state=((B, D), "f32"), y=(shape, io), marks=((B, M, D), "f32"), dr=(shape, io), di=(shape, io), du=(shape, io),
                dz=(shape, io), drate=((D,), "f32"), dr_bias=((D,), "f32"), di_bias=((D,), "f32"), dfirst=((B, D), "f32"))
    o, clean = {}, {}
    for k, (s, t) in spec.items():
        o[k], clean[k] = guarded(s, t, before=36 if t == "f32" else 40, after=after)
    lh.gated_prefill(state=o["state"], y=o["y"], marks=o["marks"], **c)
    assert [k for k, f in clean.items() if not f()] == []
    lh.gated_backward(dev(r.normal(size=shape), io), marks=o["marks"], **{k: o[k] for k in spec if k[0] == "d"}, **c)
    assert [k for k, f in clean.items() if not f()] == []
    t = {k: v[:, 0] if v.dim() == 3 else v for k, v in c.items() if k != "lengths"}
    y, ok = guarded((B, D), io, after=after)
    lh.gated_step(t["rate"], t["r"], t["i"], t["u"], o["state"], y, r_bias=t["r_bias"], i_bias=t["i_bias"], z=t["z"])
    assert ok() and clean["state"]()
