"""GPU parity of the gated recurrence (prompts, single tokens, gradients) against the float64
oracle ``oracle.model``, whose bounds (in units of 2^-24, carried along with the values) are
the tolerances; a bfloat16 output adds its rounding, 2^-8 of the value."""
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


def rows(a, io, front=1, pad=2):
    """The values as a slice of wider rows that starts and ends inside them, the rest NaN."""
    t = dev(a, io)
    wide = torch.full((*t.shape[:-1], front + t.shape[-1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    wide[..., front:front + t.shape[-1]] = t
    return wide[..., front:front + t.shape[-1]]


def np64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def nan_like(shape, io="f32"):
    return torch.full(shape, float("nan"), dtype=IO[io], device="cuda")


def check(got, ref, bound, io="f32", name=""):
    got = np64(got)
    tol = bound * U + (2.0 ** -8 * (np.abs(ref) + bound * U) if io == "bf16" else 0) + 1e-30
    bad = ~(np.abs(got - ref) <= tol)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} off, first at {i}: {got[i]} against {ref[i]}, tolerance {tol[i]}")


def case(B, T, D, io, seed=0, gate=True, bias=True, lengths=None, strided=False):
    r = gen(seed + 7 * B + 11 * T + D)
    make = rows if strided else dev
    c = dict(rate=dev(np.exp(r.uniform(-6, 1.5, D))))
    if bias:
        c.update(r_bias=dev(0.5 * r.normal(size=D)), i_bias=dev(0.5 * r.normal(size=D)))
    for k in ("r", "i", "u") + (("z",) if gate else ()):
        c[k] = make(r.normal(size=(B, T, D)), io)
    if lengths is not None:
        c["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    return c


def ref_args(c):
    return {k: v.cpu().numpy() if k == "lengths" else np64(v) for k, v in c.items()}


SHAPES = [(1, 1, 1), (1, 2, 3), (2, 7, 64), (3, 64, 65), (2, 65, 70), (1, 127, 130), (1, 128, 64), (2, 129, 67), (1, 700, 100),
          (5, 300, 33), (400, 3, 64), (2, 1025, 5), (390, 140, 10),
          (1, 256, 64), (1, 257, 64), (1, 2200, 3), (159, 390, 7), (160, 390, 7)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_prompt(shape, io):
    B, T, D = shape
    c = case(B, T, D, io, gate=T % 2 == 0)
    y, state = nan_like(shape, io), nan_like((B, D))
    marks = nan_like((B, -(-T // lh.GATED_MARK), D))
    lh.gated_prefill(state=state, y=y, marks=marks, **c)
    ry, rh, ey, eh, before, eb = om.gated(**ref_args(c))
    check(y, ry, ey, io, "y")
    check(state, rh, eh, name="state")
    check(marks, before[:, ::lh.GATED_MARK], eb[:, ::lh.GATED_MARK], name="marks")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(7, 70, 100), (4, 520, 65), (3, 128, 64)], ids=str)
def test_ragged_strided_resumed_prompt(shape, io):
    B, T, D = shape
    n = [T, 0, T + 5, 1, -3, T // 2, 64][:B]
    c = case(B, T, D, io, seed=3, lengths=n, strided=True)
    start = gen(4).normal(size=(B, D))
    # what lies past a row's tokens is not read
    for b, m in enumerate(n):
        for k in ("r", "i", "u", "z"):
            c[k][b, max(m, 0):] = float("nan")
    y, state, marks = nan_like(shape, io), dev(start), nan_like((B, -(-T // lh.GATED_MARK), D))
    args = ref_args(c)
    lh.gated_prefill(state=state, y=y, resume=True, marks=marks, **c)
    ry, rh, ey, eh, before, eb = om.gated(state=np64(dev(start)), **args)
    check(y, ry, ey, io, "y")
    check(state, rh, eh, name="state")
    m = marks.cpu()
    for b, k in enumerate(n):
        k = min(max(k, 0), T)
        used = -(-k // lh.GATED_MARK)
        assert torch.isnan(m[b, used:]).all()
        check(m[b, :used], before[b, :k:lh.GATED_MARK], eb[b, :k:lh.GATED_MARK], name="marks")


def test_no_biases_no_marks_and_no_tokens():
    c = case(2, 33, 40, "f32", bias=False, gate=False)
    y, state = nan_like((2, 33, 40)), nan_like((2, 40))
    lh.gated_prefill(state=state, y=y, **c)
    ry, rh, ey, eh, *_ = om.gated(**ref_args(c))
    check(y, ry, ey)
    check(state, rh, eh)
    c = case(2, 0, 40, "bf16")
    kept = dev(gen(1).normal(size=(2, 40)))
    state = kept.clone()
    lh.gated_prefill(state=state, y=nan_like((2, 0, 40), "bf16"), resume=True, **c)
    assert torch.equal(state, kept)
    lh.gated_prefill(state=state, y=nan_like((2, 0, 40), "bf16"), **c)
    assert not state.any()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (3, 64), (64, 2048), (5, 257), (300, 70)], ids=str)
def test_step_is_a_prompt_of_one_token(shape, io):
    B, D = shape
    c = case(B, 1, D, io, seed=5, gate=B != 3, strided=True)
    start = gen(6).normal(size=shape)
    y, state = nan_like((B, D), io), dev(start)
    t = {k: v[:, 0] if v.dim() == 3 else v for k, v in c.items()}
    lh.gated_step(t["rate"], t["r"], t["i"], t["u"], state, y, r_bias=t["r_bias"], i_bias=t["i_bias"], z=t.get("z"))
    ry, rh, ey, eh, *_ = om.gated(state=np64(dev(start)), **ref_args(c))
    check(y, ry[:, 0], ey[:, 0], io, "y")
    check(state, rh, eh, name="state")


def grads(c, io, B, T, D):
    g = {k: nan_like((B, T, D), io) for k in ("dr", "di", "du") + (("dz",) if "z" in c else ())}
    g.update(drate=nan_like((D,)), dfirst=nan_like((B, D)))
    if "r_bias" in c:
        g.update(dr_bias=nan_like((D,)), di_bias=nan_like((D,)))
    return g


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradients(shape, io):
    B, T, D = shape
    c = case(B, T, D, io, seed=8, gate=T % 2 == 1, bias=D != 65)
    dy = dev(gen(9).normal(size=shape), io)
    marks = nan_like((B, -(-T // lh.GATED_MARK), D))
    lh.gated_prefill(state=nan_like((B, D)), y=nan_like(shape, io), marks=marks, **c)
    g = grads(c, io, B, T, D)
    lh.gated_backward(dy, marks=marks, **c, **g)
    out, err = om.gated_grad(np64(dy), **ref_args(c))
    for k, t in g.items():
        check(t, out[k], err[k], io if t.dtype == torch.bfloat16 else "f32", k)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_ragged_resumed_gradients_with_the_states(io):
    B, T, D = 7, 200, 70
    n = [T, 0, T + 5, 1, -3, 97, 64]
    c = case(B, T, D, io, seed=10, lengths=n, strided=True)
    for b, m in enumerate(n):
        for k in ("r", "i", "u", "z"):
            c[k][b, max(m, 0):] = float("nan")
    start, dlast = dev(gen(11).normal(size=(B, D))), dev(gen(12).normal(size=(B, D)))
    dy = dev(gen(13).normal(size=(B, T, D)), io)
    for b, m in enumerate(n):
        dy[b, max(m, 0):] = float("nan")
    marks = nan_like((B, -(-T // lh.GATED_MARK), D))
    lh.gated_prefill(state=start.clone(), y=nan_like((B, T, D), io), marks=marks, resume=True, **c)
    g = grads(c, io, B, T, D)
    lh.gated_backward(dy, marks=marks, dlast=dlast, **c, **g)
    out, err = om.gated_grad(np64(dy), state=np64(start), dlast=np64(dlast), **ref_args(c))
    for k, t in g.items():
        check(t, out[k], err[k], io if t.dtype == torch.bfloat16 else "f32", k)
    assert torch.equal(g["dfirst"][1], dlast[1]) and torch.equal(g["dfirst"][4], dlast[4])


def test_gradients_of_no_tokens():
    c = case(2, 0, 30, "f32")
    g, dlast = grads(c, "f32", 2, 0, 30), dev(gen(1).normal(size=(2, 30)))
    lh.gated_backward(nan_like((2, 0, 30)), marks=nan_like((2, 0, 30)), dlast=dlast, **c, **g)
    assert torch.equal(g["dfirst"], dlast)
    assert not any(g[k].any() for k in ("drate", "dr_bias", "di_bias"))


def test_gradients_against_differences():
    """The gradient along a direction against the change of a float64 sum of the outputs, whose
    float32 outputs are off by their bounds."""
    B, T, D = 2, 90, 33
    c = case(B, T, D, "f32", seed=20)
    dy = dev(gen(21).normal(size=(B, T, D)))
    marks = nan_like((B, -(-T // lh.GATED_MARK), D))

    def value(c):
        y = nan_like((B, T, D))
        lh.gated_prefill(state=nan_like((B, D)), y=y, marks=marks, **c)
        return (y.double() * dy.double()).sum().item()

    g = grads(c, "f32", B, T, D)
    value(c)
    lh.gated_backward(dy, marks=marks.clone(), **c, **g)
    _, _, ey, *_ = om.gated(**ref_args(c))
    noise = (ey * np.abs(np64(dy))).sum() * U
    for k in ("rate", "r", "i", "u", "z", "r_bias", "i_bias"):
        step = 2.0 ** -7 * c[k].abs() if k == "rate" else torch.full_like(c[k], 2.0 ** -8)
        hi, lo = value({**c, k: c[k] + step}), value({**c, k: c[k] - step})
        slope = (g["d" + k].double() * step.double()).sum().item()
        # second differences: a third of the step cubed times third derivatives, here by halving the step
        hi2, lo2 = value({**c, k: c[k] + step / 2}), value({**c, k: c[k] - step / 2})
        first, second = (hi - lo) / 2, hi2 - lo2
        best = (4 * second - first) / 3
        assert abs(best - slope) <= 4 * noise + 2 * abs(second - first) * 2.0 ** -4 + 1e-6 * abs(slope), (k, best, slope, noise)


def test_rates_at_their_ends():
    B, T, D = 1, 150, 6
    c = case(B, T, D, "f32", seed=30, gate=False)
    c["rate"] = torch.tensor([0.0, 1e-30, 1e-7, 50.0, 3e38, 1.0], device="cuda")
    c["r"][0, 3] = float("-inf")  # f = 0: the state is held, nothing comes in
    c["r"][0, 5] = float("inf")
    c["i"][0, 7], c["i"][0, 9] = float("-inf"), float("inf")
    start = dev(np.ones((B, D)))
    y, state, marks = nan_like((B, T, D)), start.clone(), nan_like((B, -(-T // lh.GATED_MARK), D))
    lh.gated_prefill(state=state, y=y, resume=True, marks=marks, **c)
    args = ref_args(c)
    args["rate"] = np.minimum(args["rate"], 2e38)
    ry, rh, ey, eh, *_ = om.gated(state=np.ones((B, D)), **args)
    # (a rate of 1e-30 lets in sqrt(2 rate f), 10^-15 of the state)
    check(y, ry, ey + np.array([0, 8, 0, 0, 0, 0]), name="y")
    assert torch.equal(y[0, :, 0], torch.ones(T, device="cuda")) and torch.equal(y[0, 3], y[0, 2])
    dy = dev(gen(31).normal(size=(B, T, D)))
    g = grads(c, "f32", B, T, D)
    lh.gated_backward(dy, marks=marks, **c, **g)
    assert all(torch.isfinite(v).all() for v in g.values())
    assert g["drate"][0] == 0 and not g["dr"][0, :, 0].any() and not g["du"][0, :, 0].any()
    c["rate"] = torch.full((D,), -0.5, device="cuda")
    lh.gated_prefill(state=state, y=y, **c)
    assert torch.isnan(y[0, 0]).all()


def test_values_that_are_not_finite_stay_in_their_channel_and_later():
    B, T, D = 2, 300, 70
    c = case(B, T, D, "bf16", seed=40)
    y0, y1 = nan_like((B, T, D), "bf16"), nan_like((B, T, D), "bf16")
    s0, s1 = nan_like((B, D)), nan_like((B, D))
    lh.gated_prefill(state=s0, y=y0, **c)
    c["u"][1, 140, 9] = float("inf")
    c["r"][0, 200, 3] = float("nan")
    lh.gated_prefill(state=s1, y=y1, **c)
    same = torch.ones((B, T, D), dtype=torch.bool, device="cuda")
    same[1, 140:, 9] = False
    same[0, 200:, 3] = False
    assert torch.equal(y0[same], y1[same]) and not torch.isfinite(y1[~same]).any()
    assert not torch.isfinite(s1[1, 9]) and not torch.isfinite(s1[0, 3])


def test_a_prompt_in_parts_is_the_prompt():
    """Long prompts are cut into chunks; in parts, each continued from the last one's state, they
    are cut elsewhere.  Both are within the oracle's bound of a float64 evaluation, so within
    twice that of each other; 3 decays a step of the channel's memory."""
    B, T, D = 2, 5000, 70
    c = case(B, T, D, "f32", seed=50)
    c["rate"] = c["rate"].clamp(min=0.05)
    y, s = nan_like((B, T, D)), nan_like((B, D))
    lh.gated_prefill(state=s, y=y, **c)
    parts, s2 = [], nan_like((B, D))
    for k, (i, j) in enumerate([(0, 1), (1, 1300), (1300, 1364), (1364, 4999), (4999, 5000)]):
        part = {n: v[:, i:j].contiguous() if v.dim() == 3 else v for n, v in c.items()}
        parts.append(nan_like((B, j - i, D)))
        lh.gated_prefill(state=s2, y=parts[-1], resume=k > 0, **part)
    # G = 3 x 6 + 8 for |x| < 6: a state of magnitude M is off by at most (2 G + 35 + (G + 9) (M / |v|)) units of |v| a
    # token of its memory: 1 / (1 - e^-0.01) = 100 tokens of |v| < 1, M < 20
    tol = 2 * 100 * (2 * 26 + 35 + 35 * 20) * U
    assert (torch.cat(parts, 1) - y).abs().max().item() <= tol * c["z"].abs().max().item()
    assert (s - s2).abs().max().item() <= tol


def test_offsets_past_32_bits():
    """Tensors of more than 2^31 elements: the last tokens against the same tokens on their own."""
    T, D, tail = (1 << 21) + 70, 1056, 100
    g = torch.Generator(device="cuda").manual_seed(1)
    u = torch.empty((1, T, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    rate, bias = dev(np.exp(gen(2).uniform(-2, 1, D))), dev(gen(3).normal(size=D))
    M = lh.GATED_MARK
    y, marks, s = torch.empty_like(u), torch.empty((1, -(-T // M), D), device="cuda"), nan_like((1, D))
    lh.gated_prefill(rate, u, u, u, s, y, r_bias=bias, marks=marks)
    k = (T - tail) // M  # a mark
    n = T - M * k
    state, part, m2 = marks[:, k].clone(), torch.empty((1, n, D), dtype=torch.bfloat16, device="cuda"), nan_like((1, -(-n // M), D))
    x = u[:, M * k:].contiguous()
    lh.gated_prefill(rate, x, x, x, state, part, r_bias=bias, resume=True, marks=m2)
    # the same tokens from the same state, cut elsewhere: 2^-8 of the outputs' rounding, and of their scale
    assert (part.float() - y[:, M * k:].float()).abs().max().item() <= 2.0 ** -7 * part.float().abs().max().item()
    assert (state - s).abs().max().item() <= 1e-4 * s.abs().max().item()
    # gradients that only the last tokens get
    dy = torch.zeros_like(u)
    dy[:, -tail:] = 1
    big = [torch.empty_like(u) for _ in range(3)]
    dr = [nan_like((D,)) for _ in range(2)]
    lh.gated_backward(dy, rate, u, u, u, marks, dr[0], *big, r_bias=bias)
    small = [torch.empty_like(x) for _ in range(3)]
    lh.gated_backward(dy[:, M * k:].contiguous(), rate, x, x, x, m2, dr[1], *small, r_bias=bias)
    for a, b in zip(big, small):
        a = a[:, M * k:]
        assert (a.float() - b.float()).abs().max().item() <= 2.0 ** -6 * b.float().abs().max().item()
