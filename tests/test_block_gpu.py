"""GPU parity of the selective block (layer norm, short causal convolution, selective
scan; prompts, single tokens, gradients) against the float64 oracle ``oracle.block``.

Tolerances, fixed from the arithmetic: a float32 evaluation with at most ``k`` roundings
on the way of any term differs from the exact value by at most ``k 2^-24`` times the sum
of the terms' magnitudes, which the oracle gives (``magnitude=True``).  The counts:

  layer norm    128: a lane adds at most 64 values, 6 + 4 tree levels, a dozen products;
                the statistics' own error reaches y through rstd: 64 (1 + max|s| rstd)
                of the normalised value
  convolution   K + 16 (gradient 3 K + 24; its sums over tokens one more per token)
  scan          3 T + N + 64: two or three roundings a step, the exponent's relative
                error (about 16) times E e^-E < 0.4
  its gradient  8 B T + D + N + 128: both recurrences, and sums over tokens and channels

A bfloat16 output adds its rounding, 2^-8 of the value.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.block as ob
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


def rows(a, io, pad=3, front=1):
    """The values as a slice of wider rows that starts and ends inside them, the rest NaN."""
    t = dev(a, io)
    lead, row = (t.shape[:2], t.shape[2:]) if t.dim() > 2 else (t.shape[:1], t.shape[1:])
    n = int(np.prod(row))
    wide = torch.full((*lead, front + n + pad), float("nan"), dtype=t.dtype, device="cuda")
    wide[..., front:front + n] = t.reshape(*lead, n)
    return wide[..., front:front + n].unflatten(-1, tuple(row)) if len(row) > 1 else wide[..., front:front + n]


def np64(t):
    return t.detach().double().cpu().numpy()


def nan_like(shape, io="f32"):
    return torch.full(shape, float("nan"), dtype=IO[io], device="cuda")


def check(got, ref, mag, k, io="f32", name=""):
    got = np64(got)
    tol = k * U * mag + (2.0 ** -8 * np.abs(ref) if io == "bf16" else 0) + 1e-30
    bad = ~(np.abs(got - ref) <= tol)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} off, first at {i}: {got[i]} against {ref[i]}, tolerance {tol[i]}")


# ---- layer norm

NORM = [(1, 1), (1, 7), (3, 64), (5, 100), (2, 513), (64, 2048), (3, 1001), (2500, 130), (2100, 2048), (600, 3000),
        (2, 4099), (3, 8192), (2, 9001), (2, 20000), (1, 40001), (2049, 37)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("res", [False, True])
@pytest.mark.parametrize("shape", NORM, ids=str)
def test_layer_norm(shape, res, io):
    R, D = shape
    r = gen(R * 7 + D)
    x, w, b = dev(2 + r.normal(size=shape), io), dev(r.normal(size=D)), dev(r.normal(size=D))
    residual = dev(r.normal(size=shape), io) if res else None
    y, mean, rstd = nan_like(shape, io), nan_like((R,)), nan_like((R,))
    total = nan_like(shape, io) if res else None
    lh.layer_norm(x, w, b, y, residual=residual, total=total, mean=mean, rstd=rstd)
    args = (np64(x), np64(w), np64(b), np64(residual) if res else None)
    ref, s, m, rs = ob.layer_norm(*args)
    mag, smag, top, _ = ob.layer_norm(*args, magnitude=True)
    spread = (1 + top * rs)[:, None]
    check(y, ref, mag + 0.5 * spread * np.abs(ref - args[2]), 128, io, "y")
    check(mean, m, top, 128, name="mean")
    check(rstd, rs, rs * spread[:, 0], 128, name="rstd")
    if res:
        check(total, s, smag, 1, io, "total")


def test_layer_norm_without_bias_total_in_place_and_eps():
    r = gen(3)
    for alias in ("x", "residual"):
        x, res, w = dev(r.normal(size=(9, 300))), dev(r.normal(size=(9, 300))), dev(r.normal(size=300))
        args = (np64(x), np64(w), None, np64(res))
        ref, s, _, _ = ob.layer_norm(*args, eps=0.5)
        y = nan_like((9, 300))
        total = x if alias == "x" else res
        lh.layer_norm(x, w, None, y, residual=res, total=total, eps=0.5)
        check(y, ref, ob.layer_norm(*args, eps=0.5, magnitude=True)[0], 192, name="y")
        check(total, s, np.abs(s) + 1, 1, name="total")
    x = torch.full((2, 50), 3.0, device="cuda")  # no variance at all
    y = nan_like((2, 50))
    lh.layer_norm(x, dev(r.normal(size=50)), None, y)
    assert not y.any()
    y = nan_like((0, 50))
    lh.layer_norm(y, dev(r.normal(size=50)), None, y.clone())  # no rows


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("extra", [False, True])
@pytest.mark.parametrize("shape", NORM, ids=str)
def test_layer_norm_backward(shape, extra, io):
    R, D = shape
    r = gen(R * 5 + D)
    x, dy, w = dev(1 + r.normal(size=shape), io), dev(r.normal(size=shape), io), dev(r.normal(size=D))
    dtotal = dev(r.normal(size=shape), io) if extra else None
    _, _, m, rs = ob.layer_norm(np64(x), np64(w), None)
    mean, rstd = dev(m), dev(rs)
    args = (np64(dy), np64(x), np64(w), np64(mean), np64(rstd), np64(dtotal) if extra else None)
    ref = ob.layer_norm_grad(*args)
    mag = ob.layer_norm_grad(*args, magnitude=True)
    dx, dw, db = nan_like(shape, io), nan_like((D,)), nan_like((D,))
    lh.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, dtotal=dtotal)
    check(dx, ref[0], mag[0], 192, io, "dx")
    check(dw, ref[1], mag[1], 16 + R, name="dw")
    check(db, ref[2], mag[2], 16 + R, name="db")
    if extra:  # in place, without db
        lh.layer_norm_backward(dy, x, w, mean, rstd, dtotal, dw, None, dtotal=dtotal)
        assert torch.equal(dtotal, dx)


def test_layer_norm_backward_of_no_rows():
    e, z = torch.empty((0, 33), device="cuda"), torch.empty((0,), device="cuda")
    dw, db = nan_like((33,)), nan_like((33,))
    lh.layer_norm_backward(e, e.clone(), torch.ones(33, device="cuda"), z, z.clone(), e.clone(), dw, db)
    assert not dw.any() and not db.any()


# ---- short convolution

CONV = [  # B, T, D, K, lengths
    (1, 1, 1, 1, None), (2, 3, 5, 4, None), (3, 9, 130, 3, [9, 0, 2]), (1, 70, 64, 2, None),
    (2, 130, 33, 8, [1, 129]), (4, 40, 17, 5, [40, 3, -5, 1000]), (2, 20, 1001, 4, None), (1, 5, 24, 6, [4]),
    (2, 6, 40, 7, None), (2, 0, 12, 4, None),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("resume", [False, True])
@pytest.mark.parametrize("case", CONV, ids=str)
def test_short_conv_prefill(case, resume, silu, io):
    B, T, D, K, lengths = case
    r = gen(B + 10 * T + D)
    x = rows(r.normal(size=(B, T, D)), io)
    w, bias = dev(r.normal(size=(D, K))), dev(r.normal(size=D)) if K % 2 else None
    state = dev(r.normal(size=(B, K - 1, D)), io) if resume else nan_like((B, K - 1, D), io)
    args = dict(x=np64(x), w=np64(w), bias=None if bias is None else np64(bias), silu=silu,
                state=np64(state) if resume else None, lengths=lengths)
    ref, sref = ob.short_conv(**args)
    mag, _ = ob.short_conv(**args, magnitude=True)
    n = None
    if lengths is not None:
        n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        for b, c in enumerate(lengths):
            x[b, max(c, 0):] = float("nan")  # what lies past a row's tokens is not read
    y = nan_like((B, T, D), io)
    lh.short_conv_prefill(x, w, bias, state, y, silu=silu, lengths=n, resume=resume)
    check(y, ref, mag, K + 16, io, "y")
    assert np.array_equal(np64(state), sref)


@pytest.mark.parametrize("K", [4, 5, 6, 8])
def test_short_conv_resumes_with_long_filters_on_many_rows(K):
    """The inputs before the first tokens come from the state as it was, whichever part of
    a row runs first: few threads (the shortest runs) over many rows, against one row each."""
    B, T, D = 64, 23, 24
    r = gen(K + 50)
    x, w = dev(r.normal(size=(B, T, D))), dev(r.normal(size=(D, K)))
    old = dev(r.normal(size=(B, K - 1, D)))
    ref, sref = ob.short_conv(np64(x), np64(w), None, False, state=np64(old))
    mag, _ = ob.short_conv(np64(x), np64(w), None, False, state=np64(old), magnitude=True)
    for _ in range(5):
        state, y = old.clone(), nan_like((B, T, D))
        lh.short_conv_prefill(x, w, None, state, y, silu=False, resume=True)
        check(y, ref, mag, K + 16, name="y")
        assert np.array_equal(np64(state), sref)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("K", [1, 2, 4, 8])
def test_short_conv_steps_continue_a_prefill(K, io):
    B, T, D = 3, 12, 37
    r = gen(K)
    x, w, bias = dev(r.normal(size=(B, T, D)), io), dev(r.normal(size=(D, K))), dev(r.normal(size=D))
    ref = nan_like((B, T, D), io)
    full = nan_like((B, K - 1, D), io)
    lh.short_conv_prefill(x, w, bias, full, ref)
    y, state = nan_like((B, T, D), io), nan_like((B, K - 1, D), io)
    lh.short_conv_prefill(x[:, :5].contiguous(), w, bias, state, first := nan_like((B, 5, D), io))
    y[:, :5] = first
    for t in range(5, T):
        y_t = nan_like((B, D), io)
        lh.short_conv_step(x[:, t], w, bias, state, y_t)  # a slice of rows
        y[:, t] = y_t
    assert torch.equal(y, ref) and torch.equal(state, full)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("case", CONV, ids=str)
def test_short_conv_backward(case, silu, io):
    B, T, D, K, lengths = case
    r = gen(B + 20 * T + D)
    x, dy = rows(r.normal(size=(B, T, D)), io), dev(r.normal(size=(B, T, D)), io)
    w, bias = dev(r.normal(size=(D, K))), dev(r.normal(size=D)) if K % 2 else None
    args = dict(dy=np64(dy), x=np64(x), w=np64(w), bias=None if bias is None else np64(bias), silu=silu, lengths=lengths)
    ref, mag = ob.short_conv_grad(**args), ob.short_conv_grad(**args, magnitude=True)
    n = None
    if lengths is not None:
        n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        for b, c in enumerate(lengths):
            x[b, max(c, 0):] = float("nan")
            dy[b, max(c, 0):] = float("nan")
    dx, dw, db = nan_like((B, T, D), io), nan_like((D, K)), nan_like((D,))
    lh.short_conv_backward(dy, x, w, bias, dx, dw, db, silu=silu, lengths=n)
    k = 3 * K + 24
    check(dx, ref[0], mag[0], k, io, "dx")
    check(dw, ref[1], mag[1], k + B * T, name="dw")
    check(db, ref[2], mag[2], k + B * T, name="dbias")


# ---- selective scan

SCAN = [  # B, T, D, N, G, lengths
    (1, 1, 1, 1, 1, None), (2, 5, 3, 2, 1, None), (3, 17, 70, 16, 1, [17, 0, 3]), (2, 33, 130, 12, 2, None),
    (1, 300, 96, 16, 1, None), (2, 200, 65, 7, 5, [200, 131]), (1, 130, 33, 5, 33, None), (2, 40, 20, 20, 1, None),
    (1, 70, 12, 33, 2, [65]), (1, 129, 8, 48, 1, None), (1, 65, 70, 64, 1, None), (1, 40, 5, 96, 1, None),
    (2, 35, 6, 128, 3, [-1, 35]), (1, 40, 9, 101, 1, None), (2, 0, 6, 4, 1, None), (1, 64, 64, 3, 1, None),
]


def scan_case(case, io, gate=True, seed=0, strided=True):
    B, T, D, N, G, lengths = case
    r = gen(B * 3 + T * 5 + D * 7 + N + seed)
    f = (lambda *s: rows(r.normal(size=s), io)) if strided else (lambda *s: dev(r.normal(size=s), io))
    c = dict(A=dev(-np.exp(r.normal(size=(D, N)))), dt=f(B, T, D), Bm=f(B, T, G, N), Cm=f(B, T, G, N), u=f(B, T, D),
             h0=dev(r.normal(size=D)), dt_bias=dev(r.normal(size=D) - 2))
    if gate:
        c["z"] = f(B, T, D)
    return c


def poison(c, lengths, names):
    """NaN into what lies past the rows' tokens."""
    for k in names:
        for b, n in enumerate(lengths):
            c[k][b, max(n, 0):] = float("nan")


def device_lengths(lengths):
    return None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")


def host(c):
    return {k: np64(v) for k, v in c.items()}


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("resume", [False, True])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("case", SCAN, ids=str)
def test_selective_prefill(case, gate, resume, io):
    B, T, D, N, G, lengths = case
    c = scan_case(case, io, gate)
    state = dev(gen(T).normal(size=(B, D, N))) if resume else nan_like((B, D, N))
    args = dict(host(c), state=np64(state) if resume else None, lengths=lengths)
    ref, xref = ob.selective(**args)
    mag, xmag = ob.selective(**args, magnitude=True)
    if lengths is not None:
        poison(c, lengths, [k for k in ("dt", "Bm", "Cm", "u", "z") if k in c])
    y = nan_like((B, T, D), io)
    lh.selective_prefill(state=state, y=y, lengths=device_lengths(lengths), resume=resume, **c)
    k = 3 * T + N + 64
    check(y, ref, mag, k, io, "y")
    check(state, xref, xmag, k, name="state")


# prompts that are cut into more chunks than carry by themselves, and into a few
LONG = [(1, 1200, 20, 16, 1, None), (2, 1100, 10, 8, 1, [1100, 530]), (1, 560, 70, 4, 2, None), (1, 1030, 6, 33, 3, [1017])]


@pytest.mark.parametrize("resume", [False, True])
@pytest.mark.parametrize("case", LONG, ids=str)
def test_selective_prefill_in_chunks(case, resume):
    B, T, D, N, G, lengths = case
    assert lh.selective_workspace_bytes(B, T, D, N, G) > 0
    c = scan_case(case, "f32", seed=3)
    state = dev(gen(T).normal(size=(B, D, N))) if resume else nan_like((B, D, N))
    args = dict(host(c), state=np64(state) if resume else None, lengths=lengths)
    ref, xref = ob.selective(**args)
    mag, xmag = ob.selective(**args, magnitude=True)
    if lengths is not None:
        poison(c, lengths, ("dt", "Bm", "Cm", "u", "z"))
    y = nan_like((B, T, D))
    lh.selective_prefill(state=state, y=y, lengths=device_lengths(lengths), resume=resume, **c)
    check(y, ref, mag, 3 * T + N + 64, name="y")
    check(state, xref, xmag, 3 * T + N + 64, name="state")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 3, 4, 6, 8, 13, 16, 31, 32, 64, 100, 128])
def test_selective_steps(N, io):
    B, T, D, G = 3, 4, 38, 2
    c = scan_case((B, T, D, N, G, None), io)
    x0 = dev(gen(N).normal(size=(B, D, N)))
    args = dict(host(c), state=np64(x0))
    ref, xref = ob.selective(**args)
    mag, xmag = ob.selective(**args, magnitude=True)
    state = x0.clone()
    y = nan_like((B, T, D), io)
    for t in range(T):
        y_t = nan_like((B, D), io)
        lh.selective_step(c["A"], c["dt"][:, t], c["Bm"][:, t], c["Cm"][:, t], c["u"][:, t], state, y_t, h0=c["h0"],
                          dt_bias=c["dt_bias"], z=c["z"][:, t])
        y[:, t] = y_t
    k = 3 * T + N + 64
    check(y, ref, mag, k, io, "y")
    check(state, xref, xmag, k, name="state")


def test_selective_without_options():
    case = (2, 20, 9, 4, 1, None)
    c = scan_case(case, "f32", gate=False)
    del c["h0"], c["dt_bias"]
    ref, mag = ob.selective(**host(c)), ob.selective(**host(c), magnitude=True)
    state, y = nan_like((2, 9, 4)), nan_like((2, 20, 9))
    lh.selective_prefill(state=state, y=y, **c)
    check(y, ref[0], mag[0], 128, name="y")
    check(state, ref[1], mag[1], 128, name="state")
    state.zero_()
    y_t = nan_like((2, 9))
    lh.selective_step(c["A"], c["dt"][:, 0], c["Bm"][:, 0], c["Cm"][:, 0], c["u"][:, 0], state, y_t)
    check(y_t, ref[0][:, 0], mag[0][:, 0], 128, name="y_t")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("case", SCAN, ids=str)
def test_selective_backward(case, gate, io):
    B, T, D, N, G, lengths = case
    c = scan_case(case, io, gate, seed=1)
    dy = dev(gen(T + 1).normal(size=(B, T, D)), io)
    args = dict(host(c), dy=np64(dy), lengths=lengths)
    ref, mag = ob.selective_grad(**args), ob.selective_grad(**args, magnitude=True)
    if lengths is not None:
        poison(dict(c, dy=dy), lengths, [k for k in ("dt", "Bm", "Cm", "u", "z", "dy") if k in c or k == "dy"])
    out = dict(dA=nan_like((D, N)), ddt=nan_like((B, T, D), io), dBm=nan_like((B, T, G, N), io),
               dCm=nan_like((B, T, G, N), io), du=nan_like((B, T, D), io), dh0=nan_like((D,)), ddt_bias=nan_like((D,)))
    if gate:
        out["dz"] = nan_like((B, T, D), io)
    lh.selective_backward(dy=dy, lengths=device_lengths(lengths), **c, **out)
    for k, v in out.items():
        check(v, ref[k], mag[k], 8 * B * T + D + N + 128, io if v.dtype is torch.bfloat16 else "f32", k)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_large_steps_and_slow_poles(io):
    # steps from e^-20 to 20, poles from none to immediate decay, gates far out on both sides
    B, T, D, N = 2, 40, 70, 16
    c = scan_case((B, T, D, N, 1, None), io, strided=False)
    r = gen(77)
    c["dt"] = dev(r.uniform(-20, 20, size=(B, T, D)), io)
    c["A"] = dev(-np.exp(r.uniform(-12, 5, size=(D, N))))
    c["z"] = dev(r.uniform(-120, 120, size=(B, T, D)), io)
    ref, mag = ob.selective(**host(c)), ob.selective(**host(c), magnitude=True)
    state, y = nan_like((B, D, N)), nan_like((B, T, D), io)
    lh.selective_prefill(state=state, y=y, **c)
    # 30 more: the bias is added to dt up to 20 in size, where delta keeps 24 of its 2^-24
    check(y, ref[0], mag[0], 3 * T + N + 94, io, "y")
    check(state, ref[1], mag[1], 3 * T + N + 94, name="state")


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("N", [3, 16])
def test_an_input_that_is_not_finite_stays_in_its_channel(value, N):
    B, T, D = 2, 200, 70
    c = scan_case((B, T, D, N, 1, None), "f32", strided=False)
    y0, s0 = nan_like((B, T, D)), nan_like((B, D, N))
    lh.selective_prefill(state=s0, y=y0, **c)
    c["u"][1, 90, 5] = value
    y, s = nan_like((B, T, D)), nan_like((B, D, N))
    lh.selective_prefill(state=s, y=y, **c)
    assert not torch.isfinite(y[1, 90:, 5]).any() and not torch.isfinite(s[1, 5]).all()
    y[1, 90:, 5], y0[1, 90:, 5] = 0, 0
    s[1, 5], s0[1, 5] = 0, 0
    assert torch.equal(y, y0) and torch.equal(s, s0)


# ---- gradients against differences of the kernels' own outputs

def _directional(loss, x, v, eps):
    """Central difference of loss along v, which perturbs x in place."""
    x0 = x.clone()
    x.copy_(x0 + eps * v)
    hi = loss()
    x.copy_(x0 - eps * v)
    lo = loss()
    x.copy_(x0)
    return (hi - lo) / (2 * eps)


def _check_directions(loss, pairs, eps=2.0 ** -6):
    # truncation eps^2 / 6 of the third derivative and rounding 1e-6 / eps of the terms:
    # both below 1e-3 of the sum of |gradient x direction| for these smooth sums of N(0, 1)
    g = torch.Generator(device="cuda").manual_seed(5)
    for name, x, grad in pairs:
        v = torch.randn(x.shape, generator=g, device="cuda")
        got = _directional(loss, x, v, eps)
        want = (grad.double() * v.double())
        assert abs(got - want.sum().item()) <= 1e-2 * want.abs().sum().item(), (name, got, want.sum().item())


def test_differences():
    r = gen(11)
    # layer norm
    x, w, b, dy = (dev(r.normal(size=s)) for s in ((4, 50), 50, 50, (4, 50)))
    y, mean, rstd = nan_like((4, 50)), nan_like((4,)), nan_like((4,))
    lh.layer_norm(x, w, b, y, mean=mean, rstd=rstd)
    dx, dw, db = nan_like((4, 50)), nan_like((50,)), nan_like((50,))
    lh.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)

    def loss():
        o = nan_like((4, 50))
        lh.layer_norm(x, w, b, o)
        return (o.double() * dy.double()).sum().item()

    _check_directions(loss, [("x", x, dx), ("w", w, dw), ("b", b, db)])
    # short convolution
    x, w, b, dy = (dev(r.normal(size=s)) for s in ((2, 20, 9), (9, 4), 9, (2, 20, 9)))
    dx, dw, db = nan_like((2, 20, 9)), nan_like((9, 4)), nan_like((9,))
    lh.short_conv_backward(dy, x, w, b, dx, dw, db)

    def loss():  # noqa: F811
        o, s = nan_like((2, 20, 9)), nan_like((2, 3, 9))
        lh.short_conv_prefill(x, w, b, s, o)
        return (o.double() * dy.double()).sum().item()

    _check_directions(loss, [("x", x, dx), ("w", w, dw), ("bias", b, db)])
    # selective scan
    c = scan_case((2, 70, 9, 6, 3, None), "f32", strided=False)
    dy = dev(r.normal(size=(2, 70, 9)))
    out = {"d" + k: nan_like(v.shape) for k, v in c.items()}
    lh.selective_backward(dy=dy, **c, **out)

    def loss():  # noqa: F811
        o, s = nan_like((2, 70, 9)), nan_like((2, 9, 6))
        lh.selective_prefill(state=s, y=o, **c)
        return (o.double() * dy.double()).sum().item()

    _check_directions(loss, [(k, v, out["d" + k]) for k, v in c.items()], eps=2.0 ** -8)


# ---- calls: bits, streams, graphs, long tensors

def _block_calls(io="bf16"):
    """One call of each entry point on fixed inputs: (run, outputs, in/out states)."""
    B, T, D, N, K = 2, 150, 70, 16, 4
    r = gen(21)
    c = scan_case((B, T, D, N, 2, None), io)
    x, w, b = dev(r.normal(size=(B, T, D)), io), dev(r.normal(size=D)), dev(r.normal(size=D))
    taps, dy = dev(r.normal(size=(D, K))), dev(r.normal(size=(B, T, D)), io)
    o = {k: nan_like((B, T, D), io) for k in ("y", "dx", "cy", "cdx", "sy", "ddt", "du", "dz")}
    o.update({k: nan_like((D,)) for k in ("dw", "db", "cdb", "dh0", "ddt_bias")})
    o.update(mean=nan_like((B, T)), rstd=nan_like((B, T)), cdw=nan_like((D, K)), dA=nan_like((D, N)),
             dBm=nan_like((B, T, 2, N), io), dCm=nan_like((B, T, 2, N), io))
    cstate, sstate = nan_like((B, K - 1, D), io), nan_like((B, D, N))
    cy_t, sy_t = nan_like((B, D), io), nan_like((B, D), io)

    def run():
        lh.layer_norm(x, w, b, o["y"], mean=o["mean"], rstd=o["rstd"])
        lh.layer_norm_backward(dy, x, w, o["mean"], o["rstd"], o["dx"], o["dw"], o["db"])
        lh.short_conv_prefill(x, taps, b, cstate, o["cy"])
        lh.short_conv_step(x[:, 3], taps, b, cstate, cy_t)
        lh.short_conv_backward(dy, x, taps, b, o["cdx"], o["cdw"], o["cdb"])
        lh.selective_prefill(state=sstate, y=o["sy"], **c)
        lh.selective_step(c["A"], c["dt"][:, 3], c["Bm"][:, 3], c["Cm"][:, 3], c["u"][:, 3], sstate, sy_t, h0=c["h0"])
        lh.selective_backward(dy=dy, **c, **{k: o[k] for k in ("dA", "ddt", "dBm", "dCm", "du", "dh0", "ddt_bias", "dz")})

    return run, list(o.values()) + [cstate, sstate, cy_t, sy_t]


def _poison(outputs):
    for t in outputs:
        t.fill_(float("nan"))


def test_same_bits_again_and_on_another_stream():
    run, outputs = _block_calls()
    run()
    torch.cuda.synchronize()
    first = [t.clone() for t in outputs]
    assert all(torch.isfinite(t.float()).all() for t in first)
    _poison(outputs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, outputs))


def test_graph_replays():
    run, outputs = _block_calls()
    run()
    torch.cuda.synchronize()
    first = [t.clone() for t in outputs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(3):
        _poison(outputs)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        junk = torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outputs))
        del junk


def test_workspace_from_another_stream_and_too_small():
    c = scan_case((1, 300, 96, 16, 1, None), "f32")
    need = lh.selective_workspace_bytes(1, 300, 96, 16)
    assert need > 0
    y, s = nan_like((1, 300, 96)), nan_like((1, 96, 16))
    with pytest.raises(lh.LHError) as e:
        lh.selective_prefill(state=s, y=y, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"), **c)
    assert e.value.status == 5
    assert torch.isnan(y).all() and torch.isnan(s).all()
    lh.selective_prefill(state=s, y=y, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), **c)
    y2, s2 = nan_like((1, 300, 96)), nan_like((1, 96, 16))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    lh.selective_prefill(state=s2, y=y2, stream=side, **c)  # its workspace is the side stream's
    junk = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    side.synchronize()
    assert torch.equal(y, y2) and torch.equal(s, s2)
    del junk


def test_offsets_past_32_bits():
    """Tensors of more than 2^31 elements: the last tokens of a row against the same
    tokens on their own, continued from the state before them."""
    T, D, tail = (1 << 21) + 70, 1056, 100
    u = torch.empty((1, T, D), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    y = torch.empty_like(u)
    w, b = dev(gen(1).normal(size=D)), dev(gen(2).normal(size=D))
    lh.layer_norm(u, w, b, y)
    args = (np64(u[0, -tail:]), np64(w), np64(b))
    ref = ob.layer_norm(*args)[0]
    mag, _, top, rs = ob.layer_norm(*args, magnitude=True)
    check(y[0, -tail:], ref, mag + 0.5 * (1 + top * rs)[:, None] * np.abs(ref - args[2]), 128, "bf16", "y")
    part = torch.empty((1, tail, D), dtype=torch.bfloat16, device="cuda")
    taps = dev(gen(3).normal(size=(D, 4)))
    state, end = (torch.empty((1, 3, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lh.short_conv_prefill(u, taps, b, end, y)
    state.copy_(u[:, -tail - 3:-tail])
    lh.short_conv_prefill(u[:, -tail:], taps, b, state, part, resume=True)
    assert torch.equal(y[:, -tail:], part) and torch.equal(state, end)
    r = gen(4)
    bc = torch.empty((1, T, 1, 8), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    A, bias = dev(-np.exp(r.normal(size=(D, 4)))), dev(r.normal(size=D) - 2)
    args = lambda t: dict(dt=u[:, t], Bm=bc[:, t, :, :4], Cm=bc[:, t, :, 4:], u=u[:, t], A=A, dt_bias=bias)  # noqa: E731
    x, x2 = nan_like((1, D, 4)), nan_like((1, D, 4))
    lh.selective_prefill(state=x, y=y, **args(slice(None)))
    n = torch.tensor([T - tail], dtype=torch.int32, device="cuda")
    last = y[:, -tail:].clone()
    lh.selective_prefill(state=x2, y=y, lengths=n, **args(slice(None)))
    assert not y[:, -tail:].any()
    lh.selective_prefill(state=x2, y=part, resume=True, **args(slice(T - tail, None)))
    # the two cut the tokens into chunks differently: 3 tail + N + 64 roundings of the state's scale
    scale = x.abs().amax().item()
    assert (x - x2).abs().amax().item() <= 400 * U * scale
    assert (part.float() - last.float()).abs().amax().item() <= 2.0 ** -7 * last.float().abs().amax().item()
