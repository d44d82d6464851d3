"""The selective block's calls at sizes whose offsets pass 32 bits, against the oracle on the
last rows.  Tolerances are those derived in ``test_block_gpu``."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.block as ob
import paper_2310_18780_amd as lh
from test_block_gpu import check, dev, gen, host, np64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    lh.lib()
    yield


def randn(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)


def test_a_step_of_many_sessions():
    B, D, N = 32768, 2048, 16  # 4.3 GB of state
    r = gen(40)
    c = dict(A=dev(-abs(r.normal(size=(D, N))) - 0.1), h0=dev(r.normal(size=D)), dt_bias=dev(r.normal(size=D) - 2))
    rows = dict(dt=randn(1, B, D), u=randn(2, B, D), z=randn(3, B, D), Bm=randn(4, B, 1, N), Cm=randn(5, B, 1, N))
    state = randn(6, B, D, N, dtype=torch.float32)
    last = slice(B - 2, B)
    args = dict(host(c), **{k: np64(v[last])[:, None] for k, v in rows.items()}, state=np64(state[last]))
    ref, xref = ob.selective(**args)
    mag, xmag = ob.selective(**args, magnitude=True)
    y = torch.full((B, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    lh.selective_step(c["A"], rows["dt"], rows["Bm"], rows["Cm"], rows["u"], state, y, h0=c["h0"], dt_bias=c["dt_bias"],
                      z=rows["z"])
    check(y[last], ref[:, 0], mag[:, 0], 3 + N + 64, "bf16", "y")
    check(state[last], xref, xmag, 3 + N + 64, name="state")
    assert torch.isfinite(y).all()


def test_steps_and_a_gradient_on_rows_far_apart():
    """Tokens taken as slices of a long buffer: rows 2^26 elements and more apart."""
    B, D, N, far = 2, 70, 16, (1 << 26) + 5
    r = gen(41)
    wide = torch.full((B * far,), float("nan"), dtype=torch.bfloat16, device="cuda").view(B, far)
    rows = {}
    at = 3
    for k, n in (("dt", D), ("u", D), ("Bm", N), ("Cm", N)):
        wide[:, at:at + n] = dev(r.normal(size=(B, n)), "bf16")
        rows[k] = wide[:, at:at + n]
        at += n + 1
    rows["Bm"], rows["Cm"] = rows["Bm"].unflatten(1, (1, N)), rows["Cm"].unflatten(1, (1, N))
    c = dict(A=dev(-abs(r.normal(size=(D, N)))), h0=dev(r.normal(size=D)), dt_bias=dev(r.normal(size=D) - 2))
    state = dev(r.normal(size=(B, D, N)))
    args = dict(host(c), **{k: np64(v)[:, None] for k, v in rows.items()})
    ref, xref = ob.selective(**args, state=np64(state))
    mag, xmag = ob.selective(**args, state=np64(state), magnitude=True)
    y = torch.empty((B, D), dtype=torch.bfloat16, device="cuda")
    lh.selective_step(c["A"], rows["dt"], rows["Bm"], rows["Cm"], rows["u"], state, y, h0=c["h0"], dt_bias=c["dt_bias"])
    check(y, ref[:, 0], mag[:, 0], 3 + N + 64, "bf16", "y")
    check(state, xref, xmag, 3 + N + 64, name="state")
    one = {k: v[:, None] for k, v in rows.items()}  # prompts of one token
    dy = dev(r.normal(size=(B, 1, D)), "bf16")
    out = {"d" + k: torch.full(v.shape, float("nan"), dtype=v.dtype, device="cuda") for k, v in {**c, **one}.items()}
    lh.selective_backward(dy=dy, **c, **one, **out)
    gref, gmag = ob.selective_grad(np64(dy), **args), ob.selective_grad(np64(dy), **args, magnitude=True)
    for k, v in out.items():
        check(v, gref[k], gmag[k], 8 * B + D + N + 128, "bf16" if v.dtype is torch.bfloat16 else "f32", k)


def test_gradients_past_32_bits():
    """Tensors of more than 2^31 elements: the last tokens' gradients against the oracle on
    those tokens and enough before them."""
    T, D, N, tail, keep = (1 << 21) + 70, 1056, 2, 160, 40
    dy, x = randn(1, 1, T, D), randn(2, 1, T, D)
    last, own = slice(T - tail, T), slice(tail - keep, tail)
    # layer norm: rows are independent
    w, mean, rstd = dev(gen(1).normal(size=D)), torch.zeros((1, T), device="cuda"), torch.ones((1, T), device="cuda")
    dx, dw = torch.empty_like(x), torch.empty(D, device="cuda")
    lh.layer_norm_backward(dy, x, w, mean, rstd, dx, dw)
    args = (np64(dy[0, last]), np64(x[0, last]), np64(w), np64(mean[0, last]), np64(rstd[0, last]))
    check(dx[0, last], ob.layer_norm_grad(*args)[0], ob.layer_norm_grad(*args, magnitude=True)[0], 192, "bf16", "dx")
    # convolution: a token's gradient needs K - 1 tokens on both sides
    K = 4
    taps, bias, dtaps = dev(gen(2).normal(size=(D, K))), dev(gen(3).normal(size=D)), torch.empty((D, K), device="cuda")
    lh.short_conv_backward(dy, x, taps, bias, dx, dtaps)
    args = dict(dy=np64(dy[:, last]), x=np64(x[:, last]), w=np64(taps), bias=np64(bias), silu=True)
    ref, mag = ob.short_conv_grad(**args)[0], ob.short_conv_grad(**args, magnitude=True)[0]
    check(dx[:, last][:, own], ref[:, own], mag[:, own], 3 * K + 24, "bf16", "dx")
    # scan: steps of softplus(4 + N(0, 1)) > 0.1 and poles below -8 leave less than e^-90 of a
    # state after 120 tokens
    r = gen(4)
    A, dt_bias, h0 = dev(-8 - r.random(size=(D, N))), dev(np.full(D, 4.0)), dev(r.normal(size=D))
    rows = randn(3, 1, T, 1, 2 * N)
    c = dict(A=A, dt=x, Bm=rows[..., :N], Cm=rows[..., N:], u=dy, h0=h0, dt_bias=dt_bias)
    out = dict(dA=torch.empty((D, N), device="cuda"), ddt=dx, du=torch.empty_like(x), dh0=torch.empty(D, device="cuda"),
               ddt_bias=torch.empty(D, device="cuda"),
               **{k: torch.empty((1, T, 1, N), dtype=torch.bfloat16, device="cuda") for k in ("dBm", "dCm")})
    lh.selective_backward(dy=dy, **c, **out)
    args = {k: np64(v[:, last]) if k in ("dt", "u", "Bm", "Cm") else np64(v) for k, v in c.items()}
    ref, mag = ob.selective_grad(np64(dy[:, last]), **args), ob.selective_grad(np64(dy[:, last]), **args, magnitude=True)
    for k in ("ddt", "du", "dBm", "dCm"):
        check(out[k][:, last][:, own], ref[k][:, own], mag[k][:, own], 8 * tail + D + N + 128, "bf16", k)
