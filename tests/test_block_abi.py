"""What the selective block's entry points refuse, on the host and before any device
work (no GPU needed: the addresses are made up, and only calls that must be refused
are made)."""
from __future__ import annotations

import ctypes

import pytest

import paper_2310_18780_amd as lh

A = 0x7F0000000000
MB = 1 << 20
BAD = ctypes.c_size_t(-1).value
INVALID, OVERLAP, DTYPE, WORKSPACE = 1, 2, 3, 5


def refused(status, call, *words):
    assert call() == status
    text = lh.lib().lh_last_error().decode()
    for w in words:
        assert w in text, text


def norm(**kw):
    a = dict(x=A, residual=None, w=A + MB, b=A + 2 * MB, rows=4, D=64, eps=1e-5, io=0, y=A + 3 * MB, total=None,
             mean=None, rstd=None, stream=None)
    a.update(kw)
    return lambda: lh.lib().lh_layer_norm(*a.values())


def norm_backward(**kw):
    a = dict(dy=A, x=A + MB, w=A + 2 * MB, mean=A + 3 * MB, rstd=A + 4 * MB, dtotal=None, rows=4, D=64, io=0,
             dx=A + 5 * MB, dw=A + 6 * MB, db=A + 7 * MB, ws=A + 8 * MB, ws_bytes=MB, stream=None)
    a.update(kw)
    return lambda: lh.lib().lh_layer_norm_backward(*a.values())


def test_layer_norm_refusals():
    refused(INVALID, norm(rows=-1), "rows")
    refused(INVALID, norm(D=0), "D")
    refused(INVALID, norm(rows=1 << 40, D=1 << 26), "overflow")
    refused(INVALID, norm(rows=1, D=1 << 30), "threads")
    refused(INVALID, norm(x=None), "NULL")
    refused(INVALID, norm(w=None), "NULL")
    refused(INVALID, norm(eps=-1.0), "eps")
    refused(INVALID, norm(eps=float("nan")), "eps")
    refused(INVALID, norm(total=A + 9 * MB), "residual")
    refused(INVALID, norm(x=A + 2), "aligned")
    refused(DTYPE, norm(io=7), "io_dtype")
    refused(OVERLAP, norm(y=A), "y overlaps x")
    refused(OVERLAP, norm(residual=A + 9 * MB, total=A + 9 * MB + 256), "total overlaps residual")
    refused(OVERLAP, norm(residual=A + 9 * MB, total=A + 3 * MB), "overlaps")
    refused(OVERLAP, norm(mean=A + 3 * MB), "overlaps")


def test_layer_norm_backward_refusals():
    refused(INVALID, norm_backward(dw=None), "NULL")
    refused(INVALID, norm_backward(mean=None), "NULL")
    refused(WORKSPACE, norm_backward(ws=None), "NULL")
    refused(WORKSPACE, norm_backward(ws_bytes=64), "needed")
    refused(INVALID, norm_backward(ws=A + 8 * MB + 64), "aligned")
    refused(OVERLAP, norm_backward(dx=A), "dx overlaps dy")
    refused(OVERLAP, norm_backward(dtotal=A + 9 * MB, dx=A + 9 * MB + 16), "dx overlaps dtotal")
    assert lh.lib().lh_layer_norm_backward_workspace_bytes(-1, 4) == BAD
    assert lh.lib().lh_layer_norm_backward_workspace_bytes(0, 4) == 0


def conv(**kw):
    a = dict(x=A, ld=8, w=A + MB, bias=A + 2 * MB, lengths=None, B=2, T=3, D=8, K=4, io=0, silu=1, resume=0,
             state=A + 3 * MB, y=A + 4 * MB, stream=None)
    a.update(kw)
    return lambda: lh.lib().lh_short_conv_prefill(*a.values())


def test_short_conv_refusals():
    refused(INVALID, conv(B=0), "B")
    refused(INVALID, conv(T=-1), "T")
    refused(INVALID, conv(D=0), "D")
    refused(INVALID, conv(K=0), "K")
    refused(INVALID, conv(K=9), "K")
    refused(INVALID, conv(ld=7), "ld_x")
    refused(INVALID, conv(B=1 << 20, D=1 << 20, T=0), "threads")
    refused(INVALID, conv(state=None), "NULL")
    refused(INVALID, conv(y=None), "NULL")
    refused(INVALID, conv(lengths=A + 5 * MB + 2), "aligned")
    refused(DTYPE, conv(io=2))
    refused(OVERLAP, conv(y=A + 64), "y overlaps x")
    refused(OVERLAP, conv(ld=16, y=A + 32), "y overlaps x")  # between the rows of x
    refused(OVERLAP, conv(state=A + MB), "state overlaps w")
    L = lh.lib()
    assert L.lh_short_conv_step(A, 8, A + MB, None, 2, 8, 9, 0, 1, A + 2 * MB, A + 3 * MB, None) == INVALID
    assert L.lh_short_conv_step(A, 8, A + MB, None, 2, 8, 4, 0, 1, None, A + 3 * MB, None) == INVALID
    assert L.lh_short_conv_step(A, 8, A + MB, None, 2, 8, 4, 0, 1, A + 2 * MB, A, None) == OVERLAP
    back = lambda ws, n: L.lh_short_conv_backward(A, A + MB, 8, A + 2 * MB, None, None, 2, 3, 8, 4, 0, 1,  # noqa: E731
                                                  A + 3 * MB, A + 4 * MB, None, ws, n, None)
    assert back(None, 0) == WORKSPACE and back(A + 5 * MB, 16) == WORKSPACE
    assert L.lh_short_conv_backward_workspace_bytes(2, 3, 8, 9) == BAD


def inputs(**kw):
    s = lh._SelectiveInputs()
    a = dict(A=A, dt_bias=A + MB, h0=A + 2 * MB, dt=A + 3 * MB, u=A + 4 * MB, z=A + 5 * MB, Bm=A + 6 * MB, Cm=A + 7 * MB,
             lengths=None, ld_dt=8, ld_u=8, ld_z=8, ld_B=8, ld_C=8, B=2, T=3, D=8, N=4, G=2, io_dtype=0)
    a.update(kw)
    for k, v in a.items():
        setattr(s, k, v)
    return s


def scan(state=A + 8 * MB, y=A + 9 * MB, ws=None, ws_bytes=0, **kw):
    s = inputs(**kw)
    return lambda: lh.lib().lh_selective_prefill(ctypes.byref(s), 0, state, y, ws, ws_bytes, None)


def test_selective_refusals():
    assert lh.lib().lh_selective_prefill(None, 0, A, A + MB, None, 0, None) == INVALID
    refused(INVALID, scan(B=0), "B")
    refused(INVALID, scan(T=-1), "T")
    refused(INVALID, scan(N=0), "N")
    refused(INVALID, scan(N=129), "N")
    refused(INVALID, scan(G=3), "multiple")
    refused(INVALID, scan(G=0), "G")
    refused(INVALID, scan(G=16), "multiple")
    refused(INVALID, scan(B=1 << 20, D=1 << 20, ld_dt=1 << 20, ld_u=1 << 20, ld_z=1 << 20), "threads")
    refused(INVALID, scan(A=None), "A")
    refused(INVALID, scan(Bm=None), "NULL")
    refused(INVALID, scan(state=None), "NULL")
    refused(INVALID, scan(ld_B=7), "ld_B")
    refused(INVALID, scan(ld_C=1 << 26), "2^26")
    refused(INVALID, scan(ld_z=7), "ld_z")
    refused(DTYPE, scan(io_dtype=5))
    refused(OVERLAP, scan(y=A + 3 * MB), "y overlaps dt")
    refused(OVERLAP, scan(state=A + 4 * MB), "state overlaps u")
    refused(OVERLAP, scan(state=A + 9 * MB + 4), "overlaps")
    refused(WORKSPACE, scan(T=1000, state=A + 20 * MB, y=A + 30 * MB), "NULL")
    s = inputs()
    assert lh.lib().lh_selective_step(ctypes.byref(s), A + 8 * MB, A + 9 * MB, None) == INVALID  # T = 3
    s = inputs(T=1, lengths=A + 10 * MB)
    assert lh.lib().lh_selective_step(ctypes.byref(s), A + 8 * MB, A + 9 * MB, None) == INVALID
    assert lh.lib().lh_selective_workspace_bytes(1, 1, 8, 129, 1) == BAD


def test_selective_backward_refusals():
    need = lh.selective_backward_workspace_bytes(2, 3, 8, 4, 2)
    assert need > 0 and lh.lib().lh_selective_backward_workspace_bytes(2, 3, 8, 4, 3) == BAD

    def back(ws=A + 40 * MB, ws_bytes=need, inp=None, **kw):
        s, g = inputs(**(inp or {})), lh._SelectiveGrads()
        a = {k: A + (20 + i) * MB for i, k in enumerate(("dy", "ddt", "du", "dz", "dBm", "dCm", "dA", "dh0", "ddt_bias"))}
        a.update(kw)
        for k, v in a.items():
            setattr(g, k, v)
        return lambda: lh.lib().lh_selective_backward(ctypes.byref(s), ctypes.byref(g), ws, ws_bytes, None)

    refused(INVALID, back(dA=None), "dA")
    refused(INVALID, back(dy=None), "NULL")
    refused(INVALID, back(dz=None), "dz")
    refused(INVALID, back(inp=dict(z=None)), "dz")
    refused(INVALID, back(inp=dict(h0=None)), "dh0")
    refused(WORKSPACE, back(ws=None), "NULL")
    refused(WORKSPACE, back(ws_bytes=need - 1), "needed")
    refused(OVERLAP, back(du=A + 20 * MB), "du overlaps dy")
    refused(OVERLAP, back(du=A + 21 * MB), "overlaps")


def test_binding_refuses_tensors_off_the_device():
    import torch

    x, w = torch.zeros((2, 8)), torch.ones(8)
    with pytest.raises(ValueError, match="HIP device"):
        lh.layer_norm(x, w, None, torch.zeros_like(x))
    with pytest.raises(ValueError, match="HIP device"):
        lh.short_conv_step(x, torch.zeros((8, 4)), None, torch.zeros((2, 3, 8)), torch.zeros_like(x))
    with pytest.raises(lh.LHError):
        lh.selective_workspace_bytes(1, 1, 8, 300)
