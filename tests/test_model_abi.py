"""What the entry points of the gated recurrence, the embedding, the distillation of logits
and the verification of drafts refuse, on the host and before any device work (no GPU
needed: the addresses are made up, and only calls that must be refused are made)."""
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


def inputs(**kw):
    s = lh._GatedInputs()
    a = dict(rate=A, r_bias=A + MB, i_bias=A + 2 * MB, r=A + 3 * MB, i=A + 4 * MB, u=A + 5 * MB, z=A + 6 * MB, lengths=None,
             ld_r=8, ld_i=8, ld_u=8, ld_z=8, B=2, T=3, D=8, io_dtype=0)
    a.update(kw)
    for k, v in a.items():
        setattr(s, k, v)
    return s


def gated(state=A + 8 * MB, y=A + 9 * MB, marks=None, ws=None, ws_bytes=0, **kw):
    s = inputs(**kw)
    return lambda: lh.lib().lh_gated_prefill(ctypes.byref(s), 0, state, y, marks, ws, ws_bytes, None)


def test_gated_refusals():
    L = lh.lib()
    assert L.lh_gated_prefill(None, 0, A, A + MB, None, None, 0, None) == INVALID
    refused(INVALID, gated(B=0), "B")
    refused(INVALID, gated(T=-1), "T")
    refused(INVALID, gated(D=0), "D")
    refused(INVALID, gated(B=1 << 16, D=1 << 16, T=1, ld_r=1 << 16, ld_i=1 << 16, ld_u=1 << 16, ld_z=1 << 16), "threads")
    refused(INVALID, gated(B=1 << 30, D=1 << 30), "overflow")
    refused(INVALID, gated(rate=None), "rate")
    refused(INVALID, gated(i=None), "NULL")
    refused(INVALID, gated(state=None), "NULL")
    refused(INVALID, gated(y=None), "NULL")
    refused(INVALID, gated(ld_i=7), "ld_i")
    refused(INVALID, gated(ld_z=7), "ld_z")
    refused(INVALID, gated(ld_u=1 << 26), "2^26")
    refused(INVALID, gated(r=A + 3 * MB + 2), "aligned")
    refused(INVALID, gated(lengths=A + 10 * MB + 1), "aligned")
    refused(DTYPE, gated(io_dtype=2))
    refused(OVERLAP, gated(y=A + 5 * MB), "y overlaps u")
    refused(OVERLAP, gated(ld_u=16, y=A + 5 * MB + 32), "y overlaps u")  # between the rows of u
    refused(OVERLAP, gated(state=A + 9 * MB + 4), "overlaps")
    refused(OVERLAP, gated(marks=A + 8 * MB), "overlaps")
    need = lh.gated_workspace_bytes(1, 4096, 64)
    assert need > 0
    refused(WORKSPACE, gated(B=1, T=4096, D=64, ld_r=64, ld_i=64, ld_u=64, ld_z=64, r=A + 20 * MB, i=A + 30 * MB,
                             u=A + 40 * MB, z=A + 50 * MB, y=A + 60 * MB), "NULL")
    assert L.lh_gated_workspace_bytes(0, 1, 1) == BAD and L.lh_gated_workspace_bytes(1, 1, 1) == 0
    step = lambda **kw: L.lh_gated_step(ctypes.byref(inputs(**kw)), A + 8 * MB, A + 9 * MB, None)  # noqa: E731
    assert step() == INVALID  # T = 3
    assert step(T=1, lengths=A + 10 * MB) == INVALID
    assert L.lh_gated_step(ctypes.byref(inputs(T=1)), A + 8 * MB, None, None) == INVALID
    assert L.lh_gated_step(ctypes.byref(inputs(T=1)), A + 8 * MB, A + 8 * MB, None) == OVERLAP


def test_gated_backward_refusals():
    need = lh.gated_backward_workspace_bytes(2, 3, 8)
    assert need > 0 and lh.lib().lh_gated_backward_workspace_bytes(2, -3, 8) == BAD

    def back(ws=A + 40 * MB, ws_bytes=need, inp=None, **kw):
        s, g = inputs(**(inp or {})), lh._GatedGrads()
        a = {k: A + (20 + j) * MB for j, (k, _) in enumerate(lh._GatedGrads._fields_)}
        a.update(kw)
        for k, v in a.items():
            setattr(g, k, v)
        return lambda: lh.lib().lh_gated_backward(ctypes.byref(s), ctypes.byref(g), ws, ws_bytes, None)

    refused(INVALID, back(drate=None), "drate")
    refused(INVALID, back(marks=None), "marks")
    refused(INVALID, back(dy=None), "NULL")
    refused(INVALID, back(dz=None), "dz")
    refused(INVALID, back(inp=dict(z=None)), "dz")
    refused(INVALID, back(inp=dict(r_bias=None)), "dr_bias")
    refused(WORKSPACE, back(ws=None), "NULL")
    refused(WORKSPACE, back(ws_bytes=need - 1), "needed")
    refused(INVALID, back(ws=A + 40 * MB + 4), "aligned")
    refused(OVERLAP, back(du=A + 20 * MB), "du overlaps dy")
    refused(OVERLAP, back(dfirst=A + 22 * MB), "dfirst overlaps dlast")
    refused(OVERLAP, back(dr=A + 24 * MB), "overlaps")
    refused(OVERLAP, back(dr=A + 3 * MB), "dr overlaps r")


def test_embed_refusals():
    L = lh.lib()

    def embed(W=A, ids=A + 10 * MB, n=4, V=16, D=8, table=0, io=0, y=A + 20 * MB):
        return lambda: L.lh_embed(W, ids, n, V, D, table, io, 1.0, y, None)

    refused(INVALID, embed(n=-1), "n")
    refused(INVALID, embed(V=0), "V")
    refused(INVALID, embed(D=0), "D")
    refused(INVALID, embed(n=1 << 31), "2^31")
    refused(INVALID, embed(V=1 << 31), "2^31")
    refused(INVALID, embed(V=1 << 30, D=1 << 30), "overflow")
    refused(INVALID, embed(W=None), "NULL")
    refused(INVALID, embed(ids=None), "NULL")
    refused(INVALID, embed(y=None), "NULL")
    refused(INVALID, embed(ids=A + 10 * MB + 2), "aligned")
    refused(DTYPE, embed(table=3))
    refused(DTYPE, embed(io=-1))
    refused(OVERLAP, embed(y=A + 64), "y overlaps W")
    need = lh.embed_backward_workspace_bytes(4, 16, 8)
    assert need > 0 and L.lh_embed_backward_workspace_bytes(4, 0, 8) == BAD
    assert L.lh_embed_backward_workspace_bytes(0, 16, 8) == 0

    def back(dy=A, ids=A + 10 * MB, n=4, V=16, D=8, io=0, dW=A + 20 * MB, ws=A + 30 * MB, ws_bytes=need):
        return lambda: L.lh_embed_backward(dy, ids, n, V, D, io, 1.0, 0, dW, ws, ws_bytes, None)

    refused(INVALID, back(dW=None), "NULL")
    refused(INVALID, back(dy=None), "NULL")
    refused(INVALID, back(dy=A + 1), "aligned")
    refused(DTYPE, back(io=2))
    refused(WORKSPACE, back(ws=None), "NULL")
    refused(WORKSPACE, back(ws_bytes=need - 1), "needed")
    refused(INVALID, back(ws=A + 30 * MB + 128), "aligned")
    refused(OVERLAP, back(dW=A), "dW overlaps dy")
    refused(OVERLAP, back(dW=A + 30 * MB), "overlaps")


def test_distill_logits_refusals():
    L = lh.lib()

    def loss(logits=A, ld=32, values=A + 10 * MB, ids=A + 11 * MB, scale=None, rows=4, V=32, K=3, io=0, tau=1.0,
             loss=A + 12 * MB, lse=None, dlogits=None, ld_d=0):
        return lambda: L.lh_distill_logits(logits, ld, values, ids, scale, rows, V, K, io, tau, loss, lse, dlogits, ld_d,
                                           None, 0, None)

    refused(INVALID, loss(rows=-1), "rows")
    refused(INVALID, loss(V=0), "V")
    refused(INVALID, loss(V=1 << 31, ld=1 << 31), "2^31")
    refused(INVALID, loss(K=0), "K")
    refused(INVALID, loss(K=1025), "K")
    refused(INVALID, loss(ld=31), "ld_logits")
    refused(INVALID, loss(tau=0.0), "tau")
    refused(INVALID, loss(tau=-1.0), "tau")
    refused(INVALID, loss(tau=float("inf")), "tau")
    refused(INVALID, loss(tau=float("nan")), "tau")
    refused(INVALID, loss(values=None), "NULL")
    refused(INVALID, loss(loss=None), "loss")
    refused(INVALID, loss(dlogits=A + 13 * MB, ld_d=16), "ld_dlogits")
    refused(DTYPE, loss(io=9))
    refused(OVERLAP, loss(dlogits=A + 128, ld_d=32), "dlogits overlaps logits")
    refused(OVERLAP, loss(ld=40, dlogits=A, ld_d=32), "dlogits overlaps logits")  # other rows of the same buffer
    refused(OVERLAP, loss(lse=A + 12 * MB), "overlaps")
    refused(OVERLAP, loss(loss=A + 10 * MB), "loss overlaps values")
    assert L.lh_distill_logits_workspace_bytes(4, 32, 0) == BAD

    def back(dloss=A + 14 * MB, lse=A + 15 * MB, dlogits=A + 16 * MB, ld_d=32, **kw):
        a = dict(logits=A, ld=32, values=A + 10 * MB, ids=A + 11 * MB, scale=None)
        a.update(kw)
        return lambda: L.lh_distill_logits_backward(dloss, *a.values(), lse, 4, 32, 3, 0, 1.0, dlogits, ld_d, None)

    refused(INVALID, back(dloss=None), "NULL")
    refused(INVALID, back(lse=None), "NULL")
    refused(INVALID, back(dlogits=None), "NULL")
    refused(OVERLAP, back(dlogits=A + 11 * MB), "dlogits overlaps ids")


def test_verify_draft_refusals():
    L = lh.lib()
    need = lh.verify_draft_workspace_bytes(2, 3, 100)
    assert need > 0 and L.lh_verify_draft_workspace_bytes(2, 65, 100) == BAD

    def verify(ws_bytes=need, **kw):
        a = dict(drafted=A, lengths=None, draft_p=A + 10 * MB, ld_d=100, target_p=A + 20 * MB, ld_t=100, u=A + MB,
                 u_last=A + 2 * MB, B=2, K=3, V=100, io=0, accepted=A + 3 * MB, tokens=A + 4 * MB, ws=A + 5 * MB)
        a.update(kw)
        return lambda: L.lh_verify_draft(*a.values(), ws_bytes, None)

    refused(INVALID, verify(B=0), "B")
    refused(INVALID, verify(K=0), "K")
    refused(INVALID, verify(K=65), "K")
    refused(INVALID, verify(V=0), "V")
    refused(INVALID, verify(V=1 << 31, ld_d=1 << 31, ld_t=1 << 31), "2^31")
    refused(INVALID, verify(ld_d=99), "ld_draft")
    refused(INVALID, verify(ld_t=99), "ld_target")
    refused(INVALID, verify(u=None), "NULL")
    refused(INVALID, verify(tokens=None), "NULL")
    refused(INVALID, verify(accepted=A + 3 * MB + 2), "aligned")
    refused(DTYPE, verify(io=4))
    refused(WORKSPACE, verify(ws=None), "NULL")
    refused(WORKSPACE, verify(ws_bytes=need - 1), "needed")
    refused(OVERLAP, verify(tokens=A), "tokens overlaps drafted")
    refused(OVERLAP, verify(accepted=A + 4 * MB), "overlaps")


def test_binding_refuses_tensors_off_the_device():
    import torch

    x, i = torch.zeros((2, 8)), torch.zeros((2,), dtype=torch.int32)
    with pytest.raises(ValueError, match="HIP device"):
        lh.gated_step(torch.zeros(8), x, x, x, torch.zeros((2, 8)), torch.zeros((2, 8)))
    with pytest.raises(ValueError, match="HIP device"):
        lh.embed(x, i, torch.zeros((2, 8)))
    with pytest.raises(ValueError, match="HIP device"):
        lh.embed_backward(x, i, torch.zeros((4, 8)))
    with pytest.raises(ValueError, match="HIP device"):
        lh.distill_logits(x, x, i, torch.zeros(2))
    with pytest.raises(TypeError, match="dlogits"):
        lh.distill_logits_backward(torch.zeros(2), x, x, i, torch.zeros(2), None)
    with pytest.raises(ValueError, match="HIP device"):
        lh.verify_draft(torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 4, 8)), x, x, i, i)
    with pytest.raises(lh.LHError):
        lh.verify_draft_workspace_bytes(1, 0, 8)


def test_the_binding_knows_the_headers_constants():
    import os
    import re

    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "lh.h")).read()
    assert int(re.search(r"#define LH_GATED_MARK (\d+)", text).group(1)) == lh.GATED_MARK
