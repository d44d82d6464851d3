"""Sizes that the selective block's entry points take (no GPU needed: a call whose sizes
pass is refused for a later reason, here an output over an input)."""
from __future__ import annotations

import ctypes

import paper_2310_18780_amd as lh

A = 1 << 44
INVALID, OVERLAP = 1, 2
BAD = ctypes.c_size_t(-1).value


def inputs(B, T, D, N, G=1, gap=1 << 40, **kw):
    s = lh._SelectiveInputs()
    a = dict(A=A, dt=A + gap, u=A + 2 * gap, Bm=A + 3 * gap, Cm=A + 4 * gap, ld_dt=D, ld_u=D, ld_B=G * N, ld_C=G * N, B=B, T=T,
             D=D, N=N, G=G, io_dtype=1)
    a.update(kw)
    for k, v in a.items():
        setattr(s, k, v)
    return s


def step(*sizes, **kw):
    return lh.lib().lh_selective_step(ctypes.byref(inputs(sizes[0], 1, *sizes[1:], **kw)), A + 5 * (1 << 40), A + (1 << 40), None)


def prefill(*sizes, **kw):
    return lh.lib().lh_selective_prefill(ctypes.byref(inputs(*sizes, **kw)), 0, A + 5 * (1 << 40), A + (1 << 40), None, 0, None)


def test_many_sessions_take_a_step():
    # 32768 sessions of 2048 channels with 16 states (4.3 GB of state): 2^28 threads
    assert step(32768, 2048, 16) == OVERLAP
    assert step(1 << 20, 2048, 4) == OVERLAP  # 2^31 threads
    assert step(1 << 20, 4096, 4) == INVALID and b"threads" in lh.lib().lh_last_error()  # 2^32
    assert step(1 << 17, 2048, 128) == INVALID  # 2^28 rows of 32 lanes


def test_large_batches_take_a_prompt_and_a_gradient():
    # 4 wavefronts to each of 2^20 tiles
    assert prefill(32768, 1, 2048, 16) == OVERLAP
    assert lh.selective_workspace_bytes(32768, 1, 2048, 16) == 0
    assert prefill(1 << 19, 1, 2048, 16) == INVALID and b"threads" in lh.lib().lh_last_error()
    assert 0 < lh.selective_backward_workspace_bytes(32768, 1, 2048, 16) < BAD
    # the gradient's carry: two threads to each of 2^31 states
    assert lh.lib().lh_selective_backward_workspace_bytes(1 << 16, 1, 2048, 16, 1) == BAD


def test_rows_far_apart():
    # token t of [B, 65536, 2048]: its rows lie 2^27 elements apart
    far = dict(ld_dt=1 << 27, ld_u=1 << 27, ld_B=1 << 27, ld_C=1 << 27)
    assert step(2, 2048, 16, **far) == OVERLAP
    assert prefill(2, 1, 2048, 16, **far) == INVALID and b"2^26" in lh.lib().lh_last_error()
    g = lh._SelectiveGrads()
    for i, k in enumerate(("dy", "ddt", "du", "dBm", "dCm", "dA")):
        setattr(g, k, A + (6 + i) * (1 << 40))
    g.du = A + (1 << 40)  # over dt
    need = lh.selective_backward_workspace_bytes(2, 1, 2048, 16)
    assert lh.lib().lh_selective_backward(ctypes.byref(inputs(2, 1, 2048, 16, **far)), ctypes.byref(g), A + (13 << 40), need,
                                          None) == OVERLAP


def test_prompts_of_many_states_are_cut_where_that_is_faster():
    # 2048 steps and channels, us in one pass and in chunks: 64 states, 4 rows 436 and 389; 128
    # states, 2 rows 786 and 379, 4 rows 792 and 711; 32 states, 8 rows 275 and 328
    cut = lambda B, N: lh.selective_workspace_bytes(B, 2048, 2048, N) > 0  # noqa: E731
    assert cut(4, 64) and cut(2, 128) and cut(4, 128)
    assert not cut(8, 32) and not cut(8, 64) and not cut(8, 128)
    # up to 16 states: 4 rows 199 and 133, 8 rows 199 and 232
    assert cut(4, 16) and not cut(8, 16)
