"""Workspaces and limits of the embedding's gradient and of the distillation as include/lh.h states them
(no GPU needed)."""
from __future__ import annotations

import ctypes

import pytest

import paper_2310_18780_amd as lh

BAD = ctypes.c_size_t(-1).value


def up(x):
    return -(-x // 256) * 256


@pytest.mark.parametrize("D", [1, 3, 64, 1025, 2048])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 75, 8192, 8193, 65536, 131073, 1 << 20])
def test_embedding_gradient_takes_what_the_header_says(n, D):
    arrays, parts = 4 * up(4 * n), 8 * D * -(-n // (16 if n <= 8192 else 64))
    for V in (1, 500, 50000, 200000, (1 << 31) // D - 1):
        need = lh.embed_backward_workspace_bytes(n, V, D)
        counts = need - arrays - parts
        assert counts == 0 if n <= 8192 else 0 < counts <= 256 << 10 and counts % 256 == 0


@pytest.mark.parametrize("D,n", [(1, 1 << 28), (1024, 1 << 28), (1025, 1 << 27), (2048, 1 << 27)])
def test_embedding_gradients_largest_number_of_tokens(D, n):
    call = lh.lib().lh_embed_backward_workspace_bytes
    assert call(n - 64, 1000, D) != BAD
    assert call(n, 1000, D) == BAD and "threads" in lh.lib().lh_last_error().decode()


def test_distillation_takes_none():
    for rows, V, K in ((0, 1, 1), (1, 1, 1), (8192, 50000, 64), (17, 200007, 1024)):
        assert lh.distill_logits_workspace_bytes(rows, V, K) == 0


def test_gated_prompts_take_one_where_workgroups_share_them():
    # below 160 tiles of 64 channels, from three blocks of 128 steps on
    need = lh.gated_workspace_bytes
    assert need(1, 256, 64) == 0 and need(1, 257, 64) > 0
    assert need(159, 1000, 64) > 0 and need(160, 1000, 64) == 0
    assert need(2, 0, 64) == 0
    # a word of 8 bytes for each channel and block, and 4 bytes for each tile, in whole words
    assert need(3, 1000, 100) == 3 * 8 * 8 * 100 + 4 * 6
    assert need(1, 1000, 64) == 8 * 8 * 64 + 8
