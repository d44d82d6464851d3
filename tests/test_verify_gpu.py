"""GPU parity of the verification of drafted tokens against the float64 oracle
``oracle.model``: whole numbers, equal.  (A border that falls within 10^-13 of a cumulative sum
could go either way; the random numbers here have 24 bits, so none of these does but by design,
where the sums are exact.)"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.model as om
import paper_2310_18780_amd as lh

pytestmark = pytest.mark.gpu

IO = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    lh.lib()
    yield


def gen(seed):
    return np.random.default_rng(seed)


def f32(a, io="f32"):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.float32))).to(IO[io]).cuda()


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def run(drafted, target_p, u, u_last, draft_p=None, lengths=None):
    B, K = drafted.shape
    accepted, tokens = torch.full((B,), -9, dtype=torch.int32, device="cuda"), torch.full((B, K + 1), -9, dtype=torch.int32, device="cuda")
    lh.verify_draft(drafted, target_p, u, u_last, accepted, tokens, draft_p=draft_p, lengths=lengths)
    a, t = om.verify(drafted.cpu().numpy(), np64(target_p), u.cpu().numpy(), u_last.cpu().numpy(), np64(draft_p),
                     None if lengths is None else lengths.cpu().numpy())
    assert accepted.tolist() == a.tolist()
    assert tokens.tolist() == t.tolist()
    return accepted, tokens


def probabilities(r, shape, noise=None, sharp=1.3):
    x = -sharp * np.log(r.random(shape) + 1e-9) if noise is None else noise[0] + noise[1] * r.normal(size=shape)
    p = np.exp(x - x.max(-1, keepdims=True))
    return x, p / p.sum(-1, keepdims=True)


def case(B, K, V, io, seed, certain=False, top=0, ragged=False):
    r = gen(seed + B + K + V)
    x, p = probabilities(r, (B, K + 1, V))
    _, q = probabilities(r, (B, K, V), (x[:, :K], 0.4))
    if top:
        for t in (p, q):
            t[t < np.sort(t, -1)[..., -min(top, V)][..., None]] = 0
    c = dict(target_p=f32(p, io), u=f32(r.random((B, K), np.float32)), u_last=f32(r.random(B, np.float32)))
    if certain:
        c["drafted"] = i32(p[:, :K].argmax(-1))
    else:
        c["draft_p"] = f32(q, io)
        c["drafted"] = i32((np.cumsum(q, -1) > r.random((B, K, 1)) * q.sum(-1, keepdims=True)).argmax(-1))
    if ragged:
        c["lengths"] = i32(np.r_[K, 0, K + 3, -2, r.integers(0, K + 1, max(B - 4, 0))][:B])
    return c


SIZES = [(1, 1, 1), (2, 1, 2), (3, 4, 7), (8, 5, 100), (5, 3, 2047), (5, 3, 2048), (5, 3, 2049), (16, 4, 5000), (4, 64, 301),
         (3, 7, 50001), (2, 2, 140000)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_against_the_definition(size, io):
    B, K, V = size
    some = 0
    for seed in range(4):
        a, _ = run(**case(B, K, V, io, seed, certain=seed == 2, top=(0, 20, 0, 3)[seed], ragged=seed % 2 == 1))
        some += int(a.sum())
    assert some > 0 or V < 3 or B < 3


def test_rows_that_lie_apart():
    c = case(6, 4, 333, "bf16", 1)
    for k, extra in (("target_p", 5), ("draft_p", 3)):
        wide = torch.full((*c[k].shape[:2], 333 + extra), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[..., 1:334] = c[k]
        c[k] = wide[..., 1:334]
    run(**c)


def test_borders_go_to_the_lowest_token_past_them():
    # exact sums: 1/8 a token
    V = 8
    p = f32(np.full((9, 2, V), 0.125))
    q = f32(np.full((9, 1, V), 0.125))
    last = f32([k / 8 for k in range(8)] + [1 - 2.0 ** -24])
    a, t = run(i32(np.zeros((9, 1))), p, f32(np.zeros((9, 1))), last, q)
    assert t[:, 1].tolist() == [0, 1, 2, 3, 4, 5, 6, 7, 7]
    # zeros are never drawn, whatever the number
    p = np.zeros((4, 2, 5000))
    p[:, :, [700, 2500, 4999]] = [0.25, 0.5, 0.25]
    a, t = run(i32(np.full((4, 1), 700)), f32(p), f32(np.zeros((4, 1))), f32([0, 0.25, 0.75, 1.0]), f32(p[:, :1]))
    assert t[:, 1].tolist() == [700, 2500, 4999, 4999]


def test_many_tokens_of_equal_weight():
    """A border in every part of a long row, sums exact: 2^-17 a token."""
    V = 1 << 17
    n = 64
    u = (np.arange(n) * 2053 % V) / V
    p = f32(np.full((n, 2, V), 2.0 ** -17))
    _, t = run(i32(np.zeros((n, 1))), p, f32(np.full((n, 1), 0.5)), f32(u), None)
    # a certain draft of token 0 with u = 1/2 is refused: what is left are the tokens from 1 on
    want = np.searchsorted(np.arange(1, V), u * (V - 1), side="right") + 1
    assert t[:, 0].tolist() == want.tolist()


def test_nothing_left():
    V = 3000
    z, one = np.zeros((2, V)), np.eye(V)[5]
    p = np.stack([np.stack([one, z[0]]), z, np.stack([z[0], one]), z])
    q = np.stack([one, z[0], one, one])[:, None]
    # 0: accepted, then nothing to draw; 1: refused (0 < 0 is false), nothing at all; 2: refused, all of q above p, p empty
    a, t = run(i32([[5], [5], [7], [5]]), f32(p), f32([[0.5], [0.0], [0.5], [0.5]]), f32([0.5] * 4), f32(q))
    assert a.tolist() == [1, 0, 0, 0] and t.tolist() == [[5, -1], [-1, -1], [-1, -1], [-1, -1]]
    # refused where p is nowhere above q: drawn from p itself
    p = np.stack([np.stack([0.5 * one, one])])
    a, t = run(i32([[5]]), f32(p), f32([[0.75]]), f32([0.5]), f32(one[None, None]))
    assert a.tolist() == [0] and t.tolist() == [[5, -1]]


def test_odd_entries():
    V = 600
    r = gen(3)
    p, q = (r.random((4, k, V)) for k in (3, 2))
    p[0, 0, ::3] = -1.0        # negative and NaN entries count as nothing
    p[1, 0, ::2] = np.nan
    q[2, 0, 1::2] = np.nan
    # tokens outside the table are not accepted and not read
    run(i32([[V, 1], [-1, 1], [2 ** 31 - 1, 1], [-2 ** 31, 1]]), f32(p), f32(np.zeros((4, 2))), f32(r.random(4)), f32(q))
    run(i32([[V, 1], [-1, 1], [2 ** 31 - 1, 1], [-2 ** 31, 1]]), f32(p), f32(np.zeros((4, 2))), f32(r.random(4)))
    a, _ = run(i32([[1, 1], [1, V], [2, 1], [1, -1]]), f32(p), f32(np.zeros((4, 2))), f32(r.random(4)), f32(q))
    assert a.tolist() == [2, 1, 2, 1]


def test_offsets_past_32_bits():
    B, K, V = 17, 3, 40_000_003
    p = torch.zeros((B, K + 1, V), dtype=torch.bfloat16, device="cuda")
    assert p.numel() > 1 << 31
    p[..., V - 2], p[..., 9] = 0.5, 0.5
    drafted = torch.full((B, K), V - 2, dtype=torch.int32, device="cuda")
    drafted[B - 1, 2] = 8
    accepted, tokens = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty((B, K + 1), dtype=torch.int32, device="cuda")
    u = torch.full((B, K), 0.25, device="cuda")
    lh.verify_draft(drafted, p, u, torch.full((B,), 0.75, device="cuda"), accepted, tokens)
    assert accepted.tolist() == [3] * (B - 1) + [2]
    assert tokens[0].tolist() == [V - 2] * 4 and tokens[-1].tolist() == [V - 2, V - 2, V - 2, -1]
