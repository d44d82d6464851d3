"""GPU parity of the embedding lookup and of its table's gradient.  A lookup is one float32
product and one rounding, which torch's elementary operations give bit for bit; a gradient
sums a row's tokens in float32, one rounding a token (``oracle.model.embed_grad``'s bound)."""
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


def ids_of(a):
    return torch.from_numpy(np.asarray(a, np.int32)).cuda()


def nan_like(shape, io="f32"):
    return torch.full(shape, float("nan"), dtype=IO[io], device="cuda")


@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (5, 9, 3), (64, 100, 2048), (3, 50, 8), (2, 50, 7), (700, 33, 1001), (4099, 500, 70),
                                   (2048, 10, 515), (7, 20, 5000)])
def test_lookup(n, V, D, io, table):
    r = gen(n + D)
    W = dev(r.normal(size=(V, D)), table)
    ids = ids_of(np.where(r.random(n) < 0.2, r.choice([-1, V, 2 ** 31 - 1, -2 ** 31], n), r.integers(0, V, n)))
    y = nan_like((n, D), io)
    lh.embed(W, ids, y, scale=1.7)
    inside = (ids >= 0) & (ids < V)
    ref = torch.where(inside[:, None], W[ids.long().clamp(0, V - 1)].float() * torch.tensor(1.7, device="cuda"), 0.0).to(IO[io])
    assert torch.equal(y, ref)


def test_lookup_shapes_and_rows_that_start_anywhere():
    W = dev(gen(1).normal(size=(30, 40)), "bf16")
    ids = ids_of(gen(2).integers(0, 30, (2, 3, 5)))
    y = nan_like((2, 3, 5, 40), "bf16")
    lh.embed(W, ids, y)
    assert torch.equal(y, W[ids.long()])
    lh.embed(W, ids[:0], y[:0])
    # a table and an output at the odd elements of a buffer
    store, out = torch.empty(30 * 41 + 1, dtype=torch.bfloat16, device="cuda"), torch.empty(15 * 41 + 1, dtype=torch.bfloat16, device="cuda")
    W2, y2 = store[1:].view(30, 41), out[1:].view(15, 41)
    W2.normal_()
    lh.embed(W2, ids.view(-1)[:15].contiguous(), y2)
    assert torch.equal(y2, W2[ids.view(-1)[:15].long()])


def check_gradient(dy, ids, V, scale, dW0=None):
    dW = nan_like((V, dy.shape[-1])) if dW0 is None else dW0.clone()
    lh.embed_backward(dy, ids, dW, scale=scale, accumulate=dW0 is not None)
    ref, bound = om.embed_grad(dy.double().cpu().numpy(), ids.cpu().numpy(), V, scale, None if dW0 is None else dW0.double().cpu().numpy())
    got = dW.double().cpu().numpy()
    bad = ~(np.abs(got - ref) <= bound * U + 1e-30)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[0], got[bad][0], ref[bad][0])
    return dW


# (tokens, rows, columns): placed by counting, or by a sort of one to three digits (more than 8192, where windows are of 64
# tokens and not of 16)
SIZES = [(1, 1, 1), (1, 1000, 5), (2, 3, 8), (16, 4, 70), (17, 2, 3), (300, 40, 130), (4096, 300, 9), (4097, 300, 9), (5000, 7, 33),
         (8191, 4000, 6), (8192, 300, 9), (8193, 300, 9),
         (9000, 5000, 20), (20000, 70000, 4), (12345, 300000, 2), (70000, 513, 5), (3000, 2, 600)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient(size, io):
    n, V, D = size
    r = gen(n + V)
    ids = np.minimum((V * r.random(n) ** 4).astype(np.int64), V - 1)  # a few tokens are most of them
    ids = np.where(r.random(n) < 0.1, -1, ids)
    check_gradient(dev(r.normal(size=(n, D)), io), ids_of(ids), V, 0.3)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 64, 1000, 8192, 8193, 20000])
def test_gradient_of_one_token_over_and_over(n):
    dy = dev(gen(n).normal(size=(n, 12)))
    for ids in (np.zeros(n), np.full(n, 4), np.full(n, -1), np.full(n, 5)):
        check_gradient(dy, ids_of(ids), 5, -2.0)


def test_gradient_adds_to_what_is_there():
    r = gen(5)
    for n, V, D, io in ((50, 300, 33, "bf16"), (9000, 300, 1001, "f32"), (300, 5, 37, "bf16")):
        ids = ids_of(np.where(r.random(n) < 0.3, V + 1, r.integers(0, V // 2 + 1, n)))
        dW0 = dev(r.normal(size=(V, D)))
        dW0[V - 1] = float("inf")  # no token is its: not touched
        ids[ids == V - 1] = 0
        dy = dev(r.normal(size=(n, D)), io)
        dW = check_gradient(dy, ids, V, 0.7, dW0.clamp(max=1e30))
        keep = dW0.clone()
        lh.embed_backward(dy, ids, keep, scale=0.7, accumulate=True)
        assert torch.equal(keep[V - 1], dW0[V - 1]) and torch.equal(keep[:V - 1], dW[:V - 1])


def test_gradient_without_tokens_and_at_odd_addresses():
    dW = nan_like((9, 33))
    lh.embed_backward(nan_like((0, 33)), ids_of(np.zeros(0)), dW)
    assert not dW.any()
    keep = dev(gen(1).normal(size=(9, 33)))
    dW = keep.clone()
    lh.embed_backward(nan_like((0, 33)), ids_of(np.zeros(0)), dW, accumulate=True)
    assert torch.equal(dW, keep)
    for off in (1, 2, 3):  # the zeros are stored in pieces of 16 bytes
        store = nan_like((off + 5 * 7 + 4,))
        lh.embed_backward(dev(np.ones((2, 7))), ids_of([1, 3]), store[off:off + 35].view(5, 7))
        assert store[off:off + 35].view(5, 7).sum(1).tolist() == [0, 7, 0, 7, 0]
        assert torch.isnan(store[:off]).all() and torch.isnan(store[off + 35:]).all()


def test_gradient_adds_in_the_order_of_the_tokens():
    """Sums in float32 depend on their order: two calls, and a call whose other tokens differ,
    give a row the same bits."""
    r = gen(6)
    n, V, D = 30000, 50, 64
    dy = dev(r.normal(size=(n, D)))
    ids = ids_of(np.minimum((V * r.random(n) ** 2).astype(np.int64), V - 1))
    a, b = nan_like((V, D)), nan_like((V, D))
    lh.embed_backward(dy, ids, a)
    for _ in range(3):
        lh.embed_backward(dy, ids, b.fill_(float("nan")))
        assert torch.equal(a, b)


def test_values_that_are_not_finite_stay_in_their_row():
    n, V, D = 5000, 40, 16
    r = gen(7)
    ids = r.integers(0, V, n)
    ids[100] = ids[3000] = 11
    dy = dev(r.normal(size=(n, D)))
    clean, dW = nan_like((V, D)), nan_like((V, D))
    lh.embed_backward(dy, ids_of(ids), clean)
    dy[100, 3], dy[3000, 4] = float("nan"), float("inf")
    lh.embed_backward(dy, ids_of(ids), dW)
    same = torch.ones((V, D), dtype=torch.bool, device="cuda")
    same[11, 3:5] = False
    assert torch.equal(clean[same], dW[same]) and not torch.isfinite(dW[~same]).any()


def test_gradient_against_differences():
    """The lookup is linear in the table: along any direction the change is the gradient's product."""
    r = gen(8)
    n, V, D = 500, 60, 33
    W, d, dy = (dev(r.normal(size=s)) for s in ((V, D), (V, D), (n, D)))
    ids = ids_of(r.integers(-1, V, n))
    y, y2, dW = nan_like((n, D)), nan_like((n, D)), nan_like((V, D))
    lh.embed(W, ids, y, scale=0.5)
    lh.embed(W + d, ids, y2, scale=0.5)
    lh.embed_backward(dy, ids, dW, scale=0.5)
    got = ((y2 - y).double() * dy.double()).sum().item()
    want = (dW.double() * d.double()).sum().item()
    # three roundings of a value of at most |W| + |d|, and the sums of at most 30 tokens a row
    size = ((W.abs() + d.abs()).double()[ids.long().clamp(min=0)] * dy.abs().double()).sum().item()
    assert abs(got - want) <= 40 * U * size


def test_offsets_past_32_bits():
    V, D, n = (1 << 20) + 5, 2112, (1 << 20) + 9
    W = torch.empty((V, D), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    ids = torch.arange(n, device="cuda", dtype=torch.int32) % V
    ids[-1] = V - 1
    y = torch.empty((n, D), dtype=torch.bfloat16, device="cuda")
    lh.embed(W, ids, y)
    assert torch.equal(y[-1], W[-1]) and torch.equal(y[V - 3:V], W[V - 3:]) and torch.equal(y[-5:-1], W[ids[-5:-1].long()])
    dW = torch.empty((V, D), device="cuda")
    lh.embed_backward(y, ids, dW)
    assert torch.equal(dW[-1], 2 * W[-1].float()) and torch.equal(dW[5:V - 1], W[5:-1].float())
