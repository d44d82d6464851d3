"""The gated recurrence, the embedding, the distillation of logits and the verification of
drafts together, as a model uses them: trained (gradients against a float64 evaluation by
torch's elementary operations) and served; the same bits again, on another stream and from
replayed graphs; workspaces."""
from __future__ import annotations

import copy
import os
import sys

import numpy as np
import pytest
import torch

import paper_2310_18780_amd as lh

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    lh.lib()
    yield


def plain_loss(student, teacher, ids, tau=1.5):
    """The example's loss in float64 on the CPU, by elementary operations and autograd."""
    s = copy.deepcopy(student).cpu().double()
    x = s.table[ids.long()] * s.width ** 0.5
    norm = lambda x, k: torch.nn.functional.layer_norm(x, (s.width,), s.norms[k], s.shifts[k])  # noqa: E731
    for k in range(s.layers):
        r, i, u, z = (norm(x, k) @ s.w_in[k].T).split(s.width, -1)
        a = torch.exp(-torch.exp(s.log_rate[k]) * torch.sigmoid(r + s.r_bias[k]))
        v = torch.sqrt(1 - a * a) * torch.sigmoid(i + s.i_bias[k]) * u
        h, hs = torch.zeros_like(v[:, 0]), []
        for t in range(ids.shape[1]):
            h = a[:, t] * h + v[:, t]
            hs.append(h)
        x = x + (torch.stack(hs, 1) * torch.nn.functional.silu(z)) @ s.w_out[k].T
    logits = (norm(x, s.layers) @ s.table.T)[:, 1:]
    table = teacher.table.cpu().double()
    values, top = torch.topk(table[0][ids[:, :-1].long()] + table[1][ids[:, 1:].long()], 8)
    logp = torch.log_softmax(values / tau, -1)
    logq = torch.gather(torch.log_softmax(logits / tau, -1), -1, top)
    loss = tau ** 2 * (logp.exp() * (logp - logq)).sum(-1).mean()
    loss.backward()
    return loss.item(), {n: p.grad for n, p in s.named_parameters()}


def test_a_students_gradients():
    import recurrent_student as ex

    torch.manual_seed(1)
    teacher, student = ex.Teacher(40, "cuda"), ex.Student(40, 48).to("cuda")
    ids = teacher.text(3, 70)
    loss = ex.loss_of(student, teacher, ids)
    loss.backward()
    want, grads = plain_loss(student, teacher, ids.cpu())
    assert abs(loss.item() - want) <= 1e-5 * want
    for n, p in student.named_parameters():
        # float32 throughout: about 2^-24 times some 100 roundings of the sums' scale
        scale = grads[n].abs().max().item()
        assert (p.grad.double().cpu() - grads[n]).abs().max().item() <= 3e-5 * scale, n


def test_the_example_trains_and_drafts():
    import recurrent_student as ex

    losses, kept, worst = ex.run(steps=30)
    assert all(np.isfinite(losses)) and len(kept) == 6 and all(0 <= k <= 4 for k in kept)
    # float32 on both sides, states of order 1, some 100 roundings
    assert worst < 1e-4


def calls(io=torch.bfloat16, shared=None):
    """One call of each entry point on fixed inputs: (run, outputs, what to put back before)."""
    g = torch.Generator(device="cuda").manual_seed(5)
    rn = lambda *s, dtype=torch.float32: torch.randn(s, generator=g, device="cuda", dtype=dtype)  # noqa: E731
    B, T, D, V, K = 2, 1500, 200, 5003, 6
    n = 9001
    x = rn(B, T, 4 * D, dtype=io)
    rate, rb, ib = torch.exp(rn(D) - 2), rn(D), rn(D)
    r, i, u, z = x.split(D, -1)
    dy, dlast = rn(B, T, D, dtype=io), rn(B, D)
    lengths = torch.tensor([T, 777], dtype=torch.int32, device="cuda")
    ids = torch.randint(-3, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[::3] = 17
    W, de = rn(V, D), rn(n, D, dtype=io)
    logits, values = rn(7, V, dtype=io), rn(7, K)
    top = torch.randint(0, V, (7, K), generator=g, device="cuda", dtype=torch.int32)
    up = rn(7)
    p, q = torch.softmax(3 * rn(B, K + 1, V), -1), torch.softmax(3 * rn(B, K, V), -1)
    drafted = p[:, :K].argmax(-1).int()
    un, last = torch.full((B, K), 0.4, device="cuda"), torch.full((B,), 0.7, device="cuda")
    e = lambda *s, dtype=torch.float32: torch.empty(s, device="cuda", dtype=dtype)  # noqa: E731
    o = dict(y=e(B, T, D, dtype=io), state=e(B, D), marks=e(B, -(-T // lh.GATED_MARK), D), yt=e(B, D, dtype=io), drate=e(D), drb=e(D),
             dib=e(D), dfirst=e(B, D), emb=e(n, D, dtype=io), dW=e(V, D), dW2=e(V, D), loss=e(7), lse=e(7), loss2=e(7),
             dl=e(7, V, dtype=io), dl2=e(7, V, dtype=io))
    o.update({k: e(B, T, D, dtype=io) for k in ("dr", "di", "du", "dz")})
    acc, tok = e(B, dtype=torch.int32), e(B, K + 1, dtype=torch.int32)
    ws = shared if shared is not None else torch.empty(max(
        lh.gated_workspace_bytes(B, T, D), lh.gated_backward_workspace_bytes(B, T, D), lh.embed_backward_workspace_bytes(n, V, D),
        lh.distill_logits_workspace_bytes(7, V, K), lh.verify_draft_workspace_bytes(B, K, V)), dtype=torch.uint8, device="cuda")
    bias = dict(r_bias=rb, i_bias=ib)

    def run():
        lh.gated_prefill(rate, r, i, u, o["state"], o["y"], z=z, lengths=lengths, marks=o["marks"], workspace=ws, **bias)
        lh.gated_backward(dy, rate, r, i, u, o["marks"], o["drate"], o["dr"], o["di"], o["du"], dr_bias=o["drb"],
                          di_bias=o["dib"], z=z, dz=o["dz"], lengths=lengths, dlast=dlast, dfirst=o["dfirst"], workspace=ws, **bias)
        lh.gated_step(rate, r[:, 3], i[:, 3], u[:, 3], o["state"], o["yt"], z=z[:, 3], **bias)
        lh.embed(W, ids, o["emb"], scale=3.0)
        lh.embed_backward(de, ids, o["dW"], scale=3.0, workspace=ws)
        lh.embed_backward(de, ids, o["dW2"], workspace=ws)
        lh.embed_backward(o["emb"], ids, o["dW2"], accumulate=True, workspace=ws)
        lh.distill_logits(logits, values, top, o["loss"], dlogits=o["dl"], tau=2.0, workspace=ws)
        lh.distill_logits(logits, values, top, o["loss2"], lse=o["lse"], tau=2.0, workspace=ws)
        lh.distill_logits_backward(up, logits, values, top, o["lse"], o["dl2"], tau=2.0)
        lh.verify_draft(drafted, p, un, last, acc, tok, draft_p=q, workspace=ws)

    return run, [*o.values(), acc, tok], ws


def poison(outputs):
    for t in outputs:
        t.fill_(float("nan") if t.is_floating_point() else -9)


def differing(a, b):
    """The outputs that differ (marks past a row's tokens are not written: NaN on both sides)."""
    return [i for i, (x, y) in enumerate(zip(a, b)) if not torch.equal(torch.nan_to_num(x), torch.nan_to_num(y))]


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16], ids=str)
def test_same_bits_again_and_on_another_stream(io):
    run, outputs, _ = calls(io)
    poison(outputs)
    run()
    torch.cuda.synchronize()
    first = [t.clone() for t in outputs]
    assert sum(torch.isnan(t).any().item() for t in first if t.is_floating_point()) == 1  # marks
    poison(outputs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    assert not differing(first, outputs)


def test_graph_replays_of_two_graphs_that_share_a_workspace():
    run, outputs, ws = calls()
    poison(outputs)
    run()
    torch.cuda.synchronize()
    first = [t.clone() for t in outputs]
    run2, outputs2, _ = calls(shared=ws)
    graphs = []
    for f in (run, run2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    for _ in range(3):
        poison(outputs)
        poison(outputs2)
        ws.fill_(255)
        torch.cuda.synchronize()
        for g in graphs:  # one after the other on one stream
            g.replay()
        torch.cuda.synchronize()
        junk = torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        assert not differing(first, outputs) and not differing(first, outputs2)
        del junk


def test_two_streams_at_once():
    a, b = calls(), calls()
    poison(a[1])
    poison(b[1])
    a[0]()
    torch.cuda.synchronize()
    first = [t.clone() for t in a[1]]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, c in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                c[0]()
    torch.cuda.synchronize()
    assert not differing(first, a[1]) and not differing(first, b[1])


def test_a_workspace_that_is_too_small_is_refused_untouched():
    x, rate = torch.randn(1, 4096, 64, device="cuda"), torch.rand(64, device="cuda")
    y, s = torch.full_like(x, float("nan")), torch.full((1, 64), float("nan"), device="cuda")
    need = lh.gated_workspace_bytes(1, 4096, 64)
    assert need > 0
    with pytest.raises(lh.LHError) as e:
        lh.gated_prefill(rate, x, x, x, s, y, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 5 and torch.isnan(y).all() and torch.isnan(s).all()
    ids, dW = torch.zeros(100, dtype=torch.int32, device="cuda"), torch.full((5, 64), float("nan"), device="cuda")
    need = lh.embed_backward_workspace_bytes(100, 5, 64)
    with pytest.raises(lh.LHError):
        lh.embed_backward(x[0, :100].contiguous(), ids, dW, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert torch.isnan(dW).all()
    lh.embed_backward(x[0, :100].contiguous(), ids, dW, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    assert torch.isfinite(dW).all()


def test_a_workspace_of_the_calls_own_on_another_stream():
    rate, x = torch.rand(96, device="cuda"), torch.randn(1, 3000, 96, device="cuda")
    y, s, y2, s2 = torch.empty_like(x), torch.empty(1, 96, device="cuda"), torch.empty_like(x), torch.empty(1, 96, device="cuda")
    lh.gated_prefill(rate, x, x, x, s, y)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    lh.gated_prefill(rate, x, x, x, s2, y2, stream=side)
    junk = [torch.full((lh.gated_workspace_bytes(1, 3000, 96),), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    side.synchronize()
    assert torch.equal(y, y2) and torch.equal(s, s2)
    del junk


def test_binding_refuses_wrong_types_and_shapes():
    x, i = torch.zeros((2, 8), device="cuda"), torch.zeros((2,), dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        lh.embed(x, i.long(), torch.zeros((2, 8), device="cuda"))
    with pytest.raises(TypeError):
        lh.embed(x.half(), i, torch.zeros((2, 8), device="cuda"))
    with pytest.raises(ValueError):
        lh.embed(x, i, torch.zeros((3, 8), device="cuda"))
    with pytest.raises(ValueError):
        lh.gated_step(x[0], x[:, ::2], x, x, x.clone(), x.clone())
    with pytest.raises(TypeError):
        lh.gated_backward(x[None], x[0], x[None], x[None], x[None], None, x[0], x[None], x[None], x[None])
    with pytest.raises(ValueError):
        lh.distill_logits(x, torch.zeros((2, 3), device="cuda"), torch.zeros((2, 4), dtype=torch.int32, device="cuda"),
                          torch.zeros(2, device="cuda"))
    with pytest.raises(lh.LHError):
        lh.distill_logits(x, torch.zeros((2, 3), device="cuda"), torch.zeros((2, 3), dtype=torch.int32, device="cuda"),
                          torch.zeros(2, device="cuda"), tau=0.0)
    with pytest.raises(lh.LHError) as e:
        lh.embed(x, i, x[:, :8])  # the output over the table
    assert e.value.status == 2
