"""The measured work of the operators at the two ends of a recurrent language model and of
its gated recurrence: embedding, gated linear recurrence, distillation from a teacher's
top logits, verification of drafted tokens.

A case names one call (``kind``) and its sizes:

  gated         the gated linear recurrence over a prompt ``[B, T, D]`` (``gate``: the output
                is multiplied by ``silu(z)``; ``resume``: continued from a state)
  gated_step    one token per row, state in place
  gated_train   the prompt's outputs, then its gradients
  embed         rows of a table ``[V, D]`` (type ``table``) times a scale, ``n`` tokens
  embed_grad    the table's gradient, dense (``add``: added to one that is there, as with
                a table that the output layer shares)
  distill       loss against a teacher's top ``K`` logits of ``rows`` tokens and its
                gradient, in one call
  distill_two   the loss first, the gradient from an upstream gradient in a second call
  verify        ``K`` drafted tokens for each of ``B`` sessions against the target's
                probabilities (``top``: both sides keep that many tokens; ``greedy``: the
                draft has no probabilities)

``ragged``: row ``b`` of the prompt (of the draft) has ``lengths[b]`` tokens, an empty row
among them.  Inputs of the recurrence are slices of one projection's rows ``[.., 4 D]``.
Token frequencies fall as 1 / rank.  The widths 768 / 1024 / 2048 and prompts are those of the
package's workloads; vocabularies are round numbers and odd ones.

The plain forms are elementary torch operations in float32; in float64 are the recurrence's
decays, states and sums over tokens (a decay near 1 counts for thousands of tokens; a scan by
doubling) and the cumulative sums of probabilities, whose borders decide a token.  ``exact``
evaluates the definitions in float64.
"""
import math

import torch

own = False

IO = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gated(name, B, T, D, io, gate=True, ragged=False, resume=False, kind="gated"):
    return dict(name=name, kind=kind, B=B, T=T, D=D, io=io, gate=gate, ragged=ragged, resume=resume)


def _embed(name, n, V, D, io, table, kind="embed", add=False, pad=False):
    return dict(name=name, kind=kind, n=n, V=V, D=D, io=io, table=table, add=add, pad=pad)


def _distill(name, rows, V, K, io, tau, masked, kind="distill"):
    return dict(name=name, kind=kind, rows=rows, V=V, K=K, io=io, tau=tau, masked=masked)


def _verify(name, B, K, V, io, ragged=False, top=0, greedy=False):
    return dict(name=name, kind="verify", B=B, K=K, V=V, io=io, ragged=ragged, top=top, greedy=greedy)


def listed():
    return [
        # one generated token of 64 sessions, one layer: the latency of a call
        _gated("gated_step_b64_d2048", 64, 1, 2048, "bf16", kind="gated_step"),
        # a batch of ordinary prompts at the 1.3B width
        _gated("gated_b16_t4096_d2048", 16, 4096, 2048, "bf16"),
        # one long document, continued from a state
        _gated("gated_b1_t65536_d1024", 1, 65536, 1024, "bf16", gate=False, resume=True),
        # a training batch
        _gated("gated_train_b4_t4096_d2048", 4, 4096, 2048, "bf16", kind="gated_train"),
        # fine-tuning on right-padded texts of different lengths, odd sizes
        _gated("gated_train_b7_t1999_d1000", 7, 1999, 1000, "f32", ragged=True, kind="gated_train"),
        # the next token of 64 sessions
        _embed("embed_n64_d2048", 64, 50000, 2048, "bf16", "bf16"),
        # a training batch of 16 x 4096 tokens from the optimiser's float32 table
        _embed("embed_n65536_d2048", 65536, 50000, 2048, "bf16", "f32"),
        # its gradient
        _embed("embed_grad_n65536_d2048", 65536, 50000, 2048, "bf16", "f32", kind="embed_grad"),
        # a training batch, the teacher's top 64
        _distill("distill_r8192_v50000_k64", 8192, 50000, 64, "bf16", 2.0, True),
        # a small batch with an odd vocabulary, loss and gradient apart
        _distill("distill_two_r517_v32003_k13", 517, 32003, 13, "f32", 1.0, True, kind="distill_two"),
        # 64 sessions, four drafted tokens each
        _verify("verify_b64_k4_v50000", 64, 4, 50000, "f32"),
        # three sessions with drafts of different lengths, a large vocabulary cut to its top tokens
        _verify("verify_b3_k7_v100003", 3, 7, 100003, "bf16", ragged=True, top=50),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    d = _log(rng, 64, 2560)
    return (d + 63) // 64 * 64 if rng.random() < 0.6 else d


def draw(rng):
    kind = rng.choice(["gated", "gated", "gated_step", "gated_train", "gated_train", "embed", "embed_grad", "embed_grad",
                       "distill", "distill_two", "verify", "verify"])
    io = rng.choice(["f32", "bf16", "bf16"])
    flag = lambda p: rng.random() < p  # noqa: E731
    if kind.startswith("gated"):
        step = kind == "gated_step"
        cap = {"gated": 1 << 27, "gated_step": 1 << 20, "gated_train": 1 << 25}[kind]
        B, T, D = _log(rng, 1, 256 if step else 64), 1 if step else _log(rng, 1, 65536), _width(rng)
        while B * T * D > cap:
            if T > 16 * B:
                T = max(1, int(T / 1.9))
            else:
                B = max(1, int(B / 1.9))
        return dict(kind=kind, B=B, T=T, D=D, io=io, gate=flag(0.5), ragged=not step and flag(0.3),
                    resume=kind == "gated" and flag(0.3))
    if kind.startswith("embed"):
        n, V, D = _log(rng, 1, 1 << 17), _log(rng, 1000, 200000), _width(rng)
        while n * D > 1 << 27:
            n = int(n / 1.9)
        while V * D > 1 << 27:
            V = int(V / 1.9)
        return dict(kind=kind, n=n, V=V, D=D, io=io, table=rng.choice([io, "f32"]), add=kind == "embed_grad" and flag(0.3),
                    pad=flag(0.3))
    V = _log(rng, 1000, 200000)
    if kind == "verify":
        B, K = _log(rng, 1, 128), rng.randint(1, 12)
        while B * K * V > 1 << 25:
            B = max(1, int(B / 1.9)) if B > 1 else B
            V = int(V / 1.5) if B == 1 else V
        return dict(kind=kind, B=B, K=K, V=V, io=io, ragged=flag(0.4), top=rng.choice([0, 0, 20, 100]), greedy=flag(0.2))
    rows, K = _log(rng, 1, 16384), _log(rng, 1, 256)
    while rows * V > 1 << 28:
        rows = int(rows / 1.9)
    return dict(kind=kind, rows=rows, V=V, K=K, io=io, tau=rng.choice([1.0, 1.0, 2.0, 3.5]), masked=flag(0.5))


# ---- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _gated_inputs(case, randn, rand):
    B, T, D = case["B"], case["T"], case["D"]
    io = IO[case["io"]]
    s = {}
    if case["ragged"]:
        n = (rand(B) * (T + 1)).int().clamp_(max=T)
        n[0], n[B // 2] = T, T if B == 1 else 0
        s["lengths"] = n
    rows = (B,) if case["kind"] == "gated_step" else (B, T)
    proj = randn(*rows, 4 * D, dtype=io)
    s["r"], s["i"], s["u"] = proj[..., :D], proj[..., D:2 * D], proj[..., 2 * D:3 * D]
    if case["gate"]:
        s["z"] = proj[..., 3 * D:]
    # a channel forgets within 1 to 2000 tokens
    s["rate"] = torch.exp(math.log(1e-3) + math.log(2e3) * rand(D))
    s["r_bias"], s["i_bias"] = 0.5 * randn(D), 0.5 * randn(D)
    if case["kind"] == "gated_train":
        s["dy"] = randn(B, T, D, dtype=io)
    else:
        s["state"] = randn(B, D)
    return s


def _tokens(rand, V, n):
    """n tokens, frequencies falling as 1 / rank."""
    c = torch.cumsum(1 / (torch.arange(V, device="cuda", dtype=torch.float64) + 3), 0)
    return torch.searchsorted(c, rand(n).double() * c[-1]).clamp_(max=V - 1).int()


def _embed_inputs(case, randn, rand):
    n, V, D = case["n"], case["V"], case["D"]
    s = {"ids": _tokens(rand, V, n), "scale": math.sqrt(D)}
    if case["pad"]:
        s["ids"][rand(n) < 0.2] = -1
    if case["kind"] == "embed":
        s["W"] = randn(V, D, dtype=IO[case["table"]]).mul_(1 / math.sqrt(D))
    else:
        s["dy"] = randn(n, D, dtype=IO[case["io"]])
        if case["add"]:
            s["dW"] = randn(V, D)
    return s


def _distill_inputs(case, randn, rand):
    rows, V, K = case["rows"], case["V"], case["K"]
    s = {"logits": randn(rows, V, dtype=IO[case["io"]]).mul_(2)}
    s["values"] = torch.empty((rows, K), device="cuda")
    s["ids"] = torch.empty((rows, K), dtype=torch.int32, device="cuda")
    for i in range(0, rows, 1024):  # a teacher that agrees with the student in part
        t = 0.7 * s["logits"][i:i + 1024].float()
        t += 1.5 * randn(*t.shape)
        v, j = torch.topk(t, K)
        s["values"][i:i + 1024], s["ids"][i:i + 1024] = v, j
    s["scale"] = torch.full((rows,), 1 / rows, device="cuda")
    if case["masked"]:  # prompts' tokens take no part, and some rows came with fewer entries
        s["scale"][rand(rows) < 0.15] = 0
        s["ids"][:, K // 2:].masked_fill_((rand(rows) < 0.2)[:, None], -1)
    if case["kind"] == "distill_two":
        s["dloss"] = 1 + 0.1 * randn(rows)
    return s


def _verify_inputs(case, randn, rand):
    B, K, V = case["B"], case["K"], case["V"]
    io = IO[case["io"]]
    # probabilities fall as rank^-1.3, the draft's are near the target's
    base = -1.3 * torch.log(rand(B, K + 1, V) + 1e-9)
    other = base[:, :K] + 0.4 * randn(B, K, V)

    def probabilities(x):
        if case["top"]:
            least = torch.topk(x, min(case["top"], V))[0][..., -1:]
            x = x.masked_fill(x < least, float("-inf"))
        return torch.softmax(x, -1)

    s = {"target_p": probabilities(base).to(io)}
    q = probabilities(other)
    if case["greedy"]:
        s["drafted"] = q.argmax(-1).int()
    else:
        s["draft_p"] = q.to(io)
        c = torch.cumsum(q.double(), -1)
        s["drafted"] = torch.searchsorted(c, rand(B, K, 1).double() * c[..., -1:])[..., 0].clamp_(max=V - 1).int()
    if case["ragged"]:
        n = (rand(B) * (K + 1)).int().clamp_(max=K)
        n[0], n[B // 2] = K, K if B == 1 else 0
        s["lengths"] = n
    s["u"], s["u_last"] = rand(B, K), rand(B)
    return s


def _inputs(case, seed):
    g = _generator(seed)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype)

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    make = {"gated": _gated_inputs, "embed": _embed_inputs, "distill": _distill_inputs, "verify": _verify_inputs}
    s = make[case["kind"].split("_")[0]](case, randn, rand)
    s["case"] = case
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_2310_18780_amd as lh

    # what a program holds beside its inputs: outputs and scratch
    def like(x, *names, shape=None):
        for n in names:
            s[n] = torch.empty(x.shape if shape is None else shape, dtype=x.dtype, device="cuda")

    def workspace(n):
        return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None

    kind = case["kind"]
    if kind.startswith("gated"):
        B, T, D = case["B"], case["T"], case["D"]
        like(s["u"], "y")
        if kind == "gated":
            s["ws"] = workspace(lh.gated_workspace_bytes(B, T, D))
        if kind == "gated_train":
            like(s["u"], *("dr", "di", "du", "dz")[:3 + case["gate"]])
            like(s["rate"], "drate", "dr_bias", "di_bias")
            like(s["rate"], "state", shape=(B, D))
            like(s["rate"], "marks", shape=(B, -(-T // lh.GATED_MARK), D))
            s["ws"] = workspace(max(lh.gated_workspace_bytes(B, T, D), lh.gated_backward_workspace_bytes(B, T, D)))
    elif kind == "embed":
        s["y"] = torch.empty((case["n"], case["D"]), dtype=IO[case["io"]], device="cuda")
    elif kind == "embed_grad":
        if not case["add"]:
            s["dW"] = torch.empty((case["V"], case["D"]), device="cuda")
        s["ws"] = workspace(lh.embed_backward_workspace_bytes(case["n"], case["V"], case["D"]))
    elif kind.startswith("distill"):
        like(s["scale"], "loss", "lse")
        like(s["logits"], "dlogits")
        s["ws"] = workspace(lh.distill_logits_workspace_bytes(case["rows"], case["V"], case["K"]))
    else:
        like(s["drafted"], "accepted", shape=(case["B"],))
        like(s["drafted"], "tokens", shape=(case["B"], case["K"] + 1))
        s["ws"] = workspace(lh.verify_draft_workspace_bytes(case["B"], case["K"], case["V"]))
    return s


# ---- the framework's calls

GRADS = ("drate", "dr", "di", "du", "dr_bias", "di_bias", "dz")


def _run_own(s):
    import paper_2310_18780_amd as lh

    case, kind = s["case"], s["case"]["kind"]
    if kind.startswith("gated"):
        more = {k: s[k] for k in ("r_bias", "i_bias", "z", "lengths") if k in s}
        args = (s["rate"], s["r"], s["i"], s["u"])
        if kind == "gated_step":
            lh.gated_step(*args, s["state"], s["y"], **more)
            return {"y": s["y"], "state": s["state"]}
        lh.gated_prefill(*args, s["state"], s["y"], resume=case["resume"], marks=s.get("marks"), workspace=s["ws"], **more)
        if kind == "gated":
            return {"y": s["y"], "state": s["state"]}
        lh.gated_backward(s["dy"], *args, s["marks"], s["drate"], s["dr"], s["di"], s["du"], dr_bias=s["dr_bias"],
                          di_bias=s["di_bias"], dz=s.get("dz"), workspace=s["ws"], **more)
        return {k: s[k] for k in ("y", "state") + GRADS if k in s}
    if kind == "embed":
        lh.embed(s["W"], s["ids"], s["y"], scale=s["scale"])
        return {"y": s["y"]}
    if kind == "embed_grad":
        lh.embed_backward(s["dy"], s["ids"], s["dW"], scale=s["scale"], accumulate=case["add"], workspace=s["ws"])
        return {"dW": s["dW"]}
    if kind == "distill":
        lh.distill_logits(s["logits"], s["values"], s["ids"], s["loss"], dlogits=s["dlogits"], scale=s["scale"],
                          tau=case["tau"], workspace=s["ws"])
        return {"loss": s["loss"], "dlogits": s["dlogits"]}
    if kind == "distill_two":
        lh.distill_logits(s["logits"], s["values"], s["ids"], s["loss"], lse=s["lse"], scale=s["scale"], tau=case["tau"],
                          workspace=s["ws"])
        lh.distill_logits_backward(s["dloss"], s["logits"], s["values"], s["ids"], s["lse"], s["dlogits"],
                                   scale=s["scale"], tau=case["tau"])
        return {"loss": s["loss"], "dlogits": s["dlogits"]}
    lh.verify_draft(s["drafted"], s["target_p"], s["u"], s["u_last"], s["accepted"], s["tokens"],
                    draft_p=s.get("draft_p"), lengths=s.get("lengths"), workspace=s["ws"])
    return {"accepted": s["accepted"], "tokens": s["tokens"]}


# ---- plain forms: float32 (float64 where that loses what matters), rounded once

def _gates(s):
    """Gates of all tokens: f, p in float32, a, g in float64."""
    f = torch.sigmoid(s["r"].float() + s["r_bias"])
    p = torch.sigmoid(s["i"].float() + s["i_bias"])
    L = s["rate"].double() * f
    return f, p, torch.exp(-L), torch.sqrt(-torch.expm1(-2 * L))


def _valid(s):
    """[B, T, 1] truth values of the tokens in a right-padded batch, or None."""
    if "lengths" not in s:
        return None
    return (torch.arange(s["case"]["T"], device="cuda") < s["lengths"][:, None])[..., None]


def _keep(x, valid, other=0.0):
    return x if valid is None else torch.where(valid, x, torch.full((), other, dtype=x.dtype, device="cuda"))


def _double(a, v):
    """All states of h <- a h + v over the second axis, from zero, by doubling; in place."""
    k = 1
    while k < a.shape[1]:
        v[:, k:] += a[:, k:] * v[:, :-k]
        if 2 * k < a.shape[1]:
            a[:, k:] = a[:, k:] * a[:, :-k]
        k *= 2
    return v


def _states(s, a, v, start):
    """States of all tokens; a padded token leaves the state alone."""
    valid = _valid(s)
    a, v = _keep(a, valid, 1.0).clone(), _keep(v, valid).clone()
    if start is not None:
        v[:, 0] += a[:, 0] * start
    return _double(a, v)


def _silu(x):
    return x * torch.sigmoid(x)


def _plain_gated(s):
    case = s["case"]
    _, p, a, g = _gates(s)
    h = _states(s, a, g * p * s["u"].float(), s["state"] if case["resume"] else None)
    y = h * _silu(s["z"].float()) if "z" in s else h
    s["state"].copy_(h[:, -1])
    return {"y": _keep(y, _valid(s)).to(s["u"].dtype), "state": s["state"]}


def _plain_gated_step(s):
    _, p, a, g = _gates(s)
    h = a * s["state"] + g * p * s["u"].float()
    y = h * _silu(s["z"].float()) if "z" in s else h
    s["state"].copy_(h)
    return {"y": y.to(s["u"].dtype), "state": s["state"]}


def _plain_gated_train(s):
    io, valid = s["u"].dtype, _valid(s)
    f, p, a, g = _gates(s)
    u = s["u"].float()
    h = _states(s, a, g * p * u, None)
    out = {"state": h[:, -1].float()}
    dy = s["dy"].double()
    if "z" in s:
        z = s["z"].float()
        sz = torch.sigmoid(z)
        out["dz"] = _keep(dy * h * sz * (1 + z * (1 - sz)), valid).to(io)
        out["y"] = _keep(h * z * sz, valid).to(io)
        dy = dy * z * sz
    else:
        out["y"] = _keep(h, valid).to(io)
    # dh_t = dy_t + a_(t+1) dh_(t+1), the same recurrence backwards in time
    later = torch.cat([_keep(a, valid, 1.0)[:, 1:], torch.ones_like(a[:, :1])], 1).flip(1)
    dh = _double(later.contiguous(), _keep(dy, valid).flip(1).contiguous()).flip(1)
    before = torch.cat([torch.zeros_like(h[:, :1]), h[:, :-1]], 1)
    dL = _keep(dh * (p * u * a * a / g - a * before), valid)
    dr, di = dL * s["rate"] * f * (1 - f), _keep(dh * g * u * p * (1 - p), valid)
    out.update(drate=(dL * f).sum((0, 1)).float(), dr=dr.to(io), di=di.to(io), du=_keep(dh * g * p, valid).to(io),
               dr_bias=dr.sum((0, 1)).float(), di_bias=di.sum((0, 1)).float())
    return {k: out[k] for k in ("y", "state") + GRADS if k in out}


def _plain_embed(s):
    ids = s["ids"].long()
    y = s["W"][ids.clamp(min=0)].float() * s["scale"]
    return {"y": torch.where((ids >= 0)[:, None], y, torch.zeros((), device="cuda")).to(IO[s["case"]["io"]])}


def _plain_embed_grad(s):
    case, ids = s["case"], s["ids"].long()
    sums = torch.zeros((case["V"], case["D"]), device="cuda")
    sums.index_add_(0, ids.clamp(min=0), torch.where((ids >= 0)[:, None], s["dy"].float(), torch.zeros((), device="cuda")))
    sums *= s["scale"]
    return {"dW": s["dW"].add_(sums) if case["add"] else sums}


def _plain_distill(s):
    case, io = s["case"], s["logits"].dtype
    tau, scale = case["tau"], s["scale"]
    x = s["logits"].float() / tau
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    valid = s["ids"] >= 0
    ids = s["ids"].long().clamp(min=0)
    t = torch.where(valid, s["values"] / tau, torch.full((), -1e30, device="cuda"))
    t = t - t.amax(-1, keepdim=True)
    w = torch.exp(t) * valid
    ws = w.sum(-1, keepdim=True).clamp(min=1e-30)  # (a row without entries has loss and gradient 0)
    p = w / ws
    each = p * ((t - torch.log(ws)) - (torch.gather(x, 1, ids) - top - torch.log(total)))
    loss = scale * tau * tau * torch.where(p > 0, each, torch.zeros((), device="cuda")).sum(-1)
    d = e.div_(total).scatter_add_(1, ids, -p)
    c = scale * tau * valid.any(-1) * (s["dloss"] if "dloss" in s else 1)
    return {"loss": loss, "dlogits": d.mul_(c[:, None]).to(io)}


def _plain_verify(s):
    case = s["case"]
    B, K, V = case["B"], case["K"], case["V"]
    rows, at = torch.arange(B, device="cuda"), torch.arange(K + 1, device="cuda")
    n = s["lengths"].long() if "lengths" in s else torch.full((B,), K, device="cuda")
    t = s["drafted"].long()
    p = torch.gather(s["target_p"][:, :K], 2, t[..., None])[..., 0].double()
    q = torch.gather(s["draft_p"], 2, t[..., None])[..., 0].double() if "draft_p" in s else torch.ones_like(p)
    taken = (s["u"].double() * q < p) & (at[:K] < n[:, None])
    m = torch.cumprod(taken.int(), 1).sum(1)
    w = s["target_p"][rows, m].double()
    last = torch.clamp(m, max=K - 1)
    if "draft_p" in s:
        minus = s["draft_p"][rows, last].double()
    else:
        minus = torch.zeros_like(w).scatter_(1, t[rows, last][:, None], float("inf"))
    rest = torch.clamp(w - minus, min=0)
    w = torch.where(((m < n) & (rest.sum(1) > 0))[:, None], rest, w)
    c = torch.cumsum(w, 1)
    drawn = (c <= s["u_last"].double()[:, None] * c[:, -1:]).sum(1)
    tokens = torch.where(at < m[:, None], torch.nn.functional.pad(s["drafted"], (0, 1)), torch.full((), -1, device="cuda"))
    tokens = torch.where(at == m[:, None], drawn.clamp(max=V - 1)[:, None], tokens)
    return {"accepted": m.int(), "tokens": tokens.int()}


PLAIN = {"gated": _plain_gated, "gated_step": _plain_gated_step, "gated_train": _plain_gated_train, "embed": _plain_embed,
         "embed_grad": _plain_embed_grad, "distill": _plain_distill, "distill_two": _plain_distill, "verify": _plain_verify}


def run(s):
    return _run_own(s) if own else PLAIN[s["case"]["kind"]](s)


# ---- the work that a call cannot do without

def work(case):
    kind = case["kind"]
    es = 2 if case["io"] == "bf16" else 4
    if kind.startswith("gated"):
        B, T, D, gate = case["B"], case["T"], case["D"], case["gate"]
        n = B * T * D
        reads = kind == "gated_step" or case["resume"]
        out = {"bytes": es * n * (5 if gate else 4) + 12 * D + 4 * B * D * (2 if reads else 1), "flops": n * (22 if gate else 18)}
        if kind == "gated_train":  # the inputs once for both calls; dy in, dr, di, du (dz) out
            out["bytes"] += es * n * (5 if gate else 4) + 12 * D
            out["flops"] += n * (40 if gate else 30)
        return out
    if kind.startswith("embed"):
        n, V, D = case["n"], case["V"], case["D"]
        if kind == "embed":
            et = 2 if case["table"] == "bf16" else 4
            # rows that recur are read once: the expected number of different tokens
            f = 1 / (torch.arange(V, dtype=torch.float64) + 3)
            rows = int((1 - torch.exp(n * (0.8 if case["pad"] else 1) * torch.log1p(-f / f.sum()))).sum()) + 1
            return {"bytes": n * D * es + rows * D * et + 4 * n, "flops": n * D}
        return {"bytes": n * D * es + V * D * (8 if case["add"] else 4) + 4 * n, "flops": n * D + V * D}
    if kind.startswith("distill"):
        n = case["rows"] * case["V"]
        return {"bytes": 2 * es * n + 8 * case["rows"] * case["K"] + 8 * case["rows"], "flops": 7 * n}
    B, K, V = case["B"], case["K"], case["V"]
    return {"bytes": es * B * V * (1 if case["greedy"] else 2) + 16 * B * K, "flops": 3 * B * V}


# ---- float64, from the definitions

def _logistic(x):
    return 1 / (1 + torch.exp(-x))


def _exact_gates(s):
    """float64, time first: f, p, a, g, u, h0 of a row's tokens; a padded token has a = 1, no input."""
    step = s["case"]["kind"] == "gated_step"
    d = {k: (s[k][:, None] if step else s[k]).double().transpose(0, 1) for k in ("r", "i", "u", "z", "dy") if k in s}
    f = _logistic(d["r"] + s["r_bias"].double())
    d["f"], d["p"] = f, _logistic(d["i"] + s["i_bias"].double())
    d["a"] = torch.exp(-s["rate"].double() * f)
    d["g"] = torch.sqrt(-torch.expm1(-2 * s["rate"].double() * f))
    d["v"] = d["g"] * d["p"] * d["u"]
    if "lengths" in s:
        d["out"] = (torch.arange(s["case"]["T"], device="cuda")[:, None] >= s["lengths"])[..., None]
        d["a"] = d["a"].masked_fill(d["out"], 1.0)
        for k in ("v", "dy"):
            if k in d:
                d[k] = d[k].masked_fill(d["out"], 0.0)
    return d


def _exact_gated(s):
    case = s["case"]
    d = _exact_gates(s)
    T, train = case["T"], case["kind"] == "gated_train"
    h = torch.zeros((case["B"], case["D"]), dtype=torch.float64, device="cuda")
    if case["kind"] == "gated_step" or case["resume"]:
        h = s["state"].double()
    states = torch.empty_like(d["v"])
    for t in range(T):
        h = torch.addcmul(d["v"][t], d["a"][t], h)
        states[t] = h
    out = {"state": h}
    sz = _logistic(d["z"]) if "z" in d else None
    y = states * d["z"] * sz if "z" in d else states
    hide = lambda x: x.masked_fill(d["out"], 0.0) if "out" in d else x  # noqa: E731
    y = hide(y).transpose(0, 1)
    out["y"] = y[:, 0] if case["kind"] == "gated_step" else y
    if not train:
        return {"y": out["y"], "state": out["state"]}
    if "z" in d:
        out["dz"] = d["dy"] * states * sz * (1 + d["z"] * (1 - sz))
        down = d["dy"] * d["z"] * sz
    else:
        down = d["dy"]
    dh = torch.empty_like(down)
    b = torch.zeros_like(h)
    for t in reversed(range(T)):
        b = down[t] + b
        dh[t] = b
        b = b * d["a"][t]
    before = torch.cat([torch.zeros_like(states[:1]), states[:-1]])
    dL = hide(dh * (d["p"] * d["u"] * d["a"] ** 2 / d["g"] - d["a"] * before))
    out["dr"] = dL * s["rate"].double() * d["f"] * (1 - d["f"])
    out["di"] = hide(dh * d["g"] * d["u"] * d["p"] * (1 - d["p"]))
    out["du"] = hide(dh * d["g"] * d["p"])
    out["drate"], out["dr_bias"], out["di_bias"] = (dL * d["f"]).sum((0, 1)), out["dr"].sum((0, 1)), out["di"].sum((0, 1))
    for k in ("dr", "di", "du", "dz"):
        if k in out:
            out[k] = out[k].transpose(0, 1)
    return {k: out[k] for k in ("y", "state") + GRADS if k in out}


def _exact_embed(s):
    table = torch.cat([s["W"].double() * s["scale"], torch.zeros((1, s["W"].shape[1]), dtype=torch.float64, device="cuda")])
    return {"y": table[s["ids"].long()]}  # id -1: the row of zeros


def _exact_embed_grad(s):
    case, ids = s["case"], s["ids"].long()
    order = torch.argsort(ids, stable=True)
    sums = torch.zeros((case["V"] + 1, case["D"]), dtype=torch.float64, device="cuda")
    for i in range(0, len(order), 8192):
        k = order[i:i + 8192]
        sums.index_add_(0, ids[k] % (case["V"] + 1), s["dy"][k].double())
    sums = sums[:-1] * s["scale"]
    return {"dW": sums + s["dW"].double() if case["add"] else sums}


def _exact_distill(s):
    case, tau = s["case"], s["case"]["tau"]
    loss, grad = [], []
    for i in range(0, case["rows"], 512):
        r = slice(i, i + 512)
        logq = torch.log_softmax(s["logits"][r].double() / tau, -1)
        ids = s["ids"][r].long()
        logp = torch.log_softmax((s["values"][r].double() / tau).masked_fill(ids < 0, -1e300), -1)
        p = torch.exp(logp).masked_fill(ids < 0, 0.0)
        slots = ids.clamp(min=0)
        gap = torch.where(p > 0, logp - torch.gather(logq, 1, slots), torch.zeros_like(p))
        scale = s["scale"][r].double()
        loss.append(scale * tau ** 2 * (p * gap).sum(-1))
        d = torch.exp(logq)
        d.scatter_add_(1, slots, -p)
        up = s["dloss"][r].double() if "dloss" in s else torch.ones_like(scale)
        up = up.masked_fill((ids < 0).all(-1), 0.0)
        grad.append(d * (scale * tau * up)[:, None])
    return {"loss": torch.cat(loss), "dlogits": torch.cat(grad)}


def exact(case, seed):
    kind = case["kind"]
    if kind == "verify":
        return None  # whole numbers
    s = _inputs(case, seed)
    if kind.startswith("gated"):
        return _exact_gated(s)
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad}.get(kind, _exact_distill)(s)
