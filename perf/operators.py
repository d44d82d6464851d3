"""The measured work of the selective block's operators: layer norm, the short causal
convolution and the selective state-space scan, for prompts, single tokens and gradients.

A case names one call (``kind``) and its sizes:

  norm          layer norm of ``rows`` rows of ``D`` channels, with the residual sum of a
                pre-norm block where ``res``
  norm_grad     its gradients: rows, weight and bias (``res``: the gradient that comes
                down the residual stream is added)
  conv          depthwise causal convolution of ``K`` taps over a prompt ``[B, T, D]``
                (SiLU where ``silu``), and the last ``K - 1`` inputs as state
  conv_step     the same for one token per row, state in place
  conv_grad     its gradients
  scan          the selective scan over a prompt: ``N`` states per channel, input and
                output rows of ``G`` channel groups, gated where ``gate``
  scan_step     one token per row, state in place
  scan_grad     its gradients

``ragged``: a right-padded batch, row ``b`` of the prompt has ``lengths[b]`` tokens (an
empty row among them).  ``resume``: the call continues from a state.

Inputs lie as the projections of a block leave them: the convolution's input and the
gate are halves of one ``[B T, 2 D]`` product, the scan's input and output rows slices of
another.  The widths 768 / 1024 / 2048, orders 16 / 32 and prompts are those of the
package's workloads.

The plain forms are elementary torch operations in float32 (a scan in time blocks by
doubling); ``exact`` evaluates the definitions in float64, step by step.
"""
import math

import torch

own = False

IO = {"f32": torch.float32, "bf16": torch.bfloat16}


def _norm(name, rows, D, io, res, kind="norm"):
    return dict(name=name, kind=kind, rows=rows, D=D, io=io, res=res)


def _conv(name, B, T, D, K, io, silu=True, ragged=False, resume=False, kind="conv"):
    return dict(name=name, kind=kind, B=B, T=T, D=D, K=K, io=io, silu=silu, ragged=ragged, resume=resume)


def _scan(name, B, T, D, N, io, G=1, gate=True, ragged=False, resume=False, kind="scan"):
    return dict(name=name, kind=kind, B=B, T=T, D=D, N=N, G=G, io=io, gate=gate, ragged=ragged, resume=resume)


def listed():
    return [
        # one token of 64 sessions at the 1.3B width: the latency of a call
        _norm("norm_token_b64_d2048", 64, 2048, "bf16", True),
        # a ragged batch of prompts, a width that no power of two divides
        _norm("norm_r13993_d1001", 13993, 1001, "f32", False),
        # a training batch: 16 sequences of 4096 tokens
        _norm("norm_grad_r65536_d2048", 65536, 2048, "bf16", True, "norm_grad"),
        # the package's headline prompt batch
        _conv("conv_b64_t4096_d2048", 64, 4096, 2048, 4, "bf16"),
        # one generated token of 64 sessions
        _conv("conv_step_b64_d2048", 64, 1, 2048, 4, "bf16", kind="conv_step"),
        # a training batch at the 125M width, three taps without activation
        _conv("conv_grad_b16_t2048_d768", 16, 2048, 768, 3, "f32", silu=False, kind="conv_grad"),
        # one generated token of 64 sessions, one layer
        _scan("scan_step_b64_d2048_n16", 64, 1, 2048, 16, "bf16", kind="scan_step"),
        # one short prompt: time to the first token of a single session
        _scan("scan_one_t512_d768_n16", 1, 512, 768, 16, "f32"),
        # a batch of ordinary prompts at the 1.3B width
        _scan("scan_b16_t4096_d2048_n16", 16, 4096, 2048, 16, "bf16"),
        # one long document, two groups, continued from a state
        _scan("scan_b1_t65536_d1024_n16", 1, 65536, 1024, 16, "f32", G=2, resume=True),
        # right-padded prompts of different lengths, odd sizes, no gate
        _scan("scan_b7_t1999_d1000_n12", 7, 1999, 1000, 12, "bf16", gate=False, ragged=True),
        # a training batch
        _scan("scan_grad_b4_t4096_d2048_n16", 4, 4096, 2048, 16, "bf16", kind="scan_grad"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _shape(rng, cap, B=64, T=65536):
    """Batch, prompt and width of at most ``cap`` values; most widths are multiples of 64."""
    b, t, d = _log(rng, 1, B), _log(rng, 1, T), _log(rng, 64, 2560)
    if rng.random() < 0.6:
        d = (d + 63) // 64 * 64
    while b * t * d > cap:
        if t > 16 * b:
            t = max(1, int(t / 1.9))
        else:
            b = max(1, int(b / 1.9))
    return b, t, d


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "conv", "conv_step", "conv_grad",
                       "scan", "scan", "scan", "scan_step", "scan_grad", "scan_grad"])
    io = rng.choice(["f32", "bf16", "bf16"])
    flag = lambda p: rng.random() < p  # noqa: E731
    if kind.startswith("norm"):
        rows, _, D = _shape(rng, 1 << 27, 65536, 1)
        return dict(kind=kind, rows=rows, D=D, io=io, res=flag(0.5))
    if kind.startswith("conv"):
        cap = {"conv": 1 << 28, "conv_step": 1 << 20, "conv_grad": 1 << 27}[kind]
        B, T, D = _shape(rng, cap, 256 if kind == "conv_step" else 64, 1 if kind == "conv_step" else 65536)
        return dict(kind=kind, B=B, T=T, D=D, K=rng.choice([2, 3, 4, 4, 6]), io=io, silu=flag(0.7),
                    ragged=kind != "conv_step" and flag(0.3), resume=kind == "conv" and flag(0.3))
    N = rng.choice([16, 16, 32, 64, _log(rng, 4, 64)])
    cap = {"scan": 1 << 31, "scan_step": 1 << 26, "scan_grad": 1 << 29}[kind] // N
    B, T, D = _shape(rng, min(cap, 1 << 27), 256 if kind == "scan_step" else 64, 1 if kind == "scan_step" else 65536)
    G = rng.choice([1, 1, 2, 4])
    while D % G:
        G //= 2
    return dict(kind=kind, B=B, T=T, D=D, N=N, G=G, io=io, gate=flag(0.7),
                ragged=kind != "scan_step" and flag(0.3), resume=kind == "scan" and flag(0.3))


# ---- inputs

def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    io = IO[case["io"]]
    D = case["D"]
    s = {"case": case}

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype)

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    kind = case["kind"]
    if kind.startswith("norm"):
        rows = case["rows"]
        s["w"], s["b"] = 1 + 0.1 * randn(D), 0.1 * randn(D)
        # residual streams have channels of different scales and an offset per row
        scale = torch.exp(0.5 * randn(D)).to(io)
        s["x"] = randn(rows, D, dtype=io).mul_(scale).add_(0.2 * randn(rows, 1).to(io))
        if kind == "norm" and case["res"]:
            s["residual"] = randn(rows, D, dtype=io)
        if kind == "norm_grad":
            s["dy"] = randn(rows, D, dtype=io)
            if case["res"]:
                s["dtotal"] = randn(rows, D, dtype=io)
            # the statistics that the forward pass kept
            s["mean"], s["rstd"] = (torch.empty(rows, device="cuda") for _ in range(2))
            for i in range(0, rows, 8192):
                x = s["x"][i:i + 8192].float()
                s["mean"][i:i + 8192] = x.mean(-1)
                s["rstd"][i:i + 8192] = torch.rsqrt(x.var(-1, unbiased=False) + 1e-5)
        return s
    B, T = case["B"], case["T"]
    step = kind.endswith("step")
    if case["ragged"]:
        n = (rand(B) * (T + 1)).int().clamp_(max=T)
        n[0], n[B // 2] = T, T if B == 1 else 0
        s["lengths"] = n
    # [.., 2 D]: convolution input (or the gate's neighbour) and gate of one projection
    rows = (B,) if step else (B, T)
    if kind.startswith("conv"):
        K = case["K"]
        s["x"] = randn(*rows, 2 * D, dtype=io)[..., :D]
        s["w"], s["bias"] = randn(D, K) / math.sqrt(K), 0.1 * randn(D)
        if kind == "conv_grad":
            s["dy"] = randn(*rows, D, dtype=io)
        else:
            s["state"] = randn(B, K - 1, D, dtype=io)
        return s
    N, G = case["N"], case["G"]
    # A = -(1 .. N), spread by training; steps between 1e-3 and 1e-1 before the input's part
    s["A"] = -torch.arange(1, N + 1, device="cuda") * torch.exp(0.1 * randn(D, N))
    step0 = torch.exp(math.log(1e-3) + math.log(100.0) * rand(D))
    s["dt_bias"] = step0 + torch.log(-torch.expm1(-step0))
    s["h0"] = randn(D)
    s["u"] = randn(*rows, D, dtype=io)
    s["dt"] = randn(*rows, D, dtype=io)
    rank = max(1, D // 16)
    proj = randn(*rows, rank + 2 * G * N, dtype=io)
    s["Bm"] = proj[..., rank:rank + G * N].unflatten(-1, (G, N))
    s["Cm"] = proj[..., rank + G * N:].unflatten(-1, (G, N))
    if case["gate"]:
        s["z"] = randn(*rows, 2 * D, dtype=io)[..., D:]
    if kind == "scan_grad":
        s["dy"] = randn(*rows, D, dtype=io)
    else:
        s["state"] = randn(B, D, N)
    return s


def _workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_2310_18780_amd as lh

    # what a program holds beside its inputs: outputs and scratch
    kind, D = case["kind"], case["D"]

    def like(x, *names):
        for n in names:
            s[n] = torch.empty(x.shape, dtype=x.dtype, device="cuda")

    if kind == "norm":
        like(s["x"], "y")
        if case["res"]:
            like(s["x"], "total")
    elif kind == "norm_grad":
        like(s["x"], "dx")
        like(s["w"], "dw", "db")
        s["ws"] = _workspace(lh.layer_norm_backward_workspace_bytes(case["rows"], D))
    elif kind.startswith("conv"):
        if kind == "conv_grad":
            like(s["x"], "dx")
            like(s["w"], "dw")
            like(s["bias"], "dbias")
            s["ws"] = _workspace(lh.short_conv_backward_workspace_bytes(case["B"], case["T"], D, case["K"]))
        else:
            like(s["x"], "y")
    else:
        sizes = (case["B"], case["T"], D, case["N"], case["G"])
        if kind == "scan_grad":
            like(s["u"], "du", "ddt")
            like(s["Bm"], "dBm", "dCm")
            like(s["A"], "dA")
            like(s["h0"], "dh0", "ddt_bias")
            if case["gate"]:
                like(s["u"], "dz")
            s["ws"] = _workspace(lh.selective_backward_workspace_bytes(*sizes))
        else:
            like(s["u"], "y")
            if kind == "scan":
                s["ws"] = _workspace(lh.selective_workspace_bytes(*sizes))
    return s


# ---- the framework's calls

def _run_own(s):
    import paper_2310_18780_amd as lh

    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        lh.layer_norm(s["x"], s["w"], s["b"], s["y"], residual=s.get("residual"), total=s.get("total"))
        return {k: s[k] for k in ("y", "total") if k in s}
    if kind == "norm_grad":
        lh.layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"],
                               dtotal=s.get("dtotal"), workspace=s["ws"])
        return {k: s[k] for k in ("dx", "dw", "db")}
    lengths = s.get("lengths")
    if kind == "conv":
        lh.short_conv_prefill(s["x"], s["w"], s["bias"], s["state"], s["y"], silu=case["silu"], lengths=lengths,
                              resume=case["resume"])
        return {"y": s["y"], "state": s["state"]}
    if kind == "conv_step":
        lh.short_conv_step(s["x"], s["w"], s["bias"], s["state"], s["y"], silu=case["silu"])
        return {"y": s["y"], "state": s["state"]}
    if kind == "conv_grad":
        lh.short_conv_backward(s["dy"], s["x"], s["w"], s["bias"], s["dx"], s["dw"], s["dbias"], silu=case["silu"],
                               lengths=lengths, workspace=s["ws"])
        return {k: s[k] for k in ("dx", "dw", "dbias")}
    if kind == "scan":
        lh.selective_prefill(s["A"], s["dt"], s["Bm"], s["Cm"], s["u"], s["state"], s["y"], h0=s["h0"],
                             dt_bias=s["dt_bias"], z=s.get("z"), lengths=lengths, resume=case["resume"],
                             workspace=s["ws"])
        return {"y": s["y"], "state": s["state"]}
    if kind == "scan_step":
        lh.selective_step(s["A"], s["dt"], s["Bm"], s["Cm"], s["u"], s["state"], s["y"], h0=s["h0"],
                          dt_bias=s["dt_bias"], z=s.get("z"))
        return {"y": s["y"], "state": s["state"]}
    lh.selective_backward(s["dy"], s["A"], s["dt"], s["Bm"], s["Cm"], s["u"], s["dA"], s["ddt"], s["dBm"], s["dCm"],
                          s["du"], h0=s["h0"], dh0=s["dh0"], dt_bias=s["dt_bias"], ddt_bias=s["ddt_bias"],
                          z=s.get("z"), dz=s.get("dz"), lengths=lengths, workspace=s["ws"])
    return {k: s[k] for k in ("dA", "ddt", "dBm", "dCm", "du", "dh0", "ddt_bias", "dz") if k in s}


# ---- plain forms: float32, rounded once

def _valid(s, T):
    """[B, T, 1] truth values of the tokens in a right-padded batch, or None."""
    if "lengths" not in s:
        return None
    return (torch.arange(T, device="cuda") < s["lengths"][:, None])[..., None]


def _keep(x, valid):
    return x if valid is None else torch.where(valid, x, torch.zeros((), dtype=x.dtype, device="cuda"))


def _plain_norm(s):
    x = s["x"].float()
    out = {}
    if "residual" in s:
        x = x + s["residual"].float()
        out["total"] = x.to(s["x"].dtype)
    c = x - x.mean(-1, keepdim=True)
    y = c * torch.rsqrt((c * c).mean(-1, keepdim=True) + 1e-5)
    out["y"] = (y * s["w"] + s["b"]).to(s["x"].dtype)
    return {k: out[k] for k in ("y", "total") if k in out}


def _plain_norm_grad(s):
    dy = s["dy"].float()
    xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["w"]
    dx = s["rstd"][:, None] * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    if "dtotal" in s:
        dx = dx + s["dtotal"].float()
    return {"dx": dx.to(s["x"].dtype), "dw": (dy * xh).sum(0), "db": dy.sum(0)}


def _silu(x):
    return x * torch.sigmoid(x)


def _silu_slope(x):
    p = torch.sigmoid(x)
    return p * (1 + x * (1 - p))


def _taps(s, xp, T):
    acc = s["bias"].expand(xp.shape[0], T, -1)
    for k in range(s["w"].shape[1]):
        acc = acc + s["w"][:, k] * xp[:, k:k + T].float()
    return acc


def _plain_conv(s):
    case = s["case"]
    B, T, D, K = case["B"], case["T"], case["D"], case["K"]
    step = case["kind"] == "conv_step"
    valid = _valid(s, T)
    x = s["x"][:, None] if step else _keep(s["x"], valid)
    past = s["state"] if step or case["resume"] else torch.zeros_like(s["state"])
    xp = torch.cat([past, x], 1)
    y = _taps(s, xp, T)
    if case["silu"]:
        y = _silu(y)
    y = _keep(y, valid).to(s["x"].dtype)
    if valid is None:
        s["state"].copy_(xp[:, T:])
    else:
        at = s["lengths"].long()[:, None] + torch.arange(K - 1, device="cuda")
        s["state"].copy_(torch.gather(xp, 1, at[..., None].expand(-1, -1, D)))
    return {"y": y[:, 0] if step else y, "state": s["state"]}


def _plain_conv_grad(s):
    case = s["case"]
    T, K = case["T"], case["K"]
    valid = _valid(s, T)
    x, g = _keep(s["x"], valid).float(), _keep(s["dy"], valid).float()
    xp = torch.nn.functional.pad(x, (0, 0, K - 1, 0))
    if case["silu"]:
        g = g * _silu_slope(_taps(s, xp, T))
    gp = torch.nn.functional.pad(g, (0, 0, 0, K - 1))
    dx = torch.zeros_like(x)
    dw = torch.empty_like(s["w"])
    for k in range(K):
        dx += s["w"][:, k] * gp[:, K - 1 - k:K - 1 - k + T]
        dw[:, k] = (g * xp[:, k:k + T]).sum((0, 1))
    return {"dx": _keep(dx, valid).to(s["x"].dtype), "dw": dw, "dbias": g.sum((0, 1))}


def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-torch.abs(x)))


def _block(case):
    """Steps of one time block: about 2^25 states at a time."""
    return max(16, min(256, (1 << 25) // (case["B"] * case["D"] * case["N"])))


def _double(a, v, x):
    """All states of x <- a x + v over the second axis, from x, by doubling."""
    v[:, 0] += a[:, 0] * x
    k = 1
    while k < a.shape[1]:
        v[:, k:] += a[:, k:] * v[:, :-k]
        if 2 * k < a.shape[1]:
            a[:, k:] = a[:, k:] * a[:, :-k]
        k *= 2
    return v


def _per_channel(m, D):
    """[B, t, G, N] rows as the [B, t, D, N] of their channels."""
    G = m.shape[2]
    return m.float()[:, :, :, None].expand(-1, -1, -1, D // G, -1).flatten(2, 3)


def _slices(s, i, j):
    """float32 inputs of the steps i .. j - 1; padded tokens leave the state alone."""
    valid = _valid(s, s["case"]["T"])
    if valid is not None:
        valid = valid[:, i:j]
    D = s["case"]["D"]
    pre = s["dt"][:, i:j].float() + s["dt_bias"]
    delta = _keep(_softplus(pre), valid)
    u = _keep(s["u"][:, i:j].float(), valid)
    v4 = None if valid is None else valid[..., None]
    return valid, pre, delta, u, _keep(_per_channel(s["Bm"][:, i:j], D), v4), _keep(_per_channel(s["Cm"][:, i:j], D), v4)


def _plain_scan(s):
    case = s["case"]
    B, T, D, N = (case[k] for k in ("B", "T", "D", "N"))
    x = s["state"] if case["resume"] else torch.zeros_like(s["state"])
    y = torch.empty((B, T, D), dtype=s["u"].dtype, device="cuda")
    step = _block(case)
    for i in range(0, T, step):
        j = min(T, i + step)
        valid, _, delta, u, Bm, Cm = _slices(s, i, j)
        states = _double(torch.exp(delta[..., None] * s["A"]), (delta * u)[..., None] * Bm, x)
        o = (Cm * states).sum(-1) + s["h0"] * u
        if "z" in s:
            o = o * _silu(s["z"][:, i:j].float())
        y[:, i:j] = _keep(o, valid)
        x = states[:, -1]
    s["state"].copy_(x)
    return {"y": y, "state": s["state"]}


def _plain_scan_step(s):
    D = s["case"]["D"]
    u = s["u"].float()
    delta = _softplus(s["dt"].float() + s["dt_bias"])
    Bm, Cm = (_per_channel(s[k][:, None], D)[:, 0] for k in ("Bm", "Cm"))
    s["state"].mul_(torch.exp(delta[..., None] * s["A"])).add_((delta * u)[..., None] * Bm)
    y = (Cm * s["state"]).sum(-1) + s["h0"] * u
    if "z" in s:
        y = y * _silu(s["z"].float())
    return {"y": y.to(s["u"].dtype), "state": s["state"]}


def _plain_scan_grad(s):
    case = s["case"]
    B, T, D, N, G = (case[k] for k in ("B", "T", "D", "N", "G"))
    io = s["u"].dtype
    step = _block(case)
    x = torch.zeros((B, D, N), device="cuda")
    entry = []  # state at the start of each block
    for i in range(0, T, step):
        _, _, delta, u, Bm, _ = _slices(s, i, min(T, i + step))
        entry.append(x)
        x = _double(torch.exp(delta[..., None] * s["A"]), (delta * u)[..., None] * Bm, x)[:, -1].clone()
    out = {k: torch.empty((B, T, D), dtype=io, device="cuda") for k in ("ddt", "du", "dz")[:2 + ("z" in s)]}
    out.update({k: torch.empty((B, T, G, N), dtype=io, device="cuda") for k in ("dBm", "dCm")})
    out["dA"] = torch.zeros((D, N), device="cuda")
    out["dh0"], out["ddt_bias"] = torch.zeros(D, device="cuda"), torch.zeros(D, device="cuda")
    back = torch.zeros((B, D, N), device="cuda")  # gradient that reaches the block's last state from later ones
    for b, i in reversed(list(enumerate(range(0, T, step)))):
        j = min(T, i + step)
        valid, pre, delta, u, Bm, Cm = _slices(s, i, j)
        a = torch.exp(delta[..., None] * s["A"])
        states = _double(a.clone(), (delta * u)[..., None] * Bm, entry[b])
        dy = _keep(s["dy"][:, i:j].float(), valid)
        if "z" in s:
            z = _keep(s["z"][:, i:j].float(), valid)
            o = (Cm * states).sum(-1) + s["h0"] * u
            out["dz"][:, i:j] = _keep(dy * o * _silu_slope(z), valid)
            dy = dy * _silu(z)
        # dx_t = C_t dy_t + a_(t+1) dx_(t+1), the same recurrence backwards in time
        later = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1).flip(1)
        dx = _double(later, (Cm * dy[..., None]).flip(1), back).flip(1)
        back = a[:, 0] * dx[:, 0]
        before = torch.cat([entry[b][:, None], states[:, :-1]], 1)
        da = dx * before * a
        out["dA"] += (da * delta[..., None]).sum((0, 1))
        db = (dx * Bm).sum(-1)
        ddt = ((da * s["A"]).sum(-1) + db * u) * torch.sigmoid(pre)
        ddt = _keep(ddt, valid)
        out["ddt"][:, i:j] = ddt
        out["ddt_bias"] += ddt.sum((0, 1))
        out["du"][:, i:j] = _keep(db * delta + s["h0"] * dy, valid)
        out["dh0"] += (dy * u).sum((0, 1))
        group = lambda m: m.unflatten(2, (G, D // G)).sum(3)  # noqa: E731
        out["dBm"][:, i:j] = group(dx * (delta * u)[..., None])
        out["dCm"][:, i:j] = group(states * dy[..., None])
    return {k: out[k] for k in ("dA", "ddt", "dBm", "dCm", "du", "dh0", "ddt_bias", "dz") if k in out}


PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "conv": _plain_conv, "conv_step": _plain_conv,
         "conv_grad": _plain_conv_grad, "scan": _plain_scan, "scan_step": _plain_scan_step,
         "scan_grad": _plain_scan_grad}


def run(s):
    return _run_own(s) if own else PLAIN[s["case"]["kind"]](s)


# ---- the work that a call cannot do without

def work(case):
    kind, D = case["kind"], case["D"]
    es = 2 if case["io"] == "bf16" else 4
    if kind == "norm":
        n = case["rows"] * D
        return {"bytes": es * n * (4 if case["res"] else 2) + 8 * D, "flops": n * (9 if case["res"] else 8)}
    if kind == "norm_grad":
        n = case["rows"] * D
        return {"bytes": es * n * (4 if case["res"] else 3) + 8 * case["rows"] + 12 * D, "flops": 14 * n}
    B, T = case["B"], case["T"]
    n = B * T * D
    if kind.startswith("conv"):
        K = case["K"]
        state = es * B * (K - 1) * D
        if kind == "conv_grad":
            return {"bytes": 3 * es * n + 8 * D * K + 8 * D, "flops": n * (4 * K + 1 + (2 * K + 8 if case["silu"] else 0))}
        reads = kind == "conv_step" or case["resume"]
        return {"bytes": 2 * es * n + state * (2 if reads else 1) + 4 * D * K + 4 * D,
                "flops": n * (2 * K + (4 if case["silu"] else 0))}
    N, G, gate = case["N"], case["G"], case["gate"]
    rows = es * B * T * G * N
    if kind == "scan_grad":
        # dx and states (9 operations), four sums over them (8), the steps' two (4); exp counted as one
        return {"bytes": es * n * (7 if gate else 5) + 4 * rows + 8 * D * N + 16 * D,
                "flops": n * (21 * N + (26 if gate else 16))}
    reads = kind == "scan_step" or case["resume"]
    return {"bytes": es * n * (4 if gate else 3) + 2 * rows + 4 * D * N + 8 * D + 4 * B * D * N * (2 if reads else 1),
            "flops": n * (7 * N + (13 if gate else 8))}


# ---- float64, from the definitions

def _exact_norm(s):
    y, total = [], []
    for i in range(0, s["case"]["rows"], 4096):
        x = s["x"][i:i + 4096].double()
        if "residual" in s:
            x = x + s["residual"][i:i + 4096].double()
            total.append(x)
        var = x.var(-1, unbiased=False, keepdim=True)
        y.append((x - x.mean(-1, keepdim=True)) / torch.sqrt(var + 1e-5) * s["w"].double() + s["b"].double())
    return {"y": torch.cat(y), "total": torch.cat(total)} if total else {"y": torch.cat(y)}


def _exact_norm_grad(s):
    D = s["case"]["D"]
    w = s["w"].double()
    dx, dw, db = [], torch.zeros_like(w), torch.zeros_like(w)
    for i in range(0, s["case"]["rows"], 4096):
        r = slice(i, i + 4096)
        dy, rstd = s["dy"][r].double(), s["rstd"][r].double()[:, None]
        xh = (s["x"][r].double() - s["mean"][r].double()[:, None]) * rstd
        dw += (dy * xh).sum(0)
        db += dy.sum(0)
        g = dy * w
        d = (D * g - g.sum(-1, keepdim=True) - xh * (g * xh).sum(-1, keepdim=True)) * rstd / D
        dx.append(d + s["dtotal"][r].double() if "dtotal" in s else d)
    return {"dx": torch.cat(dx), "dw": dw, "db": db}


def _rows64(s, b, *names):
    """Row b of a right-padded batch, its own tokens only, in float64."""
    n = int(s["lengths"][b]) if "lengths" in s else s["case"]["T"]
    return [s[k][b, :n].double() for k in names]


def _exact_conv(s):
    case = s["case"]
    B, T, D, K = case["B"], case["T"], case["D"], case["K"]
    w, bias = s["w"].double(), s["bias"].double()
    y = torch.zeros((B, T, D), dtype=torch.float64, device="cuda")
    state = torch.zeros((B, K - 1, D), dtype=torch.float64, device="cuda")
    for b in range(B):
        if case["kind"] == "conv_step":
            x = s["x"][b:b + 1].double()
        else:
            x, = _rows64(s, b, "x")
        past = s["state"][b].double()
        if case["kind"] == "conv" and not case["resume"]:
            past = past * 0
        xp = torch.cat([past, x])
        if len(x):  # windows [tokens, D, K]
            o = (xp.unfold(0, K, 1) * w).sum(-1) + bias
            y[b, :len(x)] = o / (1 + torch.exp(-o)) if case["silu"] else o
        state[b] = xp[len(x):]
    return {"y": y[:, 0] if case["kind"] == "conv_step" else y, "state": state}


def _exact_conv_grad(s):
    case = s["case"]
    B, T, D, K = case["B"], case["T"], case["D"], case["K"]
    w, bias = s["w"].double(), s["bias"].double()
    dx = torch.zeros((B, T, D), dtype=torch.float64, device="cuda")
    dw, dbias = torch.zeros_like(w), torch.zeros_like(bias)
    for b in range(B):
        x, g = _rows64(s, b, "x", "dy")
        n = len(x)
        if n == 0:
            continue
        win = torch.cat([torch.zeros((K - 1, D), dtype=torch.float64, device="cuda"), x]).unfold(0, K, 1)
        if case["silu"]:
            o = (win * w).sum(-1) + bias
            p = 1 / (1 + torch.exp(-o))
            g = g * (p + o * p * (1 - p))
        dw += (g[..., None] * win).sum(0)
        dbias += g.sum(0)
        for k in range(min(K, n)):  # input t reaches output t + k through tap K - 1 - k
            dx[b, :n - k] += g[k:] * w[:, K - 1 - k]
    return {"dx": dx, "dw": dw, "dbias": dbias}


def _exact_steps(s):
    """float64 inputs with the time first; a padded token has step 0 and zeros."""
    step = s["case"]["kind"] == "scan_step"
    one = (lambda x: x[:, None]) if step else (lambda x: x)
    pre = (one(s["dt"]).double() + s["dt_bias"].double()).transpose(0, 1)
    delta = torch.log(1 + torch.exp(-pre.abs())) + torch.relu(pre)
    delta = torch.where(pre < -30, torch.exp(pre), delta)
    d = {"pre": pre, "delta": delta}
    for k in ("u", "Bm", "Cm", "z", "dy"):
        if k in s:
            d[k] = one(s[k]).double().transpose(0, 1)
    if "lengths" in s:
        out = torch.arange(s["case"]["T"], device="cuda")[:, None] >= s["lengths"]
        for k in d:
            d[k] = d[k].masked_fill(out.reshape(out.shape + (1,) * (d[k].dim() - 2)), 0.0)
    return d


def _exact_scan(s):
    case = s["case"]
    B, T, D, N, G = (case[k] for k in ("B", "T", "D", "N", "G"))
    d = _exact_steps(s)
    A, h0 = s["A"].double(), s["h0"].double()
    x = s["state"].double()
    if case["kind"] == "scan" and not case["resume"]:
        x = torch.zeros_like(x)
    y = torch.empty((T, B, D), dtype=torch.float64, device="cuda")
    for t in range(T):
        x = torch.exp(d["delta"][t, ..., None] * A) * x
        du = (d["delta"][t] * d["u"][t]).view(B, G, D // G, 1)
        x = x + (du * d["Bm"][t][:, :, None]).view(B, D, N)
        y[t] = torch.matmul(x.view(B, G, D // G, N), d["Cm"][t][..., None].contiguous()).view(B, D)
    y += h0 * d["u"]
    if "z" in d:
        y *= d["z"] / (1 + torch.exp(-d["z"]))
    y = y.transpose(0, 1)
    return {"y": y[:, 0] if case["kind"] == "scan_step" else y, "state": x}


def _exact_scan_grad(s):
    case = s["case"]
    B, T, D, N, G = (case[k] for k in ("B", "T", "D", "N", "G"))
    d = _exact_steps(s)
    A, h0 = s["A"].double(), s["h0"].double()
    wide = lambda m: m.repeat_interleave(D // G, dim=1)  # noqa: E731  [B, G, N] -> [B, D, N]
    xs = torch.zeros((T + 1, B, D, N), dtype=torch.float64, device="cuda")
    for t in range(T):
        xs[t + 1] = torch.exp(d["delta"][t, ..., None] * A) * xs[t] + (d["delta"][t] * d["u"][t])[..., None] * wide(d["Bm"][t])
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out = {"dA": zeros(D, N), "ddt": zeros(T, B, D), "dBm": zeros(T, B, G, N), "dCm": zeros(T, B, G, N),
           "du": zeros(T, B, D), "dh0": zeros(D), "ddt_bias": zeros(D)}
    if "z" in d:
        out["dz"] = zeros(T, B, D)
    grad = zeros(B, D, N)  # of the state after step t
    for t in reversed(range(T)):
        u, delta, dy = d["u"][t], d["delta"][t], d["dy"][t]
        Bw, Cw = wide(d["Bm"][t]), wide(d["Cm"][t])
        if "z" in d:
            z = d["z"][t]
            p = 1 / (1 + torch.exp(-z))
            out["dz"][t] = dy * ((Cw * xs[t + 1]).sum(-1) + h0 * u) * (p + z * p * (1 - p))
            dy = dy * z * p
        grad = grad + dy[..., None] * Cw
        out["dCm"][t] = (dy[..., None] * xs[t + 1]).view(B, G, D // G, N).sum(2)
        out["dBm"][t] = (grad * (delta * u)[..., None]).view(B, G, D // G, N).sum(2)
        gb = (grad * Bw).sum(-1)
        decay = torch.exp(delta[..., None] * A)
        through = grad * decay * xs[t]
        out["dA"] += (through * delta[..., None]).sum(0)
        out["ddt"][t] = ((through * A).sum(-1) + gb * u) / (1 + torch.exp(-d["pre"][t]))
        out["du"][t] = gb * delta + h0 * dy
        out["dh0"] += (dy * u).sum(0)
        grad = grad * decay
    if "lengths" in s:
        past = torch.arange(T, device="cuda")[:, None] >= s["lengths"]
        out["ddt"][past] = 0
    out["ddt_bias"] = out["ddt"].sum((0, 1))
    for k in ("ddt", "dBm", "dCm", "du", "dz"):
        if k in out:
            out[k] = out[k].transpose(0, 1)
    return {k: out[k] for k in ("dA", "ddt", "dBm", "dCm", "du", "dh0", "ddt_bias", "dz") if k in out}


EXACT = {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "conv": _exact_conv, "conv_step": _exact_conv,
         "conv_grad": _exact_conv_grad, "scan": _exact_scan, "scan_step": _exact_scan, "scan_grad": _exact_scan_grad}


def exact(case, seed):
    return EXACT[case["kind"]](_inputs(case, seed))
