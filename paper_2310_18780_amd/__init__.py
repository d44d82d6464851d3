"""Distilled modal recurrence (Laughing Hyena) on AMD MI355X.

Thin Python binding of ``liblh.so`` (C ABI in ``include/lh.h``): it checks
tensor shapes and dtypes, marshals pointers and the current HIP stream, and
calls the library.  Every step of the computation runs in the library's HIP
kernels; there is no fallback.  PyTorch provides device memory and streams.

    prefill(lam, R, h0, u, state, y)   # y[b,t,c], t < T, and state = x_T
    prefill_plan(B, D, d, T, io="bf16")  # its plan's name ("scan", "mfma", "mfma_seg")
    prefill_path(B, D, d, T, io="bf16")  # what runs: ("mfma" or "valu", columns, segments)
    prefill_with_plan(lam, R, h0, u, state, y, plan=PLAN_MFMA)  # a named plan (tests, benchmarks)
    prefill_fft(lam, R, h0, u, state, y)  # the same results by FFT convolution
    step(lam, R, h0, state, u_t, y_t)  # y_t from x_t, then x_{t+1} in place

The selective block beside it (prompts, single tokens, gradients):

    layer_norm, layer_norm_backward
    short_conv_prefill, short_conv_step, short_conv_backward
    selective_prefill, selective_step, selective_backward

The gated recurrence and the two ends of a language model:

    gated_prefill, gated_step, gated_backward
    embed, embed_backward
    distill_logits, distill_logits_backward
    verify_draft

``lam``, ``R``: complex64 ``[D, d]``; ``h0``: float32 ``[D]``; ``u``, ``y``:
float32 or bfloat16 ``[B, T, D]``; ``state``: complex64 ``[B, D, d]``;
``u_t``, ``y_t``: ``[B, D]``.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

__all__ = [
    "LH_F32",
    "LH_BF16",
    "LHError",
    "lib",
    "library_path",
    "workspace_bytes",
    "prefill_plan",
    "prefill_path",
    "PREFILL_PLANS",
    "PLAN_AUTO",
    "PLAN_MFMA",
    "PLAN_MFMA_SEG",
    "prefill",
    "prefill_with_plan",
    "prefill_noalloc",
    "NOALLOC_SCRATCH_BYTES",
    "fft_workspace_bytes",
    "prefill_fft",
    "step",
    "mh_step",
    "distill",
    "companion_coeffs",
    "companion_step",
    "companion_init_workspace_bytes",
    "companion_init",
    "layer_norm",
    "layer_norm_backward_workspace_bytes",
    "layer_norm_backward",
    "short_conv_prefill",
    "short_conv_step",
    "short_conv_backward_workspace_bytes",
    "short_conv_backward",
    "selective_workspace_bytes",
    "selective_prefill",
    "selective_step",
    "selective_backward_workspace_bytes",
    "selective_backward",
    "GATED_MARK",
    "gated_workspace_bytes",
    "gated_prefill",
    "gated_step",
    "gated_backward_workspace_bytes",
    "gated_backward",
    "embed",
    "embed_backward_workspace_bytes",
    "embed_backward",
    "distill_logits_workspace_bytes",
    "distill_logits",
    "distill_logits_backward",
    "verify_draft_workspace_bytes",
    "verify_draft",
    "STATUS",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "liblh.so")

LH_F32 = 0
LH_BF16 = 1
# plan requests of prefill_with_plan (values > 0 are VALU chunk lengths)
PLAN_AUTO = 0
PLAN_MFMA = -1
PLAN_MFMA_SEG = -2
# scratch that lh_prefill_noalloc holds per GPU
NOALLOC_SCRATCH_BYTES = 64 << 20
# tokens between the states that gated_prefill leaves for gated_backward
GATED_MARK = 8
STATUS = {
    0: "LH_OK",
    1: "LH_ERR_INVALID_ARG",
    2: "LH_ERR_OVERLAP",
    3: "LH_ERR_UNSUPPORTED_DTYPE",
    4: "LH_ERR_NO_DEVICE",
    5: "LH_ERR_WORKSPACE",
    6: "LH_ERR_HIP",
}

_lib: Optional[ctypes.CDLL] = None
# torch and its current-stream lookup, set when the library is loaded
_torch = None
_raw_stream = None


class _SelectiveInputs(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("A", "dt_bias", "h0", "dt", "u", "z", "Bm", "Cm", "lengths")]
                + [(k, ctypes.c_int64) for k in ("ld_dt", "ld_u", "ld_z", "ld_B", "ld_C", "B", "T", "D", "N", "G")]
                + [("io_dtype", ctypes.c_int)])


class _SelectiveGrads(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("dy", "ddt", "du", "dz", "dBm", "dCm", "dA", "dh0", "ddt_bias")]


class _GatedInputs(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("rate", "r_bias", "i_bias", "r", "i", "u", "z", "lengths")]
                + [(k, ctypes.c_int64) for k in ("ld_r", "ld_i", "ld_u", "ld_z", "B", "T", "D")]
                + [("io_dtype", ctypes.c_int)])


class _GatedGrads(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("dy", "marks", "dlast", "dr", "di", "du", "dz", "drate", "dr_bias",
                                               "di_bias", "dfirst")]


class LHError(RuntimeError):
    def __init__(self, status: int, detail: str):
        self.status = status
        self.name = STATUS.get(status, f"status {status}")
        super().__init__(f"{self.name}: {detail}")


def library_path() -> str:
    return _LIB_PATH


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib, _torch, _raw_stream
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2310_18780_amd.build` "
            "(or __graft_entry__.build()); there is no fallback implementation")
    # torch first: it brings its own HIP runtime, and the library's dependency
    # on the HIP runtime then resolves to that same, already loaded copy.
    # Loaded the other way round, the process would hold two HIP runtimes and
    # torch's memory and streams would be unknown to the library's.
    import torch

    _torch = torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    L = ctypes.CDLL(_LIB_PATH)
    i64, vp, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
    L.lh_abi_version.argtypes = []
    L.lh_abi_version.restype = ctypes.c_int
    L.lh_status_string.argtypes = [ctypes.c_int]
    L.lh_status_string.restype = ctypes.c_char_p
    L.lh_last_error.argtypes = []
    L.lh_last_error.restype = ctypes.c_char_p
    L.lh_prefill_workspace_bytes.argtypes = [i64, i64, i64, i64]
    L.lh_prefill_workspace_bytes.restype = sz
    L.lh_prefill_with_plan_workspace_bytes.argtypes = [i64, i64, i64, i64, i64]
    L.lh_prefill_with_plan_workspace_bytes.restype = sz
    L.lh_prefill_plan.argtypes = [i64, i64, i64, i64, i64, ctypes.c_int]
    L.lh_prefill_plan.restype = ctypes.c_int
    L.lh_prefill_path.argtypes = [i64, i64, i64, i64, i64, ctypes.c_int, ctypes.POINTER(i64),
                                  ctypes.POINTER(i64)]
    L.lh_prefill_path.restype = ctypes.c_int
    L.lh_prefill.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, ctypes.c_int, vp, vp, vp, sz, vp]
    L.lh_prefill.restype = ctypes.c_int
    L.lh_prefill_with_plan.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, ctypes.c_int, vp, vp,
                                       i64, vp, sz, vp]
    L.lh_prefill_with_plan.restype = ctypes.c_int
    L.lh_prefill_noalloc.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, ctypes.c_int, vp, vp, vp]
    L.lh_prefill_noalloc.restype = ctypes.c_int
    L.lh_prefill_fft_workspace_bytes.argtypes = [i64, i64, i64, i64]
    L.lh_prefill_fft_workspace_bytes.restype = sz
    L.lh_prefill_fft.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, ctypes.c_int, vp, vp, vp, sz,
                                 vp]
    L.lh_prefill_fft.restype = ctypes.c_int
    L.lh_step.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, ctypes.c_int, vp]
    L.lh_step.restype = ctypes.c_int
    L.lh_mh_step.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, ctypes.c_int, vp]
    L.lh_mh_step.restype = ctypes.c_int
    L.lh_distill.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp]
    L.lh_distill.restype = ctypes.c_int
    L.lh_companion_coeffs.argtypes = [vp, vp, i64, i64, vp, vp, vp]
    L.lh_companion_coeffs.restype = ctypes.c_int
    L.lh_companion_step.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, ctypes.c_int, vp]
    L.lh_companion_step.restype = ctypes.c_int
    L.lh_companion_init_workspace_bytes.argtypes = [i64, i64, i64]
    L.lh_companion_init_workspace_bytes.restype = sz
    L.lh_companion_init.argtypes = [vp, vp, i64, i64, i64, i64, ctypes.c_int, vp, vp, sz, vp]
    L.lh_companion_init.restype = ctypes.c_int
    ci, cf = ctypes.c_int, ctypes.c_float
    L.lh_layer_norm.argtypes = [vp, vp, vp, vp, i64, i64, cf, ci, vp, vp, vp, vp, vp]
    L.lh_layer_norm.restype = ci
    L.lh_layer_norm_backward_workspace_bytes.argtypes = [i64, i64]
    L.lh_layer_norm_backward_workspace_bytes.restype = sz
    L.lh_layer_norm_backward.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, ci, vp, vp, vp, vp, sz, vp]
    L.lh_layer_norm_backward.restype = ci
    L.lh_short_conv_prefill.argtypes = [vp, i64, vp, vp, vp, i64, i64, i64, i64, ci, ci, ci, vp, vp, vp]
    L.lh_short_conv_prefill.restype = ci
    L.lh_short_conv_step.argtypes = [vp, i64, vp, vp, i64, i64, i64, ci, ci, vp, vp, vp]
    L.lh_short_conv_step.restype = ci
    L.lh_short_conv_backward_workspace_bytes.argtypes = [i64, i64, i64, i64]
    L.lh_short_conv_backward_workspace_bytes.restype = sz
    L.lh_short_conv_backward.argtypes = [vp, vp, i64, vp, vp, vp, i64, i64, i64, i64, ci, ci, vp, vp, vp, vp, sz, vp]
    L.lh_short_conv_backward.restype = ci
    for name in ("lh_selective_workspace_bytes", "lh_selective_backward_workspace_bytes"):
        getattr(L, name).argtypes = [i64, i64, i64, i64, i64]
        getattr(L, name).restype = sz
    L.lh_selective_prefill.argtypes = [vp, ci, vp, vp, vp, sz, vp]
    L.lh_selective_prefill.restype = ci
    L.lh_selective_step.argtypes = [vp, vp, vp, vp]
    L.lh_selective_step.restype = ci
    L.lh_selective_backward.argtypes = [vp, vp, vp, sz, vp]
    L.lh_selective_backward.restype = ci
    cf = ctypes.c_float
    for name in ("lh_gated_workspace_bytes", "lh_gated_backward_workspace_bytes", "lh_embed_backward_workspace_bytes",
                 "lh_distill_logits_workspace_bytes", "lh_verify_draft_workspace_bytes"):
        getattr(L, name).argtypes = [i64, i64, i64]
        getattr(L, name).restype = sz
    for name, args in (
            ("lh_gated_prefill", [vp, ci, vp, vp, vp, vp, sz, vp]),
            ("lh_gated_step", [vp, vp, vp, vp]),
            ("lh_gated_backward", [vp, vp, vp, sz, vp]),
            ("lh_embed", [vp, vp, i64, i64, i64, ci, ci, cf, vp, vp]),
            ("lh_embed_backward", [vp, vp, i64, i64, i64, ci, cf, ci, vp, vp, sz, vp]),
            ("lh_distill_logits", [vp, i64, vp, vp, vp, i64, i64, i64, ci, cf, vp, vp, vp, i64, vp, sz, vp]),
            ("lh_distill_logits_backward", [vp, vp, i64, vp, vp, vp, vp, i64, i64, i64, ci, cf, vp, i64, vp]),
            ("lh_verify_draft", [vp, vp, vp, i64, vp, i64, vp, vp, i64, i64, i64, ci, vp, vp, vp, sz, vp])):
        getattr(L, name).argtypes = args
        getattr(L, name).restype = ci
    _lib = L
    return L


def _torch_loaded():
    lib()
    return _torch


def _check(status: int) -> None:
    if status != 0:
        raise LHError(status, lib().lh_last_error().decode(errors="replace"))


def workspace_bytes(B: int, D: int, d: int, T: int, plan: int = PLAN_AUTO) -> int:
    """Workspace bytes of ``prefill`` (``lh_prefill_workspace_bytes``), or of
    ``prefill_with_plan`` with this plan request
    (``lh_prefill_with_plan_workspace_bytes``)."""
    if plan == PLAN_AUTO:
        n = lib().lh_prefill_workspace_bytes(B, D, d, T)
    else:
        n = lib().lh_prefill_with_plan_workspace_bytes(B, D, d, T, plan)
    if n == ctypes.c_size_t(-1).value:
        raise LHError(1, f"invalid sizes B={B} D={D} d={d} T={T} plan={plan}")
    return int(n)


PREFILL_PLANS = ("scan", "mfma", "mfma_seg")


def prefill_plan(B: int, D: int, d: int, T: int, plan: int = PLAN_AUTO, io: str = "f32") -> str:
    """The name of a prefill's plan, which fixes its workspace (``lh_prefill_plan``):
    "scan", "mfma" (matrix cores, whole prompt) or "mfma_seg" (segmented).
    ``prefill_path`` tells what runs."""
    k = lib().lh_prefill_plan(B, D, d, T, plan, {"f32": 0, "bf16": 1}[io])
    if k < 0:
        raise LHError(1, f"no prefill plan for B={B} D={D} d={d} T={T} plan={plan} io={io}")
    return PREFILL_PLANS[k]


def prefill_path(B: int, D: int, d: int, T: int, plan: int = PLAN_AUTO, io: str = "f32"):
    """What a prefill executes (``lh_prefill_path``): ("mfma" or "valu", chunks of a
    row side by side in a matrix product, time segments in parallel)."""
    columns, segments = ctypes.c_int64(), ctypes.c_int64()
    k = lib().lh_prefill_path(B, D, d, T, plan, {"f32": 0, "bf16": 1}[io], ctypes.byref(columns),
                              ctypes.byref(segments))
    if k < 0:
        raise LHError(1, f"no prefill plan for B={B} D={D} d={d} T={T} plan={plan} io={io}")
    return ("valu", "mfma")[k], columns.value, segments.value


def _io_dtype(t) -> int:
    if t.dtype is _torch.float32:
        return LH_F32
    if t.dtype is _torch.bfloat16:
        return LH_BF16
    raise TypeError(f"u / y must be float32 or bfloat16, got {t.dtype}")


def _need(t, name, dtype, shape):
    # one test of all properties; which one fails is found out only then
    if (isinstance(t, _torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == shape
            and t.is_contiguous()):
        return
    if not isinstance(t, _torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a HIP device, got {t.device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _stream(dev, stream):
    """(torch stream object, raw hipStream_t handle) of ``stream``: None is the
    device's current stream; a raw handle is wrapped as an external stream."""
    if stream is None:
        stream = _torch.cuda.current_stream(dev)
    elif not isinstance(stream, _torch.cuda.Stream):
        stream = _torch.cuda.ExternalStream(int(stream), device=dev)
    return stream, int(stream.cuda_stream)


def _handle(t, stream) -> int:
    """Raw hipStream_t handle of ``stream``; None is the current stream of ``t``'s
    device, whose handle is read without building a stream object where torch
    offers that (1.7 us less per call)."""
    if stream is None and _raw_stream is not None:
        return _raw_stream(t.get_device())
    return _stream(t.device, stream)[1]


def _scratch(need: int, workspace, dev, stream):
    """The caller's workspace, or a new one when ``workspace`` is None.  A
    workspace allocated here comes from torch's caching allocator, whose blocks
    belong to the current stream; the library enqueues on ``stream``, so the
    block is marked as used there (record_stream) and is not handed out again
    before that stream's work on it has completed."""
    if need > 0 and workspace is None:
        workspace = _torch.empty(need, dtype=_torch.uint8, device=dev)
        stream, handle = _stream(dev, stream)
        if handle != _torch.cuda.current_stream(dev).cuda_stream:
            workspace.record_stream(stream)
    if workspace is None:
        return workspace, None, 0
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _prefill_args(lam, R, h0, u, state, y):
    torch = _torch_loaded()
    B, T, D = u.shape
    d = lam.shape[1]
    _need(lam, "lam", torch.complex64, (D, d))
    _need(R, "R", torch.complex64, (D, d))
    _need(h0, "h0", torch.float32, (D,))
    _need(u, "u", u.dtype, (B, T, D))
    _need(state, "state", torch.complex64, (B, D, d))
    _need(y, "y", u.dtype, (B, T, D))
    return B, D, d, T, _io_dtype(u)


def prefill(lam, R, h0, u, state, y, workspace=None, stream=None) -> None:
    """Prompt outputs ``y`` and post-prompt state ``state`` (both overwritten),
    with the library's automatic plan (``lh_prefill``).

    ``workspace``: a uint8 CUDA tensor of at least ``workspace_bytes(...)``
    bytes, or None to have one allocated here with torch."""
    B, D, d, T, io = _prefill_args(lam, R, h0, u, state, y)
    handle = _handle(u, stream)
    workspace, ws_ptr, ws_len = _scratch(workspace_bytes(B, D, d, T), workspace, u.device, stream)
    _check(lib().lh_prefill(lam.data_ptr(), R.data_ptr(), h0.data_ptr(), u.data_ptr(), B, D, d, T,
                            io, state.data_ptr(), y.data_ptr(), ws_ptr, ws_len, handle))


def prefill_with_plan(lam, R, h0, u, state, y, plan: int, workspace=None, stream=None) -> None:
    """``prefill`` with a named plan (``lh_prefill_with_plan``): ``PLAN_AUTO``,
    ``PLAN_MFMA``, ``PLAN_MFMA_SEG`` or a VALU chunk length > 0."""
    B, D, d, T, io = _prefill_args(lam, R, h0, u, state, y)
    handle = _handle(u, stream)
    workspace, ws_ptr, ws_len = _scratch(workspace_bytes(B, D, d, T, plan), workspace, u.device,
                                         stream)
    _check(lib().lh_prefill_with_plan(lam.data_ptr(), R.data_ptr(), h0.data_ptr(), u.data_ptr(), B,
                                      D, d, T, io, state.data_ptr(), y.data_ptr(), plan, ws_ptr,
                                      ws_len, handle))


def prefill_noalloc(lam, R, h0, u, state, y, stream=None) -> None:
    """``prefill`` without a workspace (``lh_prefill_noalloc``): the library's
    static per-GPU scratch serves the plan, so nothing is allocated.  Sizes
    needing more than ``NOALLOC_SCRATCH_BYTES`` of scratch raise; calls that
    overlap on one GPU race on that scratch."""
    B, D, d, T, io = _prefill_args(lam, R, h0, u, state, y)
    _check(lib().lh_prefill_noalloc(lam.data_ptr(), R.data_ptr(), h0.data_ptr(), u.data_ptr(), B,
                                    D, d, T, io, state.data_ptr(), y.data_ptr(),
                                    _handle(u, stream)))


def fft_workspace_bytes(B: int, D: int, d: int, T: int) -> int:
    n = lib().lh_prefill_fft_workspace_bytes(B, D, d, T)
    if n == ctypes.c_size_t(-1).value:
        raise LHError(1, f"invalid sizes for the FFT prefill B={B} D={D} d={d} T={T}")
    return int(n)


def prefill_fft(lam, R, h0, u, state, y, workspace=None, stream=None) -> None:
    """``prefill``'s results by FFT convolution with the materialised filter
    and a Vandermonde contraction for the state (``lh_prefill_fft``)."""
    B, D, d, T, io = _prefill_args(lam, R, h0, u, state, y)
    handle = _handle(u, stream)
    workspace, ws_ptr, ws_len = _scratch(fft_workspace_bytes(B, D, d, T), workspace, u.device,
                                         stream)
    _check(lib().lh_prefill_fft(lam.data_ptr(), R.data_ptr(), h0.data_ptr(), u.data_ptr(), B, D,
                                d, T, io, state.data_ptr(), y.data_ptr(), ws_ptr, ws_len, handle))


def step(lam, R, h0, state, u_t, y_t, stream=None) -> None:
    """One decode step: ``y_t`` from the current state, then the state update
    in place."""
    torch = _torch_loaded()
    B, D = u_t.shape
    d = lam.shape[1]
    _need(lam, "lam", torch.complex64, (D, d))
    _need(R, "R", torch.complex64, (D, d))
    _need(h0, "h0", torch.float32, (D,))
    _need(state, "state", torch.complex64, (B, D, d))
    _need(u_t, "u_t", u_t.dtype, (B, D))
    _need(y_t, "y_t", u_t.dtype, (B, D))
    io = _io_dtype(u_t)
    _check(lib().lh_step(lam.data_ptr(), R.data_ptr(), h0.data_ptr(), state.data_ptr(),
                         u_t.data_ptr(), y_t.data_ptr(), B, D, d, io,
                         _handle(u_t, stream)))


def mh_step(lam, R, h0, state, q, k, v, y, stream=None) -> None:
    """One multi-head decode step (``lh_mh_step``): ``y`` from the current
    per-entry states of the ``M`` heads, then the state update in place.

    ``lam``, ``R``: ``[M, d]`` complex64; ``h0``: ``[M]``; ``state``:
    ``[B, M, N, N, d]`` complex64; ``q``, ``k``, ``v``, ``y``: ``[B, M N]``.
    """
    torch = _torch_loaded()
    B, M, N, _, d = state.shape
    _need(lam, "lam", torch.complex64, (M, d))
    _need(R, "R", torch.complex64, (M, d))
    _need(h0, "h0", torch.float32, (M,))
    _need(state, "state", torch.complex64, (B, M, N, N, d))
    for name, t in (("q", q), ("k", k), ("v", v), ("y", y)):
        _need(t, name, q.dtype, (B, M * N))
    io = _io_dtype(q)
    _check(lib().lh_mh_step(lam.data_ptr(), R.data_ptr(), h0.data_ptr(), state.data_ptr(),
                            q.data_ptr(), k.data_ptr(), v.data_ptr(), y.data_ptr(), B, M, N, d,
                            io, _handle(q, stream)))


def distill(A, theta, R, target, loss, dA, dtheta, dR, hhat=None, stream=None) -> None:
    """Distillation objective (``lh_distill``): ``loss [D]`` and the gradients
    ``dA, dtheta [D, d]`` (float32), ``dR [D, d]`` (complex64,
    ``d/dRe R + i d/dIm R``) of the squared l2 error between the modal filter
    of polar poles ``A e^{i theta}`` and residues ``R`` and ``target [D, L]``;
    optionally the materialised filter ``hhat [D, L]``."""
    torch = _torch_loaded()
    D, d = A.shape
    L = target.shape[1]
    _need(A, "A", torch.float32, (D, d))
    _need(theta, "theta", torch.float32, (D, d))
    _need(R, "R", torch.complex64, (D, d))
    _need(target, "target", torch.float32, (D, L))
    _need(loss, "loss", torch.float32, (D,))
    _need(dA, "dA", torch.float32, (D, d))
    _need(dtheta, "dtheta", torch.float32, (D, d))
    _need(dR, "dR", torch.complex64, (D, d))
    if hhat is not None:
        _need(hhat, "hhat", torch.float32, (D, L))
    _check(lib().lh_distill(A.data_ptr(), theta.data_ptr(), R.data_ptr(), target.data_ptr(), D, d,
                            L, loss.data_ptr(), dA.data_ptr(), dtheta.data_ptr(), dR.data_ptr(),
                            hhat.data_ptr() if hhat is not None else None,
                            _handle(A, stream)))


def companion_coeffs(lam, R, a, beta, stream=None) -> None:
    """Rational coefficients of the filters' companion form
    (``lh_companion_coeffs``): ``a, beta [D, 2d]`` float64 from ``lam, R [D, d]``."""
    torch = _torch_loaded()
    D, d = lam.shape
    _need(lam, "lam", torch.complex64, (D, d))
    _need(R, "R", torch.complex64, (D, d))
    _need(a, "a", torch.float64, (D, 2 * d))
    _need(beta, "beta", torch.float64, (D, 2 * d))
    _check(lib().lh_companion_coeffs(lam.data_ptr(), R.data_ptr(), D, d, a.data_ptr(),
                                     beta.data_ptr(), _handle(lam, stream)))


def companion_step(a, beta, h0, state, u_t, y_t, stream=None) -> None:
    """One companion decode step (``lh_companion_step``); ``state [B, D, 2d]``
    float64 in place."""
    torch = _torch_loaded()
    B, D, order = state.shape
    _need(a, "a", torch.float64, (D, order))
    _need(beta, "beta", torch.float64, (D, order))
    _need(h0, "h0", torch.float32, (D,))
    _need(state, "state", torch.float64, (B, D, order))
    _need(u_t, "u_t", u_t.dtype, (B, D))
    _need(y_t, "y_t", u_t.dtype, (B, D))
    if order % 2:
        raise ValueError(f"companion order must be even (2d), got {order}")
    _check(lib().lh_companion_step(a.data_ptr(), beta.data_ptr(), h0.data_ptr(), state.data_ptr(),
                                   u_t.data_ptr(), y_t.data_ptr(), B, D, order // 2,
                                   _io_dtype(u_t), _handle(u_t, stream)))


def companion_init_workspace_bytes(D: int, d: int, T: int) -> int:
    n = lib().lh_companion_init_workspace_bytes(D, d, T)
    if n == ctypes.c_size_t(-1).value:
        raise LHError(1, f"invalid sizes for the companion initialisation D={D} d={d} T={T}")
    return int(n)


def companion_init(a, u, state, workspace=None, stream=None) -> None:
    """Companion state after the prompt ``u [B, T, D]`` (``lh_companion_init``,
    Proposition "fast_init")."""
    torch = _torch_loaded()
    B, T, D = u.shape
    order = a.shape[1]
    _need(a, "a", torch.float64, (D, order))
    _need(u, "u", u.dtype, (B, T, D))
    _need(state, "state", torch.float64, (B, D, order))
    if order % 2:
        raise ValueError(f"companion order must be even (2d), got {order}")
    handle = _handle(u, stream)
    workspace, ws_ptr, ws_len = _scratch(companion_init_workspace_bytes(D, order // 2, T), workspace,
                                         u.device, stream)
    _check(lib().lh_companion_init(a.data_ptr(), u.data_ptr(), B, D, order // 2, T, _io_dtype(u),
                                   state.data_ptr(), ws_ptr, ws_len, handle))


# ---- the selective block

def _ptr(t):
    return None if t is None else t.data_ptr()


def _need_rows(t, name, dtype, shape, lead, width) -> int:
    """Checks ``t`` of this shape, the first ``lead`` axes (batch, or batch and time) of
    which count rows of ``width`` contiguous elements, a fixed distance apart; returns
    that distance in elements."""
    # one test of all properties, as in _need
    if isinstance(t, _torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == shape:
        if t.is_contiguous():
            return width
        strides = t.stride()
        n = 1
        for i in range(len(shape) - 1, lead - 1, -1):
            if strides[i] != n and shape[i] > 1:
                raise ValueError(f"{name} must have contiguous rows")
            n *= shape[i]
        # (the stride of an axis of one says nothing)
        if lead == 1 or shape[1] == 1:
            ld = strides[0] if shape[0] > 1 else width
        else:
            ld = strides[1]
            if shape[0] > 1 and strides[0] != shape[1] * ld:
                raise ValueError(f"{name}: the rows of its batches must follow one another")
        if ld < width:
            raise ValueError(f"{name} must have rows that do not overlap")
        return ld
    if not isinstance(t, _torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a HIP device, got {t.device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _need_lengths(lengths, B):
    if lengths is not None:
        _need(lengths, "lengths", _torch.int32, (B,))


def _block_bytes(name, *sizes) -> int:
    n = getattr(lib(), name)(*sizes)
    if n == ctypes.c_size_t(-1).value:
        raise LHError(1, lib().lh_last_error().decode(errors="replace"))
    return int(n)


def layer_norm(x, w, b, y, residual=None, total=None, mean=None, rstd=None, eps: float = 1e-5,
               stream=None) -> None:
    """Layer norm over the last axis of ``x`` (``lh_layer_norm``), of ``x + residual``
    where a residual is given; ``total`` receives that sum (it may be ``x`` or
    ``residual`` itself).  ``mean``, ``rstd``: float32, one per row, for the gradient.
    ``w``, ``b``: float32 ``[D]`` (``b`` may be None)."""
    torch = _torch_loaded()
    shape, D = x.shape, x.shape[-1]
    rows = x.numel() // D if D else 0
    _need(x, "x", x.dtype, shape)
    _need(w, "w", torch.float32, (D,))
    if b is not None:
        _need(b, "b", torch.float32, (D,))
    _need(y, "y", x.dtype, shape)
    for name, t in (("residual", residual), ("total", total)):
        if t is not None:
            _need(t, name, x.dtype, shape)
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t is not None:
            _need(t, name, torch.float32, shape[:-1])
    _check(lib().lh_layer_norm(x.data_ptr(), _ptr(residual), w.data_ptr(), _ptr(b), rows, D, eps,
                               _io_dtype(x), y.data_ptr(), _ptr(total), _ptr(mean), _ptr(rstd),
                               _handle(x, stream)))


def layer_norm_backward_workspace_bytes(rows: int, D: int) -> int:
    return _block_bytes("lh_layer_norm_backward_workspace_bytes", rows, D)


def layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db=None, dtotal=None, workspace=None,
                        stream=None) -> None:
    """Gradients of ``layer_norm`` (``lh_layer_norm_backward``): ``x`` is what was
    normalised (the total), ``dtotal`` the gradient that reaches it from elsewhere,
    which is added to ``dx`` (and may be ``dx`` itself)."""
    torch = _torch_loaded()
    shape, D = x.shape, x.shape[-1]
    rows = x.numel() // D if D else 0
    _need(x, "x", x.dtype, shape)
    _need(dy, "dy", x.dtype, shape)
    _need(dx, "dx", x.dtype, shape)
    if dtotal is not None:
        _need(dtotal, "dtotal", x.dtype, shape)
    _need(w, "w", torch.float32, (D,))
    _need(dw, "dw", torch.float32, (D,))
    if db is not None:
        _need(db, "db", torch.float32, (D,))
    _need(mean, "mean", torch.float32, shape[:-1])
    _need(rstd, "rstd", torch.float32, shape[:-1])
    handle = _handle(x, stream)
    workspace, ws_ptr, ws_len = _scratch(layer_norm_backward_workspace_bytes(rows, D), workspace,
                                         x.device, stream)
    _check(lib().lh_layer_norm_backward(dy.data_ptr(), x.data_ptr(), w.data_ptr(), mean.data_ptr(),
                                        rstd.data_ptr(), _ptr(dtotal), rows, D, _io_dtype(x),
                                        dx.data_ptr(), dw.data_ptr(), _ptr(db), ws_ptr, ws_len,
                                        handle))


def _conv_args(x, w, bias, lead):
    torch = _torch_loaded()
    D, K = w.shape
    ld = _need_rows(x, "x", x.dtype, (*lead, D), len(lead), D)
    _need(w, "w", torch.float32, (D, K))
    if bias is not None:
        _need(bias, "bias", torch.float32, (D,))
    return ld, D, K, _io_dtype(x)


def _conv_state(state, dtype, B, K, D):
    """Pointer of the state ``[B, K - 1, D]``; None is no state, which one tap leaves."""
    if state is None and K == 1:
        return None
    _need(state, "state", dtype, (B, K - 1, D))
    return state.data_ptr()


def short_conv_prefill(x, w, bias, state, y, silu: bool = True, lengths=None, resume: bool = False,
                       stream=None) -> None:
    """Short causal convolution of the prompt ``x [B, T, D]`` with the taps ``w [D, K]``
    (``lh_short_conv_prefill``); ``state [B, K - 1, D]`` receives the last inputs, and is
    what the prompt continues from where ``resume`` (None is taken with one tap).  ``x`` may
    be a slice of rows."""
    B, T = x.shape[:2]
    ld, D, K, io = _conv_args(x, w, bias, (B, T))
    state_ptr = _conv_state(state, x.dtype, B, K, D)
    _need(y, "y", x.dtype, (B, T, D))
    _need_lengths(lengths, B)
    _check(lib().lh_short_conv_prefill(x.data_ptr(), ld, w.data_ptr(), _ptr(bias), _ptr(lengths), B,
                                       T, D, K, io, silu, resume, state_ptr, y.data_ptr(),
                                       _handle(x, stream)))


def short_conv_step(x_t, w, bias, state, y_t, silu: bool = True, stream=None) -> None:
    """One token per row, ``x_t``, ``y_t`` ``[B, D]``, ``state`` in place (None is taken with
    one tap) (``lh_short_conv_step``)."""
    B = x_t.shape[0]
    ld, D, K, io = _conv_args(x_t, w, bias, (B,))
    state_ptr = _conv_state(state, x_t.dtype, B, K, D)
    _need(y_t, "y_t", x_t.dtype, (B, D))
    _check(lib().lh_short_conv_step(x_t.data_ptr(), ld, w.data_ptr(), _ptr(bias), B, D, K, io, silu,
                                    state_ptr, y_t.data_ptr(), _handle(x_t, stream)))


def short_conv_backward_workspace_bytes(B: int, T: int, D: int, K: int) -> int:
    return _block_bytes("lh_short_conv_backward_workspace_bytes", B, T, D, K)


def short_conv_backward(dy, x, w, bias, dx, dw, dbias=None, silu: bool = True, lengths=None,
                        workspace=None, stream=None) -> None:
    """Gradients of ``short_conv_prefill`` from zero inputs before the prompt
    (``lh_short_conv_backward``)."""
    torch = _torch_loaded()
    B, T = x.shape[:2]
    ld, D, K, io = _conv_args(x, w, bias, (B, T))
    _need(dy, "dy", x.dtype, (B, T, D))
    _need(dx, "dx", x.dtype, (B, T, D))
    _need(dw, "dw", torch.float32, (D, K))
    if dbias is not None:
        _need(dbias, "dbias", torch.float32, (D,))
    _need_lengths(lengths, B)
    handle = _handle(x, stream)
    workspace, ws_ptr, ws_len = _scratch(short_conv_backward_workspace_bytes(B, T, D, K), workspace,
                                         x.device, stream)
    _check(lib().lh_short_conv_backward(dy.data_ptr(), x.data_ptr(), ld, w.data_ptr(), _ptr(bias),
                                        _ptr(lengths), B, T, D, K, io, silu, dx.data_ptr(),
                                        dw.data_ptr(), _ptr(dbias), ws_ptr, ws_len, handle))


def _selective_args(A, dt, Bm, Cm, u, h0, dt_bias, z, lengths, lead):
    torch = _torch_loaded()
    D, N = A.shape
    G = Bm.shape[-2]
    dtype, k = u.dtype, len(lead)
    rows, sel = (*lead, D), (*lead, G, N)
    _need(A, "A", torch.float32, (D, N))
    ld_dt = _need_rows(dt, "dt", dtype, rows, k, D)
    ld_u = _need_rows(u, "u", dtype, rows, k, D)
    ld_B = _need_rows(Bm, "Bm", dtype, sel, k, G * N)
    ld_C = _need_rows(Cm, "Cm", dtype, sel, k, G * N)
    ld_z = pz = pb = ph = pl = None
    if z is not None:
        ld_z, pz = _need_rows(z, "z", dtype, rows, k, D), z.data_ptr()
    if dt_bias is not None:
        _need(dt_bias, "dt_bias", torch.float32, (D,))
        pb = dt_bias.data_ptr()
    if h0 is not None:
        _need(h0, "h0", torch.float32, (D,))
        ph = h0.data_ptr()
    if lengths is not None:
        _need_lengths(lengths, lead[0])
        pl = lengths.data_ptr()
    return _SelectiveInputs(A.data_ptr(), pb, ph, dt.data_ptr(), u.data_ptr(), pz, Bm.data_ptr(), Cm.data_ptr(), pl,
                            ld_dt, ld_u, ld_z or 0, ld_B, ld_C, lead[0], lead[1] if k > 1 else 1, D, N, G,
                            _io_dtype(u))


def selective_workspace_bytes(B: int, T: int, D: int, N: int, G: int = 1) -> int:
    return _block_bytes("lh_selective_workspace_bytes", B, T, D, N, G)


def selective_prefill(A, dt, Bm, Cm, u, state, y, h0=None, dt_bias=None, z=None, lengths=None,
                      resume: bool = False, workspace=None, stream=None) -> None:
    """Selective scan of a prompt (``lh_selective_prefill``): ``dt``, ``u``, ``z``
    ``[B, T, D]``, ``Bm``, ``Cm`` ``[B, T, G, N]`` (all may be slices of rows), ``A [D, N]``,
    ``h0``, ``dt_bias`` ``[D]`` and ``state [B, D, N]`` float32; writes ``y [B, T, D]`` and the
    state, which the prompt continues from where ``resume``."""
    B, T = u.shape[:2]
    s = _selective_args(A, dt, Bm, Cm, u, h0, dt_bias, z, lengths, (B, T))
    _need(state, "state", _torch.float32, (B, s.D, s.N))
    _need(y, "y", u.dtype, (B, T, s.D))
    handle = _handle(u, stream)
    workspace, ws_ptr, ws_len = _scratch(selective_workspace_bytes(B, T, s.D, s.N, s.G), workspace,
                                         u.device, stream)
    _check(lib().lh_selective_prefill(ctypes.byref(s), resume, state.data_ptr(), y.data_ptr(), ws_ptr,
                                      ws_len, handle))


def selective_step(A, dt_t, Bm_t, Cm_t, u_t, state, y_t, h0=None, dt_bias=None, z=None,
                   stream=None) -> None:
    """One token per row (``lh_selective_step``): ``dt_t``, ``u_t``, ``z`` ``[B, D]``,
    ``Bm_t``, ``Cm_t`` ``[B, G, N]``, ``state`` in place."""
    B = u_t.shape[0]
    s = _selective_args(A, dt_t, Bm_t, Cm_t, u_t, h0, dt_bias, z, None, (B,))
    _need(state, "state", _torch.float32, (B, s.D, s.N))
    _need(y_t, "y_t", u_t.dtype, (B, s.D))
    _check(lib().lh_selective_step(ctypes.byref(s), state.data_ptr(), y_t.data_ptr(),
                                   _handle(u_t, stream)))


def selective_backward_workspace_bytes(B: int, T: int, D: int, N: int, G: int = 1) -> int:
    return _block_bytes("lh_selective_backward_workspace_bytes", B, T, D, N, G)


def selective_backward(dy, A, dt, Bm, Cm, u, dA, ddt, dBm, dCm, du, h0=None, dh0=None, dt_bias=None,
                       ddt_bias=None, z=None, dz=None, lengths=None, workspace=None,
                       stream=None) -> None:
    """Gradients of ``selective_prefill`` from a zero state (``lh_selective_backward``),
    from its inputs and ``dy [B, T, D]``."""
    torch = _torch_loaded()
    B, T = u.shape[:2]
    s = _selective_args(A, dt, Bm, Cm, u, h0, dt_bias, z, lengths, (B, T))
    D, N, G = s.D, s.N, s.G
    g = _SelectiveGrads()
    for name, t, dtype, shape in (
            ("dy", dy, u.dtype, (B, T, D)), ("ddt", ddt, u.dtype, (B, T, D)), ("du", du, u.dtype, (B, T, D)),
            ("dz", dz, u.dtype, (B, T, D)), ("dBm", dBm, u.dtype, (B, T, G, N)),
            ("dCm", dCm, u.dtype, (B, T, G, N)), ("dA", dA, torch.float32, (D, N)),
            ("dh0", dh0, torch.float32, (D,)), ("ddt_bias", ddt_bias, torch.float32, (D,))):
        if t is not None:
            _need(t, name, dtype, shape)
            setattr(g, name, t.data_ptr())
        elif name not in ("dz", "dh0", "ddt_bias"):
            raise TypeError(f"{name} must be a torch.Tensor")
    handle = _handle(u, stream)
    workspace, ws_ptr, ws_len = _scratch(selective_backward_workspace_bytes(B, T, D, N, G), workspace,
                                         u.device, stream)
    _check(lib().lh_selective_backward(ctypes.byref(s), ctypes.byref(g), ws_ptr, ws_len, handle))


# ---- the gated recurrence

def _gated_args(rate, r, i, u, r_bias, i_bias, z, lengths, lead):
    torch = _torch_loaded()
    D, = rate.shape
    dtype, k, rows = u.dtype, len(lead), (*lead, D)
    _need(rate, "rate", torch.float32, (D,))
    ld_r = _need_rows(r, "r", dtype, rows, k, D)
    ld_i = _need_rows(i, "i", dtype, rows, k, D)
    ld_u = _need_rows(u, "u", dtype, rows, k, D)
    ld_z = pz = pr = pi = pl = None
    if z is not None:
        ld_z, pz = _need_rows(z, "z", dtype, rows, k, D), z.data_ptr()
    if r_bias is not None:
        _need(r_bias, "r_bias", torch.float32, (D,))
        pr = r_bias.data_ptr()
    if i_bias is not None:
        _need(i_bias, "i_bias", torch.float32, (D,))
        pi = i_bias.data_ptr()
    if lengths is not None:
        _need_lengths(lengths, lead[0])
        pl = lengths.data_ptr()
    return _GatedInputs(rate.data_ptr(), pr, pi, r.data_ptr(), i.data_ptr(), u.data_ptr(), pz, pl, ld_r, ld_i, ld_u,
                        ld_z or 0, lead[0], lead[1] if k > 1 else 1, D, _io_dtype(u))


def gated_workspace_bytes(B: int, T: int, D: int) -> int:
    return _block_bytes("lh_gated_workspace_bytes", B, T, D)


def gated_prefill(rate, r, i, u, state, y, r_bias=None, i_bias=None, z=None, lengths=None, resume: bool = False,
                  marks=None, workspace=None, stream=None) -> None:
    """Gated linear recurrence over a prompt (``lh_gated_prefill``): ``r``, ``i``, ``u``, ``z``
    ``[B, T, D]`` (all may be slices of rows), ``rate``, ``r_bias``, ``i_bias`` ``[D]`` and
    ``state [B, D]`` float32; writes ``y [B, T, D]`` and the state, which the prompt continues
    from where ``resume``.  ``marks [B, ceil(T / GATED_MARK), D]`` float32 receives the states
    that ``gated_backward`` takes."""
    B, T = u.shape[:2]
    s = _gated_args(rate, r, i, u, r_bias, i_bias, z, lengths, (B, T))
    _need(state, "state", _torch.float32, (B, s.D))
    _need(y, "y", u.dtype, (B, T, s.D))
    if marks is not None:
        _need(marks, "marks", _torch.float32, (B, -(-T // GATED_MARK), s.D))
    handle = _handle(u, stream)
    workspace, ws_ptr, ws_len = _scratch(gated_workspace_bytes(B, T, s.D), workspace, u.device, stream)
    _check(lib().lh_gated_prefill(ctypes.byref(s), resume, state.data_ptr(), y.data_ptr(), _ptr(marks), ws_ptr, ws_len,
                                  handle))


def gated_step(rate, r_t, i_t, u_t, state, y_t, r_bias=None, i_bias=None, z=None, stream=None) -> None:
    """One token per row (``lh_gated_step``): ``r_t``, ``i_t``, ``u_t``, ``z``, ``y_t`` ``[B, D]``,
    ``state`` in place."""
    B = u_t.shape[0]
    s = _gated_args(rate, r_t, i_t, u_t, r_bias, i_bias, z, None, (B,))
    _need(state, "state", _torch.float32, (B, s.D))
    _need(y_t, "y_t", u_t.dtype, (B, s.D))
    _check(lib().lh_gated_step(ctypes.byref(s), state.data_ptr(), y_t.data_ptr(), _handle(u_t, stream)))


def gated_backward_workspace_bytes(B: int, T: int, D: int) -> int:
    return _block_bytes("lh_gated_backward_workspace_bytes", B, T, D)


def gated_backward(dy, rate, r, i, u, marks, drate, dr, di, du, r_bias=None, dr_bias=None, i_bias=None, di_bias=None,
                   z=None, dz=None, lengths=None, dlast=None, dfirst=None, workspace=None, stream=None) -> None:
    """Gradients of ``gated_prefill`` (``lh_gated_backward``) from its inputs, the ``marks`` it
    left and ``dy [B, T, D]``.  ``dlast [B, D]`` is the gradient of the state after the prompt
    (None: 0), ``dfirst [B, D]`` receives that of the state before it."""
    torch = _torch_loaded()
    B, T = u.shape[:2]
    s = _gated_args(rate, r, i, u, r_bias, i_bias, z, lengths, (B, T))
    D, g, f32 = s.D, _GatedGrads(), torch.float32
    for name, t, dtype, shape in (
            ("dy", dy, u.dtype, (B, T, D)), ("marks", marks, f32, (B, -(-T // GATED_MARK), D)),
            ("dlast", dlast, f32, (B, D)), ("dr", dr, u.dtype, (B, T, D)), ("di", di, u.dtype, (B, T, D)),
            ("du", du, u.dtype, (B, T, D)), ("dz", dz, u.dtype, (B, T, D)), ("drate", drate, f32, (D,)),
            ("dr_bias", dr_bias, f32, (D,)), ("di_bias", di_bias, f32, (D,)), ("dfirst", dfirst, f32, (B, D))):
        if t is not None:
            _need(t, name, dtype, shape)
            setattr(g, name, t.data_ptr())
        elif name in ("dy", "marks", "dr", "di", "du", "drate"):
            raise TypeError(f"{name} must be a torch.Tensor")
    handle = _handle(u, stream)
    workspace, ws_ptr, ws_len = _scratch(gated_backward_workspace_bytes(B, T, D), workspace, u.device, stream)
    _check(lib().lh_gated_backward(ctypes.byref(s), ctypes.byref(g), ws_ptr, ws_len, handle))


# ---- the ends of a language model

def embed(W, ids, y, scale: float = 1.0, stream=None) -> None:
    """Rows of the table ``W [V, D]`` times ``scale`` (``lh_embed``): ``y [*ids.shape, D]`` for
    int32 ``ids``; zeros where an id is outside the table.  ``W`` and ``y`` may differ in type."""
    torch = _torch_loaded()
    V, D = W.shape
    _need(W, "W", W.dtype, (V, D))
    _need(ids, "ids", torch.int32, ids.shape)
    _need(y, "y", y.dtype, (*ids.shape, D))
    _check(lib().lh_embed(W.data_ptr(), ids.data_ptr(), ids.numel(), V, D, _io_dtype(W), _io_dtype(y), scale,
                          y.data_ptr(), _handle(y, stream)))


def embed_backward_workspace_bytes(n: int, V: int, D: int) -> int:
    return _block_bytes("lh_embed_backward_workspace_bytes", n, V, D)


def embed_backward(dy, ids, dW, scale: float = 1.0, accumulate: bool = False, workspace=None, stream=None) -> None:
    """Gradient of ``embed`` (``lh_embed_backward``): ``dW [V, D]`` float32, written, or added to
    where ``accumulate``, from ``dy [*ids.shape, D]``."""
    torch = _torch_loaded()
    V, D = dW.shape
    _need(dW, "dW", torch.float32, (V, D))
    _need(ids, "ids", torch.int32, ids.shape)
    _need(dy, "dy", dy.dtype, (*ids.shape, D))
    n = ids.numel()
    handle = _handle(dy, stream)
    workspace, ws_ptr, ws_len = _scratch(embed_backward_workspace_bytes(n, V, D), workspace, dy.device, stream)
    _check(lib().lh_embed_backward(dy.data_ptr(), ids.data_ptr(), n, V, D, _io_dtype(dy), scale, accumulate,
                                   dW.data_ptr(), ws_ptr, ws_len, handle))


def _distill_args(logits, values, ids, scale, dlogits):
    torch = _torch_loaded()
    rows, V = logits.shape
    K = values.shape[-1]
    ld = _need_rows(logits, "logits", logits.dtype, (rows, V), 1, V)
    _need(values, "values", torch.float32, (rows, K))
    _need(ids, "ids", torch.int32, (rows, K))
    if scale is not None:
        _need(scale, "scale", torch.float32, (rows,))
    ld_d = 0 if dlogits is None else _need_rows(dlogits, "dlogits", logits.dtype, (rows, V), 1, V)
    return rows, V, K, ld, ld_d, _io_dtype(logits)


def distill_logits_workspace_bytes(rows: int, V: int, K: int) -> int:
    return _block_bytes("lh_distill_logits_workspace_bytes", rows, V, K)


def distill_logits(logits, values, ids, loss, dlogits=None, lse=None, scale=None, tau: float = 1.0, workspace=None,
                   stream=None) -> None:
    """Distillation from a teacher's top logits (``lh_distill_logits``): ``values``, ``ids``
    ``[rows, K]`` float32 and int32, ``logits [rows, V]`` (rows may lie apart); writes
    ``loss [rows]``, where given the gradient ``dlogits`` of the losses' sum (it may be
    ``logits`` itself) and ``lse [rows]``, which ``distill_logits_backward`` takes.  ``scale
    [rows]`` multiplies each row's loss; rows of scale 0 take no part."""
    rows, V, K, ld, ld_d, io = _distill_args(logits, values, ids, scale, dlogits)
    for name, t in (("loss", loss), ("lse", lse)):
        if t is not None or name == "loss":
            _need(t, name, _torch.float32, (rows,))
    handle = _handle(logits, stream)
    workspace, ws_ptr, ws_len = _scratch(distill_logits_workspace_bytes(rows, V, K), workspace, logits.device, stream)
    _check(lib().lh_distill_logits(logits.data_ptr(), ld, values.data_ptr(), ids.data_ptr(), _ptr(scale), rows, V, K, io,
                                   tau, loss.data_ptr(), _ptr(lse), _ptr(dlogits), ld_d, ws_ptr, ws_len, handle))


def distill_logits_backward(dloss, logits, values, ids, lse, dlogits, scale=None, tau: float = 1.0, stream=None) -> None:
    """Gradient of ``distill_logits`` for an upstream gradient ``dloss [rows]`` of its losses
    (``lh_distill_logits_backward``)."""
    if dlogits is None:
        raise TypeError("dlogits must be a torch.Tensor")
    rows, V, K, ld, ld_d, io = _distill_args(logits, values, ids, scale, dlogits)
    _need(dloss, "dloss", _torch.float32, (rows,))
    _need(lse, "lse", _torch.float32, (rows,))
    _check(lib().lh_distill_logits_backward(dloss.data_ptr(), logits.data_ptr(), ld, values.data_ptr(), ids.data_ptr(),
                                            _ptr(scale), lse.data_ptr(), rows, V, K, io, tau, dlogits.data_ptr(), ld_d,
                                            _handle(logits, stream)))


def verify_draft_workspace_bytes(B: int, K: int, V: int) -> int:
    return _block_bytes("lh_verify_draft_workspace_bytes", B, K, V)


def verify_draft(drafted, target_p, u, u_last, accepted, tokens, draft_p=None, lengths=None, workspace=None,
                 stream=None) -> None:
    """Verification of drafted tokens (``lh_verify_draft``): ``drafted [B, K]`` int32 against
    ``target_p [B, K + 1, V]``, with the draft's own probabilities ``draft_p [B, K, V]`` (None: it
    was certain; rows of both may lie apart) and random numbers ``u [B, K]``, ``u_last [B]`` in
    [0, 1); writes ``accepted [B]`` and ``tokens [B, K + 1]`` (the accepted, the next, then -1)."""
    torch = _torch_loaded()
    B, K = drafted.shape
    V, dtype, i32, f32 = target_p.shape[-1], target_p.dtype, torch.int32, torch.float32
    _need(drafted, "drafted", i32, (B, K))
    ld_t = _need_rows(target_p, "target_p", dtype, (B, K + 1, V), 2, V)
    ld_d = 0 if draft_p is None else _need_rows(draft_p, "draft_p", dtype, (B, K, V), 2, V)
    _need_lengths(lengths, B)
    for name, t, want, shape in (("u", u, f32, (B, K)), ("u_last", u_last, f32, (B,)), ("accepted", accepted, i32, (B,)),
                                 ("tokens", tokens, i32, (B, K + 1))):
        _need(t, name, want, shape)
    handle = _handle(target_p, stream)
    workspace, ws_ptr, ws_len = _scratch(verify_draft_workspace_bytes(B, K, V), workspace, target_p.device, stream)
    _check(lib().lh_verify_draft(drafted.data_ptr(), _ptr(lengths), _ptr(draft_p), ld_d, target_p.data_ptr(), ld_t,
                                 u.data_ptr(), u_last.data_ptr(), B, K, V, _io_dtype(target_p), accepted.data_ptr(),
                                 tokens.data_ptr(), ws_ptr, ws_len, handle))
