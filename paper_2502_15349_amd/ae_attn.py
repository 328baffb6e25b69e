"""ctypes binding of libae_attn.so: argument marshalling only.

Names mirror the C ABI (include/ae_attn.h): ae_attn_create, ae_attn_forward,
ae_attn_destroy, ae_attn_query.  Every step of the attention path runs in the
HIP kernels; PyTorch supplies device memory and the stream, nothing else.
Importing this module fails if the library has not been built
(`python -m paper_2502_15349_amd.build`): there is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Optional, Sequence

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libae_attn.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(
        f"{_LIB_PATH} is missing: build it with `python -m paper_2502_15349_amd.build` "
        "(the HIP library is the only implementation; there is no fallback)")
_lib = C.CDLL(_LIB_PATH)

AE_OK, AE_ERR_INVALID_ARG, AE_ERR_UNSUPPORTED, AE_ERR_HIP, AE_ERR_NOMEM = range(5)
SCORE_MODS = {"none": 0, "bias": 1, "head_decay": 2, "relu": 3, "bias_tensor": 4}
NORMS = {"softmax": 0, "sigmoid": 1, "abssum": 2, "abs_of_sum": 3, "none": 4}
MASKS = {"none": 0, "causal": 1, "sliding_window": 2}
OUT_DTYPES = {"f32": 0, "bf16": 1}


class ae_attn_desc_t(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("H_q", C.c_int32), ("H_kv", C.c_int32), ("L_q", C.c_int32),
        ("L_k", C.c_int32), ("D_qk", C.c_int32), ("D_v", C.c_int32),
        ("score_mod", C.c_int), ("bias", C.c_float), ("gamma", C.POINTER(C.c_float)),
        ("norm", C.c_int), ("mask", C.c_int), ("scale", C.c_float), ("out_dtype", C.c_int),
        ("window", C.c_int32), ("kv_splits", C.c_int32),
        ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3),
        ("v_stride", C.c_int64 * 3), ("o_stride", C.c_int64 * 3),
        ("bias_stride", C.c_int64 * 3),
    ]


_lib.ae_attn_create.argtypes = [C.POINTER(ae_attn_desc_t), C.POINTER(C.c_void_p)]
_lib.ae_attn_create.restype = C.c_int
_lib.ae_attn_forward.argtypes = [C.c_void_p] * 6
_lib.ae_attn_forward.restype = C.c_int
_lib.ae_attn_forward_stats.argtypes = [C.c_void_p] * 7
_lib.ae_attn_forward_stats.restype = C.c_int
_lib.ae_attn_forward_bias.argtypes = [C.c_void_p] * 8
_lib.ae_attn_forward_bias.restype = C.c_int
_lib.ae_attn_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
_lib.ae_attn_workspace_bytes.restype = C.c_int
_lib.ae_attn_forward_split.argtypes = [C.c_void_p] * 7 + [C.c_size_t, C.c_void_p]
_lib.ae_attn_forward_split.restype = C.c_int
_lib.ae_attn_forward_split_static.argtypes = [C.c_void_p] * 7
_lib.ae_attn_forward_split_static.restype = C.c_int
_lib.ae_attn_backward_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
_lib.ae_attn_backward_workspace_bytes.restype = C.c_int
_lib.ae_attn_backward.argtypes = [C.c_void_p] * 11 + [C.c_size_t, C.c_void_p]
_lib.ae_attn_backward.restype = C.c_int
_lib.ae_attn_backward_bias.argtypes = [C.c_void_p] * 12 + [C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
_lib.ae_attn_backward_bias.restype = C.c_int


class ae_recurrent_desc_t(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("L", C.c_int32), ("D_qk", C.c_int32), ("D_v", C.c_int32),
                ("chunk", C.c_int32), ("scale", C.c_float), ("gamma", C.POINTER(C.c_float)), ("out_dtype", C.c_int)]


_lib.ae_recurrent_create.argtypes = [C.POINTER(ae_recurrent_desc_t), C.POINTER(C.c_void_p)]
_lib.ae_recurrent_create.restype = C.c_int
_lib.ae_recurrent_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
_lib.ae_recurrent_workspace_bytes.restype = C.c_int
_lib.ae_recurrent_forward.argtypes = [C.c_void_p] * 6 + [C.c_size_t, C.c_void_p]
_lib.ae_recurrent_forward.restype = C.c_int
_lib.ae_recurrent_forward_state.argtypes = [C.c_void_p] * 8 + [C.c_size_t, C.c_void_p]
_lib.ae_recurrent_forward_state.restype = C.c_int
_lib.ae_recurrent_step.argtypes = [C.c_void_p] * 7
_lib.ae_recurrent_step.restype = C.c_int
_lib.ae_recurrent_destroy.argtypes = [C.c_void_p]
_lib.ae_recurrent_destroy.restype = C.c_int
_lib.ae_attn_destroy.argtypes = [C.c_void_p]
_lib.ae_attn_destroy.restype = C.c_int
_lib.ae_attn_query.argtypes = [C.c_void_p] + [C.POINTER(C.c_int32)] * 5
_lib.ae_attn_query.restype = C.c_int
_lib.ae_attn_kernel_name.argtypes = [C.c_void_p]
_lib.ae_attn_kernel_name.restype = C.c_char_p
_lib.ae_calib_mfma_bf16.argtypes = [C.c_void_p, C.c_size_t, C.c_int32, C.c_int32, C.POINTER(C.c_double), C.c_void_p]
_lib.ae_calib_mfma_bf16.restype = C.c_int
_lib.ae_attn_last_error.argtypes = []
_lib.ae_attn_last_error.restype = C.c_char_p
_lib.ae_attn_version.argtypes = []
_lib.ae_attn_version.restype = C.c_int32


class AeAttnError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"ae_attn status {status}: {message}")
        self.status = status


def ae_attn_last_error() -> str:
    return _lib.ae_attn_last_error().decode()


def ae_attn_version() -> int:
    return int(_lib.ae_attn_version())


def _check(status: int) -> None:
    if status != AE_OK:
        raise AeAttnError(status, ae_attn_last_error())


def ae_attn_create(*, B: int, H_q: int, H_kv: int, L_q: int, L_k: int, D_qk: int, D_v: int,
                   scale: float, score_mod="none", bias: float = 0.0,
                   gamma: Optional[Sequence[float]] = None, norm="softmax", mask="none",
                   q_stride=(0, 0, 0), k_stride=(0, 0, 0), v_stride=(0, 0, 0), o_stride=(0, 0, 0),
                   out_dtype="f32", window: int = 0, kv_splits: int = 0, bias_stride=(0, 0, 0)) -> int:
    """Returns an opaque handle (int).  Enum arguments accept names or raw ints."""
    d = ae_attn_desc_t()
    d.B, d.H_q, d.H_kv, d.L_q, d.L_k, d.D_qk, d.D_v = B, H_q, H_kv, L_q, L_k, D_qk, D_v
    d.score_mod = SCORE_MODS[score_mod] if isinstance(score_mod, str) else int(score_mod)
    d.norm = NORMS[norm] if isinstance(norm, str) else int(norm)
    d.mask = MASKS[mask] if isinstance(mask, str) else int(mask)
    d.bias, d.scale = float(bias), float(scale)
    d.out_dtype = OUT_DTYPES[out_dtype] if isinstance(out_dtype, str) else int(out_dtype)
    d.window = int(window)
    d.kv_splits = int(kv_splits)
    keep = None
    if gamma is not None:
        keep = (C.c_float * len(gamma))(*[float(x) for x in gamma])
        d.gamma = C.cast(keep, C.POINTER(C.c_float))
    for name, val in (("q_stride", q_stride), ("k_stride", k_stride), ("v_stride", v_stride), ("o_stride", o_stride),
                      ("bias_stride", bias_stride)):
        setattr(d, name, (C.c_int64 * 3)(*[int(x) for x in val]))
    h = C.c_void_p()
    _check(_lib.ae_attn_create(C.byref(d), C.byref(h)))
    return h.value


def ae_attn_workspace_bytes(handle: int) -> int:
    n = C.c_size_t(0)
    _check(_lib.ae_attn_workspace_bytes(handle, C.byref(n)))
    return int(n.value)


def ae_attn_forward_split(handle: int, Q: int, K: int, V: int, O: int, stats: int, workspace: int,
                          workspace_bytes: int, stream: int = 0) -> None:
    """Forward of a handle created with kv_splits > 1; stats may be 0 (not written)."""
    _check(_lib.ae_attn_forward_split(handle, Q, K, V, O, stats, workspace, workspace_bytes, stream))


def ae_attn_forward_split_static(handle: int, Q: int, K: int, V: int, O: int, stats: int = 0, stream: int = 0) -> None:
    """ae_attn_forward_split with the partial results in the library's static device scratch (no workspace, no allocation)."""
    _check(_lib.ae_attn_forward_split_static(handle, Q, K, V, O, stats, stream))


AE_ATTN_STATIC_SCRATCH_BYTES = 4 << 20


def ae_attn_backward_workspace_bytes(handle: int) -> int:
    """Bytes of device workspace ae_attn_backward needs for this handle."""
    n = C.c_size_t(0)
    _check(_lib.ae_attn_backward_workspace_bytes(handle, C.byref(n)))
    return int(n.value)


def ae_attn_backward(handle: int, Q: int, K: int, V: int, O: int, dO: int, stats: int, dQ: int, dK: int, dV: int,
                     workspace: int, workspace_bytes: int, stream: int = 0) -> None:
    """Device addresses throughout: dQ, dK, dV (fp32, contiguous) receive the gradients for the upstream
    gradient dO (bf16, contiguous); O and stats are what ae_attn_forward_stats wrote."""
    _check(_lib.ae_attn_backward(handle, Q, K, V, O, dO, stats, dQ, dK, dV, workspace, workspace_bytes, stream))


def ae_attn_backward_bias(handle: int, Q: int, K: int, V: int, bias: int, O: int, dO: int, stats: int, dQ: int, dK: int,
                          dV: int, dBias: int, dbias_row_stride: int, workspace: int, workspace_bytes: int,
                          stream: int = 0) -> None:
    """ae_attn_backward for a handle created with score_mod "bias_tensor" (bias: device address of the tensor; dBias:
    0, or the address of a zero-filled bf16 buffer [B, H_q, L_q, dbias_row_stride] for the bias gradient)."""
    _check(_lib.ae_attn_backward_bias(handle, Q, K, V, bias, O, dO, stats, dQ, dK, dV, dBias, dbias_row_stride, workspace,
                                      workspace_bytes, stream))


def ae_attn_forward_bias(handle: int, Q: int, K: int, V: int, bias: int, O: int, stats: int = 0, stream: int = 0) -> None:
    """Forward of a handle created with score_mod "bias_tensor"; bias is the device address of the bf16 bias tensor,
    stats may be 0 (not written)."""
    _check(_lib.ae_attn_forward_bias(handle, Q, K, V, bias, O, stats, stream))


def ae_attn_forward_stats(handle: int, Q: int, K: int, V: int, O: int, stats: int, stream: int = 0) -> None:
    """ae_attn_forward that also writes the row statistic (fp32 [B, H_q, L_q]) to `stats`."""
    _check(_lib.ae_attn_forward_stats(handle, Q, K, V, O, stats, stream))


def ae_attn_forward(handle: int, Q: int, K: int, V: int, O: int, stream: int = 0) -> None:
    """Q, K, V, O are device addresses (tensor.data_ptr()); stream is a raw hipStream_t."""
    _check(_lib.ae_attn_forward(handle, Q, K, V, O, stream))


def ae_calib_mfma_bf16(sink: int, sink_bytes: int, workgroups: int, iters: int, stream: int = 0) -> float:
    """Enqueues the pure-MFMA calibration kernel; returns the flop it performs."""
    flop = C.c_double(0.0)
    _check(_lib.ae_calib_mfma_bf16(sink, sink_bytes, workgroups, iters, C.byref(flop), stream))
    return float(flop.value)


def ae_attn_destroy(handle: Optional[int]) -> None:
    _check(_lib.ae_attn_destroy(handle))


def ae_attn_query(handle: int) -> dict:
    v = [C.c_int32() for _ in range(5)]
    _check(_lib.ae_attn_query(handle, *[C.byref(x) for x in v]))
    keys = ("block_m", "block_n", "lds_bytes", "grid_size", "block_threads")
    out = {k: int(x.value) for k, x in zip(keys, v)}
    out["kernel"] = _lib.ae_attn_kernel_name(handle).decode()
    return out


# ---- convenience for torch callers (still marshalling only) -------------------
def ae_recurrent_create(*, B: int, H: int, L: int, D_qk: int, D_v: int, chunk: int, scale: float,
                        gamma: Optional[Sequence[float]], out_dtype="f32") -> int:
    """Handle for chunk-parallel recurrent retention (h_t = gamma h_{t-1} + k_t^T v_t, o_t = scale q_t h_t)."""
    d = ae_recurrent_desc_t(B=B, H=H, L=L, D_qk=D_qk, D_v=D_v, chunk=chunk, scale=scale,
                            out_dtype=OUT_DTYPES[out_dtype] if isinstance(out_dtype, str) else int(out_dtype))
    keep = None
    if gamma is not None:
        keep = (C.c_float * len(gamma))(*[float(g) for g in gamma])
        d.gamma = C.cast(keep, C.POINTER(C.c_float))
    out = C.c_void_p()
    _check(_lib.ae_recurrent_create(C.byref(d), C.byref(out)))
    return out.value


def ae_recurrent_workspace_bytes(handle: int) -> int:
    n = C.c_size_t()
    _check(_lib.ae_recurrent_workspace_bytes(handle, C.byref(n)))
    return n.value


def ae_recurrent_forward(handle: int, Q: int, K: int, V: int, O: int, workspace: int, workspace_bytes: int,
                         stream: int = 0) -> None:
    _check(_lib.ae_recurrent_forward(handle, Q, K, V, O, workspace, workspace_bytes, stream))


def ae_recurrent_forward_state(handle: int, Q: int, K: int, V: int, h_in: int, O: int, h_out: int, workspace: int,
                               workspace_bytes: int, stream: int = 0) -> None:
    """ae_recurrent_forward with the state in front of the first token (h_in, 0: zero) and the state after the last
    one (h_out, 0: not computed), both fp32 [B, H, D_qk, D_v] device addresses."""
    _check(_lib.ae_recurrent_forward_state(handle, Q, K, V, h_in, O, h_out, workspace, workspace_bytes, stream))


def ae_recurrent_step(handle: int, q: int, k: int, v: int, state: int, o: int, stream: int = 0) -> None:
    """One token: state <- gamma state + k^T v (fp32 [B, H, D_qk, D_v], in place), o = scale q state (fp32 [B, H, D_v])."""
    _check(_lib.ae_recurrent_step(handle, q, k, v, state, o, stream))


def ae_recurrent_destroy(handle: Optional[int]) -> None:
    _check(_lib.ae_recurrent_destroy(handle))


def _memory_of(stream):
    """What a call allocates belongs to the stream that it writes on: memory of another one may still be in use there, or be given away
    there while this one writes it."""
    if stream is None:
        return contextlib.nullcontext()
    import torch

    return torch.cuda.stream(stream)


def retention_recurrent(Q, K, V, *, scale, gamma, chunk=256, out=None, workspace=None, stream=None, h_in=None,
                        return_state=False, out_dtype=None):
    """Recurrent retention on contiguous bf16 device tensors Q, K [B, H, L, D_qk], V [B, H, L, D_v];
    returns O [B, H, L, D_v] fp32 (bf16 with out_dtype=torch.bfloat16 or a bf16 `out`).  workspace: device byte tensor of ae_recurrent_workspace_bytes() bytes
    (allocated here if not given).  h_in: optional contiguous fp32 device tensor [B, H, D_qk, D_v], the state in
    front of the first token; return_state: also return the state after the last token (same layout)."""
    import torch

    for t in (Q, K, V):
        if not t.is_cuda or t.dtype != torch.bfloat16 or t.dim() != 4 or not t.is_contiguous():
            raise ValueError("Q, K, V must be contiguous 4-D bf16 device tensors; there is no CPU path")
    B, H, L, D_qk = Q.shape
    D_v = V.shape[3]
    if K.shape != Q.shape or V.shape[:3] != Q.shape[:3]:
        raise ValueError("K / V shape does not match Q")
    if out is None:
        with _memory_of(stream):
            out = torch.empty((B, H, L, D_v), dtype=out_dtype or torch.float32, device=Q.device)
    if out.dtype not in (torch.float32, torch.bfloat16) or tuple(out.shape) != (B, H, L, D_v) or not out.is_contiguous():
        raise ValueError("O must be a contiguous fp32 or bf16 tensor [B, H, L, D_v]")
    h = ae_recurrent_create(B=B, H=H, L=L, D_qk=D_qk, D_v=D_v, chunk=chunk, scale=scale, gamma=gamma,
                            out_dtype="bf16" if out.dtype == torch.bfloat16 else "f32")
    try:
        s = torch.cuda.current_stream(Q.device) if stream is None else stream
        with torch.cuda.device(Q.device), _memory_of(stream):
            need = ae_recurrent_workspace_bytes(h)
            if workspace is None:
                workspace = torch.empty(need, dtype=torch.uint8, device=Q.device)
            if h_in is not None and (h_in.dtype != torch.float32 or tuple(h_in.shape) != (B, H, D_qk, D_v)
                                     or not h_in.is_contiguous() or not h_in.is_cuda):
                raise ValueError("h_in must be a contiguous fp32 device tensor [B, H, D_qk, D_v]")
            h_out = torch.empty((B, H, D_qk, D_v), dtype=torch.float32, device=Q.device) if return_state else None
            ae_recurrent_forward_state(h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), 0 if h_in is None else h_in.data_ptr(),
                                       out.data_ptr(), 0 if h_out is None else h_out.data_ptr(), workspace.data_ptr(),
                                       workspace.numel(), s.cuda_stream)
    finally:
        ae_recurrent_destroy(h)
    return (out, h_out) if return_state else out


def attention_forward(Q, K, V, *, scale, score_mod="none", bias=0.0, gamma=None, norm="softmax",
                      mask="none", out=None, stream=None, out_dtype=None, stats=None, window=0, kv_splits=0,
                      workspace=None, bias_tensor=None):
    """Runs the HIP operator on CUDA/HIP bf16 tensors laid out [B, H, L, D]
    (last dim contiguous) and returns O [B, H_q, L_q, D_v]: fp32, or bf16 if `out` is a
    bf16 tensor or out_dtype is torch.bfloat16.  stats: optional contiguous fp32 device
    tensor [B, H_q, L_q] that receives the row statistic of the normalization.  window: keys
    per query for mask="sliding_window".  kv_splits > 1: the keys are cut into that many ranges
    (few query rows, many keys); `workspace` is then a device byte tensor of at least
    ae_attn_workspace_bytes() bytes (allocated here if not given).  bias_tensor: for score_mod
    "bias_tensor", a bf16 device tensor [B or 1, H_q or 1, L_q, L_k] (last dimension contiguous)."""
    import torch

    if not (Q.is_cuda and K.is_cuda and V.is_cuda):
        raise ValueError("attention_forward needs device tensors; there is no CPU path")
    for t in (Q, K, V):
        if t.dtype != torch.bfloat16 or t.dim() != 4 or t.stride(3) != 1:
            raise ValueError("Q, K, V must be 4-D bf16 with a contiguous last dimension")
    B, H_q, L_q, D_qk = Q.shape
    _, H_kv, L_k, D_v = V.shape
    if K.shape != (B, H_kv, L_k, D_qk):
        raise ValueError("K shape does not match Q / V")
    if out is None:
        with _memory_of(stream):
            out = torch.empty((B, H_q, L_q, D_v), dtype=out_dtype or torch.float32, device=Q.device)
    if out.dtype not in (torch.float32, torch.bfloat16) or out.stride(3) != 1:
        raise ValueError("O must be fp32 or bf16 with a contiguous last dimension")
    _rows_apart(Q, K, V, out)
    h = ae_attn_create(B=B, H_q=H_q, H_kv=H_kv, L_q=L_q, L_k=L_k, D_qk=D_qk, D_v=D_v, scale=scale,
                       score_mod=score_mod, bias=bias, gamma=gamma, norm=norm, mask=mask,
                       q_stride=Q.stride()[:3], k_stride=K.stride()[:3], v_stride=V.stride()[:3],
                       o_stride=out.stride()[:3], out_dtype="bf16" if out.dtype == torch.bfloat16 else "f32",
                       window=window, kv_splits=kv_splits, bias_stride=_bias_strides(bias_tensor, B, H_q, L_q, L_k))
    try:
        s = torch.cuda.current_stream(Q.device) if stream is None else stream
        with torch.cuda.device(Q.device), _memory_of(stream):
            if stats is not None and (stats.dtype != torch.float32 or tuple(stats.shape) != (B, H_q, L_q)
                                      or not stats.is_contiguous()):
                raise ValueError("stats must be a contiguous fp32 tensor [B, H_q, L_q]")
            need = ae_attn_workspace_bytes(h)
            if bias_tensor is not None:
                ae_attn_forward_bias(h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), bias_tensor.data_ptr(), out.data_ptr(),
                                     0 if stats is None else stats.data_ptr(), s.cuda_stream)
            elif need:
                if workspace is None:
                    workspace = torch.empty(need, dtype=torch.uint8, device=Q.device)
                ae_attn_forward_split(h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(),
                                      0 if stats is None else stats.data_ptr(), workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(), s.cuda_stream)
            elif stats is None:
                ae_attn_forward(h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(), s.cuda_stream)
            else:
                if stats.dtype != torch.float32 or tuple(stats.shape) != (B, H_q, L_q) or not stats.is_contiguous():
                    raise ValueError("stats must be a contiguous fp32 tensor [B, H_q, L_q]")
                ae_attn_forward_stats(h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(), stats.data_ptr(),
                                      s.cuda_stream)
    finally:
        ae_attn_destroy(h)
    return out


def _rows_apart(*tensors):
    """Strides of zero in batch, head and row mean contiguous to the C ABI: a vector expanded over all three must not reach it."""
    for t in tensors:
        if not any(t.stride()[:3]) and t.shape[0] * t.shape[1] * t.shape[2] > 1:
            raise ValueError("Q, K, V and O must not be a vector expanded over batch, heads and rows; make a contiguous copy")


def _bias_strides(bias_tensor, B, H_q, L_q, L_k):
    """Element strides {batch, head, row} of a bias tensor [B or 1, H_q or 1, L_q, L_k]; a dimension of size 1 is
    shared (stride 0)."""
    if bias_tensor is None:
        return (0, 0, 0)
    import torch
    t = bias_tensor
    if (t.dtype != torch.bfloat16 or t.dim() != 4 or t.shape[0] not in (1, B) or t.shape[1] not in (1, H_q)
            or tuple(t.shape[2:]) != (L_q, L_k) or t.stride(3) != 1 or not t.is_cuda):
        raise ValueError("bias_tensor must be a bf16 device tensor [B or 1, H_q or 1, L_q, L_k] with a contiguous last dimension")
    if L_q > 1 and t.stride(2) == 0:
        raise ValueError("the rows of bias_tensor must not be expanded; make a contiguous copy")
    # (a single row's stride is not looked at, but three zeros would mean contiguous)
    row = t.stride(2) or -(-L_k // 8) * 8
    return (0 if t.shape[0] == 1 else t.stride(0), 0 if t.shape[1] == 1 else t.stride(1), row)


def attention_backward(Q, K, V, O, dO, stats, *, scale, score_mod="none", bias=0.0, gamma=None, norm="softmax",
                       mask="none", window=0, stream=None, workspace=None, bias_tensor=None, want_dbias=False):
    """Runs the HIP backward pass on device tensors: Q, K, V bf16 [B, H, L, D] (last dim contiguous), O the
    forward output (fp32 or bf16), dO bf16 contiguous, stats the fp32 row statistic of the forward pass (O and
    stats may be None for sigmoid and no normalization); window: keys per query for mask="sliding_window".  Returns (dQ, dK, dV)
    as contiguous fp32 tensors; with want_dbias also the bias gradient, bf16 [B, H_q, L_q, L_k] (per batch and head)."""
    import torch

    if not (Q.is_cuda and K.is_cuda and V.is_cuda and dO.is_cuda):
        raise ValueError("attention_backward needs device tensors; there is no CPU path")
    B, H_q, L_q, D_qk = Q.shape
    _, H_kv, L_k, D_v = V.shape
    if dO.dtype != torch.bfloat16 or tuple(dO.shape) != (B, H_q, L_q, D_v) or not dO.is_contiguous():
        raise ValueError("dO must be a contiguous bf16 tensor [B, H_q, L_q, D_v]")
    if stats is not None and (stats.dtype != torch.float32 or tuple(stats.shape) != (B, H_q, L_q) or not stats.is_contiguous()):
        raise ValueError("stats must be a contiguous fp32 tensor [B, H_q, L_q]")
    _rows_apart(Q, K, V, *(() if O is None else (O,)))
    o_dtype, o_stride = ("f32", (0, 0, 0)) if O is None else ("bf16" if O.dtype == torch.bfloat16 else "f32", O.stride()[:3])
    h = ae_attn_create(B=B, H_q=H_q, H_kv=H_kv, L_q=L_q, L_k=L_k, D_qk=D_qk, D_v=D_v, scale=scale,
                       score_mod=score_mod, bias=bias, gamma=gamma, norm=norm, mask=mask, q_stride=Q.stride()[:3],
                       k_stride=K.stride()[:3], v_stride=V.stride()[:3], o_stride=o_stride, out_dtype=o_dtype,
                       window=window, bias_stride=_bias_strides(bias_tensor, B, H_q, L_q, L_k))
    try:
        s = torch.cuda.current_stream(Q.device) if stream is None else stream
        with torch.cuda.device(Q.device), _memory_of(stream):
            dQ = torch.empty((B, H_q, L_q, D_qk), dtype=torch.float32, device=Q.device)
            dK = torch.empty((B, H_kv, L_k, D_qk), dtype=torch.float32, device=Q.device)
            dV = torch.empty((B, H_kv, L_k, D_v), dtype=torch.float32, device=Q.device)
            need = ae_attn_backward_workspace_bytes(h)
            if workspace is None:
                workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=Q.device)
            tail = (0 if O is None else O.data_ptr(), dO.data_ptr(), 0 if stats is None else stats.data_ptr(), dQ.data_ptr(),
                    dK.data_ptr(), dV.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                    s.cuda_stream)
            dB = None
            if bias_tensor is not None:
                ld = (L_k + 3) // 4 * 4
                if want_dbias:
                    # (unmasked, every entry is written: clearing it first cost 9 of 72 us at 2 x 12 x 1023 x 1201)
                    make = torch.empty if mask == "none" else torch.zeros
                    dB = make((B, H_q, L_q, ld), dtype=torch.bfloat16, device=Q.device)
                ae_attn_backward_bias(h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), bias_tensor.data_ptr(), *tail[:6],
                                      0 if dB is None else dB.data_ptr(), ld, *tail[6:])
            else:
                ae_attn_backward(h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), *tail)
    finally:
        ae_attn_destroy(h)
    if want_dbias:
        return dQ, dK, dV, dB[..., :L_k]
    return dQ, dK, dV


def run_workload(w, Q, K, V, out=None, out_dtype=None, stats=None, kv_splits=0, bias_tensor=None):
    """attention_forward with the parameters of a workloads.Workload."""
    return attention_forward(Q, K, V, scale=w.scale_value, score_mod=w.score_mod, bias=w.bias,
                             gamma=w.gamma(), norm=w.norm, mask=w.mask, out=out, out_dtype=out_dtype, stats=stats,
                             window=w.window, kv_splits=kv_splits, bias_tensor=bias_tensor)


# ---- recurrent pattern with per-token gates (gated retention, Mamba2 SSM) ------------------------------------
class ae_gated_desc_t(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("H_qk", C.c_int32), ("L", C.c_int32), ("D_qk", C.c_int32),
                ("D_v", C.c_int32), ("scale", C.c_float), ("out_dtype", C.c_int)]


_lib.ae_gated_create.argtypes = [C.POINTER(ae_gated_desc_t), C.POINTER(C.c_void_p)]
_lib.ae_gated_create.restype = C.c_int
_lib.ae_gated_forward.argtypes = [C.c_void_p] * 10
_lib.ae_gated_forward.restype = C.c_int
_lib.ae_gated_destroy.argtypes = [C.c_void_p]
_lib.ae_gated_destroy.restype = C.c_int
_lib.ae_gated_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
_lib.ae_gated_workspace_bytes.restype = C.c_int
_lib.ae_gated_forward_segmented.argtypes = [C.c_void_p] * 10 + [C.c_size_t, C.c_void_p]
_lib.ae_gated_forward_segmented.restype = C.c_int
_lib.ae_gated_backward_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
_lib.ae_gated_backward_workspace_bytes.restype = C.c_int
_lib.ae_gated_backward.argtypes = [C.c_void_p] * 13 + [C.c_size_t, C.c_void_p]
_lib.ae_gated_backward.restype = C.c_int


def ae_gated_create(*, B: int, H: int, L: int, D_qk: int, D_v: int, scale: float, H_qk: Optional[int] = None,
                    out_dtype="f32") -> int:
    d = ae_gated_desc_t()
    d.B, d.H, d.H_qk, d.L, d.D_qk, d.D_v = B, H, H if H_qk is None else H_qk, L, D_qk, D_v
    d.scale = float(scale)
    d.out_dtype = OUT_DTYPES[out_dtype] if isinstance(out_dtype, str) else int(out_dtype)
    h = C.c_void_p()
    _check(_lib.ae_gated_create(C.byref(d), C.byref(h)))
    return h.value


def ae_gated_forward(handle: int, Q: int, K: int, V: int, log_decay: int, key_gate: int, h_in: int, O: int, h_out: int,
                     stream: int = 0) -> None:
    """Device pointers as ints; key_gate, h_in, h_out may be 0."""
    _check(_lib.ae_gated_forward(handle, Q, K, V, log_decay, key_gate, h_in, O, h_out, stream))


def ae_gated_destroy(handle: Optional[int]) -> None:
    _check(_lib.ae_gated_destroy(handle))


def ae_gated_workspace_bytes(handle: int) -> int:
    n = C.c_size_t()
    _check(_lib.ae_gated_workspace_bytes(handle, C.byref(n)))
    return n.value


def ae_gated_forward_segmented(handle: int, Q: int, K: int, V: int, log_decay: int, key_gate: int, h_in: int, O: int, h_out: int,
                               workspace: int, workspace_bytes: int, stream: int = 0) -> None:
    _check(_lib.ae_gated_forward_segmented(handle, Q, K, V, log_decay, key_gate, h_in, O, h_out, workspace, workspace_bytes, stream))


def ae_gated_backward_workspace_bytes(handle: int) -> int:
    n = C.c_size_t()
    _check(_lib.ae_gated_backward_workspace_bytes(handle, C.byref(n)))
    return n.value


def ae_gated_backward(handle: int, Q: int, K: int, V: int, log_decay: int, key_gate: int, dO: int, dQ: int, dK: int, dV: int,
                      dlog_decay: int, dkey_gate: int, workspace: int, workspace_bytes: int, stream: int = 0) -> None:
    """Device pointers as ints; key_gate and dkey_gate are 0 together."""
    _check(_lib.ae_gated_backward(handle, Q, K, V, log_decay, key_gate, dO, dQ, dK, dV, dlog_decay, dkey_gate, workspace,
                                  workspace_bytes, stream))


def gated_recurrent(Q, K, V, log_decay, key_gate=None, *, scale, h_in=None, want_state=False, out_dtype=None, stream=None,
                    segmented=False):
    """Runs the gated recurrent pattern on device tensors: Q, K bf16 [B, H_qk, L, D_qk], V bf16 [B, H, L, D_v],
    log_decay / key_gate fp32 [B, H, L] (all contiguous), h_in fp32 [B, H, D_qk, D_v] or None.  Returns O
    [B, H, L, D_v] (fp32, or bf16 with out_dtype=torch.bfloat16), and the final state when want_state.  segmented: through
    ae_gated_forward_segmented (the walks cut into segments where few heads meet a long sequence)."""
    import torch

    for t in (Q, K, V, log_decay) + (() if key_gate is None else (key_gate,)) + (() if h_in is None else (h_in,)):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("gated_recurrent needs contiguous device tensors; there is no CPU path")
    B, H_qk, L, D_qk = Q.shape
    _, H, _, D_v = V.shape
    with _memory_of(stream):
        out = torch.empty((B, H, L, D_v), dtype=out_dtype or torch.float32, device=Q.device)
        h_out = torch.empty((B, H, D_qk, D_v), dtype=torch.float32, device=Q.device) if want_state else None
    h = ae_gated_create(B=B, H=H, H_qk=H_qk, L=L, D_qk=D_qk, D_v=D_v, scale=scale,
                        out_dtype="bf16" if out.dtype == torch.bfloat16 else "f32")
    try:
        s = torch.cuda.current_stream(Q.device) if stream is None else stream
        nbytes = ae_gated_workspace_bytes(h) if segmented else 0
        with _memory_of(stream):
            ws = torch.empty(nbytes, dtype=torch.uint8, device=Q.device) if nbytes else None
        with torch.cuda.device(Q.device):
            args = (h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), log_decay.data_ptr(),
                    0 if key_gate is None else key_gate.data_ptr(), 0 if h_in is None else h_in.data_ptr(),
                    out.data_ptr(), 0 if h_out is None else h_out.data_ptr())
            if segmented:
                ae_gated_forward_segmented(*args, 0 if ws is None else ws.data_ptr(), nbytes, s.cuda_stream)
            else:
                ae_gated_forward(*args, s.cuda_stream)
    finally:
        ae_gated_destroy(h)
    return (out, h_out) if want_state else out


def gated_recurrent_backward(Q, K, V, log_decay, key_gate, dO, *, scale, stream=None):
    """Backward pass of gated_recurrent on device tensors (layouts as there, dO bf16 [B, H, L, D_v], contiguous).
    Returns (dQ, dK, dV, dlog_decay, dkey_gate or None), all fp32; dQ and dK have the shape of Q."""
    import torch

    for t in (Q, K, V, log_decay, dO) + (() if key_gate is None else (key_gate,)):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("gated_recurrent_backward needs contiguous device tensors; there is no CPU path")
    B, H_qk, L, D_qk = Q.shape
    _, H, _, D_v = V.shape
    f32 = dict(dtype=torch.float32, device=Q.device)
    with _memory_of(stream):
        dQ, dK, dV = torch.empty(Q.shape, **f32), torch.empty(K.shape, **f32), torch.empty(V.shape, **f32)
        dla = torch.empty((B, H, L), **f32)
        dkg = None if key_gate is None else torch.empty((B, H, L), **f32)
    h = ae_gated_create(B=B, H=H, H_qk=H_qk, L=L, D_qk=D_qk, D_v=D_v, scale=scale)
    try:
        nbytes = ae_gated_backward_workspace_bytes(h)
        with _memory_of(stream):
            ws = torch.empty(nbytes, dtype=torch.uint8, device=Q.device)
        s = torch.cuda.current_stream(Q.device) if stream is None else stream
        with torch.cuda.device(Q.device):
            ae_gated_backward(h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), log_decay.data_ptr(),
                              0 if key_gate is None else key_gate.data_ptr(), dO.data_ptr(), dQ.data_ptr(), dK.data_ptr(),
                              dV.data_ptr(), dla.data_ptr(), 0 if dkg is None else dkg.data_ptr(), ws.data_ptr(), nbytes,
                              s.cuda_stream)
    finally:
        ae_gated_destroy(h)
    return dQ, dK, dV, dla, dkg


# ---- rotary positions, paged key/value cache (include/ae_serving.h) -----------------------------------------------------
ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}
CACHE_DTYPES = {"bf16": 0, "e4m3": 1}


class ae_rotary_desc_t(C.Structure):
    _fields_ = [("B", C.c_int32), ("H_q", C.c_int32), ("H_k", C.c_int32), ("L", C.c_int32), ("D", C.c_int32), ("rot_dim", C.c_int32),
                ("layout", C.c_int), ("dtype", C.c_int), ("frequencies", C.POINTER(C.c_double)), ("amplitude", C.c_double),
                ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3), ("q_out_stride", C.c_int64 * 3),
                ("k_out_stride", C.c_int64 * 3), ("position_stride", C.c_int64)]


class ae_cache_desc_t(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("page_size", C.c_int32), ("H_kv", C.c_int32), ("D_qk", C.c_int32), ("D_v", C.c_int32),
                ("dtype", C.c_int)]


class ae_cached_desc_t(C.Structure):
    _fields_ = [("B", C.c_int32), ("H_q", C.c_int32), ("n_new", C.c_int32), ("table_width", C.c_int32), ("max_length", C.c_int32),
                ("prefix_length", C.c_int32), ("chunk", C.c_int32), ("scale", C.c_float), ("out_dtype", C.c_int),
                ("q_stride", C.c_int64 * 3), ("o_stride", C.c_int64 * 3)]


_strides_t = C.c_int64 * 3
_lib.ae_cached_create.argtypes = [C.c_void_p, C.POINTER(ae_cached_desc_t), C.POINTER(C.c_void_p)]
_lib.ae_cached_create.restype = C.c_int
_lib.ae_cached_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
_lib.ae_cached_workspace_bytes.restype = C.c_int
_lib.ae_cached_init_workspace.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
_lib.ae_cached_init_workspace.restype = C.c_int
_lib.ae_cached_forward.argtypes = [C.c_void_p] * 12 + [C.c_size_t, C.c_void_p]
_lib.ae_cached_forward.restype = C.c_int
_lib.ae_cached_query.argtypes = [C.c_void_p] + [C.POINTER(C.c_int32)] * 4
_lib.ae_cached_query.restype = C.c_int
_lib.ae_cached_destroy.argtypes = [C.c_void_p]
_lib.ae_cached_destroy.restype = C.c_int
_lib.ae_rotary_create.argtypes = [C.POINTER(ae_rotary_desc_t), C.POINTER(C.c_void_p)]
_lib.ae_rotary_create.restype = C.c_int
_lib.ae_rotary_forward.argtypes = [C.c_void_p] * 7
_lib.ae_rotary_forward.restype = C.c_int
_lib.ae_rotary_backward.argtypes = [C.c_void_p] * 7
_lib.ae_rotary_backward.restype = C.c_int
_lib.ae_rotary_destroy.argtypes = [C.c_void_p]
_lib.ae_rotary_destroy.restype = C.c_int
_lib.ae_cache_create.argtypes = [C.POINTER(ae_cache_desc_t), C.POINTER(C.c_void_p)]
_lib.ae_cache_create.restype = C.c_int
_lib.ae_cache_append.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int64), C.c_void_p, C.POINTER(C.c_int64), C.c_int32, C.c_int32,
                                 C.c_void_p, C.c_int64] + [C.c_void_p] * 5
_lib.ae_cache_append.restype = C.c_int
_lib.ae_cache_read.argtypes = [C.c_void_p] * 5 + [C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.POINTER(C.c_int64),
                                                  C.c_void_p, C.POINTER(C.c_int64), C.c_void_p]
_lib.ae_cache_read.restype = C.c_int
_lib.ae_cache_destroy.argtypes = [C.c_void_p]
_lib.ae_cache_destroy.restype = C.c_int


def ae_rotary_create(*, B: int, H_q: int, H_k: int, L: int, D: int, frequencies: Sequence[float], amplitude: float = 1.0, layout="half",
                     dtype="bf16", q_stride=(0, 0, 0), k_stride=(0, 0, 0), q_out_stride=(0, 0, 0), k_out_stride=(0, 0, 0),
                     position_stride: int = 0) -> int:
    """Handle for turning the first 2 len(frequencies) elements of the rows of Q [B, H_q, L, D] and K [B, H_k, L, D]."""
    f = (C.c_double * len(frequencies))(*[float(x) for x in frequencies])
    d = ae_rotary_desc_t(B=B, H_q=H_q, H_k=H_k, L=L, D=D, rot_dim=2 * len(frequencies),
                         layout=ROTARY_LAYOUTS[layout] if isinstance(layout, str) else int(layout),
                         dtype={"bf16": 0, "f32": 1}[dtype] if isinstance(dtype, str) else int(dtype),
                         frequencies=C.cast(f, C.POINTER(C.c_double)), amplitude=float(amplitude), position_stride=int(position_stride))
    for name, val in (("q_stride", q_stride), ("k_stride", k_stride), ("q_out_stride", q_out_stride), ("k_out_stride", k_out_stride)):
        setattr(d, name, _strides_t(*[int(x) for x in val]))
    h = C.c_void_p()
    _check(_lib.ae_rotary_create(C.byref(d), C.byref(h)))
    return h.value


def ae_rotary_forward(handle: int, Q: int, K: int, positions: int, Q_out: int, K_out: int, stream: int = 0) -> None:
    """Device addresses; K and K_out are 0 exactly when the handle has H_k = 0."""
    _check(_lib.ae_rotary_forward(handle, Q, K, positions, Q_out, K_out, stream))


def ae_rotary_backward(handle: int, dQ_out: int, dK_out: int, positions: int, dQ: int, dK: int, stream: int = 0) -> None:
    _check(_lib.ae_rotary_backward(handle, dQ_out, dK_out, positions, dQ, dK, stream))


def ae_rotary_destroy(handle: Optional[int]) -> None:
    _check(_lib.ae_rotary_destroy(handle))


def ae_cache_create(*, n_pages: int, page_size: int, H_kv: int, D_qk: int, D_v: int, dtype="bf16") -> int:
    d = ae_cache_desc_t(n_pages=n_pages, page_size=page_size, H_kv=H_kv, D_qk=D_qk, D_v=D_v,
                        dtype=CACHE_DTYPES[dtype] if isinstance(dtype, str) else int(dtype))
    h = C.c_void_p()
    _check(_lib.ae_cache_create(C.byref(d), C.byref(h)))
    return h.value


def ae_cache_append(handle: int, K: int, k_stride, V: int, v_stride, B: int, L: int, slots: int, slot_stride: int, K_pages: int, V_pages: int,
                    K_exp: int = 0, V_exp: int = 0, stream: int = 0) -> None:
    """Device addresses; strides {batch, head, row} in elements."""
    _check(_lib.ae_cache_append(handle, K, _strides_t(*k_stride), V, _strides_t(*v_stride), B, L, slots, slot_stride, K_pages, V_pages, K_exp,
                                V_exp, stream))


def ae_cache_read(handle: int, K_pages: int, V_pages: int, K_exp: int, V_exp: int, B: int, L: int, slots: int, slot_stride: int, K: int,
                  k_stride, V: int, v_stride, stream: int = 0) -> None:
    _check(_lib.ae_cache_read(handle, K_pages, V_pages, K_exp, V_exp, B, L, slots, slot_stride, K, _strides_t(*k_stride), V,
                              _strides_t(*v_stride), stream))


def ae_cache_destroy(handle: Optional[int]) -> None:
    _check(_lib.ae_cache_destroy(handle))


def ae_cached_create(cache: int, *, B: int, H_q: int, n_new: int, table_width: int, max_length: int, scale: float, prefix_length: int = 0,
                     chunk: int = 0, out_dtype="f32", q_stride=(0, 0, 0), o_stride=(0, 0, 0)) -> int:
    """Handle for attention of the newest n_new tokens of B sequences over a paged cache (cache: its handle)."""
    d = ae_cached_desc_t(B=B, H_q=H_q, n_new=n_new, table_width=table_width, max_length=max_length, prefix_length=prefix_length, chunk=chunk,
                         scale=float(scale), out_dtype=OUT_DTYPES[out_dtype] if isinstance(out_dtype, str) else int(out_dtype))
    d.q_stride, d.o_stride = _strides_t(*[int(x) for x in q_stride]), _strides_t(*[int(x) for x in o_stride])
    h = C.c_void_p()
    _check(_lib.ae_cached_create(cache, C.byref(d), C.byref(h)))
    return h.value


def ae_cached_workspace_bytes(handle: int) -> int:
    n = C.c_size_t()
    _check(_lib.ae_cached_workspace_bytes(handle, C.byref(n)))
    return n.value


def ae_cached_init_workspace(handle: int, workspace: int, workspace_bytes: int, stream: int = 0) -> None:
    """Once before the first call that uses the workspace (and after anything else has written there)."""
    _check(_lib.ae_cached_init_workspace(handle, workspace, workspace_bytes, stream))


def ae_cached_forward(handle: int, Q: int, K_pages: int, V_pages: int, K_exp: int, V_exp: int, table: int, lengths: int, prefix_table: int,
                      O: int, stats: int, workspace: int, workspace_bytes: int, stream: int = 0) -> None:
    """Device addresses; K_exp, V_exp (16-bit cache), prefix_table (no prefix), stats and workspace (0 bytes) may be 0."""
    _check(_lib.ae_cached_forward(handle, Q, K_pages, V_pages, K_exp, V_exp, table, lengths, prefix_table, O, stats, workspace,
                                  workspace_bytes, stream))


def ae_cached_query(handle: int) -> dict:
    """What create chose: wavefronts of a workgroup, keys of a range (own lists, prefix), launches of a call."""
    v = [C.c_int32() for _ in range(4)]
    _check(_lib.ae_cached_query(handle, *[C.byref(x) for x in v]))
    return {k: int(x.value) for k, x in zip(("waves", "own_chunk", "prefix_chunk", "launches"), v)}


def ae_cached_destroy(handle: Optional[int]) -> None:
    _check(_lib.ae_cached_destroy(handle))


def rotary_frequencies(rot_dim: int, base: float = 10000.0, *, scaling="none", factor: float = 1.0, original_length: int = 4096,
                       slow_turns: float = 1.0, fast_turns: float = 32.0):
    """Frequencies of rot_dim / 2 pairs (radians a position) and the amplitude of the rotated part, as (list, float).
    scaling, for contexts `factor` times as long as the original_length that a model was trained with:
      "none"      base^(-2 i / rot_dim);
      "linear"    all of them divided by the factor (positions shrink);
      "ntk"       the base grows by factor^(rot_dim / (rot_dim - 2)): the slowest pair shrinks by the factor, the fastest stays;
      "by_parts"  pairs that turn at most slow_turns times in original_length positions shrink by the factor, those that turn at
                  least fast_turns times stay, the ones between blend linearly; the amplitude is 0.1 ln(factor) + 1."""
    import math

    if rot_dim < 2 or rot_dim % 2:
        raise ValueError("rot_dim must be even and at least 2")
    if not (base > 0 and factor >= 1.0):
        raise ValueError("base must be positive and factor at least 1")
    half = rot_dim // 2
    if scaling == "ntk":
        if rot_dim == 2:
            raise ValueError("ntk scaling needs two pairs or more")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = [base ** (-i / half) for i in range(half)]
    if scaling in ("none", "ntk"):
        return f, 1.0
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "by_parts":
        if not fast_turns > slow_turns:
            raise ValueError("fast_turns must exceed slow_turns")
        keep = [min(1.0, max(0.0, (original_length * x / (2 * math.pi) - slow_turns) / (fast_turns - slow_turns))) for x in f]
        return [x * k + x / factor * (1.0 - k) for x, k in zip(f, keep)], 0.1 * math.log(factor) + 1.0
    raise ValueError(f"unknown scaling {scaling!r}")


ONE_ROW = -2 ** 63  # AE_ONE_ROW


def _row_strides(t):
    """Element strides {batch, head, row} as the C ABI takes them, where three zeros mean contiguous: a tensor whose rows are all one
    (expanded from a vector) says so."""
    s = t.stride()[:3]
    return s if any(s) or t.shape[0] * t.shape[1] * t.shape[2] <= 1 else (ONE_ROW, 0, 0)


def _shape_of(t):
    return (t.shape, t.stride(), t.dtype, t.device)


def _enqueue(call, device, stream, *args):
    """call(*args, raw stream) with `device` current, on `stream` (None: the device's current one).  The step of a decoding loop pays for
    this every time: asking for a stream object takes 1.9 us, for its address 0.1, and setting the current device again 1.3."""
    import torch

    index = device.index
    raw = _raw_stream(index) if stream is None else stream.cuda_stream
    if torch.cuda.current_device() == index:
        call(*args, raw)
    else:
        with torch.cuda.device(index):
            call(*args, raw)


def _raw_stream(index):
    import torch

    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(index) if get is not None else torch.cuda.current_stream(index).cuda_stream


class RotaryPlan:
    """A rotary handle for calls of one shape: the step of a loop keeps it.  Made from the first call's tensors (Q [B, H_q, L, D], K
    [B, H_k, L, D] or None, positions int32 [L] or [B, L], outputs of the same shapes; bf16 or fp32, last dimension contiguous);
    forward() and backward() take tensors of the same shapes, strides, type and device.  backward(dQ_out, dK_out, positions, dQ, dK)
    goes from the outputs' layout to the inputs'."""

    def __init__(self, Q, K, positions, Q_out, K_out, *, freqs, amplitude=1.0, layout="half"):
        import torch

        self.handle = None
        some = [t for t in (Q, K, Q_out, K_out) if t is not None]
        if (K is None) != (K_out is None):
            raise ValueError("K and its output come together")
        for t in some:
            if not t.is_cuda or t.dim() != 4 or t.stride(3) != 1 or t.dtype != Q.dtype or t.device != Q.device:
                raise ValueError("Q, K and the outputs must be 4-D device tensors of one type and device with a contiguous last dimension; there is no CPU path")
        if Q.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("rotary positions come in bf16 and fp32")
        B, H_q, L, D = Q.shape
        if Q_out.shape != Q.shape or (K is not None and (K_out.shape != K.shape or K.shape[0] != B or tuple(K.shape[2:]) != (L, D))):
            raise ValueError("K / output shapes do not match Q")
        if (not positions.is_cuda or positions.device != Q.device or positions.dtype != torch.int32 or tuple(positions.shape) not in ((L,), (B, L))
                or (L > 1 and positions.stride(-1) != 1)):
            raise ValueError("positions must be an int32 device tensor [L] or [B, L] with contiguous rows")
        self._shared = _expanded(Q_out, K_out), _expanded(Q, K)  # (expanded tensors can be read, not written)
        zero = (0, 0, 0)
        self.handle = ae_rotary_create(
            B=B, H_q=H_q, H_k=0 if K is None else K.shape[1], L=L, D=D, frequencies=freqs, amplitude=amplitude, layout=layout,
            dtype="f32" if Q.dtype == torch.float32 else "bf16", q_stride=_row_strides(Q), k_stride=zero if K is None else _row_strides(K),
            q_out_stride=_row_strides(Q_out), k_out_stride=zero if K is None else _row_strides(K_out),
            position_stride=positions.stride(0) if positions.dim() == 2 else 0)
        self._specs = [None if t is None else _shape_of(t) for t in (Q, K, positions, Q_out, K_out)]
        self.device = Q.device

    def _run(self, call, specs, tensors, shared, stream):
        if shared:
            raise ValueError("an output must not be an expanded tensor")
        if [t if t is None else _shape_of(t) for t in tensors] != specs:
            raise ValueError("a tensor differs from the plan's in shape, strides, type or device")
        _enqueue(call, self.device, stream, self.handle, *[0 if t is None else t.data_ptr() for t in tensors])

    def forward(self, Q, K, positions, Q_out, K_out, *, stream=None):
        self._run(ae_rotary_forward, self._specs, (Q, K, positions, Q_out, K_out), self._shared[0], stream)

    def backward(self, dQ_out, dK_out, positions, dQ, dK, *, stream=None):
        s = self._specs
        self._run(ae_rotary_backward, [s[3], s[4], s[2], s[0], s[1]], (dQ_out, dK_out, positions, dQ, dK), self._shared[1], stream)

    def __del__(self):
        if getattr(self, "handle", None) is not None and _lib is not None:
            _lib.ae_rotary_destroy(self.handle)
            self.handle = None


def _expanded(*tensors):
    """Whether one of them has two indices at one address."""
    return any(t is not None and 0 in t.stride() and any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride())) for t in tensors)


def _no_overlap(*outs):
    if _expanded(*outs):
        raise ValueError("an output must not be an expanded tensor")


def _rotary(Q, K, positions, freqs, amplitude, layout, out, stream, backward):
    import torch

    if out is None:
        with _memory_of(stream):
            out = (torch.empty(Q.shape, dtype=Q.dtype, device=Q.device), None if K is None else torch.empty(K.shape, dtype=K.dtype, device=K.device))
    q, k = out
    # the handle's "inputs" are the layout that the backward pass writes
    a, b = ((q, k), (Q, K)) if backward else ((Q, K), (q, k))
    plan = RotaryPlan(a[0], a[1], positions, b[0], b[1], freqs=freqs, amplitude=amplitude, layout=layout)
    (plan.backward if backward else plan.forward)(Q, K, positions, q, k, stream=stream)
    return q, k


def rotary_forward(Q, K, positions, *, freqs, amplitude=1.0, layout="half", out=None, stream=None):
    """Rotary positions on device tensors Q [B, H_q, L, D] and K [B, H_k, L, D] (or None), bf16 or fp32, last dimension contiguous:
    pair i of a row at position p is turned by p freqs[i] and stretched by amplitude (rotary_frequencies() makes both); elements from
    2 len(freqs) on are copied.  layout "half" pairs element i with i + len(freqs), "interleaved" 2 i with 2 i + 1.  positions: int32
    [L] or [B, L].  out: a pair of output tensors (the inputs themselves: in place).  Returns (Q', K'); what is allocated for them belongs
    to the stream that the call is on (stream, else the current one)."""
    return _rotary(Q, K, positions, freqs, amplitude, layout, out, stream, False)


def rotary_backward(dQ, dK, positions, *, freqs, amplitude=1.0, layout="half", out=None, stream=None):
    """Gradients of Q and K for the gradients of rotary_forward's outputs (arguments as there): pairs are turned back."""
    return _rotary(dQ, dK, positions, freqs, amplitude, layout, out, stream, True)


class PagedCache:
    """The paged key/value cache of one layer: K pages [n_pages, H_kv, page, D_qk] and V pages [n_pages, H_kv, page, D_v], bf16 or
    float8_e4m3fn (then with exponent bytes k_exp, v_exp, uint8 [n_pages, H_kv, page]), contiguous device tensors of the caller.  A position of
    the cache is the slot page_number * page + place."""

    def __init__(self, k, v, k_exp=None, v_exp=None):
        import torch

        self.handle = None
        e4m3 = k.dtype == torch.float8_e4m3fn
        if k.dtype not in (torch.bfloat16, torch.float8_e4m3fn) or v.dtype != k.dtype:
            raise ValueError("pages must be bf16 or float8_e4m3fn")
        if (k_exp is None) == e4m3 or (v_exp is None) == e4m3:
            raise ValueError("exponents belong to an 8-bit cache, and only to it")
        if k.dim() != 4 or v.dim() != 4 or k.shape[:3] != v.shape[:3]:
            raise ValueError("pages must be [n_pages, H_kv, page, D]")
        for t in (k, v) + ((k_exp, v_exp) if e4m3 else ()):
            if not t.is_cuda or not t.is_contiguous() or t.device != k.device:
                raise ValueError("the cache's buffers must be contiguous tensors of one device; there is no CPU path")
        if e4m3 and any(t.dtype != torch.uint8 or t.shape != k.shape[:3] for t in (k_exp, v_exp)):
            raise ValueError("exponents must be uint8 [n_pages, H_kv, page]")
        self.k, self.v, self.k_exp, self.v_exp, self.device = k, v, k_exp, v_exp, k.device
        self.n_pages, self.H_kv, self.page_size, self.D_qk = k.shape
        self.D_v = v.shape[3]
        self._bf16, self._int = torch.bfloat16, torch.int32
        self.handle = ae_cache_create(n_pages=self.n_pages, page_size=self.page_size, H_kv=self.H_kv, D_qk=self.D_qk, D_v=self.D_v,
                                      dtype="e4m3" if e4m3 else "bf16")

    @classmethod
    def empty(cls, n_pages, H_kv, page_size, D_qk, D_v, *, dtype="bf16", device="cuda"):
        """A cache with buffers of its own (contents undefined until written)."""
        import torch

        e4m3 = {"bf16": False, "e4m3": True}[dtype]
        t = torch.float8_e4m3fn if e4m3 else torch.bfloat16
        k, v = (torch.empty(n_pages, H_kv, page_size, d, dtype=t, device=device) for d in (D_qk, D_v))
        e = [torch.empty(n_pages, H_kv, page_size, dtype=torch.uint8, device=device) if e4m3 else None for _ in range(2)]
        return cls(k, v, *e)

    def pointers(self):
        return (self.k.data_ptr(), self.v.data_ptr(), 0 if self.k_exp is None else self.k_exp.data_ptr(),
                0 if self.v_exp is None else self.v_exp.data_ptr())

    def _slots(self, slots, B, L):
        if (slots.dtype != self._int or slots.shape not in (((L,), (B, L)) if B == 1 else ((B, L),)) or slots.device != self.device
                or (L > 1 and slots.stride(-1) != 1)):
            raise ValueError("slots must be an int32 device tensor [B, L] (or [L] for B = 1) with contiguous rows")
        return slots.data_ptr(), slots.stride(0) if slots.dim() == 2 else 0

    def _rows(self, K, V, B, L):
        """Strides of K and V [B, H_kv, L, D]."""
        strides = []
        for t, d in ((K, self.D_qk), (V, self.D_v)):
            st = t.stride()
            if t.dtype != self._bf16 or t.shape != (B, self.H_kv, L, d) or st[3] != 1 or t.device != self.device:
                raise ValueError("K and V must be bf16 [B, H_kv, L, D] on the cache's device with a contiguous last dimension")
            strides.append(st[:3] if st[0] or st[1] or st[2] else _row_strides(t))
        return strides

    def append(self, K, V, slots, *, stream=None):
        """Writes the rows of K [B, H_kv, L, D_qk] and V [B, H_kv, L, D_v] (bf16, last dimension contiguous) to the slots int32 [B, L];
        rows whose slot is outside the cache (-1) are skipped, the others' slots must differ."""
        B, _, L, _ = K.shape
        ks, vs = self._rows(K, V, B, L)
        at, stride = self._slots(slots, B, L)
        _enqueue(ae_cache_append, self.device, stream, self.handle, K.data_ptr(), ks, V.data_ptr(), vs, B, L, at, stride, *self.pointers())

    def _empty_rows(self, B, L):
        import torch

        return tuple([torch.empty((B, self.H_kv, L, d), dtype=self._bf16, device=self.device) for d in (self.D_qk, self.D_v)])

    def read(self, slots, *, out=None, stream=None):
        """The rows at slots int32 [B, L] (or [L]: B = 1) as bf16 K [B, H_kv, L, D_qk] and V [B, H_kv, L, D_v]; zeros for a slot outside the
        cache.  out: a pair of tensors to write to (else they are allocated, on the stream that the call is on)."""
        B, L = (1, slots.shape[0]) if slots.dim() == 1 else slots.shape
        if out is None:
            if stream is None:  # (a step of a loop: entering no context takes 0.4 us of 17)
                out = self._empty_rows(B, L)
            else:
                with _memory_of(stream):
                    out = self._empty_rows(B, L)
            ks = vs = (0, 0, 0)  # (contiguous)
        else:
            ks, vs = self._rows(*out, B, L)
            _no_overlap(*out)
        at, stride = self._slots(slots, B, L)
        _enqueue(ae_cache_read, self.device, stream, self.handle, *self.pointers(), B, L, at, stride, out[0].data_ptr(), ks, out[1].data_ptr(), vs)
        return out

    def __del__(self):
        if getattr(self, "handle", None) is not None and _lib is not None:
            _lib.ae_cache_destroy(self.handle)
            self.handle = None


class CachedAttentionPlan:
    """A handle for attention of the newest tokens over a PagedCache, for calls of one shape: the step of a decoding loop keeps it, and
    its workspace.  Q [B, H_q, n, D_qk] bf16 and out [B, H_q, n, D_v] (bf16 or fp32) give shapes, strides and device; max_length: no
    sequence has more keys of its own; table_width: pages in a row of the table; prefix_length: keys that all sequences share.
    Calls of one plan must not overlap (they share its workspace, which is prepared on the stream that is current when the plan is
    made: another stream waits for that one before its first call); the plan may be dropped while a call still runs, on whichever stream.
    A captured graph keeps using the plan's buffers, so the plan has to outlive it, and a plan made while a graph is captured is of use to
    that graph alone."""

    def __init__(self, cache, Q, out, *, max_length, table_width, scale, prefix_length=0, chunk=0):
        import torch

        self.handle = None
        for t in (Q, out):
            if not t.is_cuda or t.dim() != 4 or t.stride(3) != 1 or t.device != cache.device:
                raise ValueError("Q and O must be 4-D tensors on the cache's device with a contiguous last dimension; there is no CPU path")
        B, H_q, n, D = Q.shape
        if Q.dtype != torch.bfloat16 or D != cache.D_qk:
            raise ValueError("Q must be bf16 [B, H_q, n, D_qk]")
        if out.dtype not in (torch.float32, torch.bfloat16) or tuple(out.shape) != (B, H_q, n, cache.D_v):
            raise ValueError("O must be fp32 or bf16 [B, H_q, n, D_v]")
        _no_overlap(out)
        self.handle = ae_cached_create(cache.handle, B=B, H_q=H_q, n_new=n, table_width=table_width, max_length=max_length, scale=scale,
                                       prefix_length=prefix_length, chunk=chunk, out_dtype="bf16" if out.dtype == torch.bfloat16 else "f32",
                                       q_stride=_row_strides(Q), o_stride=_row_strides(out))
        self.cache, self.device, self.shape, self._f32 = cache, Q.device, (B, H_q, n), torch.float32
        self._q, self._o = _shape_of(Q), _shape_of(out)
        self._table, self._prefix = (B, table_width), -(-prefix_length // cache.page_size)
        self.workspace_bytes = ae_cached_workspace_bytes(self.handle)
        self.workspace = None
        if self.workspace_bytes:
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=Q.device)
            self._streams = {_raw_stream(Q.device.index)}  # those that the allocator knows to use it
            _enqueue(ae_cached_init_workspace, Q.device, None, self.handle, self.workspace.data_ptr(), self.workspace_bytes)

    def forward(self, Q, table, lengths, out, *, stats=None, prefix_table=None, stream=None):
        """table int32 [B, table_width], lengths int32 [B] (device), prefix_table int32 [pages of the prefix]; stats: fp32 [B, H_q, n] that
        receives ln sum exp.  Writes and returns out."""
        if _shape_of(Q) != self._q or _shape_of(out) != self._o:
            raise ValueError("Q or O differs from the plan's in shape, strides, type or device")
        if (prefix_table is None) == bool(self._prefix):
            raise ValueError("a prefix's table is given exactly where the plan has a prefix")
        ints = ((table, self._table), (lengths, self._table[:1])) + (((prefix_table, (self._prefix,)),) if self._prefix else ())
        for t, shape in ints:
            if t.dtype != self.cache._int or t.shape != shape or not t.is_contiguous() or t.device != self.device:
                raise ValueError(f"tables and lengths must be contiguous int32 device tensors (here {shape})")
        if stats is not None and (stats.dtype != self._f32 or stats.shape != self.shape or not stats.is_contiguous() or stats.device != self.device):
            raise ValueError("stats must be a contiguous fp32 tensor [B, H_q, n]")
        if self.workspace is not None:
            self._use_workspace(stream)
        _enqueue(ae_cached_forward, self.device, stream, self.handle, Q.data_ptr(), *self.cache.pointers(), table.data_ptr(), lengths.data_ptr(),
                 0 if prefix_table is None else prefix_table.data_ptr(), out.data_ptr(), 0 if stats is None else stats.data_ptr(),
                 0 if self.workspace is None else self.workspace.data_ptr(), self.workspace_bytes)
        return out

    def _use_workspace(self, stream):
        """Its memory belongs to the stream that was current when the plan was made; given back, it must not serve that one before a call on
        another is done."""
        import torch

        raw = _raw_stream(self.device.index) if stream is None else stream.cuda_stream
        if raw not in self._streams:
            self.workspace.record_stream(torch.cuda.current_stream(self.device) if stream is None else stream)
            self._streams.add(raw)

    def __del__(self):
        if getattr(self, "handle", None) is not None and _lib is not None:
            _lib.ae_cached_destroy(self.handle)
            self.handle = None


def attention_cached(Q, cache, table, lengths, *, scale, max_length=None, prefix_table=None, prefix_length=0, out=None, out_dtype=None,
                     stats=None, chunk=0, stream=None):
    """Softmax attention of the newest n tokens of each sequence, Q bf16 [B, H_q, n, D_qk], over everything a PagedCache holds for
    them: position j of sequence b lies on page table[b, j // page] (int32 [B, width]), lengths int32 [B] counts its keys, the newest n
    among them; token t sees the first lengths[b] - n + 1 + t.  max_length: no sequence is longer (None: the table's room).
    prefix_table / prefix_length: keys in front of every sequence's own that the whole batch shares; they are read once for all.
    Returns O [B, H_q, n, D_v], fp32 or bf16 (out / out_dtype); stats: optional fp32 [B, H_q, n] that receives ln sum exp."""
    import torch

    with _memory_of(stream):  # (the workspace, too, belongs to the stream that uses it)
        if out is None:
            out = torch.empty(Q.shape[:3] + (cache.D_v,), dtype=out_dtype or torch.float32, device=Q.device)
        plan = CachedAttentionPlan(cache, Q, out, max_length=table.shape[1] * cache.page_size if max_length is None else max_length,
                                   table_width=table.shape[1], scale=scale, prefix_length=prefix_length, chunk=chunk)
        return plan.forward(Q, table, lengths, out, stats=stats, prefix_table=prefix_table)
