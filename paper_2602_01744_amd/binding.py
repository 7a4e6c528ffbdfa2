"""ctypes binding for libsla.so: argument marshalling only.

The functions ``sla_*`` mirror the C ABI one to one (raw integer addresses in,
status code out).  ``forward`` is the convenience wrapper the tests and the
benchmark use: it takes torch CUDA tensors, allocates the outputs with torch and
passes ``data_ptr()``s and the current stream to ``sla_forward``.
"""
from __future__ import annotations

import ctypes
import functools
import os
import sys
from typing import Optional, Tuple

RETNET, GLA, GDN = 0, 1, 2
FLAG_HEAD_MAJOR = 1
F32, BF16 = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libsla.so")
_lib = None


class SlaError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"libsla: {text} (status {status})")
        self.status = status


class SlaParams(ctypes.Structure):
    _fields_ = [
        ("variant", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("B", ctypes.c_int32),
        ("T", ctypes.c_int32),
        ("H", ctypes.c_int32),
        ("dk", ctypes.c_int32),
        ("dv", ctypes.c_int32),
        ("dv_split", ctypes.c_int32),
        ("flags", ctypes.c_int32),
        ("segments", ctypes.c_int32),
    ]


class SlaRotaryParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "B", "T", "Hq", "Hk", "d", "rotary", "flags")] + [
        ("magnitude", ctypes.c_float)]


class SlaNormGateParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "B", "T", "H", "dv", "gate", "flags")] + [("eps", ctypes.c_float)]


class SlaJoinNormParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "x_dtype", "B", "T", "D")] + [
        ("scale", ctypes.c_float), ("eps", ctypes.c_float)]


FLAG_ADJACENT_PAIRS, FLAG_TOKEN_POSITIONS = 2, 4  # sla_rotary_params.flags
FLAG_HEAD_WEIGHTS = 2  # sla_norm_gate_params.flags
GATES = {"none": 0, "silu": 1, "sigmoid": 2}


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libsla.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2602_01744_amd.build` "
            "(or __graft_entry__.build()); there is no CPU fallback"
        )
    lib = ctypes.CDLL(_LIB_PATH)
    vp = ctypes.c_void_p
    pp = ctypes.POINTER(SlaParams)
    lib.sla_forward.restype = ctypes.c_int
    lib.sla_forward.argtypes = [pp] + [vp] * 11
    lib.sla_forward_ws.restype = ctypes.c_int
    lib.sla_forward_ws.argtypes = [pp] + [vp] * 11 + [ctypes.c_size_t, vp]
    lib.sla_forward_static.restype = ctypes.c_int
    lib.sla_forward_static.argtypes = [pp] + [vp] * 11
    lib.sla_device_status.restype = ctypes.c_int
    lib.sla_device_status.argtypes = [ctypes.POINTER(ctypes.c_uint32), ctypes.c_int, vp]
    lib.sla_init.restype = ctypes.c_int
    lib.sla_init.argtypes = []
    lib.sla_static_scratch_bytes.restype = ctypes.c_size_t
    lib.sla_static_scratch_bytes.argtypes = []
    lib.sla_decode_step.restype = ctypes.c_int
    lib.sla_decode_step.argtypes = [pp] + [vp] * 10
    lib.sla_decode_step_fused.restype = ctypes.c_int
    lib.sla_decode_step_fused.argtypes = [pp] + [vp] * 10
    lib.sla_forward_varlen.restype = ctypes.c_int
    lib.sla_forward_varlen.argtypes = [pp] + [vp] * 12
    lib.sla_backward_varlen.restype = ctypes.c_int
    lib.sla_backward_varlen.argtypes = [pp] + [vp] * 18 + [ctypes.c_size_t, vp]
    lib.sla_backward_varlen_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_backward_varlen_workspace_bytes.argtypes = [pp]
    lib.sla_short_conv_silu.restype = ctypes.c_int
    lib.sla_short_conv_silu.argtypes = [ctypes.c_int] * 5 + [vp] * 4
    lib.sla_short_conv_silu_l2.restype = ctypes.c_int
    lib.sla_short_conv_silu_l2.argtypes = [ctypes.c_int] * 6 + [ctypes.c_float] + [vp] * 4
    lib.sla_short_conv_silu_l2_backward.restype = ctypes.c_int
    lib.sla_short_conv_silu_l2_backward.argtypes = [ctypes.c_int] * 6 + [ctypes.c_float] + [vp] * 6 + [ctypes.c_size_t, vp]
    lib.sla_short_conv_silu_l2_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_short_conv_silu_l2_backward_workspace_bytes.argtypes = [ctypes.c_int] * 4
    lib.sla_gate_logits_backward.restype = ctypes.c_int
    lib.sla_gate_logits_backward.argtypes = [pp] + [vp] * 6 + [ctypes.c_size_t, vp]
    lib.sla_gate_logits_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_gate_logits_backward_workspace_bytes.argtypes = [pp]
    lib.sla_gate_logits.restype = ctypes.c_int
    lib.sla_gate_logits.argtypes = [pp] + [vp] * 7
    lib.sla_backward.restype = ctypes.c_int
    lib.sla_backward.argtypes = [pp] + [vp] * 17 + [ctypes.c_size_t, vp]
    lib.sla_backward_gdn.restype = ctypes.c_int
    lib.sla_backward_gdn.argtypes = [pp] + [vp] * 19 + [ctypes.c_size_t, vp]
    lib.sla_backward_gdn_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_backward_gdn_workspace_bytes.argtypes = [pp]
    lib.sla_backward_gdn_varlen.restype = ctypes.c_int
    lib.sla_backward_gdn_varlen.argtypes = [pp] + [vp] * 20 + [ctypes.c_size_t, vp]
    lib.sla_backward_gdn_varlen_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_backward_gdn_varlen_workspace_bytes.argtypes = [pp]
    lib.sla_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_backward_workspace_bytes.argtypes = [pp]
    lib.sla_backward_chunks_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_backward_chunks_workspace_bytes.argtypes = [pp, ctypes.c_int]
    lib.sla_backward_gdn_chunks_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_backward_gdn_chunks_workspace_bytes.argtypes = [pp, ctypes.c_int]
    rp, np_, jp = (ctypes.POINTER(t) for t in (SlaRotaryParams, SlaNormGateParams, SlaJoinNormParams))
    for call in (lib.sla_rotary, lib.sla_rotary_backward):
        call.restype = ctypes.c_int
        call.argtypes = [rp] + [vp] * 8
    lib.sla_norm_gate.restype = ctypes.c_int
    lib.sla_norm_gate.argtypes = [np_] + [vp] * 6
    lib.sla_norm_gate_backward.restype = ctypes.c_int
    lib.sla_norm_gate_backward.argtypes = [np_] + [vp] * 9 + [ctypes.c_size_t, vp]
    lib.sla_norm_gate_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_norm_gate_backward_workspace_bytes.argtypes = [np_, ctypes.c_int]
    lib.sla_join_norm.restype = ctypes.c_int
    lib.sla_join_norm.argtypes = [jp] + [vp] * 9
    lib.sla_join_norm_backward.restype = ctypes.c_int
    lib.sla_join_norm_backward.argtypes = [jp] + [vp] * 14 + [ctypes.c_size_t, vp]
    lib.sla_join_norm_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_join_norm_backward_workspace_bytes.argtypes = [jp, ctypes.c_int]
    lib.sla_forward_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_forward_workspace_bytes.argtypes = [pp, ctypes.c_int]
    lib.sla_workspace_bytes.restype = ctypes.c_size_t
    lib.sla_workspace_bytes.argtypes = [pp, ctypes.c_int]
    lib.sla_segments.restype = ctypes.c_int
    lib.sla_segments.argtypes = [pp, ctypes.c_int]
    lib.sla_backward_segments.restype = ctypes.c_int
    lib.sla_backward_segments.argtypes = [pp, ctypes.c_int]
    lib.sla_check_args.restype = ctypes.c_int
    lib.sla_check_args.argtypes = [pp] + [vp] * 10
    lib.sla_default_dv_split.restype = ctypes.c_int
    lib.sla_default_dv_split.argtypes = [pp, ctypes.c_int]
    lib.sla_kernel_name.restype = ctypes.c_char_p
    lib.sla_kernel_name.argtypes = [pp]
    lib.sla_status_string.restype = ctypes.c_char_p
    lib.sla_status_string.argtypes = [ctypes.c_int]
    lib.sla_version.restype = ctypes.c_int
    lib.sla_version.argtypes = []
    _lib = lib
    return lib


def _p(x) -> Optional[int]:
    return None if not x else int(x)


def _stream(t) -> int:
    """The current stream of the tensor's device, as the hipStream_t handle (no Stream object is made for it).  Refuses a
    tensor in host memory, whose device index -1 would otherwise mean the current GPU."""
    device = t.get_device()
    if device < 0:
        raise ValueError(f"expected a tensor on a GPU, but got one on: {t.device}")
    return sys.modules["torch"]._C._cuda_getCurrentRawStream(device)  # (an import statement costs a tenth of a microsecond)


def sla_status_string(status: int) -> str:
    return load_library().sla_status_string(int(status)).decode()


def sla_version() -> int:
    return int(load_library().sla_version())


def sla_default_dv_split(params: SlaParams, compute_units: int) -> int:
    return int(load_library().sla_default_dv_split(ctypes.byref(params), int(compute_units)))


def sla_workspace_bytes(params: SlaParams, compute_units: int) -> int:
    return int(load_library().sla_workspace_bytes(ctypes.byref(params), int(compute_units)))


def sla_forward_workspace_bytes(params: SlaParams, compute_units: int) -> int:
    return int(load_library().sla_forward_workspace_bytes(ctypes.byref(params), int(compute_units)))


def sla_segments(params: SlaParams, compute_units: int) -> int:
    return int(load_library().sla_segments(ctypes.byref(params), int(compute_units)))


def sla_backward_segments(params: SlaParams, compute_units: int) -> int:
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_backward_segments(pr, int(compute_units)))


def sla_kernel_name(params: SlaParams) -> Optional[str]:
    s = load_library().sla_kernel_name(ctypes.byref(params))
    return None if s is None else s.decode()


def sla_check_args(params, q, k, v, q_head_logits, k_head_logits, log_decay, beta, initial_state, out, final_state) -> int:
    """Raw call: integer addresses (0/None = NULL).  Returns the status code."""
    pr = ctypes.byref(params) if params is not None else None
    return int(
        load_library().sla_check_args(
            pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(beta),
            _p(initial_state), _p(out), _p(final_state),
        )
    )


def sla_forward(params, q, k, v, q_head_logits, k_head_logits, log_decay, beta, initial_state, out, final_state,
                stream) -> int:
    """Raw call: integer device addresses (0/None = NULL) and a hipStream_t handle.  Returns the status code."""
    pr = ctypes.byref(params) if params is not None else None
    return int(
        load_library().sla_forward(
            pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(beta),
            _p(initial_state), _p(out), _p(final_state), _p(stream),
        )
    )


def sla_forward_ws(params, q, k, v, q_head_logits, k_head_logits, log_decay, beta, initial_state, out, final_state,
                   workspace, workspace_bytes, stream) -> int:
    """Raw call of the workspace-taking entry point (same conventions as sla_forward)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(
        load_library().sla_forward_ws(
            pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(beta),
            _p(initial_state), _p(out), _p(final_state), _p(workspace), int(workspace_bytes), _p(stream),
        )
    )


def sla_init() -> int:
    return int(load_library().sla_init())


DEVICE_WAIT_EXPIRED, DEVICE_DECAY_RANGE = 1, 2


def sla_device_status(reset: bool = False, stream=None):
    """Returns (status code, device status word) of the current device; waits for ``stream`` first."""
    word = ctypes.c_uint32(0)
    rc = int(load_library().sla_device_status(ctypes.byref(word), int(bool(reset)), _p(stream)))
    return rc, int(word.value)


def sla_static_scratch_bytes() -> int:
    return int(load_library().sla_static_scratch_bytes())


def sla_forward_static(params, q, k, v, q_head_logits, k_head_logits, log_decay, beta, initial_state, out,
                       final_state, stream) -> int:
    """Raw call of the entry point that allocates nothing (same conventions as sla_forward)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(
        load_library().sla_forward_static(
            pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(beta),
            _p(initial_state), _p(out), _p(final_state), _p(stream),
        )
    )


def sla_decode_step(params, q, k, v, q_head_logits, k_head_logits, log_decay, beta, state, out, stream) -> int:
    """Raw call of the decode entry point (same conventions as sla_forward)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(
        load_library().sla_decode_step(
            pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(beta), _p(state),
            _p(out), _p(stream),
        )
    )


def sla_decode_step_fused(params, q, k, v, w_gq, w_gk, log_decay, beta, state, out, stream) -> int:
    """Raw call of the decode entry point that forms the gate logits itself."""
    pr = ctypes.byref(params) if params is not None else None
    return int(
        load_library().sla_decode_step_fused(
            pr, _p(q), _p(k), _p(v), _p(w_gq), _p(w_gk), _p(log_decay), _p(beta), _p(state), _p(out), _p(stream),
        )
    )


def sla_forward_varlen(params, q, k, v, q_head_logits, k_head_logits, log_decay, beta, cu_seqlens, initial_state, out,
                       final_state, stream) -> int:
    """Raw call of the packed variable-length forward (same conventions as sla_forward)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_forward_varlen(
        pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(beta), _p(cu_seqlens),
        _p(initial_state), _p(out), _p(final_state), _p(stream)))


def sla_backward_varlen_workspace_bytes(params: SlaParams) -> int:
    return int(load_library().sla_backward_varlen_workspace_bytes(ctypes.byref(params)))


def sla_backward_varlen(params, q, k, v, q_head_logits, k_head_logits, log_decay, cu_seqlens, initial_state, d_out,
                        d_final_state, dq, dk, dv, dq_head_logits, dk_head_logits, dlog_decay, d_initial_state,
                        workspace, workspace_bytes, stream) -> int:
    """Raw call of the packed variable-length backward (same conventions as sla_backward)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_backward_varlen(
        pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(cu_seqlens),
        _p(initial_state), _p(d_out), _p(d_final_state), _p(dq), _p(dk), _p(dv), _p(dq_head_logits),
        _p(dk_head_logits), _p(dlog_decay), _p(d_initial_state), _p(workspace), int(workspace_bytes), _p(stream)))


def forward_varlen(variant: int, q, k, v, q_head_logits, k_head_logits, log_decay, beta, cu_seqlens,
                   initial_state=None, *, want_final_state: bool = True):
    """Packed sequences: q, k [T,H,dk], v [T,H,dv], logits (beta, GDN decay) [T,H], cu_seqlens int32 [B+1] on the
    device, initial_state [B,H,dk,dv] or None.  Returns (out [T,H,dv], final_state [B,H,dk,dv] or None)."""
    import torch

    assert q.is_cuda and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
    T, H, dk = q.shape
    dv = v.shape[-1]
    assert cu_seqlens.is_cuda and cu_seqlens.dtype == torch.int32 and cu_seqlens.dim() == 1 and cu_seqlens.is_contiguous()
    B = cu_seqlens.numel() - 1
    dtype = {torch.float32: F32, torch.bfloat16: BF16}[q.dtype]
    out = torch.empty((T, H, dv), dtype=q.dtype, device=q.device)
    fin = torch.empty((B, H, dk, dv), dtype=torch.float32, device=q.device) if want_final_state else None
    params = SlaParams(variant, dtype, B, T, H, dk, dv, 0, 0, 1)
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = sla_forward_varlen(params, ptr(q), ptr(k), ptr(v), ptr(q_head_logits), ptr(k_head_logits), ptr(log_decay),
                            ptr(beta), ptr(cu_seqlens), ptr(initial_state), ptr(out), ptr(fin),
                            _stream(q))
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return out, fin


def _workspace(device, most: int, least):
    """Memory for one call: the ``most`` bytes that it runs fastest with, or the ``least()`` it needs where there is no room."""
    import torch

    try:
        return torch.empty(max(most, 16), dtype=torch.uint8, device=device)
    except torch.cuda.OutOfMemoryError:
        need = least()
        if need >= most:
            raise
        return torch.empty(max(need, 16), dtype=torch.uint8, device=device)


def backward_varlen(variant: int, q, k, v, q_head_logits, k_head_logits, log_decay, d_out, cu_seqlens,
                    initial_state=None, d_final_state=None, *, want_d_initial_state: bool = False):
    """Gradients of ``forward_varlen`` (RetNet, GLA; bfloat16 or float32); tensors packed as there.  Returns a dict
    as ``backward`` does, with d_initial_state [B,H,dk,dv]."""
    import torch

    assert q.is_cuda and q.dtype in (torch.bfloat16, torch.float32)
    T, H, dk = q.shape
    dv = v.shape[-1]
    B = cu_seqlens.numel() - 1
    dev = q.device
    g = {
        "dq": torch.empty_like(q),
        "dk": torch.empty_like(k),
        "dv": torch.empty_like(v),
        "dq_head_logits": torch.empty_like(q_head_logits),
        "dk_head_logits": None if k_head_logits is None else torch.empty_like(k_head_logits),
        "dlog_decay": torch.empty_like(log_decay) if variant == GLA else None,
        "d_initial_state": torch.empty((B, H, dk, dv), dtype=torch.float32, device=dev) if want_d_initial_state else None,
    }
    params = SlaParams(variant, BF16 if q.dtype == torch.bfloat16 else F32, B, T, H, dk, dv, 0, 0, 1)
    workspace = _workspace(dev, sla_backward_chunks_workspace_bytes(params, packed=True),
                           lambda: sla_backward_varlen_workspace_bytes(params))
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = sla_backward_varlen(
        params, ptr(q), ptr(k), ptr(v), ptr(q_head_logits), ptr(k_head_logits), ptr(log_decay), ptr(cu_seqlens),
        ptr(initial_state), ptr(d_out), ptr(d_final_state), ptr(g["dq"]), ptr(g["dk"]), ptr(g["dv"]),
        ptr(g["dq_head_logits"]), ptr(g["dk_head_logits"]), ptr(g["dlog_decay"]), ptr(g["d_initial_state"]),
        ptr(workspace), workspace.numel(), _stream(q),
    )
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return g


def sla_short_conv_silu(dtype: int, B: int, T: int, channels: int, taps: int, x, w, y, stream) -> int:
    """Raw call of the short-convolution + SiLU entry point (integer device addresses or None)."""
    return int(load_library().sla_short_conv_silu(int(dtype), int(B), int(T), int(channels), int(taps), _p(x), _p(w),
                                                   _p(y), _p(stream)))


def short_conv_silu(x, w):
    """x [B,T,C] (float32 or bfloat16), w [C,taps] float32 -> silu(causal depthwise convolution) [B,T,C]."""
    import torch

    assert x.is_cuda and x.is_contiguous() and x.dim() == 3
    B, T, C = x.shape
    assert w.dtype == torch.float32 and w.is_contiguous() and w.shape[0] == C
    y = torch.empty_like(x)
    dtype = {torch.float32: F32, torch.bfloat16: BF16}[x.dtype]
    rc = sla_short_conv_silu(dtype, B, T, C, w.shape[1], x.data_ptr(), w.data_ptr(), y.data_ptr(),
                             _stream(x))
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return y


def sla_short_conv_silu_l2(dtype, B, T, channels, taps, head_width, eps, x, w, y, stream) -> int:
    """Raw call of the feature map with the L2 option (integer device addresses or None)."""
    return int(load_library().sla_short_conv_silu_l2(int(dtype), int(B), int(T), int(channels), int(taps),
                                                      int(head_width), float(eps), _p(x), _p(w), _p(y), _p(stream)))


def sla_short_conv_silu_l2_backward_workspace_bytes(B, T, channels, taps) -> int:
    return int(load_library().sla_short_conv_silu_l2_backward_workspace_bytes(int(B), int(T), int(channels), int(taps)))


def sla_short_conv_silu_l2_backward(dtype, B, T, channels, taps, head_width, eps, x, w, dy, dx, dw, workspace,
                                    workspace_bytes, stream) -> int:
    """Raw call of the feature map's backward (integer device addresses or None)."""
    return int(load_library().sla_short_conv_silu_l2_backward(
        int(dtype), int(B), int(T), int(channels), int(taps), int(head_width), float(eps), _p(x), _p(w), _p(dy), _p(dx),
        _p(dw), _p(workspace), int(workspace_bytes), _p(stream)))


def sla_gate_logits_backward_workspace_bytes(params: SlaParams) -> int:
    return int(load_library().sla_gate_logits_backward_workspace_bytes(ctypes.byref(params)))


def sla_gate_logits_backward(params, x, w, d_head_logits, dx, dw, workspace, workspace_bytes, stream) -> int:
    """Raw call of one gate projection's backward (integer device addresses or None); dx is updated in place."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_gate_logits_backward(pr, _p(x), _p(w), _p(d_head_logits), _p(dx), _p(dw),
                                                        _p(workspace), int(workspace_bytes), _p(stream)))


def short_conv_silu_l2(x, w, head_width: int = 0, eps: float = 1e-6):
    """x [B,T,C], w [C,taps] float32 -> silu(conv) with every head of head_width channels L2-normalised."""
    import torch

    assert x.is_cuda and x.is_contiguous() and x.dim() == 3
    B, T, C = x.shape
    y = torch.empty_like(x)
    dtype = {torch.float32: F32, torch.bfloat16: BF16}[x.dtype]
    rc = sla_short_conv_silu_l2(dtype, B, T, C, w.shape[1], head_width, eps, x.data_ptr(), w.data_ptr(), y.data_ptr(),
                                _stream(x))
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return y


def short_conv_silu_l2_backward(x, w, dy, head_width: int = 0, eps: float = 1e-6):
    """Gradients (dx like x, dw [C,taps] float32) of ``short_conv_silu_l2`` for the cotangent dy."""
    import torch

    B, T, C = x.shape
    K = w.shape[1]
    dx = torch.empty_like(x)
    dw = torch.empty((C, K), dtype=torch.float32, device=x.device)
    need = sla_short_conv_silu_l2_backward_workspace_bytes(B, T, C, K)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    dtype = {torch.float32: F32, torch.bfloat16: BF16}[x.dtype]
    rc = sla_short_conv_silu_l2_backward(dtype, B, T, C, K, head_width, eps, x.data_ptr(), w.data_ptr(), dy.data_ptr(),
                                         dx.data_ptr(), dw.data_ptr(), ws.data_ptr(), ws.numel(),
                                         _stream(x))
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return dx, dw


def gate_logits_backward(x, w, d_head_logits, dx):
    """dx [B,T,H,dk] += d_head_logits[..., None] * w (in place); returns dw [H,dk] float32."""
    import torch

    B, T, H, dk = x.shape
    dtype = {torch.float32: F32, torch.bfloat16: BF16}[x.dtype]
    params = SlaParams(GLA, dtype, B, T, H, dk, 64, 0, 0, 1)
    dw = torch.empty((H, dk), dtype=torch.float32, device=x.device)
    need = sla_gate_logits_backward_workspace_bytes(params)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    rc = sla_gate_logits_backward(params, x.data_ptr(), w.data_ptr(), d_head_logits.data_ptr(), dx.data_ptr(),
                                  dw.data_ptr(), ws.data_ptr(), ws.numel(), _stream(x))
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return dw


def sla_gate_logits(params, q, k, w_gq, w_gk, q_head_logits, k_head_logits, stream) -> int:
    """Raw call of the gate-logit entry point: every pointer argument is an integer device address or None."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_gate_logits(pr, _p(q), _p(k), _p(w_gq), _p(w_gk), _p(q_head_logits),
                                               _p(k_head_logits), _p(stream)))


def gate_logits(q, k, w_gq, w_gk, *, dv: int = 0):
    """q, k [B,T,H,dk] (float32 or bfloat16; k may be None), w_gq, w_gk [H,dk] float32 -> (q_head_logits,
    k_head_logits) [B,T,H] float32 on the current CUDA(HIP) device and stream."""
    import torch

    assert q.is_cuda and q.is_contiguous()
    B, T, H, dk = q.shape
    dtype = {torch.float32: F32, torch.bfloat16: BF16}[q.dtype]
    assert w_gq.dtype == torch.float32 and tuple(w_gq.shape) == (H, dk) and w_gq.is_contiguous()
    ql = torch.empty((B, T, H), dtype=torch.float32, device=q.device)
    kl = None
    if k is not None:
        assert k.shape == q.shape and k.dtype == q.dtype and k.is_contiguous()
        assert w_gk.dtype == torch.float32 and tuple(w_gk.shape) == (H, dk) and w_gk.is_contiguous()
        kl = torch.empty_like(ql)
    params = SlaParams(GLA, dtype, B, T, H, dk, dv or dk, 0, 0, 1)
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = sla_gate_logits(params, ptr(q), ptr(k), ptr(w_gq), ptr(w_gk), ptr(ql), ptr(kl),
                         _stream(q))
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return ql, kl


def sla_backward_chunks_workspace_bytes(params: SlaParams, packed: bool = False) -> int:
    return int(load_library().sla_backward_chunks_workspace_bytes(ctypes.byref(params), int(bool(packed))))


def sla_backward_workspace_bytes(params: SlaParams) -> int:
    return int(load_library().sla_backward_workspace_bytes(ctypes.byref(params)))


def sla_backward(params, q, k, v, q_head_logits, k_head_logits, log_decay, initial_state, d_out, d_final_state,
                 dq, dk, dv, dq_head_logits, dk_head_logits, dlog_decay, d_initial_state, workspace, workspace_bytes,
                 stream) -> int:
    """Raw call of the backward entry point: every pointer argument is an integer device address or None."""
    pr = ctypes.byref(params) if params is not None else None
    return int(
        load_library().sla_backward(
            pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(initial_state),
            _p(d_out), _p(d_final_state), _p(dq), _p(dk), _p(dv), _p(dq_head_logits), _p(dk_head_logits),
            _p(dlog_decay), _p(d_initial_state), _p(workspace), int(workspace_bytes), _p(stream),
        )
    )


def backward(variant: int, q, k, v, q_head_logits, k_head_logits, log_decay, d_out, initial_state=None,
             d_final_state=None, *, want_d_initial_state: bool = False, workspace=None, head_major: bool = False,
             segments: int = 1):
    """Gradients of ``forward`` (RetNet, GLA; bfloat16 or float32) on the current CUDA(HIP) device and stream.  Returns a
    dict of new tensors: dq, dk, dv, dq_head_logits, dk_head_logits (None without k_head_logits), dlog_decay (GLA only,
    else None) and d_initial_state (None unless asked for).

    bfloat16: most calls run chunk-parallel in the workspace that is allocated here, whatever ``segments`` says; long rows with
    few heads, and calls given a ``workspace`` of sla_backward_workspace_bytes, run in that many segments per row that work in
    parallel (>= 2), or in one pass (1); 0 asks ``sla_backward_segments`` for the count that fills this device.  float32:
    ``segments`` must be 0 or 1; the library cuts rows over 128 tokens of batches with few sequences by itself, unless a
    ``workspace`` is given that only has the room of the single pass.  The schedules differ in the rounding of operands."""
    import torch

    assert q.is_cuda and q.dtype in (torch.bfloat16, torch.float32)
    if head_major:  # q, k, v, d_out, the GLA decay and their gradients are [B,H,T,d]
        B, H, T, dk = q.shape
    else:
        B, T, H, dk = q.shape
    dv = v.shape[-1]
    wide = (lambda d: (B, H, T, d)) if head_major else (lambda d: (B, T, H, d))
    for t, shape, dt in ((q, wide(dk), q.dtype), (k, wide(dk), q.dtype), (v, wide(dv), q.dtype),
                         (d_out, wide(dv), q.dtype), (q_head_logits, (B, T, H), torch.float32),
                         (k_head_logits, (B, T, H), torch.float32), (initial_state, (B, H, dk, dv), torch.float32),
                         (d_final_state, (B, H, dk, dv), torch.float32)):
        assert t is None or (tuple(t.shape) == shape and t.dtype == dt and t.is_contiguous() and t.is_cuda)
    want = {RETNET: ((H,), torch.float32), GLA: (tuple(q.shape), q.dtype)}[variant]
    assert tuple(log_decay.shape) == want[0] and log_decay.dtype == want[1] and log_decay.is_contiguous()
    dev = q.device
    g = {
        "dq": torch.empty_like(q),
        "dk": torch.empty_like(k),
        "dv": torch.empty_like(v),
        "dq_head_logits": torch.empty_like(q_head_logits),
        "dk_head_logits": None if k_head_logits is None else torch.empty_like(k_head_logits),
        "dlog_decay": torch.empty_like(log_decay) if variant == GLA else None,
        "d_initial_state": torch.empty((B, H, dk, dv), dtype=torch.float32, device=dev) if want_d_initial_state else None,
    }
    params = SlaParams(variant, BF16 if q.dtype == torch.bfloat16 else F32, B, T, H, dk, dv, 0,
                       FLAG_HEAD_MAJOR if head_major else 0, max(int(segments), 1))
    if int(segments) == 0:
        cus = torch.cuda.get_device_properties(q.device).multi_processor_count
        params.segments = max(sla_backward_segments(params, cus), 1)
    if workspace is None:
        workspace = _workspace(dev, sla_backward_chunks_workspace_bytes(params), lambda: sla_backward_workspace_bytes(params))
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = sla_backward(
        params, ptr(q), ptr(k), ptr(v), ptr(q_head_logits), ptr(k_head_logits), ptr(log_decay), ptr(initial_state),
        ptr(d_out), ptr(d_final_state), ptr(g["dq"]), ptr(g["dk"]), ptr(g["dv"]), ptr(g["dq_head_logits"]),
        ptr(g["dk_head_logits"]), ptr(g["dlog_decay"]), ptr(g["d_initial_state"]), ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(q),
    )
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return g


def sla_backward_gdn_workspace_bytes(params: SlaParams) -> int:
    return int(load_library().sla_backward_gdn_workspace_bytes(ctypes.byref(params)))


def sla_backward_gdn_chunks_workspace_bytes(params: SlaParams, packed: bool = False) -> int:
    return int(load_library().sla_backward_gdn_chunks_workspace_bytes(ctypes.byref(params), int(bool(packed))))


def sla_backward_gdn(params, q, k, v, q_head_logits, k_head_logits, log_decay, beta, initial_state, d_out,
                     d_final_state, dq, dk, dv, dq_head_logits, dk_head_logits, dlog_decay, dbeta, d_initial_state,
                     workspace, workspace_bytes, stream) -> int:
    """Raw call of the gated delta rule's backward: every pointer argument is an integer device address or None."""
    pr = ctypes.byref(params) if params is not None else None
    return int(
        load_library().sla_backward_gdn(
            pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(beta),
            _p(initial_state), _p(d_out), _p(d_final_state), _p(dq), _p(dk), _p(dv), _p(dq_head_logits),
            _p(dk_head_logits), _p(dlog_decay), _p(dbeta), _p(d_initial_state), _p(workspace),
            ctypes.c_size_t(int(workspace_bytes)), _p(stream),
        )
    )


def sla_backward_gdn_varlen_workspace_bytes(params: SlaParams) -> int:
    return int(load_library().sla_backward_gdn_varlen_workspace_bytes(ctypes.byref(params)))


def sla_backward_gdn_varlen(params, q, k, v, q_head_logits, k_head_logits, log_decay, beta, cu_seqlens, initial_state,
                            d_out, d_final_state, dq, dk, dv, dq_head_logits, dk_head_logits, dlog_decay, dbeta,
                            d_initial_state, workspace, workspace_bytes, stream) -> int:
    """Raw call of the packed variable-length backward of the gated delta rule."""
    pr = ctypes.byref(params) if params is not None else None
    return int(
        load_library().sla_backward_gdn_varlen(
            pr, _p(q), _p(k), _p(v), _p(q_head_logits), _p(k_head_logits), _p(log_decay), _p(beta), _p(cu_seqlens),
            _p(initial_state), _p(d_out), _p(d_final_state), _p(dq), _p(dk), _p(dv), _p(dq_head_logits),
            _p(dk_head_logits), _p(dlog_decay), _p(dbeta), _p(d_initial_state), _p(workspace),
            ctypes.c_size_t(int(workspace_bytes)), _p(stream),
        )
    )


def backward_gdn_varlen(q, k, v, q_head_logits, k_head_logits, log_decay, beta, d_out, cu_seqlens, initial_state=None,
                        d_final_state=None, *, want_d_initial_state: bool = False):
    """Gradients of ``forward_varlen(GDN, ...)``: q, k [T,H,dk], v, d_out [T,H,dv] bfloat16; logits, log_decay, beta
    [T,H] float32; cu_seqlens [B+1] int32 on the device; states [B,H,dk,dv].  Returns a dict as ``backward_gdn``."""
    import torch

    assert q.is_cuda and q.dtype in (torch.bfloat16, torch.float32) and q.dim() == 3
    T, H, dk = q.shape
    dv = v.shape[-1]
    B = cu_seqlens.numel() - 1
    assert cu_seqlens.dtype == torch.int32 and cu_seqlens.is_cuda
    dev = q.device
    g = {
        "dq": torch.empty_like(q),
        "dk": torch.empty_like(k),
        "dv": torch.empty_like(v),
        "dq_head_logits": torch.empty_like(q_head_logits),
        "dk_head_logits": None if k_head_logits is None else torch.empty_like(k_head_logits),
        "dlog_decay": torch.empty_like(log_decay),
        "dbeta": torch.empty_like(beta),
        "d_initial_state": torch.empty((B, H, dk, dv), dtype=torch.float32, device=dev) if want_d_initial_state else None,
    }
    params = SlaParams(GDN, BF16 if q.dtype == torch.bfloat16 else F32, B, T, H, dk, dv, 0, 0, 1)
    workspace = _workspace(dev, sla_backward_gdn_chunks_workspace_bytes(params, packed=True),
                           lambda: sla_backward_gdn_varlen_workspace_bytes(params))
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = sla_backward_gdn_varlen(
        params, ptr(q), ptr(k), ptr(v), ptr(q_head_logits), ptr(k_head_logits), ptr(log_decay), ptr(beta),
        ptr(cu_seqlens), ptr(initial_state), ptr(d_out), ptr(d_final_state), ptr(g["dq"]), ptr(g["dk"]), ptr(g["dv"]),
        ptr(g["dq_head_logits"]), ptr(g["dk_head_logits"]), ptr(g["dlog_decay"]), ptr(g["dbeta"]),
        ptr(g["d_initial_state"]), ptr(workspace), workspace.numel(), _stream(q),
    )
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return g


def backward_gdn(q, k, v, q_head_logits, k_head_logits, log_decay, beta, d_out, initial_state=None,
                 d_final_state=None, *, want_d_initial_state: bool = False, workspace=None):
    """Gradients of ``forward(GDN, ...)`` (bfloat16 or float32 q, k, v, d_out [B,T,H,d]; float32 logits, log_decay and beta
    [B,T,H]) on the current CUDA(HIP) device and stream.  Returns a dict of new tensors: dq, dk, dv,
    dq_head_logits, dk_head_logits (None without k_head_logits), dlog_decay, dbeta and d_initial_state (None unless
    asked for)."""
    import torch

    assert q.is_cuda and q.dtype in (torch.bfloat16, torch.float32)
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    for t, shape, dt in ((q, (B, T, H, dk), q.dtype), (k, (B, T, H, dk), q.dtype), (v, (B, T, H, dv), q.dtype),
                         (d_out, (B, T, H, dv), q.dtype), (q_head_logits, (B, T, H), torch.float32),
                         (k_head_logits, (B, T, H), torch.float32), (log_decay, (B, T, H), torch.float32),
                         (beta, (B, T, H), torch.float32), (initial_state, (B, H, dk, dv), torch.float32),
                         (d_final_state, (B, H, dk, dv), torch.float32)):
        assert t is None or (tuple(t.shape) == shape and t.dtype == dt and t.is_contiguous() and t.is_cuda)
    dev = q.device
    g = {
        "dq": torch.empty_like(q),
        "dk": torch.empty_like(k),
        "dv": torch.empty_like(v),
        "dq_head_logits": torch.empty_like(q_head_logits),
        "dk_head_logits": None if k_head_logits is None else torch.empty_like(k_head_logits),
        "dlog_decay": torch.empty_like(log_decay),
        "dbeta": torch.empty_like(beta),
        "d_initial_state": torch.empty((B, H, dk, dv), dtype=torch.float32, device=dev) if want_d_initial_state else None,
    }
    params = SlaParams(GDN, BF16 if q.dtype == torch.bfloat16 else F32, B, T, H, dk, dv, 0, 0, 1)
    if workspace is None:
        workspace = _workspace(dev, sla_backward_gdn_chunks_workspace_bytes(params),
                               lambda: sla_backward_gdn_workspace_bytes(params))
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = sla_backward_gdn(
        params, ptr(q), ptr(k), ptr(v), ptr(q_head_logits), ptr(k_head_logits), ptr(log_decay), ptr(beta),
        ptr(initial_state), ptr(d_out), ptr(d_final_state), ptr(g["dq"]), ptr(g["dk"]), ptr(g["dv"]),
        ptr(g["dq_head_logits"]), ptr(g["dk_head_logits"]), ptr(g["dlog_decay"]), ptr(g["dbeta"]),
        ptr(g["d_initial_state"]), ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(q),
    )
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return g


def decode_step(variant: int, q, k, v, q_head_logits, k_head_logits, log_decay, beta, state, *, out=None,
                w_gq=None, w_gk=None):
    """One recurrent step on the current CUDA(HIP) device and stream: q, k [B,H,dk], v [B,H,dv], logits / beta
    [B,H] float32, state [B,H,dk,dv] float32 (updated in place).  Returns out [B,H,dv].  With w_gq (and
    optionally w_gk) [H,dk] float32 the kernel forms the logits itself (sla_decode_step_fused) and the two logits
    arguments must be None."""
    import torch

    B, H, dk = q.shape
    dv = v.shape[-1]
    dtype = BF16 if q.dtype is torch.bfloat16 else {torch.float32: F32}[q.dtype]
    f32 = torch.float32
    assert state.dtype is f32 and state.shape == (B, H, dk, dv) and state.is_contiguous()
    if w_gq is not None:
        assert q_head_logits is None and k_head_logits is None
        for w in (w_gq, w_gk):
            assert w is None or (w.dtype is f32 and w.shape == (H, dk) and w.is_contiguous())
        call, gq, gk = load_library().sla_decode_step_fused, w_gq, w_gk
    else:
        assert q.is_cuda and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
        assert k.shape == (B, H, dk) and v.shape == (B, H, dv) and k.dtype is q.dtype and v.dtype is q.dtype
        assert q_head_logits.dtype is f32 and q_head_logits.shape == (B, H) and q_head_logits.is_contiguous()
        if k_head_logits is not None:
            assert k_head_logits.dtype is f32 and k_head_logits.shape == (B, H) and k_head_logits.is_contiguous()
        want = {RETNET: ((H,), f32), GLA: ((B, H, dk), q.dtype), GDN: ((B, H), f32)}[variant]
        assert log_decay.shape == want[0] and log_decay.dtype is want[1] and log_decay.is_contiguous()
        if beta is not None:
            assert beta.dtype is f32 and beta.shape == (B, H) and beta.is_contiguous()
        call, gq, gk = load_library().sla_decode_step, q_head_logits, k_head_logits
    if out is None:
        out = q.new_empty((B, H, dv))
    # a token's host time is part of every step: the arguments go to the C entry point without the raw wrappers between
    rc = call(ctypes.byref(SlaParams(variant, dtype, B, 1, H, dk, dv, 0, 0, 1)), q.data_ptr(),
              None if k is None else k.data_ptr(), v.data_ptr(), gq.data_ptr(), None if gk is None else gk.data_ptr(),
              None if log_decay is None else log_decay.data_ptr(),
              None if beta is None else beta.data_ptr(), state.data_ptr(), out.data_ptr(), _stream(q))
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return out


_cus = {}


def _compute_units(device) -> int:
    import torch

    i = torch.device(device).index
    i = torch.cuda.current_device() if i is None else i
    if i not in _cus:
        _cus[i] = torch.cuda.get_device_properties(i).multi_processor_count
    return _cus[i]


def forward(
    variant: int,
    q,
    k,
    v,
    q_head_logits,
    k_head_logits,
    log_decay,
    beta=None,
    initial_state=None,
    *,
    dv_split: int = 0,
    out=None,
    final_state=None,
    want_final_state: bool = True,
    segments: int = 1,
    workspace=None,
    head_major: bool = False,
) -> Tuple["torch.Tensor", Optional["torch.Tensor"]]:
    """SLA forward on the current CUDA(HIP) device and stream.  Tensors must be contiguous CUDA tensors:
    q,k [B,T,H,dk], v [B,T,H,dv] in float32 or bfloat16; logits/beta/initial_state float32.

    segments = 1 runs one fused pass (sla_forward).  segments = 0 lets the library choose the
    segment-parallel schedule, segments > 1 asks for that many segments (sla_forward_ws); the workspace
    is then taken from ``workspace`` (a CUDA tensor of at least sla_workspace_bytes bytes; sla_forward_workspace_bytes of them run
    fastest) or allocated here.

    head_major = True: q, k, v (and the GLA log_decay, and the returned out) are [B,H,T,d] (SLA_FLAG_HEAD_MAJOR)."""
    import torch

    assert q.is_cuda and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
    if head_major:
        B, H, T, dk = q.shape
    else:
        B, T, H, dk = q.shape
    dv = v.shape[-1]
    assert k.shape == q.shape and v.shape == q.shape[:3] + (dv,) and k.dtype == q.dtype and v.dtype == q.dtype
    dtype = {torch.float32: F32, torch.bfloat16: BF16}[q.dtype]
    assert q_head_logits.dtype == torch.float32 and q_head_logits.shape == (B, T, H) and q_head_logits.is_contiguous()
    if k_head_logits is not None:
        assert k_head_logits.dtype == torch.float32 and k_head_logits.shape == (B, T, H) and k_head_logits.is_contiguous()
    want = {RETNET: ((H,), torch.float32), GLA: (tuple(q.shape), q.dtype), GDN: ((B, T, H), torch.float32)}[variant]
    assert tuple(log_decay.shape) == want[0] and log_decay.dtype == want[1] and log_decay.is_contiguous()
    if beta is not None:
        assert beta.dtype == torch.float32 and beta.shape == (B, T, H) and beta.is_contiguous()
    if initial_state is not None:
        assert initial_state.dtype == torch.float32 and initial_state.shape == (B, H, dk, dv) and initial_state.is_contiguous()
    if out is None:
        out = torch.empty(tuple(v.shape), dtype=q.dtype, device=q.device)
    if final_state is None and want_final_state:
        final_state = torch.empty((B, H, dk, dv), dtype=torch.float32, device=q.device)
    params = SlaParams(variant, dtype, B, T, H, dk, dv, dv_split, FLAG_HEAD_MAJOR if head_major else 0, segments)
    ptr = lambda t: None if t is None else t.data_ptr()
    stream = _stream(q)
    if segments == 1:
        rc = sla_forward(
            params, ptr(q), ptr(k), ptr(v), ptr(q_head_logits), ptr(k_head_logits), ptr(log_decay), ptr(beta),
            ptr(initial_state), ptr(out), ptr(final_state), stream,
        )
    else:
        need = sla_forward_workspace_bytes(params, _compute_units(q.device))
        if workspace is None and need > 0:
            workspace = _workspace(q.device, need, lambda: sla_workspace_bytes(params, _compute_units(q.device)))
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        rc = sla_forward_ws(
            params, ptr(q), ptr(k), ptr(v), ptr(q_head_logits), ptr(k_head_logits), ptr(log_decay), ptr(beta),
            ptr(initial_state), ptr(out), ptr(final_state), ptr(workspace), ws_bytes, stream,
        )
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))
    return out, final_state


# ---------------------------------------------------------------------------------------------------------------------
# Around the mixer: rotary positions, the normalised and gated read-out, the join with the residual stream.
#
# Scalars (magnitude, eps, scale) are numbers; where a tensor holds one, its value is read on the host at every call.  With cu_seqlens,
# rows outside every sequence stay as they were in an output that is passed and are undefined in a new one.

def sla_rotary(params, q, k, frequencies, positions, cu_seqlens, q_out, k_out, stream) -> int:
    """Raw call: integer device addresses (0/None = NULL) and a hipStream_t handle.  Returns the status code."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_rotary(pr, _p(q), _p(k), _p(frequencies), _p(positions), _p(cu_seqlens), _p(q_out),
                                         _p(k_out), _p(stream)))


def sla_rotary_backward(params, dq_out, dk_out, frequencies, positions, cu_seqlens, dq, dk, stream) -> int:
    """Raw call of the rotary gradient (same conventions as sla_rotary)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_rotary_backward(pr, _p(dq_out), _p(dk_out), _p(frequencies), _p(positions),
                                                  _p(cu_seqlens), _p(dq), _p(dk), _p(stream)))


def sla_norm_gate(params, x, g, w, cu_seqlens, y, stream) -> int:
    """Raw call of the read-out norm (integer device addresses or None)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_norm_gate(pr, _p(x), _p(g), _p(w), _p(cu_seqlens), _p(y), _p(stream)))


def sla_norm_gate_backward_workspace_bytes(params, packed: bool = False) -> int:
    return int(load_library().sla_norm_gate_backward_workspace_bytes(ctypes.byref(params), int(bool(packed))))


def sla_norm_gate_backward(params, x, g, w, dy, cu_seqlens, dx, dg, dw, workspace, workspace_bytes, stream) -> int:
    """Raw call of the read-out norm's gradients (integer device addresses or None)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_norm_gate_backward(pr, _p(x), _p(g), _p(w), _p(dy), _p(cu_seqlens), _p(dx), _p(dg),
                                                     _p(dw), _p(workspace), int(workspace_bytes), _p(stream)))


def sla_join_norm(params, x, h, w_after, channel_scale, w_before, cu_seqlens, x_out, y, stream) -> int:
    """Raw call of the residual join (integer device addresses or None)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_join_norm(pr, _p(x), _p(h), _p(w_after), _p(channel_scale), _p(w_before),
                                            _p(cu_seqlens), _p(x_out), _p(y), _p(stream)))


def sla_join_norm_backward_workspace_bytes(params, packed: bool = False) -> int:
    return int(load_library().sla_join_norm_backward_workspace_bytes(ctypes.byref(params), int(bool(packed))))


def sla_join_norm_backward(params, x_out, h, w_after, channel_scale, w_before, dy, dx_out, cu_seqlens, dx, dh, dw_after,
                           dchannel_scale, dw_before, workspace, workspace_bytes, stream) -> int:
    """Raw call of the residual join's gradients (integer device addresses or None)."""
    pr = ctypes.byref(params) if params is not None else None
    return int(load_library().sla_join_norm_backward(
        pr, _p(x_out), _p(h), _p(w_after), _p(channel_scale), _p(w_before), _p(dy), _p(dx_out), _p(cu_seqlens), _p(dx),
        _p(dh), _p(dw_after), _p(dchannel_scale), _p(dw_before), _p(workspace), int(workspace_bytes), _p(stream)))


def _need(ok, text):
    if not ok:
        raise ValueError(text)


def _tensor(name, t, device, shape, dtype):
    """Refuses what the library could not check: a tensor of another device, type, shape or order."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on GPU {device}, but got "
                         f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _ptr(t):
    return None if t is None else t.data_ptr()


# Parameter blocks by value: a token's host time is part of every step, and building one costs a microsecond.  Fields are Python
# numbers: an object that holds one, such as a tensor, would be found again by its identity after its value has changed.
@functools.lru_cache(maxsize=1024)
def _params(kind, *fields):
    return ctypes.byref(kind(*fields))


# The fields up to the scalars, which no size depends on.
@functools.lru_cache(maxsize=1024)
def _workspace_size(kind, *fields, packed):
    query = sla_norm_gate_backward_workspace_bytes if kind is SlaNormGateParams else sla_join_norm_backward_workspace_bytes
    return max(query(kind(*fields), packed), 16)


def _workspace_bytes(workspace, like):
    _need(workspace.is_contiguous() and workspace.get_device() == like.get_device(), f"workspace: expected contiguous memory on {like.device}")
    return workspace.numel() * workspace.element_size()


def _run(call, t, *args):
    """One call of the library on the current stream of t's device, with that device the current one; raises on a status."""
    c = sys.modules["torch"]._C
    device = t.get_device()
    if device >= 0 and device == c._cuda_getDevice():
        rc = call(*args, c._cuda_getCurrentRawStream(device))
    else:
        stream = _stream(t)
        with sys.modules["torch"].cuda.device(device):
            rc = call(*args, stream)
    if rc != 0:
        raise SlaError(rc, sla_status_string(rc))


def _element(name, dtype):
    torch = sys.modules["torch"]
    if dtype is torch.bfloat16:
        return BF16
    if dtype is not torch.float32:
        raise ValueError(f"{name}: expected bfloat16 or float32, but got {dtype}")
    return F32


def _sequences(name, cu_seqlens, device):
    """The number of sequences that cu_seqlens bounds."""
    _need(cu_seqlens.dim() == 1 and cu_seqlens.numel() >= 1, f"{name}: cu_seqlens is [B+1]")
    _tensor("cu_seqlens", cu_seqlens, device, cu_seqlens.shape, sys.modules["torch"].int32)
    return cu_seqlens.numel() - 1


def _batch(name, t, cu_seqlens, head_major):
    """(B, T, H, width) of a contiguous tensor of head vectors: [B,T,H,d] ([B,H,T,d] head-major); [T,H,d] with cu_seqlens;
    [B,H,d] without: one token of each of B sequences, as decode_step has them."""
    shape = t.shape
    if cu_seqlens is not None:
        _need(len(shape) == 3 and not head_major, f"{name}: a packed batch is [T,H,d]")
        B = _sequences(name, cu_seqlens, t.get_device())
        T, H, d = shape
    elif len(shape) == 4:
        B, T, H, d = shape
        if head_major:
            T, H = H, T
    else:
        _need(len(shape) == 3 and not head_major, f"{name}: expected [B,T,H,d], [T,H,d] with cu_seqlens or [B,H,d]")
        B, H, d = shape
        T = 1
    if (B | T | H | d) >> 31 or not t.is_contiguous():
        raise ValueError(f"{name}: {tuple(shape)} with strides {t.stride()} is not contiguous or out of range")
    return B, T, H, d


def rotary_frequencies(width: int, base: float = 10000.0, *, scaling: str = "none", factor: float = 1.0,
                       original_length: int = 4096, fast: float = 32.0, slow: float = 1.0, device=None):
    """(frequencies [width/2] float64 on ``device`` (default: the current GPU), magnitude) for ``rotary``: pair i turns by
    base^(-2i/width) radians a token.  For contexts of ``factor`` times the trained ``original_length``: "linear" divides every
    frequency by factor (position interpolation); "base" multiplies base by factor^(width/(width-2)), so that the slowest pair
    is slowed by factor and the fastest not at all; "blend" slows the pairs that turn fewer than ``slow`` times in the trained
    length, keeps those over ``fast`` times, goes from one to the other linearly in the turns, and scales what is turned by
    0.1 ln(factor) + 1 (YaRN, arXiv 2309.00071)."""
    import math

    import torch

    _need(width >= 2 and width % 2 == 0, f"width: expected an even number of elements, but got {width}")
    _need(scaling in ("none", "linear", "base", "blend"), f"scaling: unknown {scaling!r}")
    _need(factor > 0 and base > 0 and (scaling != "blend" or (factor >= 1 and 0 < slow < fast and original_length > 0)),
          "factor, base, fast, slow or original_length out of range")
    if scaling == "base" and width > 2:
        base = base * factor ** (width / (width - 2))
    f = torch.tensor([base ** (-2.0 * i / width) for i in range(width // 2)], dtype=torch.float64)
    magnitude = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "blend":
        turns = f * (original_length / (2.0 * math.pi))
        keep = torch.clamp((turns - slow) / (fast - slow), 0.0, 1.0)
        f = f * keep + f / factor * (1.0 - keep)
        magnitude = 0.1 * math.log(factor) + 1.0
    return f.to(device if device is not None else "cuda"), magnitude


def _rotary(call, q, k, frequencies, start, positions, cu_seqlens, adjacent, magnitude, head_major, q_out, k_out):
    torch = sys.modules["torch"]
    device, el, Hk = q.get_device(), q.dtype, 0
    B, T, Hq, d = _batch("q", q, cu_seqlens, head_major)
    if k is not None:
        Bk, Tk, Hk, dk = _batch("k", k, cu_seqlens, head_major)
        if Bk != B or Tk != T or dk != d or k.dtype is not el or k.get_device() != device:
            raise ValueError(f"k: {k.dtype} {tuple(k.shape)} on {k.device} does not go with q: {el} {tuple(q.shape)} on {q.device}")
    pairs = frequencies.numel()
    _tensor("frequencies", frequencies, device, (pairs,), torch.float64)
    flags = (FLAG_HEAD_MAJOR if head_major else 0) | (FLAG_ADJACENT_PAIRS if adjacent else 0)
    where = start
    if start is not None:
        _need(positions is None, "start and positions: give one of them")
        _tensor("start", start, device, (B,), torch.int32)
    elif positions is not None:
        _tensor("positions", positions, device, (T,) if cu_seqlens is not None else (B, T) if q.dim() == 4 else (B,), torch.int32)
        where, flags = positions, flags | FLAG_TOKEN_POSITIONS
    fresh = q_out is None and k_out is None
    if q_out is None:
        q_out = torch.empty_like(q)
    else:
        _tensor("q's output", q_out, device, q.shape, el)
    if k is None:
        _need(k_out is None, "an output for k, but no k")
    elif k_out is None:
        k_out = torch.empty_like(k)
    else:
        _tensor("k's output", k_out, device, k.shape, el)
    if not fresh and k is not None and q.numel():
        _need(q_out.data_ptr() != k.data_ptr() and k_out.data_ptr() not in (q.data_ptr(), q_out.data_ptr()),
              "an output may lie on its own input only")
    _run(call, q, _params(SlaRotaryParams, _element("q", el), B, T, Hq, Hk, d, 2 * pairs, flags, float(magnitude)), q.data_ptr(),
         _ptr(k), frequencies.data_ptr(), _ptr(where), _ptr(cu_seqlens), q_out.data_ptr(), _ptr(k_out))
    return q_out, k_out


def rotary(q, k, frequencies, *, start=None, positions=None, cu_seqlens=None, adjacent: bool = False,
           magnitude: float = 1.0, head_major: bool = False, q_out=None, k_out=None):
    """Turns the first 2 * len(frequencies) elements of every head vector of q [B,T,Hq,d] and k [B,T,Hk,d] (or None) by
    position * frequency (sla_rotary); returns (q_out, k_out).  Head vectors may also be [B,H,T,d] (head_major), [T,H,d] with
    cu_seqlens int32 [B+1], or [B,H,d]: one token of each of B sequences.  Positions count from 0 in every sequence, or from
    start int32 [B], or are positions int32 [B,T] ([T] packed, [B] for one token each).  frequencies float64, see
    ``rotary_frequencies``.  q_out and k_out may be q and k."""
    return _rotary(load_library().sla_rotary, q, k, frequencies, start, positions, cu_seqlens, adjacent, magnitude,
                   head_major, q_out, k_out)


def rotary_backward(dq_out, dk_out, frequencies, *, start=None, positions=None, cu_seqlens=None, adjacent: bool = False,
                    magnitude: float = 1.0, head_major: bool = False, dq=None, dk=None):
    """Gradients (dq, dk) of ``rotary`` from the cotangents of its outputs (arguments as there); dq may be dq_out."""
    return _rotary(load_library().sla_rotary_backward, dq_out, dk_out, frequencies, start, positions, cu_seqlens, adjacent,
                   magnitude, head_major, dq, dk)


def _norm_gate_args(x, g, w, eps, gate, cu_seqlens, head_major):
    """The parameter block, and the shape of everything but x and dx."""
    torch = sys.modules["torch"]
    device, el, shape = x.get_device(), x.dtype, x.shape
    B, T, H, dv = _batch("x", x, cu_seqlens, head_major)
    flags = 0
    if head_major:
        shape, flags = torch.Size((B, T, H, dv)), FLAG_HEAD_MAJOR
    kind = GATES.get(gate)
    if kind is None or (g is None) != (kind == 0):
        raise ValueError(f"gate: {gate!r} {'with' if g is not None else 'without'} g; expected 'silu' or 'sigmoid' with, 'none' without")
    if g is not None:
        _tensor("g", g, device, shape, el)
    if w is not None:
        if w.dim() == 2:
            flags |= FLAG_HEAD_WEIGHTS
            _tensor("w", w, device, (H, dv), torch.float32)
        else:
            _tensor("w", w, device, (dv,), torch.float32)
    return (SlaNormGateParams, _element("x", el), B, T, H, dv, kind, flags, float(eps)), shape


def norm_gate(x, g, w, *, gate: str = "silu", eps: float = 1e-5, cu_seqlens=None, head_major: bool = False, out=None):
    """The read-out behind the mixer: y = x / sqrt(mean(x^2) + eps) * w * act(g) over every head vector (sla_norm_gate).
    x, g [B,T,H,dv] ([T,H,dv] with cu_seqlens, [B,H,dv] for one token each), w float32 [dv], [H,dv] or None; gate "silu",
    "sigmoid" or "none" (then g is None).  head_major: x is [B,H,T,dv], g and y are [B,T,H,dv].  ``out`` may be g or, without
    head_major, x.  A norm over each head divides out the mixer's read gate, which scales the head's whole vector; ``join_norm`` of
    x.view(B, T, H * dv) with h None normalises over all heads and keeps it."""
    params, shape = _norm_gate_args(x, g, w, eps, gate, cu_seqlens, head_major)
    if out is None:
        out = x.new_empty(shape) if head_major else sys.modules["torch"].empty_like(x)
    else:
        _tensor("out", out, x.get_device(), shape, x.dtype)
        _need(not head_major or out.data_ptr() != x.data_ptr() or not x.numel(), "out may not be x, which is laid out differently")
    _run(load_library().sla_norm_gate, x, _params(*params), x.data_ptr(), _ptr(g), _ptr(w), _ptr(cu_seqlens), out.data_ptr())
    return out


def norm_gate_backward(x, g, w, dy, *, gate: str = "silu", eps: float = 1e-5, cu_seqlens=None, head_major: bool = False,
                       workspace=None):
    """Gradients of ``norm_gate`` for the cotangent dy of y, as a dict of new tensors: dx like x, dg like g (or None), dw like w
    (or None).  ``workspace``: a tensor of sla_norm_gate_backward_workspace_bytes, else it is allocated here."""
    torch = sys.modules["torch"]
    params, shape = _norm_gate_args(x, g, w, eps, gate, cu_seqlens, head_major)
    _tensor("dy", dy, x.get_device(), shape, x.dtype)
    dx = torch.empty_like(x)
    dg = None if g is None else torch.empty_like(g)
    dw = None if w is None else torch.empty_like(w)
    size = 0
    if workspace is not None:
        size = _workspace_bytes(workspace, x)
    elif dw is not None:
        size = _workspace_size(*params[:-1], packed=cu_seqlens is not None)
        workspace = x.new_empty(size, dtype=torch.uint8)
    _run(load_library().sla_norm_gate_backward, x, _params(*params), x.data_ptr(), _ptr(g), _ptr(w), dy.data_ptr(),
         _ptr(cu_seqlens), dx.data_ptr(), _ptr(dg), _ptr(dw), _ptr(workspace), size)
    return {"dx": dx, "dg": dg, "dw": dw}


def _join_args(x, one, other, w_after, channel_scale, w_before, scale, eps, cu_seqlens, y_dtype=None):
    """The parameter block for the stream x [..., D] and the block's tensors ``one`` and ``other``, of one type: that of y_dtype or of
    the stream where there are none."""
    torch = sys.modules["torch"]
    device, shape, el = x.get_device(), x.shape, x.dtype
    _need(len(shape) >= 1 and x.is_contiguous(), "x: expected a contiguous tensor [..., D]")
    D = shape[-1]
    kind = y_dtype or el
    if one is not None:
        kind = one.dtype
        _tensor("h or dy", one, device, shape, kind)
        if other is not None:
            _tensor("h or y", other, device, shape, kind)
    elif other is not None:
        kind = other.dtype
        _tensor("h or y", other, device, shape, kind)
    if w_before is not None:
        _tensor("w_before", w_before, device, (D,), torch.float32)
    if w_after is not None:
        _tensor("w_after", w_after, device, (D,), torch.float32)
    if channel_scale is not None:
        _tensor("channel_scale", channel_scale, device, (D,), torch.float32)
    if cu_seqlens is not None:
        _need(len(shape) == 2, "x: a packed batch is [T,D]")
        B, T = _sequences("x", cu_seqlens, device), shape[0]
    else:
        B, T = 1, x.numel() // D if D else 0
    if (T | D) >> 31:
        raise ValueError(f"x: {tuple(shape)} is out of range")
    return SlaJoinNormParams, _element("h", kind), _element("x", el), B, T, D, float(scale), float(eps)


def join_norm(x, h, w_before, *, w_after=None, channel_scale=None, scale: float = 1.0, eps: float = 1e-5, cu_seqlens=None,
              x_out=None, y=None, y_dtype=None):
    """A block's output h joins the residual stream x, and the stream is normalised for the next block (sla_join_norm):
    u = h, or h / rms(h) * w_after;  x_out = x + scale * channel_scale * u;  y = x_out / rms(x_out) * w_before.  x, h [..., D]
    ([T,D] with cu_seqlens), x float32 or of h's type; weights float32 [D].  Returns (x_out, y).  h None: no join, x_out is x, and
    y has y_dtype (default: y's type if it is given, else x's); w_before None: no norm, y is None.  ``x_out`` may be x and ``y`` may be h."""
    torch = sys.modules["torch"]
    if h is None:
        _need(w_before is not None and w_after is None and channel_scale is None and x_out is None,
              "h: needed, unless only the norm of x is asked for")
    _need(w_before is not None or y is None, "an output y, but no w_before")
    if y_dtype is not None and w_before is not None:
        like = h if h is not None else y
        _need(like is None or like.dtype is y_dtype, "y_dtype: y has the type of h, or of the tensor given for it")
    params = _join_args(x, h, y, w_after, channel_scale, w_before, scale, eps, cu_seqlens, y_dtype)
    if y is not None and x.numel():
        _need(y.data_ptr() not in (x.data_ptr(), _ptr(x_out)), "y may lie on h only")
    if h is not None:
        if x_out is None:
            x_out = torch.empty_like(x)
        else:
            _tensor("x_out", x_out, x.get_device(), x.shape, x.dtype)
            _need(x_out.data_ptr() != h.data_ptr() or not x.numel(), "x_out may lie on x only")
    if w_before is not None and y is None:
        y = torch.empty_like(x, dtype=y_dtype) if h is None else torch.empty_like(h)
    _run(load_library().sla_join_norm, x, _params(*params), x.data_ptr(), _ptr(h), _ptr(w_after), _ptr(channel_scale),
         _ptr(w_before), _ptr(cu_seqlens), _ptr(x_out), _ptr(y))
    return (x if h is None else x_out), y


def join_norm_backward(x_out, h, w_before, dy, dx_out=None, *, w_after=None, channel_scale=None, scale: float = 1.0,
                       eps: float = 1e-5, cu_seqlens=None, workspace=None):
    """Gradients of ``join_norm`` from its x_out, for the cotangents dy of y and dx_out of x_out (None: zero), as a dict:
    dx, dh, dw_after, dchannel_scale, dw_before (None where the forward had no such input).  Without w_before (and dy) dx is
    dx_out itself.  h is read only with w_after or channel_scale; None: the forward only normalised x.  ``workspace``: a tensor of
    sla_join_norm_backward_workspace_bytes, else it is allocated here."""
    torch = sys.modules["torch"]
    _need((dy is None) == (w_before is None) and (dy is not None or dx_out is not None), "dy goes with w_before; without them dx_out")
    _need(h is not None or (w_after is None and channel_scale is None), "h: needed with w_after or channel_scale")
    params = _join_args(x_out, dy, h, w_after, channel_scale, w_before, scale, eps, cu_seqlens)
    if dx_out is not None:
        _tensor("dx_out", dx_out, x_out.get_device(), x_out.shape, x_out.dtype)
    like = torch.empty_like
    dx = dx_out if dy is None else like(x_out)
    dh = None if h is None else like(h)
    dw_after = None if w_after is None else like(w_after)
    dchannel = None if channel_scale is None else like(channel_scale)
    dw_before = None if w_before is None else like(w_before)
    if dy is not None or h is not None:
        size = 0
        if workspace is not None:
            size = _workspace_bytes(workspace, x_out)
        elif dy is not None or dw_after is not None or dchannel is not None:
            size = _workspace_size(*params[:-2], packed=cu_seqlens is not None)
            workspace = x_out.new_empty(size, dtype=torch.uint8)
        _run(load_library().sla_join_norm_backward, x_out, _params(*params), x_out.data_ptr(), _ptr(h), _ptr(w_after),
             _ptr(channel_scale), _ptr(w_before), _ptr(dy), _ptr(dx_out), _ptr(cu_seqlens), None if dy is None else dx.data_ptr(),
             _ptr(dh), _ptr(dw_after), _ptr(dchannel), _ptr(dw_before), _ptr(workspace), size)
    return {"dx": dx, "dh": dh, "dw_after": dw_after, "dchannel_scale": dchannel, "dw_before": dw_before}
