"""ctypes binding of ``include/gla.h`` (argument marshalling only).

Tensors are torch tensors on an AMD GPU; torch is used for device memory and
the current stream, nothing else.  Every arithmetic step runs inside
``libgla.so``; if that library has not been built the calls raise.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
import re
from typing import List, Optional

SCAN_ROW_FWD, SCAN_ROW_REV, SCAN_COL_FWD, SCAN_COL_REV = 0, 1, 2, 3
DT_F32, DT_BF16 = 0, 1
OPT_CHUNKS_PER_SPAN, OPT_ENGINE, OPT_CARRY, OPT_BWD_SPLIT, OPT_RANGE_FALLBACK, OPT_LOOK_BACK_POLLS, OPT_GLU_SPLIT = 0, 1, 2, 3, 4, 5, 6
CARRY_AUTO, CARRY_KERNEL, CARRY_IN_OUTPUT_PASS = 0, 1, 2
LAYOUT_BHTD, LAYOUT_BTHD = 0, 1
DECAY_HEAD, DECAY_TOKEN = 0, 1
ROPE_ADJACENT, ROPE_HALVES = 0, 1
GATE_LOG, GATE_PRE = 0, 1
ACT_SILU, ACT_GELU, ACT_GELU_TANH = 0, 1, 2
ENGINE_AUTO, ENGINE_RECURRENT, ENGINE_MFMA, ENGINE_MFMA_FP16 = 0, 1, 2, 3

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "csrc", "libgla.so")
_HEADER = os.path.join(os.path.dirname(_PKG), "include", "gla.h")
_lib = None


class GlaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"gla status {status}: {message}")
        self.status = status


def library_path() -> str:
    return _LIB_PATH


def lib_symbols() -> List[str]:
    """Names of the functions that include/gla.h declares."""
    text = open(_HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(gla_[a-z_]+)\s*\(", text)))


def load_library():
    """Load libgla.so (built by ``__graft_entry__.build()`` / ``csrc/build.py``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} is missing: build the HIP library first "
            "(python -c 'import __graft_entry__ as g; g.build()'). There is no fallback path.")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i, fp, sz = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(ctypes.c_float), ctypes.c_size_t
    shape = [i] * 8
    lib.gla_fwd.restype = i
    lib.gla_fwd.argtypes = [vp, vp, vp, vp] + shape + [vp, vp, vp]
    lib.gla_fwd_static.restype = i
    lib.gla_fwd_static.argtypes = [vp, vp, vp, vp] + shape + [vp, vp, vp]
    lib.gla_fwd_ex.restype = i
    lib.gla_fwd_ex.argtypes = [vp, vp, vp, vp] + shape + [i, i, vp, vp, vp, sz, vp]
    lib.gla_fwd_layout.restype = i
    lib.gla_fwd_layout.argtypes = [vp, vp, vp, vp] + shape + [i, i, i, vp, vp, vp, vp, sz, vp]
    lib.gla_fwd_gates.restype = i
    lib.gla_fwd_gates.argtypes = [vp, vp, vp, vp, vp] + shape + [i, i, i, vp, vp, vp, vp, sz, vp]
    lib.gla_bwd.restype = i
    lib.gla_bwd.argtypes = [vp] * 5 + shape + [i] + [vp] * 4 + [vp, sz, vp]
    lib.gla_bwd_layout.restype = i
    lib.gla_bwd_layout.argtypes = [vp] * 5 + shape + [i, i] + [vp, sz] + [vp] * 4 + [vp, sz, vp]
    lib.gla_bwd_reuse.restype = i
    lib.gla_bwd_reuse.argtypes = [vp] * 5 + shape + [i] + [vp, sz] + [vp] * 4 + [vp, sz, vp]
    lib.gla_srem_dwconv.restype = i
    lib.gla_srem_dwconv.argtypes = [vp, vp, vp] + [i] * 7 + [vp, vp]
    lib.gla_fwd_multi.restype = i
    lib.gla_fwd_multi.argtypes = [vp, vp, vp, vp] + [i] * 7 + [ctypes.c_uint, i, vp, vp, sz, vp]
    lib.gla_fwd_fused.restype = i
    lib.gla_fwd_fused.argtypes = [vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, ctypes.c_float] + shape + \
        [i, i, vp, vp, vp, sz, vp]
    lib.gla_fwd_fused_gates.restype = i
    lib.gla_fwd_fused_gates.argtypes = [vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, ctypes.c_float] + shape + \
        [i, i, vp, vp, vp, sz, vp]
    lib.gla_bwd_gates.restype = i
    lib.gla_bwd_gates.argtypes = [vp] * 7 + shape + [i] + [vp] * 5 + [vp, sz, vp]
    lib.gla_bwd_gates_workspace_bytes.restype = sz
    lib.gla_bwd_gates_workspace_bytes.argtypes = [i] * 6
    lib.gla_bwd_workspace_bytes.restype = sz
    lib.gla_bwd_workspace_bytes.argtypes = [i] * 6
    f = ctypes.c_float
    lib.gla_decay_fwd.restype = i
    lib.gla_decay_fwd.argtypes = [vp] * 4 + [i, vp] + shape + [i] * 3 + [vp] * 4 + [sz, vp]
    lib.gla_decay_bwd.restype = i
    lib.gla_decay_bwd.argtypes = [vp] * 4 + [i] + [vp] * 4 + shape + [i] * 3 + [vp] * 6 + [sz, vp]
    lib.gla_decay_step.restype = i
    lib.gla_decay_step.argtypes = [vp] * 4 + [i] * 7 + [vp] * 4
    for name in ("gla_decay_fwd_workspace_bytes", "gla_decay_bwd_workspace_bytes"):
        getattr(lib, name).restype = sz
        getattr(lib, name).argtypes = [i] * 6
    lib.gla_rope.restype = i
    lib.gla_rope.argtypes = [vp, vp, vp, ctypes.POINTER(i), i, f] + [i] * 10 + [vp] * 3
    lib.gla_norm_fwd.restype = i
    lib.gla_norm_fwd.argtypes = [vp] * 3 + [f, vp] + [i] * 7 + [vp] * 2
    lib.gla_norm_bwd.restype = i
    lib.gla_norm_bwd.argtypes = [vp] * 4 + [f, vp] + [i] * 7 + [vp] * 5 + [sz, vp]
    lib.gla_norm_bwd_workspace_bytes.restype = sz
    lib.gla_norm_bwd_workspace_bytes.argtypes = [i] * 4
    lib.gla_recur_fwd.restype = i
    lib.gla_recur_fwd.argtypes = [vp, vp, i, f, i, vp] + [i] * 8 + [vp] * 4 + [sz, vp]
    lib.gla_recur_bwd.restype = i
    lib.gla_recur_bwd.argtypes = [vp, vp, i, f, i] + [vp] * 4 + [i] * 8 + [vp] * 4 + [sz, vp]
    lib.gla_recur_step.restype = i
    lib.gla_recur_step.argtypes = [vp, vp, i, f] + [i] * 5 + [vp] * 4
    for name in ("gla_recur_fwd_workspace_bytes", "gla_recur_bwd_workspace_bytes"):
        getattr(lib, name).restype = sz
        getattr(lib, name).argtypes = [i] * 3
    lp, ip = ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(i)
    lib.gla_qk_norm_fwd.restype = i
    lib.gla_qk_norm_fwd.argtypes = [vp, lp, i, vp, lp, i, vp, vp, f, vp, ip, i, f] + [i] * 9 + [vp] * 3
    lib.gla_qk_norm_bwd.restype = i
    lib.gla_qk_norm_bwd.argtypes = [vp, lp, i, vp, lp, i] + [vp] * 4 + [f, vp, ip, i, f] + [i] * 9 + [vp] * 5 + [sz, vp]
    lib.gla_qk_norm_bwd_workspace_bytes.restype = sz
    lib.gla_qk_norm_bwd_workspace_bytes.argtypes = [i] * 5
    lib.gla_glu_fwd.restype = i
    lib.gla_glu_fwd.argtypes = [vp] * 3 + [i] * 6 + [vp] * 3 + [sz, vp]
    lib.gla_glu_bwd.restype = i
    lib.gla_glu_bwd.argtypes = [vp] * 5 + [i] * 5 + [vp] * 4 + [sz, vp]
    for name in ("gla_glu_fwd_workspace_bytes", "gla_glu_bwd_workspace_bytes"):
        getattr(lib, name).restype = sz
        getattr(lib, name).argtypes = [i] * 4
    lib.gla_calibrate_mfma.restype = i
    lib.gla_calibrate_mfma.argtypes = [ctypes.POINTER(ctypes.c_double), vp]
    lib.gla_fwd_timed.restype = i
    lib.gla_fwd_timed.argtypes = [vp, vp, vp, vp] + shape + [i, i, vp, vp, vp, sz, vp, i, fp]
    lib.gla_fwd_workspace_bytes.restype = sz
    lib.gla_fwd_workspace_bytes.argtypes = [i] * 6
    lib.gla_set_option.restype = i
    lib.gla_set_option.argtypes = [i, i]
    lib.gla_get_option.restype = i
    lib.gla_get_option.argtypes = [i]
    lib.gla_status_string.restype = ctypes.c_char_p
    lib.gla_status_string.argtypes = [i]
    lib.gla_version.restype = i
    lib.gla_version.argtypes = []
    lib.gla_block_scan_dir.restype = i
    lib.gla_block_scan_dir.argtypes = [i, i]
    _lib = lib
    return lib


def gla_status_string(status: int) -> str:
    return load_library().gla_status_string(int(status)).decode()


def gla_version() -> int:
    return int(load_library().gla_version())


SCHEDULE_BLOCK_PROCESS, SCHEDULE_BLOCK_SCAN = 0, 1


def gla_block_scan_dir(block: int, schedule: int = SCHEDULE_BLOCK_PROCESS) -> int:
    """Scan order of DiG block `block` (1-based) under Algorithm 1's (or Algorithm 4's) transposes and flips."""
    d = int(load_library().gla_block_scan_dir(int(block), int(schedule)))
    if d < 0:
        raise GlaError(2, gla_status_string(2))
    return d


def gla_set_option(option: int, value: int) -> None:
    _check(load_library().gla_set_option(int(option), int(value)))


def gla_get_option(option: int) -> int:
    return int(load_library().gla_get_option(int(option)))


def gla_fwd_workspace_bytes(B, H, T, dk, dv, qkv_dtype=DT_BF16) -> int:
    return int(load_library().gla_fwd_workspace_bytes(B, H, T, dk, dv, qkv_dtype))


def _check(status: int) -> None:
    if status != 0:
        raise GlaError(status, gla_status_string(status))


_torch_module = None
_raw_stream = None              # device ordinal -> hipStream_t of its current stream


def _torch():
    global _torch_module, _raw_stream
    if _torch_module is None:
        import torch
        # torch.cuda.current_stream() builds a Stream object on every call (3.0 us against 0.1 us)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda ordinal: torch.cuda.current_stream(ordinal).cuda_stream)
        _torch_module = torch
    return _torch_module


_HERE = contextlib.nullcontext()


def _on_device_of(t):
    """Context in which the tensor's device is the current one; nothing to do where it already is (1.4 us less)."""
    torch = _torch()
    return _HERE if torch.cuda.current_device() == t.get_device() else torch.cuda.device(t.device)


def _like(t, dtype):
    torch = _torch()
    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


def _dt(t) -> int:
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return DT_BF16
    if t.dtype == torch.float32:
        return DT_F32
    raise TypeError(f"unsupported element type {t.dtype}")


def _prep(q, k, v, log_alpha, grid_h, grid_w):
    torch = _torch()
    for name, t in (("q", q), ("k", k), ("v", v), ("log_alpha", log_alpha)):
        if not t.is_cuda:
            raise ValueError(f"{name} must live on the GPU")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    if q.dim() != 4 or q.shape != k.shape or q.shape != log_alpha.shape:
        raise ValueError("q, k, log_alpha must be [B,H,T,dk] with equal shapes")
    if v.dim() != 4 or v.shape[:3] != q.shape[:3]:
        raise ValueError("v must be [B,H,T,dv]")
    if q.dtype != k.dtype or q.dtype != v.dtype:
        raise TypeError("q, k, v must share one element type")
    if log_alpha.dtype != torch.float32:
        raise TypeError("log_alpha must be fp32")
    B, H, T, dk = q.shape
    return B, H, T, dk, v.shape[3]


def _stream_ptr(stream, t=None) -> int:
    """The given stream, or the current one of the tensor's device (of the current device without a tensor)."""
    if stream is not None:
        return int(stream.cuda_stream)
    torch = _torch()
    return int(_raw_stream(torch.cuda.current_device() if t is None else t.get_device()))


def _elsewhere(stream, t) -> bool:
    """Whether a call on tensors like t goes to a torch stream that is not the current one (an object that only has a ``cuda_stream`` leaves the
    tensors' lives to the caller)."""
    if stream is None or not isinstance(stream, _torch().cuda.Stream):
        return False
    if stream.device_index != t.get_device():
        raise ValueError("stream must be one of the tensors' device")
    return int(stream.cuda_stream) != int(_raw_stream(stream.device_index))


def _call_on(stream, call, args):
    """call(**args) with the given stream as the current one.  What the call allocates comes from that stream's memory, where nothing of the caller's
    current stream is still at work; the tensors given are recorded on it and those returned on the caller's, so that their memory is handed
    on only when both are done with it, whenever the caller drops them."""
    torch = _torch()
    given = [t for t in args.values() if isinstance(t, torch.Tensor)]
    before = torch.cuda.current_stream(stream.device_index)
    with torch.cuda.stream(stream):
        result = call(**{**args, "stream": None})
    for t in given:
        t.record_stream(stream)
    for t in result if isinstance(result, tuple) else (result,):
        if isinstance(t, torch.Tensor):
            t.record_stream(before)
    return result


def gla_fwd(q, k, v, log_alpha, grid_h, grid_w, scan_dir=SCAN_ROW_FWD,
            want_final_state=True, out=None, final_state=None, stream=None):
    """bf16 q/k/v -> fp32 out (and fp32 final state); library-owned scratch."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_fwd, locals())
    torch = _torch()
    lib = load_library()
    B, H, T, dk, dv = _prep(q, k, v, log_alpha, grid_h, grid_w)
    if q.dtype != torch.bfloat16:
        raise TypeError("gla_fwd takes bf16 q/k/v; use gla_fwd_ex for fp32")
    if out is None:
        out = _like(v, torch.float32)
    if final_state is None and want_final_state:
        final_state = q.new_empty((B, H, dk, dv), dtype=torch.float32)
    with _on_device_of(q):
        _check(lib.gla_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(),
                           B, H, T, dk, dv, grid_h, grid_w, scan_dir,
                           out.data_ptr(), final_state.data_ptr() if final_state is not None else None,
                           _stream_ptr(stream, q)))
    return out, final_state


def gla_fwd_static(q, k, v, log_alpha, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, out=None, final_state=None,
                   stream=None):
    """gla_fwd with the span states in the library's static device array (no allocation inside the call):
    the caller passes ``out`` (fp32 [B,H,T,dv]) and, if wanted, ``final_state`` (fp32 [B,H,dk,dv])."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_fwd_static, locals())
    torch = _torch()
    lib = load_library()
    B, H, T, dk, dv = _prep(q, k, v, log_alpha, grid_h, grid_w)
    if q.dtype != torch.bfloat16:
        raise TypeError("gla_fwd_static takes bf16 q/k/v")
    if out is None or out.dtype != torch.float32 or tuple(out.shape) != (B, H, T, dv) or not out.is_contiguous():
        raise ValueError("out must be a contiguous fp32 GPU tensor [B,H,T,dv]")
    with _on_device_of(q):
        _check(lib.gla_fwd_static(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(),
                                  B, H, T, dk, dv, grid_h, grid_w, scan_dir,
                                  out.data_ptr(), final_state.data_ptr() if final_state is not None else None,
                                  _stream_ptr(stream, q)))
    return out, final_state


def gla_fwd_ex(q, k, v, log_alpha, grid_h, grid_w, scan_dir=SCAN_ROW_FWD,
               out_dtype=None, want_final_state=True, out=None, final_state=None,
               workspace=None, stream=None):
    """Explicit element types and caller-owned workspace (a uint8 GPU tensor)."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_fwd_ex, locals())
    torch = _torch()
    lib = load_library()
    B, H, T, dk, dv = _prep(q, k, v, log_alpha, grid_h, grid_w)
    qdt = _dt(q)
    if out is None:
        odt = torch.float32 if out_dtype is None else out_dtype
        out = _like(v, odt)
    if final_state is None and want_final_state:
        final_state = q.new_empty((B, H, dk, dv), dtype=torch.float32)
    if workspace is None:
        nbytes = gla_fwd_workspace_bytes(B, H, T, dk, dv, qdt)
        workspace = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=q.device)
    with _on_device_of(q):
        _check(lib.gla_fwd_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(),
                              B, H, T, dk, dv, grid_h, grid_w, scan_dir, qdt, _dt(out),
                              out.data_ptr(), final_state.data_ptr() if final_state is not None else None,
                              workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q)))
    return out, final_state


def gla_fwd_layout(q, k, v, log_alpha, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, layout=LAYOUT_BHTD,
                   initial_state=None, out_dtype=None, want_final_state=True, out=None, final_state=None,
                   workspace=None, stream=None):
    """gla_fwd_ex for [B,H,T,d] (LAYOUT_BHTD) or [B,T,H,d] (LAYOUT_BTHD) tensors, starting from
    ``initial_state`` ([B,H,dk,dv] fp32, or None for zero)."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_fwd_layout, locals())
    torch = _torch()
    lib = load_library()
    if layout not in (LAYOUT_BHTD, LAYOUT_BTHD):
        raise ValueError("unknown layout")
    for name, t in (("q", q), ("k", k), ("v", v), ("log_alpha", log_alpha)):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous 4-d GPU tensor")
    if q.shape != k.shape or q.shape != log_alpha.shape or v.shape[:3] != q.shape[:3]:
        raise ValueError("q, k, log_alpha must share one shape and v its first three sizes")
    if q.dtype != k.dtype or q.dtype != v.dtype or log_alpha.dtype != torch.float32:
        raise TypeError("q, k, v must share one element type and log_alpha must be fp32")
    if layout == LAYOUT_BHTD:
        B, H, T, dk = q.shape
    else:
        B, T, H, dk = q.shape
    dv = v.shape[3]
    qdt = _dt(q)
    if initial_state is not None:
        if (initial_state.dtype != torch.float32 or tuple(initial_state.shape) != (B, H, dk, dv)
                or not initial_state.is_contiguous() or not initial_state.is_cuda):
            raise ValueError("initial_state must be a contiguous fp32 GPU tensor [B,H,dk,dv]")
    if out is None:
        odt = torch.float32 if out_dtype is None else out_dtype
        out = _like(v, odt)
    if final_state is None and want_final_state:
        final_state = q.new_empty((B, H, dk, dv), dtype=torch.float32)
    if workspace is None:
        nbytes = gla_fwd_workspace_bytes(B, H, T, dk, dv, qdt)
        workspace = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=q.device)
    with _on_device_of(q):
        _check(lib.gla_fwd_layout(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(),
                                  B, H, T, dk, dv, grid_h, grid_w, scan_dir, qdt, _dt(out), layout,
                                  initial_state.data_ptr() if initial_state is not None else None,
                                  out.data_ptr(), final_state.data_ptr() if final_state is not None else None,
                                  workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q)))
    return out, final_state


def gla_fwd_gates(q, k, v, log_alpha, log_beta, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, layout=LAYOUT_BHTD,
                  initial_state=None, out_dtype=None, want_final_state=True, out=None, final_state=None,
                  workspace=None, stream=None):
    """The recurrence with the two-sided gate alpha_t^T beta_t; ``log_beta`` is fp32, shaped like v."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_fwd_gates, locals())
    torch = _torch()
    lib = load_library()
    if layout not in (LAYOUT_BHTD, LAYOUT_BTHD):
        raise ValueError("unknown layout")
    for name, t in (("q", q), ("k", k), ("v", v), ("log_alpha", log_alpha), ("log_beta", log_beta)):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous 4-d GPU tensor")
    if q.shape != k.shape or q.shape != log_alpha.shape or v.shape[:3] != q.shape[:3] or log_beta.shape != v.shape:
        raise ValueError("q, k, log_alpha must share one shape, v and log_beta another with the same first three sizes")
    if q.dtype != k.dtype or q.dtype != v.dtype or log_alpha.dtype != torch.float32 or log_beta.dtype != torch.float32:
        raise TypeError("q, k, v must share one element type and the gates must be fp32")
    if layout == LAYOUT_BHTD:
        B, H, T, dk = q.shape
    else:
        B, T, H, dk = q.shape
    dv = v.shape[3]
    qdt = _dt(q)
    if initial_state is not None:
        if (initial_state.dtype != torch.float32 or tuple(initial_state.shape) != (B, H, dk, dv)
                or not initial_state.is_contiguous() or not initial_state.is_cuda):
            raise ValueError("initial_state must be a contiguous fp32 GPU tensor [B,H,dk,dv]")
    if out is None:
        out = _like(v, torch.float32 if out_dtype is None else out_dtype)
    if final_state is None and want_final_state:
        final_state = q.new_empty((B, H, dk, dv), dtype=torch.float32)
    if workspace is None:
        nbytes = gla_fwd_workspace_bytes(B, H, T, dk, dv, qdt)
        workspace = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=q.device)
    with _on_device_of(q):
        _check(lib.gla_fwd_gates(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(), log_beta.data_ptr(),
                                 B, H, T, dk, dv, grid_h, grid_w, scan_dir, qdt, _dt(out), layout,
                                 initial_state.data_ptr() if initial_state is not None else None,
                                 out.data_ptr(), final_state.data_ptr() if final_state is not None else None,
                                 workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q)))
    return out, final_state


def gla_srem_dwconv(x, weight, bias, grid_h, grid_w, orient=0, out_dtype=None, out=None, stream=None):
    """3x3 depth-wise convolution of the SREM on tokens x [B, T, D] (canonical order); weight fp32 [D,3,3], bias
    fp32 [D] or None; ``orient`` = the scan order the paper's sequence would be in at this block."""
    if _elsewhere(stream, x):
        return _call_on(stream, gla_srem_dwconv, locals())
    torch = _torch()
    lib = load_library()
    if not x.is_cuda or not x.is_contiguous() or x.dim() != 3:
        raise ValueError("x must be a contiguous 3-d GPU tensor [B,T,D]")
    B, T, D = x.shape
    if T != grid_h * grid_w:
        raise ValueError("T != grid_h * grid_w")
    if weight.dtype != torch.float32 or tuple(weight.shape) != (D, 3, 3) or not weight.is_contiguous() or not weight.is_cuda:
        raise ValueError("weight must be a contiguous fp32 GPU tensor [D,3,3]")
    if bias is not None and (bias.dtype != torch.float32 or tuple(bias.shape) != (D,) or not bias.is_cuda):
        raise ValueError("bias must be a contiguous fp32 GPU tensor [D]")
    if out is None:
        out = torch.empty_like(x, dtype=x.dtype if out_dtype is None else out_dtype)
    with _on_device_of(x):
        _check(lib.gla_srem_dwconv(x.data_ptr(), weight.data_ptr(), bias.data_ptr() if bias is not None else None,
                                   B, grid_h, grid_w, D, orient, _dt(x), _dt(out), out.data_ptr(), _stream_ptr(stream, x)))
    return out


def gla_fwd_multi(q, k, v, log_alpha, grid_h, grid_w, scan_dirs=(SCAN_ROW_FWD, SCAN_ROW_REV), out=None,
                  workspace=None, stream=None):
    """Sum over the scan orders in ``scan_dirs`` of the forward outputs (fp32, canonical token order)."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_fwd_multi, locals())
    torch = _torch()
    lib = load_library()
    for name, t in (("q", q), ("k", k), ("v", v), ("log_alpha", log_alpha)):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous 4-d GPU tensor")
    if q.shape != k.shape or q.shape != log_alpha.shape or v.shape[:3] != q.shape[:3]:
        raise ValueError("q, k, log_alpha must share one shape and v its first three sizes")
    if q.dtype != k.dtype or q.dtype != v.dtype or log_alpha.dtype != torch.float32:
        raise TypeError("q, k, v must share one element type and log_alpha must be fp32")
    mask = 0
    for d in scan_dirs:
        if d not in (0, 1, 2, 3):
            raise ValueError("scan orders are 0..3")
        mask |= 1 << d
    B, H, T, dk = q.shape
    dv = v.shape[3]
    qdt = _dt(q)
    if out is None:
        out = _like(v, torch.float32)
    if workspace is None:
        nbytes = gla_fwd_workspace_bytes(B, H, T, dk, dv, qdt)
        workspace = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=q.device)
    with _on_device_of(q):
        _check(lib.gla_fwd_multi(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(),
                                 B, H, T, dk, dv, grid_h, grid_w, mask, qdt, out.data_ptr(),
                                 workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q)))
    return out


def gla_fwd_fused(q, k, v, z_alpha, tau, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, r_pre=None, ln_weight=None,
                  ln_bias=None, ln_eps=1e-5, out_dtype=None, want_final_state=True, out=None, final_state=None,
                  workspace=None, stream=None, _z_beta=None):
    """Forward pass with the gates taken from their pre-activations (``log_alpha = logsigmoid(z_alpha) / tau``) and,
    if ``r_pre`` is given, ``Swish(r_pre) * LayerNorm_head(o)`` stored instead of ``o``.  q, k, v, z_alpha, r_pre
    share one element type; ln_weight / ln_bias are fp32 [H, dv] or None."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_fwd_fused, locals())
    torch = _torch()
    lib = load_library()
    tensors = [("q", q), ("k", k), ("v", v), ("z_alpha", z_alpha)] + ([("r_pre", r_pre)] if r_pre is not None else [])
    if _z_beta is not None:
        tensors.append(("z_beta", _z_beta))
        if _z_beta.shape != v.shape:
            raise ValueError("z_beta must have the shape of v")
    for name, t in tensors:
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous 4-d GPU tensor")
        if t.dtype != q.dtype:
            raise TypeError("q, k, v, z_alpha and r_pre must share one element type")
    if q.shape != k.shape or q.shape != z_alpha.shape or v.shape[:3] != q.shape[:3]:
        raise ValueError("q, k, z_alpha must share one shape and v its first three sizes")
    if r_pre is not None and r_pre.shape != v.shape:
        raise ValueError("r_pre must have the shape of v")
    B, H, T, dk = q.shape
    dv = v.shape[3]
    for name, t in (("ln_weight", ln_weight), ("ln_bias", ln_bias)):
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (H, dv) or not t.is_contiguous()
                              or not t.is_cuda):
            raise ValueError(f"{name} must be a contiguous fp32 GPU tensor [H,dv]")
    qdt = _dt(q)
    if out is None:
        odt = torch.float32 if out_dtype is None else out_dtype
        out = _like(v, odt)
    if final_state is None and want_final_state:
        final_state = q.new_empty((B, H, dk, dv), dtype=torch.float32)
    if workspace is None:
        nbytes = gla_fwd_workspace_bytes(B, H, T, dk, dv, qdt)
        workspace = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=q.device)
    ptr = lambda t: t.data_ptr() if t is not None else None
    tail = (ptr(r_pre), ptr(ln_weight), ptr(ln_bias), float(ln_eps), B, H, T, dk, dv, grid_h, grid_w, scan_dir, qdt,
            _dt(out), out.data_ptr(), ptr(final_state), workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q))
    with _on_device_of(q):
        if _z_beta is not None:
            _check(lib.gla_fwd_fused_gates(q.data_ptr(), k.data_ptr(), v.data_ptr(), z_alpha.data_ptr(),
                                           _z_beta.data_ptr(), float(tau), *tail))
        else:
            _check(lib.gla_fwd_fused(q.data_ptr(), k.data_ptr(), v.data_ptr(), z_alpha.data_ptr(), float(tau), *tail))
    return out, final_state


def gla_fwd_fused_gates(q, k, v, z_alpha, z_beta, tau, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, **kwargs):
    """gla_fwd_fused with the value-side gate as well: ``log_beta = logsigmoid(z_beta) / tau``, z_beta shaped like v
    and of the element type of q, k, v.  Keyword arguments as gla_fwd_fused."""
    if z_beta is None:
        raise ValueError("z_beta is required")
    return gla_fwd_fused(q, k, v, z_alpha, tau, grid_h, grid_w, scan_dir, _z_beta=z_beta, **kwargs)


def gla_bwd_gates(q, k, v, log_alpha, log_beta, d_out, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, out_fwd=None,
                  workspace=None, stream=None):
    """Gradients of the two-sided-gate recurrence: returns (dq, dk, dv, dlog_alpha, dlog_beta), all fp32.
    ``out_fwd``: the fp32 outputs of gla_fwd_gates on the same inputs, if the caller still holds them."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_bwd_gates, locals())
    torch = _torch()
    lib = load_library()
    for name, t in (("q", q), ("k", k), ("v", v), ("log_alpha", log_alpha), ("log_beta", log_beta), ("d_out", d_out)):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous 4-d GPU tensor")
    if (q.shape != k.shape or q.shape != log_alpha.shape or v.shape[:3] != q.shape[:3] or log_beta.shape != v.shape
            or d_out.shape != v.shape):
        raise ValueError("q, k, log_alpha must share one shape; v, log_beta, d_out another with the same first three sizes")
    if q.dtype != k.dtype or q.dtype != v.dtype or d_out.dtype != q.dtype:
        raise TypeError("q, k, v, d_out must share one element type")
    if log_alpha.dtype != torch.float32 or log_beta.dtype != torch.float32:
        raise TypeError("the gates must be fp32")
    B, H, T, dk = q.shape
    dv = v.shape[3]
    qdt = _dt(q)
    if out_fwd is not None and (out_fwd.dtype != torch.float32 or out_fwd.shape != v.shape or not out_fwd.is_cuda
                                or not out_fwd.is_contiguous()):
        raise ValueError("out_fwd must be a contiguous fp32 GPU tensor shaped like v")
    dq, dk_g, dla = (_like(q, torch.float32) for _ in range(3))
    dv_g, dlb = (_like(v, torch.float32) for _ in range(2))
    if workspace is None:
        nbytes = int(lib.gla_bwd_gates_workspace_bytes(B, H, T, dk, dv, qdt))
        workspace = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=q.device)
    with _on_device_of(q):
        _check(lib.gla_bwd_gates(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(), log_beta.data_ptr(),
                                 d_out.data_ptr(), out_fwd.data_ptr() if out_fwd is not None else None,
                                 B, H, T, dk, dv, grid_h, grid_w, scan_dir, qdt,
                                 dq.data_ptr(), dk_g.data_ptr(), dv_g.data_ptr(), dla.data_ptr(), dlb.data_ptr(),
                                 workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q)))
    return dq, dk_g, dv_g, dla, dlb


def gla_bwd_gates_workspace_bytes(B, H, T, dk, dv, qkv_dtype=DT_BF16) -> int:
    return int(load_library().gla_bwd_gates_workspace_bytes(B, H, T, dk, dv, qkv_dtype))


def gla_bwd_workspace_bytes(B, H, T, dk, dv, qkv_dtype=DT_BF16) -> int:
    return int(load_library().gla_bwd_workspace_bytes(B, H, T, dk, dv, qkv_dtype))


def gla_bwd_layout(q, k, v, log_alpha, d_out, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, layout=LAYOUT_BHTD,
                   fwd_workspace=None, workspace=None, stream=None):
    """gla_bwd for [B,H,T,d] (LAYOUT_BHTD) or [B,T,H,d] (LAYOUT_BTHD) tensors; the gradients come in the same order."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_bwd_layout, locals())
    torch = _torch()
    lib = load_library()
    if layout not in (LAYOUT_BHTD, LAYOUT_BTHD):
        raise ValueError("unknown layout")
    for name, t in (("q", q), ("k", k), ("v", v), ("log_alpha", log_alpha), ("d_out", d_out)):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous 4-d GPU tensor")
    if q.shape != k.shape or q.shape != log_alpha.shape or v.shape[:3] != q.shape[:3] or d_out.shape != v.shape:
        raise ValueError("q, k, log_alpha must share one shape, v its first three sizes, d_out the shape of v")
    if q.dtype != k.dtype or q.dtype != v.dtype or q.dtype != d_out.dtype or log_alpha.dtype != torch.float32:
        raise TypeError("q, k, v, d_out must share one element type and log_alpha must be fp32")
    if layout == LAYOUT_BHTD:
        B, H, T, dk = q.shape
    else:
        B, T, H, dk = q.shape
    dv = v.shape[3]
    qdt = _dt(q)
    dq, dk_, dg = (_like(q, torch.float32) for _ in range(3))
    dv_ = _like(v, torch.float32)
    if workspace is None:
        nbytes = gla_bwd_workspace_bytes(B, H, T, dk, dv, qdt)
        workspace = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=q.device)
    with _on_device_of(q):
        _check(lib.gla_bwd_layout(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(), d_out.data_ptr(),
                                  B, H, T, dk, dv, grid_h, grid_w, scan_dir, qdt, layout,
                                  fwd_workspace.data_ptr() if fwd_workspace is not None else None,
                                  fwd_workspace.numel() if fwd_workspace is not None else 0,
                                  dq.data_ptr(), dk_.data_ptr(), dv_.data_ptr(), dg.data_ptr(),
                                  workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q)))
    return dq, dk_, dv_, dg


def gla_bwd(q, k, v, log_alpha, d_out, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, workspace=None, stream=None,
            fwd_workspace=None):
    """Gradients (dq, dk, dv, dlog_alpha), all fp32, of a loss with upstream gradient ``d_out`` = dL/d out.
    q, k, v, d_out share one element type (bf16 or fp32); [B,H,T,d] order.  ``fwd_workspace``: the workspace
    tensor of the gla_fwd_ex call on the same tensors and scan order (untouched since, same options): its span
    states are reused instead of recomputed (gla_bwd_reuse)."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_bwd, locals())
    torch = _torch()
    lib = load_library()
    B, H, T, dk, dv = _prep(q, k, v, log_alpha, grid_h, grid_w)
    if d_out.shape != v.shape or d_out.dtype != v.dtype or not d_out.is_cuda or not d_out.is_contiguous():
        raise ValueError("d_out must be a contiguous GPU tensor shaped and typed like v")
    qdt = _dt(q)
    dq, dk_, dg = (_like(q, torch.float32) for _ in range(3))
    dv_ = _like(v, torch.float32)
    if workspace is None:
        nbytes = gla_bwd_workspace_bytes(B, H, T, dk, dv, qdt)
        workspace = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=q.device)
    with _on_device_of(q):
        if fwd_workspace is None:
            _check(lib.gla_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(), d_out.data_ptr(),
                               B, H, T, dk, dv, grid_h, grid_w, scan_dir, qdt,
                               dq.data_ptr(), dk_.data_ptr(), dv_.data_ptr(), dg.data_ptr(),
                               workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q)))
        else:
            _check(lib.gla_bwd_reuse(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(), d_out.data_ptr(),
                                     B, H, T, dk, dv, grid_h, grid_w, scan_dir, qdt,
                                     fwd_workspace.data_ptr(), fwd_workspace.numel(),
                                     dq.data_ptr(), dk_.data_ptr(), dv_.data_ptr(), dg.data_ptr(),
                                     workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q)))
    return dq, dk_, dv_, dg


def gla_calibrate_mfma(stream=None):
    """TFLOP/s of a register-resident v_mfma_f32_16x16x32_bf16 loop on the current device."""
    lib = load_library()
    x = ctypes.c_double(0.0)
    _check(lib.gla_calibrate_mfma(ctypes.byref(x), _stream_ptr(stream)))
    return float(x.value)


def gla_fwd_timed(q, k, v, log_alpha, grid_h, grid_w, scan_dir, out, final_state,
                  workspace, iters=10, stream=None):
    """Mean milliseconds per call: [span-state kernel, carry kernel, output kernel, whole call]."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_fwd_timed, locals())
    torch = _torch()
    lib = load_library()
    B, H, T, dk, dv = _prep(q, k, v, log_alpha, grid_h, grid_w)
    ms = (ctypes.c_float * 4)()
    with _on_device_of(q):
        _check(lib.gla_fwd_timed(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_alpha.data_ptr(),
                                 B, H, T, dk, dv, grid_h, grid_w, scan_dir, _dt(q), _dt(out),
                                 out.data_ptr(), final_state.data_ptr() if final_state is not None else None,
                                 workspace.data_ptr(), workspace.numel(), _stream_ptr(stream, q),
                                 int(iters), ms))
    return [float(x) for x in ms]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _want(name, t, shape, dtype, gpu):
    """Raises unless t is a contiguous tensor of this shape and element type on GPU number `gpu` (-1: not on a GPU)."""
    if gpu < 0 or t.get_device() != gpu or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous GPU tensor {list(shape)} on the device of the others")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be of element type {dtype}")


def _room(nbytes, workspace, q):
    """The caller's workspace, or one of its size for this call (`nbytes` is asked for in that case only)."""
    if workspace is None:
        return _torch().empty((max(nbytes(), 16),), dtype=_torch().uint8, device=q.device)
    if workspace.get_device() != q.get_device() or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous GPU tensor on the device of the others")
    return workspace


def _prep_decay(q, k, v, log_decay, layout, seq_lens, states):
    torch = _torch()
    if layout not in (LAYOUT_BHTD, LAYOUT_BTHD):
        raise ValueError("unknown layout")
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k, v must be 4-d")
    _dt(q)
    dev = q.get_device()
    _want("q", q, q.shape, q.dtype, dev)
    _want("k", k, q.shape, q.dtype, dev)
    _want("v", v, (*q.shape[:3], v.shape[3]), q.dtype, dev)
    B, H, T, dk = q.shape if layout == LAYOUT_BHTD else (q.shape[0], q.shape[2], q.shape[1], q.shape[3])
    kind = DECAY_HEAD if log_decay.dim() == 1 else DECAY_TOKEN
    _want("log_decay", log_decay, (H,) if kind == DECAY_HEAD else q.shape[:3], torch.float32, dev)
    if seq_lens is not None:
        _want("seq_lens", seq_lens, (B,), torch.int32, dev)
    dv = v.shape[3]
    for name, t in states:
        if t is not None:
            _want(name, t, (B, H, dk, dv), torch.float32, dev)
    return kind, B, H, T, dk, dv


def gla_decay_fwd_workspace_bytes(B, H, T, dk, dv, qkv_dtype=DT_BF16) -> int:
    return int(load_library().gla_decay_fwd_workspace_bytes(B, H, T, dk, dv, qkv_dtype))


def gla_decay_bwd_workspace_bytes(B, H, T, dk, dv, qkv_dtype=DT_BF16) -> int:
    return int(load_library().gla_decay_bwd_workspace_bytes(B, H, T, dk, dv, qkv_dtype))


def gla_decay_fwd(q, k, v, log_decay, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, layout=LAYOUT_BHTD, seq_lens=None,
                  initial_state=None, out_dtype=None, want_final_state=True, out=None, final_state=None,
                  workspace=None, stream=None):
    """Linear attention with one decay a head: S_t = exp(log_decay) S_{t-1} + k_t^T v_t, o_t = q_t S_t.  log_decay fp32 [H], or a
    number for each token ([B,H,T] or [B,T,H] by ``layout``).  ``seq_lens`` int32 [B]: each sequence's own length; rows of ``out``
    behind it are left as they were.  Returns (out, final_state)."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_decay_fwd, locals())
    torch = _torch()
    lib = load_library()
    kind, B, H, T, dk, dv = _prep_decay(q, k, v, log_decay, layout, seq_lens,
                                        (("initial_state", initial_state), ("final_state", final_state)))
    if out is None:
        out = _like(v, torch.float32 if out_dtype is None else out_dtype)
    else:
        _want("out", out, v.shape, out.dtype, q.get_device())
    if final_state is None and want_final_state:
        final_state = q.new_empty((B, H, dk, dv), dtype=torch.float32)
    qdt = _dt(q)
    workspace = _room(lambda: gla_decay_fwd_workspace_bytes(B, H, T, dk, dv, qdt), workspace, q)
    with _on_device_of(q):
        _check(lib.gla_decay_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), kind, _ptr(seq_lens),
                                 B, H, T, dk, dv, grid_h, grid_w, scan_dir, qdt, _dt(out), layout, _ptr(initial_state),
                                 out.data_ptr(), _ptr(final_state), workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream_ptr(stream, q)))
    return out, final_state


def gla_decay_bwd(q, k, v, log_decay, d_out, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, layout=LAYOUT_BHTD, seq_lens=None,
                  initial_state=None, d_final_state=None, grad_dtype=None, want_d_log_decay=True, want_d_initial_state=False,
                  workspace=None, stream=None):
    """Gradients of gla_decay_fwd from those of its outputs (``d_out``, like v) and of its final state (``d_final_state`` or None).
    Returns (dq, dk, dv, dlog_decay or None, d_initial_state or None); the first three of ``grad_dtype`` (fp32)."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_decay_bwd, locals())
    torch = _torch()
    lib = load_library()
    kind, B, H, T, dk, dv = _prep_decay(q, k, v, log_decay, layout, seq_lens,
                                        (("initial_state", initial_state), ("d_final_state", d_final_state)))
    _want("d_out", d_out, v.shape, q.dtype, q.get_device())
    gdt = torch.float32 if grad_dtype is None else grad_dtype
    dq, dk_, dv_ = _like(q, gdt), _like(k, gdt), _like(v, gdt)
    dg = _like(log_decay, torch.float32) if want_d_log_decay else None
    ds = q.new_empty((B, H, dk, dv), dtype=torch.float32) if want_d_initial_state else None
    qdt = _dt(q)
    workspace = _room(lambda: gla_decay_bwd_workspace_bytes(B, H, T, dk, dv, qdt), workspace, q)
    with _on_device_of(q):
        _check(lib.gla_decay_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), kind, _ptr(seq_lens),
                                 d_out.data_ptr(), _ptr(initial_state), _ptr(d_final_state), B, H, T, dk, dv, grid_h, grid_w,
                                 scan_dir, qdt, _dt(dq), layout, dq.data_ptr(), dk_.data_ptr(), dv_.data_ptr(), _ptr(dg), _ptr(ds),
                                 workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(stream, q)))
    return dq, dk_, dv_, dg, ds


def gla_decay_step(q, k, v, log_decay, state, out_dtype=None, out=None, state_out=None, stream=None):
    """One token of gla_decay_fwd for each sequence: q, k [B,H,dk], v [B,H,dv], log_decay fp32 [H] or [B,H], state fp32 [B,H,dk,dv].
    The new state goes to ``state_out``, in place (``state``) if that is None.  Returns (out, state_out)."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_decay_step, locals())
    torch = _torch()
    lib = load_library()
    if q.dim() != 3 or v.dim() != 3:
        raise ValueError("q, k must be [B,H,dk] and v [B,H,dv]")
    B, H, dk = q.shape
    dv = v.shape[2]
    qdt, dev = _dt(q), q.get_device()
    _want("q", q, (B, H, dk), q.dtype, dev)
    _want("k", k, (B, H, dk), q.dtype, dev)
    _want("v", v, (B, H, dv), q.dtype, dev)
    kind = DECAY_HEAD if log_decay.dim() == 1 else DECAY_TOKEN
    _want("log_decay", log_decay, (H,) if kind == DECAY_HEAD else (B, H), torch.float32, dev)
    _want("state", state, (B, H, dk, dv), torch.float32, dev)
    if state_out is None:
        state_out = state
    else:
        _want("state_out", state_out, (B, H, dk, dv), torch.float32, dev)
    if out is None:
        out = _like(v, torch.float32 if out_dtype is None else out_dtype)
    else:
        _want("out", out, v.shape, out.dtype, dev)
    with _on_device_of(q):
        _check(lib.gla_decay_step(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), kind, B, H, dk, dv, qdt, _dt(out),
                                  state.data_ptr(), state_out.data_ptr(), out.data_ptr(), _stream_ptr(stream, q)))
    return out, state_out


def gla_rope(q, k, sections, grid_h=0, grid_w=0, positions=None, base=10000.0, pairing=ROPE_ADJACENT, inverse=False,
             layout=LAYOUT_BHTD, out_q=None, out_k=None, stream=None):
    """Rotary positions: the first channels of each head fall into ``sections`` (even numbers), one an axis, and pair i of a section of w
    channels is turned by position * base^(-2 i / w).  ``positions`` int32 [B,T,axes], or None: the token's number, its row and
    column, or its frame, row and column on the grid.  ``inverse`` turns back (the backward pass).  q, k [B,H,T,d] or [B,T,H,d];
    k may be None; ``out_q`` / ``out_k`` may be q / k.  Returns (q', k')."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_rope, locals())
    torch = _torch()
    lib = load_library()
    if layout not in (LAYOUT_BHTD, LAYOUT_BTHD):
        raise ValueError("unknown layout")
    if q.dim() != 4:
        raise ValueError("q must be 4-d")
    dt, dev = _dt(q), q.get_device()
    _want("q", q, q.shape, q.dtype, dev)
    if k is not None:
        _want("k", k, q.shape, q.dtype, dev)
    B, H, T, d = q.shape if layout == LAYOUT_BHTD else (q.shape[0], q.shape[2], q.shape[1], q.shape[3])
    axes = len(sections)
    if positions is not None:
        _want("positions", positions, (B, T, axes), torch.int32, dev)
    if k is None and out_k is not None:
        raise ValueError("out_k without k")
    out_q = _like(q, q.dtype) if out_q is None else out_q
    out_k = _like(k, k.dtype) if out_k is None and k is not None else out_k
    for name, t in (("out_q", out_q), ("out_k", out_k)):
        if t is not None:
            _want(name, t, q.shape, q.dtype, dev)
    secs = (ctypes.c_int * max(axes, 1))(*[int(w) for w in sections])
    with _on_device_of(q):
        _check(lib.gla_rope(q.data_ptr(), _ptr(k), _ptr(positions), secs, axes, float(base), pairing, int(bool(inverse)), B, H, T, d,
                            grid_h, grid_w, dt, layout, out_q.data_ptr(), _ptr(out_k), _stream_ptr(stream, q)))
    return out_q, out_k


def _prep_norm(x, weight, bias, r_pre, layout):
    """Sizes (B, H, T, D) of [B,H,T,D], [B,T,H,D] or [B,T,D] rows after checking the tensors."""
    torch = _torch()
    if layout not in (LAYOUT_BHTD, LAYOUT_BTHD):
        raise ValueError("unknown layout")
    if x.dim() not in (3, 4):
        raise ValueError("x must be [B,H,T,D], [B,T,H,D] or [B,T,D]")
    _dt(x)
    _want("x", x, x.shape, x.dtype, x.get_device())
    if x.dim() == 3:
        B, H, T, D = x.shape[0], 1, x.shape[1], x.shape[2]
    else:
        B, H, T, D = x.shape if layout == LAYOUT_BHTD else (x.shape[0], x.shape[2], x.shape[1], x.shape[3])
    for name, t in (("weight", weight), ("bias", bias)):
        if t is not None:
            _want(name, t, (D,) if t.dim() == 1 and H == 1 else (H, D), torch.float32, x.get_device())
    if r_pre is not None:
        _want("r_pre", r_pre, x.shape, x.dtype, x.get_device())
    return B, H, T, D


def gla_norm_fwd(x, weight=None, bias=None, eps=1e-5, r_pre=None, layout=LAYOUT_BHTD, out_dtype=None, out=None, stream=None):
    """Layer norm of each row of x ([B,H,T,D], [B,T,H,D] by ``layout``, or tokens [B,T,D]), times Swish(r_pre) if given.  weight,
    bias fp32 [H,D] ([D] for tokens) or None.  The result has ``out_dtype`` (x's)."""
    if _elsewhere(stream, x):
        return _call_on(stream, gla_norm_fwd, locals())
    lib = load_library()
    B, H, T, D = _prep_norm(x, weight, bias, r_pre, layout)
    if out is None:
        out = _like(x, x.dtype if out_dtype is None else out_dtype)
    else:
        _want("out", out, x.shape, out.dtype, x.get_device())
        if out.data_ptr() == x.data_ptr() and out.dtype != x.dtype:
            raise ValueError("in place only with one element type")
    with _on_device_of(x):
        _check(lib.gla_norm_fwd(x.data_ptr(), _ptr(weight), _ptr(bias), float(eps), _ptr(r_pre), B, H, T, D, _dt(x), _dt(out), layout,
                                out.data_ptr(), _stream_ptr(stream, x)))
    return out


def gla_norm_bwd_workspace_bytes(B, H, T, D) -> int:
    return int(load_library().gla_norm_bwd_workspace_bytes(B, H, T, D))


def gla_norm_bwd(x, d_out, weight=None, bias=None, eps=1e-5, r_pre=None, layout=LAYOUT_BHTD, grad_dtype=None, want_d_weight=None,
                 workspace=None, stream=None):
    """Gradients of gla_norm_fwd: (dx, dr or None, dweight, dbias).  dx and dr are of ``grad_dtype`` (fp32), the others fp32 [H,D] (like
    weight if that is given), or None without ``want_d_weight`` (default: whether there is a weight or a bias)."""
    if _elsewhere(stream, x):
        return _call_on(stream, gla_norm_bwd, locals())
    torch = _torch()
    lib = load_library()
    B, H, T, D = _prep_norm(x, weight, bias, r_pre, layout)
    _want("d_out", d_out, x.shape, x.dtype, x.get_device())
    gdt = torch.float32 if grad_dtype is None else grad_dtype
    dx = _like(x, gdt)
    dr = _like(x, gdt) if r_pre is not None else None
    dw = db = None
    if want_d_weight or (want_d_weight is None and (weight is not None or bias is not None)):
        like = weight if weight is not None else bias
        shape = (H, D) if like is None else like.shape
        dw, db = x.new_empty(shape, dtype=torch.float32), x.new_empty(shape, dtype=torch.float32)
    workspace = _room(lambda: gla_norm_bwd_workspace_bytes(B, H, T, D), workspace, x)
    with _on_device_of(x):
        _check(lib.gla_norm_bwd(x.data_ptr(), d_out.data_ptr(), _ptr(weight), _ptr(bias), float(eps), _ptr(r_pre), B, H, T, D, _dt(x), _dt(dx),
                                layout, dx.data_ptr(), _ptr(dr), _ptr(dw), _ptr(db), workspace.data_ptr(),
                                workspace.numel() * workspace.element_size(), _stream_ptr(stream, x)))
    return dx, dr, dw, db


_MOST = (1 << 31) - 1


def _no_int():
    raise ValueError("sizes must be below 2^31")


def _prep_recur(x, gate, gate_kind, shape, seq_lens, states):
    """Checks the tensors of a gated recurrence; x has `shape`, states its first and last size."""
    torch = _torch()
    if gate_kind not in (GATE_LOG, GATE_PRE):
        raise ValueError("unknown gate kind")
    if x.numel() > _MOST and max(shape) > _MOST:
        _no_int()
    _dt(x)
    dev = x.get_device()
    _want("x", x, shape, x.dtype, dev)
    _want("gate", gate, shape, torch.float32 if gate_kind == GATE_LOG else x.dtype, dev)
    if seq_lens is not None:
        _want("seq_lens", seq_lens, shape[:1], torch.int32, dev)
    for name, t in states:
        if t is not None:
            _want(name, t, (shape[0], shape[-1]), torch.float32, dev)


def gla_recur_fwd_workspace_bytes(B, T, D) -> int:
    return int(load_library().gla_recur_fwd_workspace_bytes(B, T, D))


def gla_recur_bwd_workspace_bytes(B, T, D) -> int:
    return int(load_library().gla_recur_bwd_workspace_bytes(B, T, D))


def gla_recur_fwd(x, gate, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, gate_kind=GATE_PRE, tau=16.0, complement=False, seq_lens=None,
                  initial_state=None, out_dtype=None, want_final_state=True, out=None, final_state=None, workspace=None, stream=None):
    """Gated recurrence of channels: h_t = a_t h_{t-1} + u_t, u = x or (``complement``) (1 - a) x.  x [B,T,D]; gate [B,T,D]: log a in fp32
    (GATE_LOG), or z of x's element type with a = sigmoid(z)^(1/tau) (GATE_PRE).  ``seq_lens`` int32 [B]: each sequence's own length; rows
    of ``out`` behind it are left as they were.  States fp32 [B,D].  The result has ``out_dtype`` (x's).  Returns (out, final_state)."""
    if _elsewhere(stream, x):
        return _call_on(stream, gla_recur_fwd, locals())
    lib = load_library()
    if x.dim() != 3:
        raise ValueError("x must be [B,T,D]")
    B, T, D = x.shape
    _prep_recur(x, gate, gate_kind, x.shape, seq_lens, (("initial_state", initial_state), ("final_state", final_state)))
    if out is None:
        out = _like(x, x.dtype if out_dtype is None else out_dtype)
    else:
        _want("out", out, x.shape, out.dtype, x.get_device())
    if final_state is None and want_final_state:
        final_state = x.new_empty((B, D), dtype=_torch().float32)
    workspace = _room(lambda: gla_recur_fwd_workspace_bytes(B, T, D), workspace, x)
    with _on_device_of(x):
        _check(lib.gla_recur_fwd(x.data_ptr(), gate.data_ptr(), gate_kind, float(tau), int(bool(complement)), _ptr(seq_lens), B, T, D, grid_h,
                                 grid_w, scan_dir, _dt(x), _dt(out), _ptr(initial_state), out.data_ptr(), _ptr(final_state),
                                 workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(stream, x)))
    return out, final_state


def gla_recur_bwd(x, gate, d_out, grid_h, grid_w, scan_dir=SCAN_ROW_FWD, gate_kind=GATE_PRE, tau=16.0, complement=False, seq_lens=None,
                  initial_state=None, d_final_state=None, grad_dtype=None, want_d_initial_state=False, workspace=None, stream=None):
    """Gradients of gla_recur_fwd from those of its outputs (``d_out``, like x) and of its final state (``d_final_state`` or None).
    Returns (dx, d_gate, d_initial_state or None); the first two of ``grad_dtype`` (fp32)."""
    if _elsewhere(stream, x):
        return _call_on(stream, gla_recur_bwd, locals())
    torch = _torch()
    lib = load_library()
    if x.dim() != 3:
        raise ValueError("x must be [B,T,D]")
    B, T, D = x.shape
    _prep_recur(x, gate, gate_kind, x.shape, seq_lens, (("initial_state", initial_state), ("d_final_state", d_final_state)))
    _want("d_out", d_out, x.shape, x.dtype, x.get_device())
    gdt = torch.float32 if grad_dtype is None else grad_dtype
    dx, dg = _like(x, gdt), _like(gate, gdt)
    ds = x.new_empty((B, D), dtype=torch.float32) if want_d_initial_state else None
    workspace = _room(lambda: gla_recur_bwd_workspace_bytes(B, T, D), workspace, x)
    with _on_device_of(x):
        _check(lib.gla_recur_bwd(x.data_ptr(), gate.data_ptr(), gate_kind, float(tau), int(bool(complement)), _ptr(seq_lens), d_out.data_ptr(),
                                 _ptr(initial_state), _ptr(d_final_state), B, T, D, grid_h, grid_w, scan_dir, _dt(x), _dt(dx), dx.data_ptr(),
                                 dg.data_ptr(), _ptr(ds), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                 _stream_ptr(stream, x)))
    return dx, dg, ds


def gla_recur_step(x, gate, state, gate_kind=GATE_PRE, tau=16.0, complement=False, out_dtype=None, out=None, state_out=None, stream=None):
    """One token of gla_recur_fwd for each sequence: x, gate [B,D], state fp32 [B,D].  The new state goes to ``state_out``, in place
    (``state``) if that is None.  Returns (out, state_out)."""
    if _elsewhere(stream, x):
        return _call_on(stream, gla_recur_step, locals())
    lib = load_library()
    if x.dim() != 2:
        raise ValueError("x must be [B,D]")
    B, D = x.shape
    if state_out is None:
        state_out = state
    _prep_recur(x, gate, gate_kind, x.shape, None, (("state", state), ("state_out", state_out)))
    if out is None:
        out = _like(x, x.dtype if out_dtype is None else out_dtype)
    else:
        _want("out", out, x.shape, out.dtype, x.get_device())
    with _on_device_of(x):
        _check(lib.gla_recur_step(x.data_ptr(), gate.data_ptr(), gate_kind, float(tau), int(bool(complement)), B, D, _dt(x), _dt(out),
                                  state.data_ptr(), state_out.data_ptr(), out.data_ptr(), _stream_ptr(stream, x)))
    return out, state_out


_Strides = ctypes.c_longlong * 3


def _want_rows(name, t, dtype, gpu):
    """Raises unless t is a 4-d tensor of this element type on GPU number `gpu` whose last dimension is dense."""
    if gpu < 0 or t.get_device() != gpu or t.dim() != 4 or (t.stride(3) != 1 and t.shape[3] > 1):
        raise ValueError(f"{name} must be a 4-d GPU tensor on the device of the others whose rows' channels lie side by side")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be of element type {dtype}")


def _row_strides(t, layout):
    """Batch, head and token strides of rows; None for dense ones."""
    if t is None or t.is_contiguous():
        return None
    s = t.stride()
    return _Strides(s[0], s[1], s[2]) if layout == LAYOUT_BHTD else _Strides(s[0], s[2], s[1])


@functools.lru_cache(maxsize=64)
def _section_array(sections):
    return (ctypes.c_int * max(len(sections), 1))(*[int(w) for w in sections])


def _prep_qk(q, k, q_weight, k_weight, positions, sections, layout):
    """Sizes (B, H, Hk, T, d) and the sections of a call on rows of queries and keys after checking the tensors."""
    torch = _torch()
    if layout not in (LAYOUT_BHTD, LAYOUT_BTHD):
        raise ValueError("unknown layout")
    dev, Hk = q.get_device(), 0
    _dt(q)
    _want_rows("q", q, q.dtype, dev)
    B, H, T, d = q.shape if layout == LAYOUT_BHTD else (q.shape[0], q.shape[2], q.shape[1], q.shape[3])
    if q.numel() > _MOST and max(q.shape) > _MOST:
        _no_int()
    if k is not None:
        _want_rows("k", k, q.dtype, dev)
        Hk = k.shape[1 if layout == LAYOUT_BHTD else 2]
        if Hk > _MOST:
            _no_int()
        if k.shape != ((B, Hk, T, d) if layout == LAYOUT_BHTD else (B, T, Hk, d)):
            raise ValueError("q and k must agree in batches, tokens and channels")
        if k_weight is not None:
            _want("k_weight", k_weight, (d,), torch.float32, dev)
    elif k_weight is not None:
        raise ValueError("k_weight without k")
    if q_weight is not None:
        _want("q_weight", q_weight, (d,), torch.float32, dev)
    if positions is not None:
        _want("positions", positions, (B, T, len(sections)), torch.int32, dev)
    return (B, H, Hk, T, d), _section_array(tuple(sections))


def gla_qk_norm_fwd(q, k, q_weight=None, k_weight=None, sections=(), eps=1e-6, grid_h=0, grid_w=0, positions=None, base=10000.0,
                    pairing=ROPE_ADJACENT, layout=LAYOUT_BHTD, out_dtype=None, out_q=None, out_k=None, stream=None):
    """Queries' and keys' rows over their root mean square, times weights fp32 [d], then turned by their positions as in gla_rope (no
    ``sections``: not turned).  q [B,H,T,d], k [B,Hk,T,d] or None, or [B,T,H,d] by ``layout``; they may be views, of a packed projection
    for instance, whose last dimension is dense.  The results are dense, of ``out_dtype`` (q's).  Returns (q', k')."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_qk_norm_fwd, locals())
    lib = load_library()
    (B, H, Hk, T, d), secs = _prep_qk(q, k, q_weight, k_weight, positions, sections, layout)
    if k is None and out_k is not None:
        raise ValueError("out_k without k")
    dt = q.dtype if out_dtype is None else out_dtype
    if out_q is None:
        out_q = _like(q, dt)
    else:
        _want("out_q", out_q, q.shape, out_q.dtype, q.get_device())
    if out_k is not None:
        _want("out_k", out_k, k.shape, out_q.dtype, q.get_device())
    elif k is not None:
        out_k = _like(k, out_q.dtype)
    with _on_device_of(q):
        _check(lib.gla_qk_norm_fwd(q.data_ptr(), _row_strides(q, layout), H, _ptr(k), _row_strides(k, layout), Hk, _ptr(q_weight), _ptr(k_weight), float(eps), _ptr(positions), secs,
                                   len(sections), float(base), pairing, B, T, d, grid_h, grid_w, _dt(q), _dt(out_q), layout, out_q.data_ptr(), _ptr(out_k),
                                   _stream_ptr(stream, q)))
    return out_q, out_k


def gla_qk_norm_bwd_workspace_bytes(B, H, Hk, T, d) -> int:
    return int(load_library().gla_qk_norm_bwd_workspace_bytes(B, H, Hk, T, d))


def gla_qk_norm_bwd(q, k, d_out_q, d_out_k, q_weight=None, k_weight=None, sections=(), eps=1e-6, grid_h=0, grid_w=0, positions=None, base=10000.0,
                    pairing=ROPE_ADJACENT, layout=LAYOUT_BHTD, grad_dtype=None, want_d_weight=True, workspace=None, stream=None):
    """Gradients of gla_qk_norm_fwd from those of its outputs (dense, of q's element type): (dq, dk or None, dq_weight or None, dk_weight or
    None); the first two dense, of ``grad_dtype`` (fp32), the others fp32 where there is a weight and ``want_d_weight``."""
    if _elsewhere(stream, q):
        return _call_on(stream, gla_qk_norm_bwd, locals())
    torch = _torch()
    lib = load_library()
    (B, H, Hk, T, d), secs = _prep_qk(q, k, q_weight, k_weight, positions, sections, layout)
    if (k is None) != (d_out_k is None):
        raise ValueError("d_out_k belongs to k")
    _want("d_out_q", d_out_q, q.shape, q.dtype, q.get_device())
    if k is not None:
        _want("d_out_k", d_out_k, k.shape, q.dtype, q.get_device())
    gdt = torch.float32 if grad_dtype is None else grad_dtype
    dq, dk = _like(q, gdt), None if k is None else _like(k, gdt)
    dqw, dkw = (w.new_empty(d) if w is not None and want_d_weight else None for w in (q_weight, k_weight))
    workspace = _room(lambda: gla_qk_norm_bwd_workspace_bytes(B, H, Hk, T, d), workspace, q)
    with _on_device_of(q):
        _check(lib.gla_qk_norm_bwd(q.data_ptr(), _row_strides(q, layout), H, _ptr(k), _row_strides(k, layout), Hk, d_out_q.data_ptr(), _ptr(d_out_k), _ptr(q_weight), _ptr(k_weight),
                                   float(eps), _ptr(positions), secs, len(sections), float(base), pairing, B, T, d, grid_h, grid_w, _dt(q), _dt(dq), layout,
                                   dq.data_ptr(), _ptr(dk), _ptr(dqw), _ptr(dkw), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                   _stream_ptr(stream, q)))
    return dq, dk, dqw, dkw


def _prep_glu(x, w_gate, w_up, pre):
    """Sizes (M, K, F) of a gated feed-forward product after checking the tensors."""
    torch = _torch()
    _dt(x)
    dev = x.get_device()
    if x.dim() < 2 or w_gate.dim() != 2:
        raise ValueError("x must be [..., K], w_gate and w_up [F, K]")
    K, F = x.shape[-1], w_gate.shape[0]
    M = x.numel() // max(K, 1)
    if M > _MOST or K > _MOST or F > _MOST:
        _no_int()
    _want("x", x, x.shape, x.dtype, dev)
    _want("w_gate", w_gate, (F, K), x.dtype, dev)
    _want("w_up", w_up, (F, K), x.dtype, dev)
    if pre is not None:
        _want("pre", pre, (2, *x.shape[:-1], F), torch.float32, dev)
    return M, K, F


def gla_glu_fwd_workspace_bytes(M, K, F, dtype=DT_BF16) -> int:
    return int(load_library().gla_glu_fwd_workspace_bytes(M, K, F, dtype))


def gla_glu_bwd_workspace_bytes(M, K, F, dtype=DT_BF16) -> int:
    return int(load_library().gla_glu_bwd_workspace_bytes(M, K, F, dtype))


def gla_glu_fwd(x, w_gate, w_up, act=ACT_SILU, out_dtype=None, out=None, pre=None, workspace=None, stream=None):
    """Gated feed-forward product act(x w_gate^T) * (x w_up^T): x [..., K], weights [F, K], result [..., F] of ``out_dtype`` (x's).  ``pre``
    fp32 [2, ..., F] takes the two products before the activation, for gla_glu_bwd."""
    if _elsewhere(stream, x):
        return _call_on(stream, gla_glu_fwd, locals())
    lib = load_library()
    M, K, F = _prep_glu(x, w_gate, w_up, pre)
    if out is None:
        out = x.new_empty((*x.shape[:-1], F), dtype=x.dtype if out_dtype is None else out_dtype)
    else:
        _want("out", out, (*x.shape[:-1], F), out.dtype, x.get_device())
    workspace = _room(lambda: gla_glu_fwd_workspace_bytes(M, K, F, _dt(x)), workspace, x)
    with _on_device_of(x):
        _check(lib.gla_glu_fwd(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), M, K, F, act, _dt(x), _dt(out), out.data_ptr(), _ptr(pre),
                               workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(stream, x)))
    return out


def gla_glu_bwd(x, w_gate, w_up, d_out, act=ACT_SILU, pre=None, want_dx=True, want_dw=True, workspace=None, stream=None):
    """Gradients of gla_glu_fwd: (dx or None, dw_gate or None, dw_up or None), of x's element type.  ``pre``: what gla_glu_fwd left there for
    the same inputs; without it the two products are formed again.  bf16 gradients are off by 1.4 times their own rounding; gla_set_option(OPT_GLU_SPLIT, 1)
    takes twice the operations of their products and leaves that rounding alone."""
    if _elsewhere(stream, x):
        return _call_on(stream, gla_glu_bwd, locals())
    lib = load_library()
    M, K, F = _prep_glu(x, w_gate, w_up, pre)
    _want("d_out", d_out, (*x.shape[:-1], F), x.dtype, x.get_device())
    dx = _like(x, x.dtype) if want_dx else None
    dwg, dwu = (_like(w_gate, x.dtype), _like(w_up, x.dtype)) if want_dw else (None, None)
    workspace = _room(lambda: gla_glu_bwd_workspace_bytes(M, K, F, _dt(x)), workspace, x)
    with _on_device_of(x):
        _check(lib.gla_glu_bwd(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), d_out.data_ptr(), _ptr(pre), M, K, F, act, _dt(x), _ptr(dx), _ptr(dwg),
                               _ptr(dwu), workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(stream, x)))
    return dx, dwg, dwu
