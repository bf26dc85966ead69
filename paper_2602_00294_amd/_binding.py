"""ctypes binding of libsata.so: argument marshalling only.

Every computation runs in the library's HIP kernels.  Torch is used for device
memory (output allocation) and for the current stream.  If the library has
not been built, loading fails with an error; there is no fallback.
"""
from __future__ import annotations

import ctypes
import functools
import os
import re
from typing import Optional, Tuple

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libsata.so")
HEADER_PATH = os.path.join(os.path.dirname(PKG_DIR), "include", "sata.h")

SATA_F32, SATA_BF16 = 0, 1
SATA_OK = 0

_lib = None


class SataError(RuntimeError):
    def __init__(self, status: int, func: str, detail: str):
        super().__init__(f"{func} failed with status {status}: {detail}")
        self.status = status


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Loads libsata.so once and declares every signature of include/sata.h."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it first with __graft_entry__.build() "
                           "or python -m paper_2602_00294_amd.build")
    lib = ctypes.CDLL(p)
    i32, i64, vp = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p
    lib.sata_feature_count.argtypes = [i32, i32]
    lib.sata_feature_count.restype = i64
    lib.sata_state_elems.argtypes = [i32, i32, i32]
    lib.sata_state_elems.restype = i64
    lib.sata_feature_index.argtypes = [i32, i32, i64, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.sata_feature_index.restype = i32
    lib.sata_feature_map.argtypes = [vp, i32, i64, i32, i32, vp, vp]
    lib.sata_feature_map.restype = i32
    lib.sata_prefill.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.sata_prefill.restype = i32
    lib.sata_prefill_grouped.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.sata_prefill_grouped.restype = i32
    lib.sata_backward.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.sata_backward.restype = i32
    lib.sata_prefill_operands.argtypes = [i32, i32, i32, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]
    lib.sata_prefill_operands.restype = i32
    lib.sata_prefill_parts.argtypes = [i32, i32, i32, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]
    lib.sata_prefill_parts.restype = i32
    lib.sata_decode_step.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.sata_decode_step.restype = i32
    lib.sata_decode_step_noalloc.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.sata_decode_step_noalloc.restype = i32
    lib.sata_residual_elems.argtypes = [i32, i32, i32]
    lib.sata_residual_elems.restype = i64
    lib.sata_decode_step_compensated.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.sata_decode_step_compensated.restype = i32
    lib.sata_decode_step_grouped.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.sata_decode_step_grouped.restype = i32
    lib.sata_decay_scratch.argtypes = [i32, i32, i32, i32, i32, i32]
    lib.sata_decay_scratch.restype = i64
    lib.sata_softmax_backward_scratch.argtypes = [i32, i32, i32, i32]
    lib.sata_softmax_backward_scratch.restype = i64
    lib.sata_softmax_step_scratch.argtypes = [i32, i32, i32, i32, i32]
    lib.sata_softmax_step_scratch.restype = i64
    lib.sata_decay_prefill.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.sata_decay_prefill.restype = i32
    lib.sata_decay_step.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.sata_decay_step.restype = i32
    lib.sata_decay_backward.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp,
                                        vp, vp, vp]
    lib.sata_decay_backward.restype = i32
    lib.sata_softmax_prefill.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.sata_softmax_prefill.restype = i32
    lib.sata_softmax_backward.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp,
                                          vp]
    lib.sata_softmax_backward.restype = i32
    lib.sata_softmax_step.argtypes = [vp, vp, i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.sata_softmax_step.restype = i32
    f32, f64 = ctypes.c_float, ctypes.c_double
    lib.sata_delta_scratch.argtypes = [i32, i32, i32, i32, i32, i32, i32, i32]
    lib.sata_delta_scratch.restype = i64
    lib.sata_delta_prefill.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.sata_delta_prefill.restype = i32
    lib.sata_delta_step.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.sata_delta_step.restype = i32
    lib.sata_delta_backward.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp,
                                        vp, vp, vp, vp, vp]
    lib.sata_delta_backward.restype = i32
    lib.sata_rotary.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, f32, i32, vp, vp, vp]
    lib.sata_rotary.restype = i32
    lib.sata_rotary_frequencies.argtypes = [i32, f64, i32, f64, f64, ctypes.POINTER(f32), ctypes.POINTER(f32)]
    lib.sata_rotary_frequencies.restype = i32
    lib.sata_packed_row_bytes.argtypes = [i32]
    lib.sata_packed_row_bytes.restype = i64
    lib.sata_packed_write.argtypes = [vp, vp, i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp]
    lib.sata_packed_write.restype = i32
    lib.sata_packed_read.argtypes = [vp, i32, vp, i32, i32, i32, i32, i32, vp, vp]
    lib.sata_packed_read.restype = i32
    lib.sata_softmax_step_packed_scratch.argtypes = [i32, i32, i32, i32, i32]
    lib.sata_softmax_step_packed_scratch.restype = i64
    lib.sata_softmax_step_packed.argtypes = [vp, vp, i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.sata_softmax_step_packed.restype = i32
    lib.sata_status_string.argtypes = [i32]
    lib.sata_status_string.restype = ctypes.c_char_p
    lib.sata_last_error.argtypes = []
    lib.sata_last_error.restype = ctypes.c_char_p
    lib.sata_release.argtypes = []
    lib.sata_release.restype = None
    if path is None:
        _lib = lib
    return lib


def header_functions(path: str = HEADER_PATH):
    """Names of the functions that include/sata.h declares."""
    text = open(path).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(sata_[a-z_]+)\s*\(", text)))


def _check(status: int, func: str):
    if status != SATA_OK:
        detail = load_library().sata_last_error().decode()
        raise SataError(status, func, detail)


def feature_count(d: int, P: int) -> int:
    return int(load_library().sata_feature_count(d, P))


def state_elems(d_k: int, d_v: int, P: int) -> int:
    return int(load_library().sata_state_elems(d_k, d_v, P))


def feature_index(d: int, P: int, f: int) -> Tuple[int, ...]:
    """Index tuple (i1 <= ... <= ip) of feature f in the library's feature order."""
    deg = ctypes.c_int(0)
    idx = (ctypes.c_int * max(1, P - 1))()
    _check(load_library().sata_feature_index(d, P, f, ctypes.byref(deg), idx), "sata_feature_index")
    return tuple(idx[j] for j in range(deg.value))


# ------------------------------------------------------------------ tensor calls

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t) -> int:
    torch, dtype = _torch(), t.dtype
    if dtype == torch.float32:
        return SATA_F32
    if dtype == torch.bfloat16:
        return SATA_BF16
    raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")


def _check_tensor(t, name: str, device=None):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _check_same_dtype(ref, **tensors):
    dtype = ref.dtype
    for name, t in tensors.items():
        if t.dtype != dtype:
            raise TypeError(f"{name} is {t.dtype}, expected {dtype} like q")


def _check_shape(t, name: str, shape):
    if t.shape != shape and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _check_state(S, shape):
    if S.dtype != _torch().float32:
        raise TypeError("S must be float32")
    _check_shape(S, "S", shape)


def _stream_ptr():
    return ctypes.c_void_p(_torch().cuda.current_stream().cuda_stream)


def _raw_stream(index: int) -> int:
    """The handle of a device's current stream.  Asked for directly it costs 0.1 us, and 2.6 us by the stream
    object, which serves where torch lacks that private function."""
    torch = _torch()
    try:
        get = torch._C._cuda_getCurrentRawStream
    except AttributeError:
        return torch.cuda.current_stream(index).cuda_stream
    return get(index)


def _invoke(name: str, device, *args):
    """Calls a function of the library on `device` and its current stream.  (A token's call is a few
    microseconds of work: the device is changed only where it has to be.)"""
    func, index = getattr(load_library(), name), device.index
    if _torch().cuda.current_device() == index:
        _check(func(*args, _raw_stream(index)), name)
    else:
        with _torch().cuda.device(device):
            _check(func(*args, _raw_stream(index)), name)


def _at(t):
    """The address that a call takes for a tensor that may be left out or hold nothing."""
    return t.data_ptr() or None if t is not None else None


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None and t.numel() > 0 else ctypes.c_void_p(None)


def _features(d: int, P: int) -> int:
    D = feature_count(d, P)
    if D < 0:
        raise ValueError(f"invalid d={d} or P={P}")
    return D


def feature_map(x, P: int, phi=None):
    """phi(x) for x [..., d] (float32 or bfloat16) -> float32 [..., D].

    A preallocated float32 output [..., D] may be passed as phi=."""
    torch = _torch()
    code = _dtype_code(x)
    d = x.shape[-1]
    rows = x.numel() // d if d else 0
    D = _features(d, P)
    if phi is not None:
        if phi.dtype != torch.float32:
            raise TypeError(f"phi is {phi.dtype}, expected torch.float32")
        _check_shape(phi, "phi", (*x.shape[:-1], D))
    _check_tensor(x, "x")
    if phi is None:
        phi = torch.empty(*x.shape[:-1], D, dtype=torch.float32, device=x.device)
    _check_tensor(phi, "phi", x.device)
    with torch.cuda.device(x.device):
        _check(load_library().sata_feature_map(_ptr(x), code, rows, d, P, _ptr(phi), _stream_ptr()),
               "sata_feature_map")
    return phi


def prefill_operands(dtype, B: int, H: int, n: int, d_k: int, d_v: int, P: int, chunk: int = 64) -> str:
    """Operand precision of the state contractions that prefill uses for these
    arguments (host only): 'bf16' (bfloat16 operands), 'split' (float32
    operands as bfloat16 hi + lo pairs, three products each) or 'f32'."""
    torch = _torch()
    code = {torch.float32: SATA_F32, torch.bfloat16: SATA_BF16}.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")
    out = ctypes.c_int(-1)
    _check(load_library().sata_prefill_operands(code, B, H, n, d_k, d_v, P, chunk, ctypes.byref(out)),
           "sata_prefill_operands")
    return {0: "f32", 1: "bf16", 2: "split"}[out.value]


def prefill_parts(dtype, B: int, H: int, n: int, d_k: int, d_v: int, P: int, chunk: int = 64) -> int:
    """Number of parts of the sequence that the chunked scan of prefill runs side by
    side for these arguments, where it runs as a scan (host only; 1: one scan from
    the first token to the last)."""
    torch = _torch()
    code = {torch.float32: SATA_F32, torch.bfloat16: SATA_BF16}.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")
    out = ctypes.c_int(-1)
    _check(load_library().sata_prefill_parts(code, B, H, n, d_k, d_v, P, chunk, ctypes.byref(out)),
           "sata_prefill_parts")
    return out.value


def prefill(q, k, v, P: int, chunk: int = 64, want_state: bool = True, y=None, S=None):
    """Causal prefill.  q, k: [B, H, n, d_k]; v: [B, H, n, d_v].

    Returns (y [B, H, n, d_v] in the input dtype, S [B, H, D, d_v+1] float32 or None).
    Preallocated outputs may be passed as y= and S=.  Shapes and dtypes are
    checked before anything is launched.
    """
    torch = _torch()
    code = _dtype_code(q)
    _check_same_dtype(q, k=k, v=v)
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k, v must be [B, H, n, d]")
    B, H, n, dk = q.shape
    dv = v.shape[-1]
    _check_shape(k, "k", (B, H, n, dk))
    _check_shape(v, "v", (B, H, n, dv))
    D = _features(dk, P)
    if y is not None:
        _check_same_dtype(q, y=y)
        _check_shape(y, "y", (B, H, n, dv))
    if S is not None:
        _check_state(S, (B, H, D, dv + 1))
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check_tensor(t, name, q.device)
    if y is None:
        y = torch.empty(B, H, n, dv, dtype=q.dtype, device=q.device)
    if want_state and S is None:
        S = torch.empty(B, H, D, dv + 1, dtype=torch.float32, device=q.device)
    _check_tensor(y, "y", q.device)
    if S is not None:
        _check_tensor(S, "S", q.device)
    with torch.cuda.device(q.device):
        _check(load_library().sata_prefill(_ptr(q), _ptr(k), _ptr(v), code, B, H, n, dk, dv, P, chunk,
                                           _ptr(y), _ptr(S) if S is not None else ctypes.c_void_p(None),
                                           _stream_ptr()), "sata_prefill")
    return y, S


def prefill_grouped(q, k, v, P: int, chunk: int = 64, want_state: bool = True, y=None, S=None):
    """Causal prefill with grouped query heads.  q: [B, H_q, n, d_k] with
    H_q = G * H_kv (query head g + G*h reads key/value head h); k: [B, H_kv, n, d_k];
    v: [B, H_kv, n, d_v].  Returns (y [B, H_q, n, d_v], S [B, H_kv, D, d_v+1] or None)."""
    torch = _torch()
    code = _dtype_code(q)
    _check_same_dtype(q, k=k, v=v)
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q [B, G*H_kv, n, d_k], k [B, H_kv, n, d_k], v [B, H_kv, n, d_v] expected")
    B, Hq, n, dk = q.shape
    Hkv = k.shape[1]
    dv = v.shape[-1]
    if Hkv < 1 or Hq % Hkv:
        raise ValueError("the query head count must be a multiple of the key/value head count")
    G = Hq // Hkv
    _check_shape(k, "k", (B, Hkv, n, dk))
    _check_shape(v, "v", (B, Hkv, n, dv))
    D = _features(dk, P)
    if y is not None:
        _check_same_dtype(q, y=y)
        _check_shape(y, "y", (B, Hq, n, dv))
    if S is not None:
        _check_state(S, (B, Hkv, D, dv + 1))
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check_tensor(t, name, q.device)
    if y is None:
        y = torch.empty(B, Hq, n, dv, dtype=q.dtype, device=q.device)
    if want_state and S is None:
        S = torch.empty(B, Hkv, D, dv + 1, dtype=torch.float32, device=q.device)
    _check_tensor(y, "y", q.device)
    if S is not None:
        _check_tensor(S, "S", q.device)
    with torch.cuda.device(q.device):
        _check(load_library().sata_prefill_grouped(_ptr(q), _ptr(k), _ptr(v), code, B, Hkv, G, n, dk, dv, P, chunk,
                                                   _ptr(y), _ptr(S) if S is not None else ctypes.c_void_p(None),
                                                   _stream_ptr()), "sata_prefill_grouped")
    return y, S


def backward(q, k, v, dy, P: int, chunk: int = 64):
    """Gradients of the causal prefill's output y for dL/dy = dy.
    q, k: [B, H, n, d_k]; v, dy: [B, H, n, d_v].  Returns (dq, dk, dv) in q's dtype."""
    torch = _torch()
    code = _dtype_code(q)
    _check_same_dtype(q, k=k, v=v, dy=dy)
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k, v, dy must be [B, H, n, d]")
    B, H, n, dk = q.shape
    dv = v.shape[-1]
    _check_shape(k, "k", (B, H, n, dk))
    _check_shape(v, "v", (B, H, n, dv))
    _check_shape(dy, "dy", (B, H, n, dv))
    _features(dk, P)
    for name, t in (("q", q), ("k", k), ("v", v), ("dy", dy)):
        _check_tensor(t, name, q.device)
    dq, dkk, dvv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    with torch.cuda.device(q.device):
        _check(load_library().sata_backward(_ptr(q), _ptr(k), _ptr(v), _ptr(dy), code, B, H, n, dk, dv, P, chunk,
                                            _ptr(dq), _ptr(dkk), _ptr(dvv), _stream_ptr()), "sata_backward")
    return dq, dkk, dvv


def decode_step(S, q, k, v, P: int, y=None):
    """One decode step in place on S [B, H, D, d_v+1]; q, k: [B, H, d_k]; v: [B, H, d_v].

    Returns y [B, H, d_v] in the input dtype.  Shapes and dtypes are checked
    before anything is launched.
    """
    torch = _torch()
    code = _dtype_code(q)
    _check_same_dtype(q, k=k, v=v)
    if q.dim() != 3 or v.dim() != 3:
        raise ValueError("q, k, v must be [B, H, d]")
    B, H, dk = q.shape
    dv = v.shape[-1]
    _check_shape(k, "k", (B, H, dk))
    _check_shape(v, "v", (B, H, dv))
    _check_state(S, (B, H, _features(dk, P), dv + 1))
    if y is not None:
        _check_same_dtype(q, y=y)
        _check_shape(y, "y", (B, H, dv))
    for name, t in (("S", S), ("q", q), ("k", k), ("v", v)):
        _check_tensor(t, name, q.device)
    if y is None:
        y = torch.empty(B, H, dv, dtype=q.dtype, device=q.device)
    _check_tensor(y, "y", q.device)
    with torch.cuda.device(q.device):
        _check(load_library().sata_decode_step(_ptr(S), _ptr(q), _ptr(k), _ptr(v), code, B, H, dk, dv, P,
                                               _ptr(y), _stream_ptr()), "sata_decode_step")
    return y


def residual_elems(d_k: int, d_v: int, P: int) -> int:
    return int(load_library().sata_residual_elems(d_k, d_v, P))


def decode_step_compensated(S, R, q, k, v, P: int, y=None):
    """decode_step with compensated summation of the normaliser column and the
    degree-0/1 rows: R [B, H, residual_elems(d_k, d_v, P)] float32, zero when
    the state is created, updated in place with S.  Returns y [B, H, d_v]."""
    torch = _torch()
    code = _dtype_code(q)
    _check_same_dtype(q, k=k, v=v)
    if q.dim() != 3 or v.dim() != 3:
        raise ValueError("q, k, v must be [B, H, d]")
    B, H, dk = q.shape
    dv = v.shape[-1]
    _check_shape(k, "k", (B, H, dk))
    _check_shape(v, "v", (B, H, dv))
    _check_state(S, (B, H, _features(dk, P), dv + 1))
    if R.dtype != torch.float32:
        raise TypeError("R must be float32")
    _check_shape(R, "R", (B, H, residual_elems(dk, dv, P)))
    if y is not None:
        _check_same_dtype(q, y=y)
        _check_shape(y, "y", (B, H, dv))
    for name, t in (("S", S), ("R", R), ("q", q), ("k", k), ("v", v)):
        _check_tensor(t, name, q.device)
    if y is None:
        y = torch.empty(B, H, dv, dtype=q.dtype, device=q.device)
    _check_tensor(y, "y", q.device)
    with torch.cuda.device(q.device):
        _check(load_library().sata_decode_step_compensated(_ptr(S), _ptr(R), _ptr(q), _ptr(k), _ptr(v), code, B, H,
                                                           dk, dv, P, _ptr(y), _stream_ptr()),
               "sata_decode_step_compensated")
    return y


def decode_step_grouped(S, q, k, v, P: int, y=None):
    """One decode step with grouped query heads, in place on S [B, H_kv, D, d_v+1].

    q: [B, H_q, d_k] with H_q = G * H_kv (query head g + G*h reads key/value
    head h); k: [B, H_kv, d_k]; v: [B, H_kv, d_v].  Returns y [B, H_q, d_v].
    """
    torch = _torch()
    code = _dtype_code(q)
    _check_same_dtype(q, k=k, v=v)
    if q.dim() != 3 or k.dim() != 3 or v.dim() != 3:
        raise ValueError("q [B, G*H_kv, d_k], k [B, H_kv, d_k], v [B, H_kv, d_v] expected")
    B, Hq, dk = q.shape
    Hkv = k.shape[1]
    dv = v.shape[-1]
    if Hkv < 1 or Hq % Hkv:
        raise ValueError("the query head count must be a multiple of the key/value head count")
    _check_shape(k, "k", (B, Hkv, dk))
    _check_shape(v, "v", (B, Hkv, dv))
    G = Hq // Hkv
    _check_state(S, (B, Hkv, _features(dk, P), dv + 1))
    if y is not None:
        _check_same_dtype(q, y=y)
        _check_shape(y, "y", (B, Hq, dv))
    for name, t in (("S", S), ("q", q), ("k", k), ("v", v)):
        _check_tensor(t, name, q.device)
    if y is None:
        y = torch.empty(B, Hq, dv, dtype=q.dtype, device=q.device)
    _check_tensor(y, "y", q.device)
    with torch.cuda.device(q.device):
        _check(load_library().sata_decode_step_grouped(_ptr(S), _ptr(q), _ptr(k), _ptr(v), code, B, Hkv, G,
                                                       dk, dv, P, _ptr(y), _stream_ptr()),
               "sata_decode_step_grouped")
    return y


# ------------------------------------------------------------------ decay and softmax attention

def _check_sizes(*sizes):
    """ctypes hands the library the low 32 bits of a size, whatever it is."""
    if max(sizes) >= 1 << 31:
        raise ValueError(f"a size of {max(sizes)} does not fit in 32 bits")


def _prompt_sizes(q, k, v):
    """(dtype code, B, H_kv, G, n, d_k, d_v) of q [B, G*H_kv, n, d_k], k [B, H_kv, n, d_k], v [B, H_kv, n, d_v]."""
    code = _dtype_code(q)
    _check_same_dtype(q, k=k, v=v)
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q [B, G*H_kv, n, d_k], k [B, H_kv, n, d_k], v [B, H_kv, n, d_v] expected")
    B, Hq, n, dk = q.shape
    Hkv, dv = k.shape[1], v.shape[-1]
    if Hkv < 1 or Hq % Hkv:
        raise ValueError("the query head count must be a multiple of the key/value head count")
    _check_shape(k, "k", (B, Hkv, n, dk))
    _check_shape(v, "v", (B, Hkv, n, dv))
    _check_sizes(B, Hq, n, dk, dv)
    return code, B, Hkv, Hq // Hkv, n, dk, dv


def _token_sizes(q, k, v):
    """(dtype code, B, H_kv, G, d_k, d_v) of q [B, G*H_kv, d_k], k [B, H_kv, d_k], v [B, H_kv, d_v]."""
    code = _dtype_code(q)
    _check_same_dtype(q, k=k, v=v)
    if q.dim() != 3 or k.dim() != 3 or v.dim() != 3:
        raise ValueError("q [B, G*H_kv, d_k], k [B, H_kv, d_k], v [B, H_kv, d_v] expected")
    B, Hq, dk = q.shape
    Hkv, dv = k.shape[1], v.shape[-1]
    if Hkv < 1 or Hq % Hkv:
        raise ValueError("the query head count must be a multiple of the key/value head count")
    _check_shape(k, "k", (B, Hkv, dk))
    _check_shape(v, "v", (B, Hkv, dv))
    _check_sizes(B, Hq, dk, dv)
    return code, B, Hkv, Hq // Hkv, dk, dv


def _check_as(t, name: str, dtype, shape):
    """Type and shape of an argument that may be left out."""
    if t is None:
        return
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {dtype}")
    _check_shape(t, name, shape)


def _check_tensors(device, **tensors):
    index = device.index  # (asked for by its number, a tensor's device takes half the time)
    for name, t in tensors.items():
        if t is not None and (t.get_device() != index or not t.is_contiguous()):
            _check_tensor(t, name, device)


def _scratch(nbytes: int, device):
    """The call's own device memory, from torch's allocator: on the current stream, and in the pool of the
    graph that a call is captured into."""
    return _torch().empty(nbytes, dtype=_torch().uint8, device=device) if nbytes > 0 else None


def decay_prefill(q, k, v, log_decay, lengths=None, S_in=None, want_state: bool = True, y=None, S=None):
    """Causal linear attention with a decay per key/value head: S_t = exp(log_decay) S_{t-1} + k_t (x) v_t,
    y_t = q_t S_t / sqrt(d_k).

    q: [B, H_q, n, d_k] with H_q = G * H_kv (query head g + G*h reads key/value head h); k: [B, H_kv, n, d_k];
    v: [B, H_kv, n, d_v]; log_decay: [H_kv] float32, at most 0; lengths: [B] int32, the tokens of each
    sequence (the rest is padding: y is zero there); S_in: the states to go on from.
    Returns (y [B, H_q, n, d_v] in the input dtype, S [B, H_kv, d_k, d_v] float32 or None).
    Preallocated outputs may be passed as y= and S=."""
    torch = _torch()
    code, B, H, G, n, dk, dv = _prompt_sizes(q, k, v)
    _check_as(log_decay, "log_decay", torch.float32, (H,))
    _check_as(lengths, "lengths", torch.int32, (B,))
    _check_as(S_in, "S_in", torch.float32, (B, H, dk, dv))
    _check_as(y, "y", q.dtype, (B, G * H, n, dv))
    _check_as(S, "S", torch.float32, (B, H, dk, dv))
    _check_tensors(q.device, q=q, k=k, v=v, log_decay=log_decay, lengths=lengths, S_in=S_in, y=y, S=S)
    if y is None:
        y = torch.empty(B, G * H, n, dv, dtype=q.dtype, device=q.device)
    if want_state and S is None:
        S = torch.empty(B, H, dk, dv, dtype=torch.float32, device=q.device)
    scratch = _scratch(load_library().sata_decay_scratch(B, H, G, n, dk, dv), q.device)
    _invoke("sata_decay_prefill", q.device, _at(q), _at(k), _at(v), _at(log_decay), code, B, H, G, n, dk, dv,
            _at(lengths), _at(S_in), _at(y), _at(S), _at(scratch))
    return y, S


def decay_step(S, q, k, v, log_decay, y=None):
    """One token of every sequence, in place on S [B, H_kv, d_k, d_v]: S = exp(log_decay) S + k (x) v,
    y = q S / sqrt(d_k).  q: [B, H_q, d_k]; k: [B, H_kv, d_k]; v: [B, H_kv, d_v].  Returns y [B, H_q, d_v]."""
    torch = _torch()
    code, B, H, G, dk, dv = _token_sizes(q, k, v)
    _check_state(S, (B, H, dk, dv))
    _check_as(log_decay, "log_decay", torch.float32, (H,))
    _check_as(y, "y", q.dtype, (B, G * H, dv))
    _check_tensors(q.device, S=S, q=q, k=k, v=v, log_decay=log_decay, y=y)
    if y is None:
        y = torch.empty(B, G * H, dv, dtype=q.dtype, device=q.device)
    _invoke("sata_decay_step", q.device, _at(S), _at(q), _at(k), _at(v), _at(log_decay), code, B, H, G, dk, dv,
            _at(y))
    return y


def decay_backward(q, k, v, log_decay, dy, lengths=None, S_in=None, dS=None):
    """Gradients of decay_prefill for dL/dy = dy [B, H_q, n, d_v] and dL/dS = dS [B, H_kv, d_k, d_v] (None: zero).
    Returns (dq, dk, dv, dS_in): the first three in q's dtype, dS_in float32, or None without S_in.
    The decay is a constant of the layer and gets no gradient."""
    torch = _torch()
    code, B, H, G, n, dk, dv = _prompt_sizes(q, k, v)
    _check_as(log_decay, "log_decay", torch.float32, (H,))
    _check_as(dy, "dy", q.dtype, (B, G * H, n, dv))
    _check_as(lengths, "lengths", torch.int32, (B,))
    _check_as(S_in, "S_in", torch.float32, (B, H, dk, dv))
    _check_as(dS, "dS", torch.float32, (B, H, dk, dv))
    _check_tensors(q.device, q=q, k=k, v=v, log_decay=log_decay, dy=dy, lengths=lengths, S_in=S_in, dS=dS)
    dq, dkk, dvv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dS_in = torch.empty_like(S_in) if S_in is not None else None
    scratch = _scratch(load_library().sata_decay_scratch(B, H, G, n, dk, dv), q.device)
    _invoke("sata_decay_backward", q.device, _at(q), _at(k), _at(v), _at(log_decay), _at(dy), code, B, H, G, n, dk,
            dv, _at(lengths), _at(S_in), _at(dS), _at(dq), _at(dkk), _at(dvv), _at(dS_in), _at(scratch))
    return dq, dkk, dvv, dS_in


def softmax_prefill(q, k, v, lengths=None, want_lse: bool = True, y=None):
    """Exact causal softmax attention, the one that the Taylor series stands for.

    q: [B, H_q, n, d_k] with H_q = G * H_kv; k: [B, H_kv, n, d_k]; v: [B, H_kv, n, d_v]; lengths: [B] int32, the
    tokens of each sequence (the rest is padding: y is zero and lse minus infinity there).
    Probabilities of bfloat16 calls are rounded to bfloat16 for their product with v; float32 calls carry 24 bits.
    Returns (y [B, H_q, n, d_v] in the input dtype, lse [B, H_q, n] float32, the logarithm of each row's sum of
    exponentials, or None)."""
    torch = _torch()
    code, B, H, G, n, dk, dv = _prompt_sizes(q, k, v)
    _check_as(lengths, "lengths", torch.int32, (B,))
    _check_as(y, "y", q.dtype, (B, G * H, n, dv))
    _check_tensors(q.device, q=q, k=k, v=v, lengths=lengths, y=y)
    if y is None:
        y = torch.empty(B, G * H, n, dv, dtype=q.dtype, device=q.device)
    lse = torch.empty(B, G * H, n, dtype=torch.float32, device=q.device) if want_lse else None
    _invoke("sata_softmax_prefill", q.device, _at(q), _at(k), _at(v), code, B, H, G, n, dk, dv, _at(lengths), _at(y),
            _at(lse))
    return y, lse


def softmax_backward(q, k, v, y, lse, dy, lengths=None):
    """Gradients of softmax_prefill for dL/dy = dy, from its outputs y and lse; the probabilities are computed
    again and, in bfloat16 calls, rounded to bfloat16 for the products.  Returns (dq, dk, dv) in q's dtype."""
    torch = _torch()
    code, B, H, G, n, dk, dv = _prompt_sizes(q, k, v)
    _check_as(y, "y", q.dtype, (B, G * H, n, dv))
    _check_as(lse, "lse", torch.float32, (B, G * H, n))
    _check_as(dy, "dy", q.dtype, (B, G * H, n, dv))
    _check_as(lengths, "lengths", torch.int32, (B,))
    _check_tensors(q.device, q=q, k=k, v=v, y=y, lse=lse, dy=dy, lengths=lengths)
    dq, dkk, dvv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    scratch = _scratch(load_library().sata_softmax_backward_scratch(B, H, G, n), q.device)
    _invoke("sata_softmax_backward", q.device, _at(q), _at(k), _at(v), _at(y), _at(lse), _at(dy), code, B, H, G, n,
            dk, dv, _at(lengths), _at(dq), _at(dkk), _at(dvv), _at(scratch))
    return dq, dkk, dvv


def softmax_step(K, V, lengths, q, k, v, y=None):
    """One token of every sequence over a cache K [B, H_kv, capacity, d_k], V [B, H_kv, capacity, d_v]: writes k and
    v as row lengths[b], then attends over rows 0..lengths[b].  lengths: [B] int32, the tokens in the cache before
    the call; it is not changed.  A sequence whose length is negative or not below the capacity is idle (its cache
    stays, its y is zero).  q: [B, H_q, d_k]; k: [B, H_kv, d_k]; v: [B, H_kv, d_v].  Returns y [B, H_q, d_v], whose
    last bits may change with the other sequences' lengths (the sums are cut by all of them)."""
    torch = _torch()
    code, B, H, G, dk, dv = _token_sizes(q, k, v)
    _check_same_dtype(q, K=K, V=V)
    if K.dim() != 4:
        raise ValueError("K must be [B, H_kv, capacity, d_k]")
    cap = K.shape[2]
    _check_sizes(cap)
    _check_shape(K, "K", (B, H, cap, dk))
    _check_shape(V, "V", (B, H, cap, dv))
    _check_as(lengths, "lengths", torch.int32, (B,))
    _check_as(y, "y", q.dtype, (B, G * H, dv))
    _check_tensors(q.device, K=K, V=V, lengths=lengths, q=q, k=k, v=v, y=y)
    if y is None:
        y = torch.empty(B, G * H, dv, dtype=q.dtype, device=q.device)
    scratch = _scratch(load_library().sata_softmax_step_scratch(B, H, G, cap, dv), q.device)
    _invoke("sata_softmax_step", q.device, _at(K), _at(V), cap, _at(lengths), _at(q), _at(k), _at(v), code, B, H, G,
            dk, dv, _at(y), _at(scratch))
    return y


# ------------------------------------------------------------------ the gated delta rule

def _delta_sizes(q, k, v, dims: int):
    """(dtype code, B, H_qk, G, n, d_k, d_v) of q, k [B, H_qk(, n), d_k] and v [B, G*H_qk(, n), d_v] of `dims` dimensions."""
    code = _dtype_code(q)
    _check_same_dtype(q, k=k, v=v)
    qs, vs = q.shape, v.shape
    if not len(qs) == len(vs) == k.dim() == dims:
        rows = ", n" if dims == 4 else ""
        raise ValueError(f"q, k [B, H_qk{rows}, d_k] and v [B, G*H_qk{rows}, d_v] expected")
    B, H, dk, Hv, dv = qs[0], qs[1], qs[-1], vs[1], vs[-1]
    if H < 1 or Hv % H or Hv < H:
        raise ValueError("the value head count must be a multiple of the query and key head count")
    n = qs[2] if dims == 4 else 1
    _check_shape(k, "k", qs)
    _check_shape(v, "v", (B, Hv, *qs[2:-1], dv))
    _check_sizes(B, Hv, n, dk, dv)
    return code, B, H, Hv // H, n, dk, dv


def delta_prefill(q, k, v, g, beta, lengths=None, S_in=None, want_state: bool = True, y=None, S=None):
    """Linear attention by the gated delta rule: S' = exp(g_t) S_{t-1}, S_t = S' + k_t (x) beta_t (v_t - k_t S'),
    y_t = q_t S_t / sqrt(d_k).

    q, k: [B, H, n, d_k]; v: [B, H_v, n, d_v] with H_v = G * H (value head g + G*h reads query and key head h);
    g (at most 0), beta: [B, H_v, n] float32; lengths: [B] int32, the tokens of each sequence (the rest is padding: y is
    zero there); S_in: the states to go on from.  Keys should be of length one or beta |k|^2 at most 2: states grow otherwise.
    Returns (y [B, H_v, n, d_v] in the input dtype, S [B, H_v, d_k, d_v] float32 or None).
    Preallocated outputs may be passed as y= and S=."""
    torch = _torch()
    code, B, H, G, n, dk, dv = _delta_sizes(q, k, v, 4)
    _check_as(g, "g", torch.float32, (B, G * H, n))
    _check_as(beta, "beta", torch.float32, (B, G * H, n))
    _check_as(lengths, "lengths", torch.int32, (B,))
    _check_as(S_in, "S_in", torch.float32, (B, G * H, dk, dv))
    _check_as(y, "y", q.dtype, (B, G * H, n, dv))
    _check_as(S, "S", torch.float32, (B, G * H, dk, dv))
    _check_tensors(q.device, q=q, k=k, v=v, g=g, beta=beta, lengths=lengths, S_in=S_in, y=y, S=S)
    if y is None:
        y = torch.empty_like(v)
    if want_state and S is None:
        S = torch.empty(B, G * H, dk, dv, dtype=torch.float32, device=q.device)
    scratch = _scratch(load_library().sata_delta_scratch(0, code, B, H, G, n, dk, dv), q.device)
    _invoke("sata_delta_prefill", q.device, _at(q), _at(k), _at(v), _at(g), _at(beta), code, B, H, G, n, dk, dv,
            _at(lengths), _at(S_in), _at(y), _at(S), _at(scratch))
    return y, S


def delta_step(S, q, k, v, g, beta, y=None):
    """One token of every sequence by the gated delta rule, in place on S [B, H_v, d_k, d_v].  q, k: [B, H, d_k];
    v: [B, H_v, d_v]; g, beta: [B, H_v] float32.  Returns y [B, H_v, d_v]."""
    torch = _torch()
    code, B, H, G, _, dk, dv = _delta_sizes(q, k, v, 3)
    _check_state(S, (B, G * H, dk, dv))
    _check_as(g, "g", torch.float32, (B, G * H))
    _check_as(beta, "beta", torch.float32, (B, G * H))
    _check_as(y, "y", q.dtype, (B, G * H, dv))
    _check_tensors(q.device, S=S, q=q, k=k, v=v, g=g, beta=beta, y=y)
    if y is None:
        y = torch.empty_like(v)
    _invoke("sata_delta_step", q.device, _at(S), _at(q), _at(k), _at(v), _at(g), _at(beta), code, B, H, G, dk, dv, _at(y))
    return y


def delta_backward(q, k, v, g, beta, dy, lengths=None, S_in=None, dS=None):
    """Gradients of delta_prefill for dL/dy = dy [B, H_v, n, d_v] and dL/dS = dS [B, H_v, d_k, d_v] (None: zero).
    Returns (dq, dk, dv, dg, dbeta, dS_in): the first three in q's dtype, the others float32, dS_in None without S_in."""
    torch = _torch()
    code, B, H, G, n, dk, dv = _delta_sizes(q, k, v, 4)
    _check_as(g, "g", torch.float32, (B, G * H, n))
    _check_as(beta, "beta", torch.float32, (B, G * H, n))
    _check_as(dy, "dy", q.dtype, (B, G * H, n, dv))
    _check_as(lengths, "lengths", torch.int32, (B,))
    _check_as(S_in, "S_in", torch.float32, (B, G * H, dk, dv))
    _check_as(dS, "dS", torch.float32, (B, G * H, dk, dv))
    _check_tensors(q.device, q=q, k=k, v=v, g=g, beta=beta, dy=dy, lengths=lengths, S_in=S_in, dS=dS)
    dq, dkk, dvv, dg, db = (torch.empty_like(x) for x in (q, k, v, g, beta))
    dS_in = torch.empty_like(S_in) if S_in is not None else None
    scratch = _scratch(load_library().sata_delta_scratch(1, code, B, H, G, n, dk, dv), q.device)
    _invoke("sata_delta_backward", q.device, _at(q), _at(k), _at(v), _at(g), _at(beta), _at(dy), code, B, H, G, n, dk, dv,
            _at(lengths), _at(S_in), _at(dS), _at(dq), _at(dkk), _at(dvv), _at(dg), _at(db), _at(dS_in), _at(scratch))
    return dq, dkk, dvv, dg, db, dS_in


# ------------------------------------------------------------------ rotary positions

ROTARY_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "by_turns": 3}


def rotary_frequencies(pairs: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                       original: float = 0.0, device="cuda"):
    """Frequencies base^(-i / pairs) of `pairs` pairs, [pairs] float32 on `device`, and the outputs' scale, for rotary().
    scaling, for contexts `factor` times as long as trained: "linear" divides all by the factor; "base" raises the
    base so that the slowest is divided by it; "by_turns" keeps those of 32 turns and more in `original` tokens, divides those
    of one and fewer, goes from the ones to the others in proportion to the turns, and scales by 0.1 ln(factor) + 1
    (weights that were trained with another way between the two need their own frequencies: rotary() takes any)."""
    if scaling not in ROTARY_SCALINGS:
        raise ValueError(f"unknown scaling {scaling!r}; one of {', '.join(ROTARY_SCALINGS)}")
    _check_sizes(pairs)
    freq, scale = (ctypes.c_float * min(max(1, pairs), 128))(), ctypes.c_float()  # (more pairs are refused)
    _check(load_library().sata_rotary_frequencies(pairs, base, ROTARY_SCALINGS[scaling], factor, original, freq,
                                                  ctypes.byref(scale)), "sata_rotary_frequencies")
    return _torch().tensor(list(freq), dtype=_torch().float32).to(device), scale.value


def _turn(q, k, positions, inv_freq, interleaved, scale, back, q_out, k_out):
    torch = _torch()
    code = _dtype_code(q)
    if q.dim() not in (3, 4):
        raise ValueError("q must be [B, H, n, d] or, for one token of every sequence, [B, H, d]")
    rows = q.shape[2:-1]
    B, Hq, n, d = q.shape[0], q.shape[1], rows[0] if rows else 1, q.shape[-1]
    Hk = 0
    if k is not None:
        _check_same_dtype(q, k=k)
        if k.dim() != q.dim():
            raise ValueError("k must have as many dimensions as q")
        Hk = k.shape[1]
        _check_shape(k, "k", (B, Hk, *rows, d))
    elif k_out is not None:
        raise ValueError("k_out without k")
    _check_as(positions, "positions", torch.int32, (B, *rows))
    if inv_freq.dim() != 1:
        raise ValueError("inv_freq must be [pairs]")
    _check_as(inv_freq, "inv_freq", torch.float32, inv_freq.shape)
    _check_as(q_out, "q_out", q.dtype, q.shape)
    _check_as(k_out, "k_out", q.dtype, k.shape if k is not None else ())
    pairs = inv_freq.shape[0]
    _check_sizes(B, Hq, Hk, n, d, pairs)
    _check_tensors(q.device, q=q, k=k, positions=positions, inv_freq=inv_freq, q_out=q_out, k_out=k_out)
    q_out = torch.empty_like(q) if q_out is None else q_out
    if Hk:
        k_out = torch.empty_like(k) if k_out is None else k_out
    elif k is not None:  # (no heads)
        k_out = torch.empty_like(k) if k_out is None else k_out
    _invoke("sata_rotary", q.device, _at(q), _at(k), _at(positions), _at(inv_freq), code, B, Hq, Hk, n, d, pairs,
            int(bool(interleaved)), float(scale), int(back), _at(q_out), _at(k_out))
    return q_out, k_out


def rotary(q, k, positions, inv_freq, interleaved: bool = False, scale: float = 1.0, q_out=None, k_out=None):
    """Queries and keys turned by their positions: pair i of the first 2 * len(inv_freq) entries of a row, entries i and
    len(inv_freq) + i, or 2 i and 2 i + 1 where interleaved, by the angle position * inv_freq[i], times scale;
    the entries behind them stay.

    q: [B, H_q, n, d] and k: [B, H_k, n, d] (or None) with positions [B, n] int32, or [B, H, d] with positions [B] for one
    token of every sequence; inv_freq: float32.  q_out and k_out may be q and k themselves.  Returns (q_out, k_out)."""
    return _turn(q, k, positions, inv_freq, interleaved, scale, False, q_out, k_out)


def rotary_backward(dq, dk, positions, inv_freq, interleaved: bool = False, scale: float = 1.0, q_out=None, k_out=None):
    """Gradients of rotary's inputs from those of its outputs: turned back by the same angles, times scale.
    Arguments and results as in rotary."""
    return _turn(dq, dk, positions, inv_freq, interleaved, scale, True, q_out, k_out)


# ------------------------------------------------------------------ caches of 4 bits an entry

@functools.lru_cache(maxsize=None)
def packed_row_bytes(d: int) -> int:
    """Bytes of a row of d entries (1 to 128) in a cache of 4 bits an entry, a scale and a least value for every 32."""
    _check_sizes(d)
    size = int(load_library().sata_packed_row_bytes(d))
    if size < 0:
        raise ValueError(f"rows of {d} entries; 1 to 128 are supported")
    return size


def _check_packed(cache, name: str, B, H, d):
    if cache.dtype != _torch().uint8:
        raise TypeError(f"{name} is {cache.dtype}, expected torch.uint8")
    if cache.dim() != 4:
        raise ValueError(f"{name} must be [B, H_kv, capacity, row bytes]")
    capacity = cache.shape[2]
    _check_sizes(capacity)
    _check_shape(cache, name, (B, H, capacity, packed_row_bytes(d)))


@functools.lru_cache(maxsize=1024)
def _packed_scratch(B: int, H: int, G: int, capacity: int, dv: int) -> int:
    """(Asked for once for a call's sizes: the question costs as much as a tenth of the call.)"""
    return int(load_library().sata_softmax_step_packed_scratch(B, H, G, capacity, dv))


def packed_write(K, V, first, k, v, counts=None):
    """Rows k [B, H, n, d_k] and v [B, H, n, d_v] into rows first[b] on of the caches K and V [B, H, capacity,
    packed_row_bytes(d)] uint8, the first counts[b] of them (None: all).  first, counts: [B] int32; first may be None
    (zero), V and v may both be None.  Rows outside of the caches are left out."""
    torch = _torch()
    code = _dtype_code(k)
    if k.dim() != 4:
        raise ValueError("k must be [B, H_kv, n, d_k]")
    B, H, n, dk = k.shape
    _check_sizes(B, H, n, dk)
    _check_packed(K, "K", B, H, dk)
    if (V is None) != (v is None):
        raise ValueError("V and v come together")
    dv = 1
    if v is not None:
        _check_same_dtype(k, v=v)
        dv = v.shape[-1]
        _check_shape(v, "v", (B, H, n, dv))
        _check_packed(V, "V", B, H, dv)
        if V.shape[2] != K.shape[2]:
            raise ValueError("K and V must have the same capacity")
    _check_as(first, "first", torch.int32, (B,))
    _check_as(counts, "counts", torch.int32, (B,))
    _check_tensors(k.device, K=K, V=V, first=first, k=k, v=v, counts=counts)
    _invoke("sata_packed_write", k.device, _at(K), _at(V), K.shape[2], _at(first), _at(k), _at(v), _at(counts), code, B, H,
            n, dk, dv)


def packed_read(cache, first, n: int, d: int, dtype, x=None):
    """What rows first[b] .. first[b] + n - 1 (first None: from 0) of a cache [B, H, capacity, packed_row_bytes(d)] stand
    for, [B, H, n, d] in dtype; zero for rows outside of the cache."""
    torch = _torch()
    if cache.dim() != 4:
        raise ValueError("cache must be [B, H_kv, capacity, row bytes]")
    B, H = cache.shape[:2]
    if n < 0:
        raise ValueError(f"n={n} < 0")
    _check_sizes(B, H, n)
    _check_packed(cache, "cache", B, H, d)
    _check_as(first, "first", torch.int32, (B,))
    _check_as(x, "x", dtype, (B, H, n, d))
    _check_tensors(cache.device, cache=cache, first=first, x=x)
    if x is None:
        x = torch.empty(B, H, n, d, dtype=dtype, device=cache.device)
    _invoke("sata_packed_read", cache.device, _at(cache), cache.shape[2], _at(first), _dtype_code(x), B, H, n, d, _at(x))
    return x


def softmax_step_packed(K, V, lengths, q, k, v, y=None):
    """softmax_step over caches of 4 bits an entry, K and V [B, H_kv, capacity, packed_row_bytes(d)] uint8: k and v are
    written as row lengths[b] in those bits and count as what they stand for, then q attends over rows 0..lengths[b].
    Arguments and result otherwise as there."""
    torch = _torch()
    code, B, H, G, dk, dv = _token_sizes(q, k, v)
    _check_packed(K, "K", B, H, dk)
    _check_packed(V, "V", B, H, dv)
    cap = K.shape[2]
    if V.shape[2] != cap:
        raise ValueError("K and V must have the same capacity")
    _check_as(lengths, "lengths", torch.int32, (B,))
    _check_as(y, "y", q.dtype, (B, G * H, dv))
    _check_tensors(q.device, K=K, V=V, lengths=lengths, q=q, k=k, v=v, y=y)
    if y is None:
        y = torch.empty(B, G * H, dv, dtype=q.dtype, device=q.device)
    scratch = _scratch(_packed_scratch(B, H, G, cap, dv), q.device)
    _invoke("sata_softmax_step_packed", q.device, _at(K), _at(V), cap, _at(lengths), _at(q), _at(k), _at(v), code, B, H, G,
            dk, dv, _at(y), _at(scratch))
    return y


def release():
    load_library().sata_release()
