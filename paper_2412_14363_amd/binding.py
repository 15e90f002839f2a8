"""Python binding of the C ABI in ``include/resq.h``.

Argument marshalling only: every function here has the name of the C entry
point it calls, takes torch tensors (device memory and streams are the only
things torch is used for), checks their dtype/device, and passes raw pointers.
All arithmetic runs in the HIP kernels.  There is no CPU fallback: if the
library cannot be loaded, importing the symbols raises.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import Optional

import torch

from . import build as _build

RESQ_OK = 0
STATUS_NAMES = {0: "RESQ_OK", 1: "RESQ_ERR_NULL", 2: "RESQ_ERR_SHAPE", 3: "RESQ_ERR_ALIGN",
                4: "RESQ_ERR_BUFFER", 5: "RESQ_ERR_HIP"}

# every symbol include/resq.h declares: name -> (restype, argtypes)
_i64, _p, _sz = C.c_int64, C.c_void_p, C.c_size_t
SYMBOLS = {
    "resq_status_string": (C.c_char_p, [C.c_int]),
    "resq_time_next_kernel": (C.c_int, [_p, _p]),
    "resq_act_hi_ld": (_i64, [_i64, _i64]),
    "resq_act_lo_ld": (_i64, [_i64, _i64]),
    "resq_packed_weight_bytes": (_sz, [_i64, _i64, _i64]),
    "resq_hadamard_block": (_i64, [_i64]),
    "resq_quantize_act": (C.c_int, [_p, _i64, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p]),
    "resq_hadamard_quantize_act": (C.c_int, [_p, _i64, _i64, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _i64, _p]),
    "resq_quantize_act_asym": (C.c_int, [_p, _i64, _i64, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _p, _p]),
    "resq_hadamard_quantize_act_asym": (C.c_int, [_p, _i64, _i64, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _p, _p, _i64, _p]),
    "resq_gemm_mixed_asym": (C.c_int, [_p, _p, _p, _p, _p, _p, _p, _i64, _p, _i64, _i64, _i64, _p, _i64, _p, _p, _p]),
    "resq_gemm_mixed_plan": (C.c_int, [_i64, _i64, _i64, _i64, C.POINTER(C.c_int), C.POINTER(C.c_int), C.POINTER(C.c_int)]),
    "resq_gemm_mixed_low_fp8": (C.c_int, [_i64, _i64, _i64, _i64]),
    "resq_quantize_gemm_mixed": (C.c_int, [_p, _i64, _i64, _p, _i64, _i64, _i64, _p, _i64, _p]),
    "resq_gemm_mixed_swiglu": (C.c_int, [_p, _p, _p, _p, _p, _i64, _p, _i64, _i64, _i64, _p, _i64, _p]),
    "resq_gram_accumulate": (C.c_int, [_p, _i64, _i64, _i64, _p, _i64, _p]),
    "resq_sym_eig_workspace_bytes": (_sz, [_i64]),
    "resq_sym_eig": (C.c_int, [_p, _i64, _i64, C.c_int, _p, _p, _i64, _p, _sz, _p]),
    "resq_sym_eig_static": (C.c_int, [_p, _i64, _i64, C.c_int, _p, _p, _i64, _p]),
    "resq_project_rows": (C.c_int, [_p, C.c_int, _i64, _i64, _i64, _p, _i64, _i64, _p, C.c_int, _i64, _p]),
    "resq_project_rows_plan": (C.c_int, [_p, C.c_int, _i64, _i64, _i64, _p, _i64, _i64, _p, C.c_int, _i64, C.POINTER(C.c_int)]),
    "resq_project_heads": (C.c_int, [_p, _i64, _i64, _i64, _p, _p, _i64, _p]),
    "resq_kv_cache_row_bytes": (_sz, [_i64, _i64]),
    "resq_quantize_kv_cache": (C.c_int, [_p, _i64, _i64, _i64, _i64, _p, _i64, _p]),
    "resq_dequantize_kv_cache": (C.c_int, [_p, _i64, _i64, _i64, _i64, _p, _i64, _p]),
    "resq_kv_slots": (C.c_int, [_p, _p, _i64, _i64, _i64, _p, _i64, _p, _p, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _p]),
    "resq_rope_frequencies": (C.c_int, [_i64, C.c_double, C.c_int, C.c_double, C.c_double, C.c_double, _i64, _p, _p]),
    "resq_rope_heads": (C.c_int, [_p, _i64, _i64, _i64, _i64, _i64, _i64, _p, _p, C.c_float, _p, _p, _i64, C.c_int, C.c_float,
                                  _p, _i64, _i64, _p]),
    "resq_append_kv_cache": (C.c_int, [_p, _i64, _i64, _p, _i64, _i64, _i64, _i64, _i64, _i64, _p, _p, _p, _i64, _i64, _i64, _i64,
                                       _i64, _p]),
    "resq_gather_kv_cache": (C.c_int, [_p, _p, _i64, _i64, _i64, _i64, _i64, _p, _i64, _i64, _i64, _i64, _p, _i64, _i64, _p, _i64,
                                       _i64, _p]),
    "resq_attend_kv_cache_workspace_bytes": (_sz, [_i64, _i64, _i64, _i64]),
    "resq_attend_kv_cache": (C.c_int, [_p, _i64, _i64, _i64, _i64, _i64, _i64, _i64, _p, _p, _i64, _i64, _p, _p, _i64, _i64, _i64, _i64,
                                       _i64, C.c_float, C.c_float, _i64, _p, _i64, _i64, _p, _p, _sz, _p]),
    "resq_attend_prompts_workspace_bytes": (_sz, [_i64] * 6),
    "resq_attend_prompts": (C.c_int, [_p, _i64, _i64, _i64, _p, _i64, _i64, _p, _i64, _i64, _i64, _p, _p, _i64, _i64, _i64, _i64, C.c_float,
                                      C.c_float, _i64, _p, _i64, _i64, _p, _p, _sz, _p]),
    "resq_attend_kv_prefix_workspace_bytes": (_sz, [_i64, _i64, _i64, _i64]),
    "resq_attend_kv_prefix": (C.c_int, [_p, _i64, _i64, _i64, _i64, _i64, _i64, _i64, _p, _p, _i64, _p, _p, _i64, _i64, _p, _p, _i64, _i64, _i64,
                                        _i64, _i64, C.c_float, C.c_float, _i64, _p, _i64, _i64, _p, _p, _sz, _p]),
    "resq_norm_residual": (C.c_int, [_p, _i64, _p, _i64, _p, _i64, C.c_int, _i64, _i64, _p, _p, C.c_float, C.c_float, C.c_float, _p, _i64, _p,
                                     _i64, _p]),
    "resq_pack_weights": (C.c_int, [_p, _i64, _i64, _i64, _i64, _p, _sz, _p]),
    "resq_unpack_weights": (C.c_int, [_p, _i64, _i64, _i64, _p, _p, _p, _p, _p]),
    "resq_gemm_mixed": (C.c_int, [_p, _p, _p, _p, _p, _i64, _p, _i64, _i64, _i64, _p, _i64, _p, _p, _p]),
    "resq_online_hadamard": (C.c_int, [_p, _p, _i64, _i64, _i64, _i64, _i64, _i64, _p]),
}

_lib = None


class ResqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().resq_status_string(status).decode()
        super().__init__(f"{where}: {msg}")


def lib() -> C.CDLL:
    """The loaded HIP library (built on first use if no library is there)."""
    global _lib
    if _lib is None:
        path = _build.ensure_built()
        handle = C.CDLL(str(path))
        for name, (res, args) in SYMBOLS.items():
            fn = getattr(handle, name)  # AttributeError if the symbol is missing
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _check(status: int, where: str) -> None:
    if status != RESQ_OK:
        raise ResqError(status, where)


def _dev(t: Optional[torch.Tensor], dtype, name: str):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _check_layer_buffers(where: str, act: "ActCodes", packed: torch.Tensor, N: int, n_out: int,
                         y: torch.Tensor, dbg=(), want_asym: bool = False) -> None:
    """Sizes the kernels rely on: a mismatch would make them read or write past a buffer."""
    M, K, r = act.M, act.K, act.r
    need = resq_packed_weight_bytes(N, K, r)
    if need == 0:
        raise ValueError(f"{where}: invalid (N, K, r) = ({N}, {K}, {r})")
    if packed.numel() < need:
        raise ValueError(f"{where}: packed holds {packed.numel()} bytes, (N, K, r) = ({N}, {K}, {r}) needs {need}")
    if act.asym != want_asym:
        raise ValueError(f"{where}: the activation codes are {'asymmetric' if act.asym else 'symmetric'}; "
                         f"use resq_gemm_mixed{'_asym' if act.asym else ''}")
    if y.shape != (M, n_out):
        raise ValueError(f"{where}: y must be [{M}, {n_out}], got {tuple(y.shape)}")
    for name, t in dbg:
        if t is not None and (tuple(t.shape) != (M, N) or not t.is_contiguous()):
            raise ValueError(f"{where}: {name} must be a contiguous [{M}, {N}] tensor")
    if act.q_hi.shape != (M, act.ld_hi) or act.q_lo.shape != (M, act.ld_lo) or act.ld_hi != resq_act_hi_ld(K, r) \
            or act.ld_lo != resq_act_lo_ld(K, r):
        raise ValueError(f"{where}: activation code buffers do not match (M, K, r) = ({M}, {K}, {r})")


# The raw handle of a device's current stream.  torch.cuda.current_stream() builds a Stream object
# around it, 2.7 us a call, a third of a small call's host time; asked for on every call all the same,
# since it is the caller's to change.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)
# The current device, without torch.cuda.current_device()'s look at whether torch has been initialized: there is a tensor
# in device memory, whose checks come first in every call (0.27 -> 0.13 us for device and stream, of 4.5 to 5.1 a call, which is
# what bounds the smallest ones).
_raw_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream(stream) -> int:
    if stream is None:
        return _raw_stream(_raw_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


# Buffers that a call makes for itself.  The allocator orders a block's uses on the stream that it was allocated on alone: one from the
# current stream's share may still be written by that stream's unfinished work when a kernel on another stream begins on it.  So
# they are allocated on the call's own stream, and what is handed out is recorded on the current one, where the caller goes on with
# it: freed, it is not handed out again before what that stream has by then is done.

def _made(make, stream, device: torch.device, handed_out: bool = True):
    """What make() allocates (a tensor, a tuple of them or an object that holds them) for a call on `stream`."""
    if stream is None or device.type != "cuda":
        return make()
    if not hasattr(stream, "cuda_stream"):   # a handle; 0 is the default stream's
        stream = torch.cuda.ExternalStream(int(stream), device) if int(stream) else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        new = make()
    if handed_out:
        current = torch.cuda.current_stream(device)
        for t in (new,) if isinstance(new, torch.Tensor) else new if isinstance(new, tuple) else vars(new).values():
            if isinstance(t, torch.Tensor):
                t.record_stream(current)
    return new


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """An output that a call makes for itself."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    return _made(lambda: torch.empty(shape, dtype=dtype, device=device), stream, device)


# ---- layout queries ---------------------------------------------------------
# Functions of their arguments alone, asked for by every GEMM call's buffer checks: the last answers
# are kept (0.1 us instead of 0.9).

@functools.lru_cache(maxsize=1024, typed=True)
def resq_act_hi_ld(K: int, r: int) -> int:
    return int(lib().resq_act_hi_ld(K, r))


@functools.lru_cache(maxsize=1024, typed=True)
def resq_act_lo_ld(K: int, r: int) -> int:
    return int(lib().resq_act_lo_ld(K, r))


@functools.lru_cache(maxsize=1024, typed=True)
def resq_packed_weight_bytes(N: int, K: int, r: int) -> int:
    return int(lib().resq_packed_weight_bytes(N, K, r))


def resq_hadamard_block(width: int) -> int:
    return int(lib().resq_hadamard_block(width))


# ---- buffers ----------------------------------------------------------------

class ActCodes:
    """Device buffers resq_quantize_act writes and resq_gemm_mixed reads."""

    def __init__(self, M: int, K: int, r: int, device="cuda"):
        self.M, self.K, self.r = M, K, r
        self.ld_hi, self.ld_lo = resq_act_hi_ld(K, r), resq_act_lo_ld(K, r)
        if self.ld_hi < 0:
            raise ValueError("invalid (K, r)")
        self.q_hi = torch.empty((M, self.ld_hi), dtype=torch.int8, device=device)
        self.q_lo = torch.empty((M, self.ld_lo), dtype=torch.uint8, device=device)
        self.s_hi = torch.empty(M, dtype=torch.float32, device=device)
        self.s_lo = torch.empty(M, dtype=torch.float32, device=device)
        self.lo_sum = torch.empty(M, dtype=torch.int32, device=device)
        # asymmetric codes only (resq_quantize_act_asym): real value of the stored code 0
        self.c_hi = torch.empty(M, dtype=torch.float32, device=device)
        self.c_lo = torch.empty(M, dtype=torch.float32, device=device)
        self.asym = False


def alloc_packed(N: int, K: int, r: int, device="cuda") -> torch.Tensor:
    nbytes = resq_packed_weight_bytes(N, K, r)
    if nbytes == 0:
        raise ValueError("invalid (N, K, r)")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


# ---- the entry points -------------------------------------------------------

def resq_quantize_act(x: torch.Tensor, r: int, out: Optional[ActCodes] = None,
                      stream=None) -> ActCodes:
    M, K = x.shape
    if x.stride(1) != 1:
        raise ValueError("x must be row-major")
    if out is None:
        out = _made(lambda: ActCodes(M, K, r, x.device), stream, x.device)
    st = lib().resq_quantize_act(_dev(x, torch.bfloat16, "x"), x.stride(0), M, K, r,
                                 out.q_hi.data_ptr() if r > 0 else None,
                                 out.q_lo.data_ptr() if K - r > 0 else None,
                                 out.s_hi.data_ptr() if r > 0 else None,
                                 out.s_lo.data_ptr() if K - r > 0 else None,
                                 out.lo_sum.data_ptr() if K - r > 0 else None, _stream(stream))
    _check(st, "resq_quantize_act")
    return out


def resq_hadamard_quantize_act(x: torch.Tensor, r: int, block: int = 0,
                               out: Optional[ActCodes] = None,
                               x_rot: Optional[torch.Tensor] = None, stream=None) -> ActCodes:
    M, K = x.shape
    if x.stride(1) != 1:
        raise ValueError("x must be row-major")
    if x_rot is not None and x_rot.stride(1) != 1:
        raise ValueError("x_rot must be row-major")
    if out is None:
        out = _made(lambda: ActCodes(M, K, r, x.device), stream, x.device)
    st = lib().resq_hadamard_quantize_act(
        _dev(x, torch.bfloat16, "x"), x.stride(0), M, K, r, block,
        out.q_hi.data_ptr() if r > 0 else None, out.q_lo.data_ptr(),
        out.s_hi.data_ptr() if r > 0 else None, out.s_lo.data_ptr(), out.lo_sum.data_ptr(),
        _dev(x_rot, torch.bfloat16, "x_rot"), x_rot.stride(0) if x_rot is not None else 0,
        _stream(stream))
    _check(st, "resq_hadamard_quantize_act")
    return out


def resq_quantize_act_asym(x: torch.Tensor, r: int, hadamard_block: int = 0,
                           out: Optional[ActCodes] = None, stream=None) -> ActCodes:
    M, K = x.shape
    if x.stride(1) != 1:
        raise ValueError("x must be row-major")
    if out is None:
        out = _made(lambda: ActCodes(M, K, r, x.device), stream, x.device)
    hi, lo = r > 0, K - r > 0
    st = lib().resq_quantize_act_asym(
        _dev(x, torch.bfloat16, "x"), x.stride(0), M, K, r, hadamard_block,
        out.q_hi.data_ptr() if hi else None, out.q_lo.data_ptr() if lo else None,
        out.s_hi.data_ptr() if hi else None, out.s_lo.data_ptr() if lo else None,
        out.c_hi.data_ptr() if hi else None, out.c_lo.data_ptr() if lo else None,
        out.lo_sum.data_ptr() if lo else None, _stream(stream))
    _check(st, "resq_quantize_act_asym")
    out.asym = True
    return out


def resq_gemm_mixed_plan(M: int, N: int, K: int, r: int):
    """(kernel, token_groups, runs) that resq_gemm_mixed uses for this shape; host only."""
    k, tg, sk = C.c_int(), C.c_int(), C.c_int()
    _check(lib().resq_gemm_mixed_plan(M, N, K, r, C.byref(k), C.byref(tg), C.byref(sk)), "resq_gemm_mixed_plan")
    return k.value, tg.value, sk.value


def resq_gemm_mixed_low_fp8(M: int, N: int, K: int, r: int) -> bool:
    """Whether the 128 x 128 tiles take the low group of this shape as fp8 numbers; host only."""
    return bool(lib().resq_gemm_mixed_low_fp8(M, N, K, r))


def resq_quantize_gemm_mixed(x: torch.Tensor, packed: torch.Tensor, N: int, r: int,
                             y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    M, K = x.shape
    if x.stride(1) != 1:
        raise ValueError("x must be row-major")
    if y is None:
        y = _empty((M, N), torch.bfloat16, x.device, stream)
    if y.stride(1) != 1:
        raise ValueError("y must be row-major")
    need = resq_packed_weight_bytes(N, K, r)
    if need == 0 or packed.numel() < need or y.shape != (M, N):
        raise ValueError(f"resq_quantize_gemm_mixed: packed ({packed.numel()} bytes, needs {need}) or y "
                         f"{tuple(y.shape)} do not match (M, N, K, r) = ({M}, {N}, {K}, {r})")
    st = lib().resq_quantize_gemm_mixed(
        _dev(x, torch.bfloat16, "x"), x.stride(0), M, _dev(packed, torch.uint8, "packed"), N, K, r,
        _dev(y, torch.bfloat16, "y"), y.stride(0), _stream(stream))
    _check(st, "resq_quantize_gemm_mixed")
    return y


def resq_hadamard_quantize_act_asym(x: torch.Tensor, r: int, block: int = 0,
                                    out: Optional[ActCodes] = None,
                                    x_rot: Optional[torch.Tensor] = None, stream=None) -> ActCodes:
    M, K = x.shape
    if x.stride(1) != 1:
        raise ValueError("x must be row-major")
    if x_rot is not None and x_rot.stride(1) != 1:
        raise ValueError("x_rot must be row-major")
    if out is None:
        out = _made(lambda: ActCodes(M, K, r, x.device), stream, x.device)
    hi = r > 0
    st = lib().resq_hadamard_quantize_act_asym(
        _dev(x, torch.bfloat16, "x"), x.stride(0), M, K, r, block,
        out.q_hi.data_ptr() if hi else None, out.q_lo.data_ptr(),
        out.s_hi.data_ptr() if hi else None, out.s_lo.data_ptr(),
        out.c_hi.data_ptr() if hi else None, out.c_lo.data_ptr(), out.lo_sum.data_ptr(),
        _dev(x_rot, torch.bfloat16, "x_rot"), x_rot.stride(0) if x_rot is not None else 0,
        _stream(stream))
    _check(st, "resq_hadamard_quantize_act_asym")
    out.asym = True
    return out


def resq_gemm_mixed_asym(act: ActCodes, packed: torch.Tensor, N: int,
                         y: Optional[torch.Tensor] = None,
                         dbg_acc_hi: Optional[torch.Tensor] = None,
                         dbg_acc_lo: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    M, K, r = act.M, act.K, act.r
    if y is None:
        y = _empty((M, N), torch.bfloat16, packed.device, stream)
    if y.stride(1) != 1:
        raise ValueError("y must be row-major")
    _check_layer_buffers("resq_gemm_mixed_asym", act, packed, N, N, y,
                         (("dbg_acc_hi", dbg_acc_hi), ("dbg_acc_lo", dbg_acc_lo)), want_asym=True)
    hi, lo = r > 0, K - r > 0
    st = lib().resq_gemm_mixed_asym(
        act.q_hi.data_ptr() if hi else None, act.q_lo.data_ptr() if lo else None,
        act.s_hi.data_ptr() if hi else None, act.s_lo.data_ptr() if lo else None,
        act.c_hi.data_ptr() if hi else None, act.c_lo.data_ptr() if lo else None,
        act.lo_sum.data_ptr() if lo else None, M, _dev(packed, torch.uint8, "packed"), N, K, r,
        _dev(y, torch.bfloat16, "y"), y.stride(0), _dev(dbg_acc_hi, torch.int32, "dbg_acc_hi"),
        _dev(dbg_acc_lo, torch.int32, "dbg_acc_lo"), _stream(stream))
    _check(st, "resq_gemm_mixed_asym")
    return y


def resq_pack_weights(w: torch.Tensor, r: int, packed: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    N, K = w.shape
    if w.stride(1) != 1:
        raise ValueError("w must be row-major [N, K]")
    if packed is None:
        packed = _made(lambda: alloc_packed(N, K, r, w.device), stream, w.device)
    st = lib().resq_pack_weights(_dev(w, torch.bfloat16, "w"), w.stride(0), N, K, r,
                                 _dev(packed, torch.uint8, "packed"), packed.numel(),
                                 _stream(stream))
    _check(st, "resq_pack_weights")
    return packed


def resq_unpack_weights(packed: torch.Tensor, N: int, K: int, r: int, stream=None):
    dev = packed.device
    need = resq_packed_weight_bytes(N, K, r)
    if need == 0 or packed.numel() < need:
        raise ValueError(f"resq_unpack_weights: packed holds {packed.numel()} bytes, (N, K, r) = ({N}, {K}, {r}) needs {need}")
    w_hi = _empty((N, r), torch.int8, dev, stream)
    w_lo = _empty((N, K - r), torch.int8, dev, stream)
    sw_hi = _empty(N, torch.int16, dev, stream)
    sw_lo = _empty(N, torch.int16, dev, stream)
    st = lib().resq_unpack_weights(_dev(packed, torch.uint8, "packed"), N, K, r,
                                   w_hi.data_ptr() if r > 0 else None,
                                   w_lo.data_ptr() if K - r > 0 else None,
                                   sw_hi.data_ptr() if r > 0 else None,
                                   sw_lo.data_ptr() if K - r > 0 else None, _stream(stream))
    _check(st, "resq_unpack_weights")
    return w_hi, w_lo, sw_hi, sw_lo


def resq_gemm_mixed(act: ActCodes, packed: torch.Tensor, N: int, y: Optional[torch.Tensor] = None,
                    dbg_acc_hi: Optional[torch.Tensor] = None,
                    dbg_acc_lo: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    M, K, r = act.M, act.K, act.r
    if y is None:
        y = _empty((M, N), torch.bfloat16, packed.device, stream)
    if y.stride(1) != 1:
        raise ValueError("y must be row-major")
    _check_layer_buffers("resq_gemm_mixed", act, packed, N, N, y,
                         (("dbg_acc_hi", dbg_acc_hi), ("dbg_acc_lo", dbg_acc_lo)))
    st = lib().resq_gemm_mixed(act.q_hi.data_ptr() if r > 0 else None,
                               act.q_lo.data_ptr() if K - r > 0 else None,
                               act.s_hi.data_ptr() if r > 0 else None,
                               act.s_lo.data_ptr() if K - r > 0 else None,
                               act.lo_sum.data_ptr() if K - r > 0 else None, M,
                               _dev(packed, torch.uint8, "packed"), N, K, r,
                               _dev(y, torch.bfloat16, "y"), y.stride(0),
                               _dev(dbg_acc_hi, torch.int32, "dbg_acc_hi"),
                               _dev(dbg_acc_lo, torch.int32, "dbg_acc_lo"), _stream(stream))
    _check(st, "resq_gemm_mixed")
    return y


def resq_gemm_mixed_swiglu(act: ActCodes, packed: torch.Tensor, N2: int,
                           y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """packed: 2F interleaved (gate, up) channels; returns y [M, F] = silu(gate) * up."""
    M, K, r = act.M, act.K, act.r
    if y is None:
        y = _empty((M, N2 // 2), torch.bfloat16, packed.device, stream)
    if y.stride(1) != 1:
        raise ValueError("y must be row-major")
    if N2 % 2:
        raise ValueError("resq_gemm_mixed_swiglu: N2 must be even (interleaved gate and up rows)")
    _check_layer_buffers("resq_gemm_mixed_swiglu", act, packed, N2, N2 // 2, y)
    hi, lo = r > 0, K - r > 0
    st = lib().resq_gemm_mixed_swiglu(
        act.q_hi.data_ptr() if hi else None, act.q_lo.data_ptr() if lo else None,
        act.s_hi.data_ptr() if hi else None, act.s_lo.data_ptr() if lo else None,
        act.lo_sum.data_ptr() if lo else None, M, _dev(packed, torch.uint8, "packed"), N2, K, r,
        _dev(y, torch.bfloat16, "y"), y.stride(0), _stream(stream))
    _check(st, "resq_gemm_mixed_swiglu")
    return y


def resq_gram_accumulate(x: torch.Tensor, c: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """c (fp32 [K, K], zeros when not given) += x^T x for x bf16 [T, K]."""
    T, K = x.shape
    if x.stride(1) != 1:
        raise ValueError("x must be row-major")
    if c is None:
        c = _made(lambda: torch.zeros((K, K), dtype=torch.float32, device=x.device), stream, x.device)   # (cleared where it is added to)
    st = lib().resq_gram_accumulate(_dev(x, torch.bfloat16, "x"), x.stride(0), T, K,
                                    _dev(c, torch.float32, "c"), c.stride(0), _stream(stream))
    _check(st, "resq_gram_accumulate")
    return c


def resq_sym_eig(c: torch.Tensor, sweeps: int = 12, stream=None):
    """Eigenvalues (decreasing, fp32 [K]) and eigenvectors (columns of fp32 [K, K]) of the symmetric c."""
    K = c.shape[0]
    nbytes = lib().resq_sym_eig_workspace_bytes(K)
    work = _made(lambda: torch.empty(max(nbytes, 1), dtype=torch.uint8, device=c.device), stream, c.device, handed_out=False)
    lam = _empty(K, torch.float32, c.device, stream)
    p = _empty((K, K), torch.float32, c.device, stream)
    st = lib().resq_sym_eig(_dev(c, torch.float32, "c"), c.stride(0), K, sweeps, lam.data_ptr(), p.data_ptr(),
                            p.stride(0), work.data_ptr(), nbytes, _stream(stream))
    _check(st, "resq_sym_eig")
    return lam, p


def resq_sym_eig_static(c: torch.Tensor, lam: torch.Tensor, p: torch.Tensor, sweeps: int = 12, stream=None):
    """resq_sym_eig into caller-provided outputs (lam fp32 [K], p fp32 [K, K]) on the library's
    built-in scratch area (K <= 512): the call itself allocates nothing."""
    K = c.shape[0]
    if tuple(lam.shape) != (K,) or tuple(p.shape) != (K, K) or p.stride(1) != 1:
        raise ValueError("lam must be [K] and p a row-major [K, K]")
    st = lib().resq_sym_eig_static(_dev(c, torch.float32, "c"), c.stride(0), K, sweeps, _dev(lam, torch.float32, "lam"),
                                   _dev(p, torch.float32, "p"), p.stride(0), _stream(stream))
    _check(st, "resq_sym_eig_static")
    return lam, p


def resq_project_rows(a: torch.Tensor, u: torch.Tensor, out: Optional[torch.Tensor] = None,
                      out_dtype=None, stream=None) -> torch.Tensor:
    """out = a @ u; a bf16 or fp32 [rows, K] (a column block of a wider matrix is fine), u fp32
    [K, J]; out bf16 or fp32 [rows, J] (a column block of a wider matrix is fine)."""
    rows, K = a.shape
    J = u.shape[1]
    if a.stride(1) != 1 or u.stride(1) != 1 or u.shape[0] != K:
        raise ValueError("a, u must be row-major with matching inner size")
    if a.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("a must be bf16 or fp32")
    if out is None:
        out = _empty((rows, J), out_dtype or a.dtype, a.device, stream)
    if out.stride(1) != 1 or out.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("out must be row-major bf16 or fp32")
    st = lib().resq_project_rows(_dev(a, a.dtype, "a"), int(a.dtype == torch.bfloat16), a.stride(0), rows, K,
                                 _dev(u, torch.float32, "u"), u.stride(0), J,
                                 _dev(out, out.dtype, "out"), int(out.dtype == torch.bfloat16), out.stride(0),
                                 _stream(stream))
    _check(st, "resq_project_rows")
    return out


def resq_project_rows_plan(a: torch.Tensor, u: torch.Tensor, out: torch.Tensor) -> int:
    """The kernel that resq_project_rows uses for these operands (0, 1 or 2, see include/resq.h); host only."""
    kernel = C.c_int()
    _check(lib().resq_project_rows_plan(a.data_ptr(), int(a.dtype == torch.bfloat16), a.stride(0), a.shape[0], a.shape[1],
                                        u.data_ptr(), u.stride(0), u.shape[1], out.data_ptr(),
                                        int(out.dtype == torch.bfloat16), out.stride(0), C.byref(kernel)),
           "resq_project_rows_plan")
    return kernel.value


def resq_project_heads(x: torch.Tensor, packed: torch.Tensor, y: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """x: bf16 [rows, d_head] (one row per token and head); packed: resq_pack_weights of the
    [d_head, d_head] matrix of output-channel rows with r = d_head; returns bf16 [rows, d_head]."""
    rows, d = x.shape
    if x.stride(1) != 1:
        raise ValueError("x must be row-major")
    if y is None:
        y = _empty((rows, d), torch.bfloat16, x.device, stream)
    if y.stride(1) != 1:
        raise ValueError("y must be row-major")
    need = resq_packed_weight_bytes(d, d, d)
    if need == 0 or packed.numel() < need or tuple(y.shape) != (rows, d):
        raise ValueError(f"resq_project_heads: packed ({packed.numel()} bytes, needs {need}) or y {tuple(y.shape)} "
                         f"do not match rows = {rows}, d_head = {d}")
    st = lib().resq_project_heads(_dev(x, torch.bfloat16, "x"), x.stride(0), rows, d,
                                  _dev(packed, torch.uint8, "packed"),
                                  _dev(y, torch.bfloat16, "y"), y.stride(0),
                                  _stream(stream))
    _check(st, "resq_project_heads")
    return y


@functools.lru_cache(maxsize=1024, typed=True)
def resq_kv_cache_row_bytes(d_head: int, r: int) -> int:
    return int(lib().resq_kv_cache_row_bytes(d_head, r))


def resq_quantize_kv_cache(x: torch.Tensor, r: int, cache: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x: bf16 [rows, d_head] (one row per token and head) -> uint8 [rows, row_bytes] compact cache rows."""
    rows, d = x.shape
    if x.stride(1) != 1:
        raise ValueError("x must be row-major")
    need = resq_kv_cache_row_bytes(d, r)
    if need == 0:
        raise ValueError(f"invalid (d_head, r) = ({d}, {r})")
    if cache is None:
        cache = _empty((rows, need), torch.uint8, x.device, stream)
    have = cache.shape   # (a new object every time it is asked for)
    if len(have) != 2 or have[0] != rows or cache.stride(1) != 1 or have[1] < need:
        raise ValueError(f"cache must be a row-major [{rows}, >= {need}] byte tensor")
    st = lib().resq_quantize_kv_cache(_dev(x, torch.bfloat16, "x"), x.stride(0), rows, d, r,
                                      _dev(cache, torch.uint8, "cache"), cache.stride(0), _stream(stream))
    _check(st, "resq_quantize_kv_cache")
    return cache


def resq_dequantize_kv_cache(cache: torch.Tensor, d_head: int, r: int, out: Optional[torch.Tensor] = None,
                             stream=None) -> torch.Tensor:
    """The reader: bf16 [rows, d_head] = code * s + z of every channel."""
    have = cache.shape
    rows = have[0]
    need = resq_kv_cache_row_bytes(d_head, r)
    if need == 0 or len(have) != 2 or cache.stride(1) != 1 or have[1] < need:
        raise ValueError(f"cache must be a row-major [rows, >= {need}] byte tensor for (d_head, r) = ({d_head}, {r})")
    if out is None:
        out = _empty((rows, d_head), torch.bfloat16, cache.device, stream)
    if out.shape != (rows, d_head) or out.stride(1) != 1:
        raise ValueError(f"out must be a row-major [{rows}, {d_head}] tensor")
    st = lib().resq_dequantize_kv_cache(_dev(cache, torch.uint8, "cache"), cache.stride(0), rows, d_head, r,
                                        _dev(out, torch.bfloat16, "out"), out.stride(0), _stream(stream))
    _check(st, "resq_dequantize_kv_cache")
    return out


# ---- the generation step: plan, position embedding, paged K/V cache, attention --------------------------------
# Sizes are checked here because the kernels rely on them; what the arrays hold (lengths, slots, table entries) is checked by the
# kernels themselves.  A step's calls are bounded by the host: each is checked in one expression, and only a call that fails it is
# looked at part by part for what to say.

_BF16, _I32, _U8 = torch.bfloat16, torch.int32, torch.uint8


def _need(ok: bool, where: str, what: str) -> None:
    if not ok:
        raise ValueError(f"{where}: {what}")


def _explain_devices(where: str, *tensors) -> None:
    """All tensors on the current device: that is where the call's kernels run."""
    for t in tensors:
        if t is not None:
            _need(t.is_cuda, where, "tensors must live in device memory")
            _need(t.get_device() == _raw_device(), where,
                  f"a tensor is on {t.device}, the current device is cuda:{_raw_device()}")


def _explain_ints(where: str, name: str, t: torch.Tensor, n: Optional[int] = None) -> None:
    _need(t.dtype == _I32 and t.dim() == 1 and t.is_contiguous() and (n is None or t.shape[0] == n), where,
          f"{name} must be a contiguous int32 vector" + (f" of {n}" if n is not None else ""))


def _explain_table(where: str, t: torch.Tensor, batch: int) -> None:
    _need(t.dtype == _I32 and t.dim() == 2 and t.shape[0] == batch and t.shape[1] > 0 and t.stride(1) == 1, where,
          f"block_table must be a row-major int32 [{batch}, pages] tensor")


def _explain_heads(where: str, name: str, t: torch.Tensor) -> None:
    _need(t.dtype == _BF16 and t.dim() == 3 and t.stride(2) == 1, where,
          f"{name} must be a bf16 [tokens, heads, d_head] tensor whose rows are contiguous")


@functools.lru_cache(maxsize=1024, typed=True)
def _page_row_bytes(d: int, r: int) -> int:
    """Bytes of a head's row in pages, 0 where there are none; r may also be an odd multiple of four there, see include/resq.h."""
    if r % 8 == 4 and 0 < r < d <= 256 and d % 8 == 0:
        return r + (d - r) // 2 + 16
    return resq_kv_cache_row_bytes(d, r)


def _explain_pages(where: str, k: torch.Tensor, v: torch.Tensor, heads: int, d: int, r: int) -> None:
    need = _page_row_bytes(d, r)
    _need(need > 0, where, f"invalid (d_head, r) = ({d}, {r})")
    _need(k.dim() == 4 and k.dtype == _U8 and v.dtype == _U8 and k.shape[1] == heads and k.shape[3] >= need and k.stride(3) == 1, where,
          f"pages must be uint8 [pages, {heads}, page_size, >= {need}] tensors whose rows are contiguous")
    _need(v.shape == k.shape and v.stride() == k.stride(), where, "k_pages and v_pages must have the same shape and strides")


class KvSlots:
    """Device buffers resq_kv_slots writes: lens [batch], cu_tokens and cu_pages [batch + 1], positions and slots [max_tokens],
    state [2] (entries of the free list gone, status).  All start at 0, slots at -1."""

    def __init__(self, batch: int, max_tokens: int, device="cuda"):
        self.batch, self.max_tokens = batch, max_tokens
        self.lens = torch.zeros(batch, dtype=torch.int32, device=device)
        self.cu_tokens = torch.zeros(batch + 1, dtype=torch.int32, device=device)
        self.cu_pages = torch.zeros(batch + 1, dtype=torch.int32, device=device)
        self.positions = torch.zeros(max_tokens, dtype=torch.int32, device=device)
        self.slots = torch.full((max_tokens,), -1, dtype=torch.int32, device=device)
        self.state = torch.zeros(2, dtype=torch.int32, device=device)
        self.device_index = self.lens.get_device()

    @property
    def pointers(self):
        return (self.lens.data_ptr(), self.cu_tokens.data_ptr(), self.cu_pages.data_ptr(), self.positions.data_ptr(),
                self.slots.data_ptr(), self.state.data_ptr())


def resq_kv_slots(lens: torch.Tensor, new_tokens: torch.Tensor, free_pages: torch.Tensor, taken: Optional[torch.Tensor],
                  block_table: torch.Tensor, page_size: int, num_pages: int, out: Optional[KvSlots] = None,
                  max_tokens: Optional[int] = None, stream=None) -> KvSlots:
    """The plan of a step: positions and slots of new_tokens[b] tokens of each request behind its lens[b], pages off the free
    list into block_table.  taken: how many of free_pages are gone (None: out.state's first entry, i.e. go on from the call
    before).  lens may be out.lens.  out.state[1] is the status, see include/resq.h."""
    batch = lens.shape[0]
    if out is None:
        _need(max_tokens is not None, "resq_kv_slots", "give out or max_tokens")
        out = _made(lambda: KvSlots(batch, max_tokens, lens.device), stream, lens.device)   # (cleared where the plan runs)
    elif not isinstance(out, KvSlots):
        raise ValueError("resq_kv_slots: out must be a KvSlots")
    if taken is None:
        taken = out.state[:1]
    cap = out.max_tokens
    dev = lens.get_device()
    ld_table, one = block_table.stride() if block_table.dim() == 2 else (0, 0)
    if not (lens.dtype == _I32 and new_tokens.dtype == _I32 and free_pages.dtype == _I32 and taken.dtype == _I32
            and block_table.dtype == _I32 and lens.shape == new_tokens.shape == (batch,) and out.batch == batch
            and free_pages.dim() == 1 and taken.shape == (1,) and lens.is_contiguous() and new_tokens.is_contiguous()
            and free_pages.is_contiguous() and one == 1 and block_table.shape[0] == batch and dev >= 0 and dev == _raw_device()
            and new_tokens.get_device() == dev and free_pages.get_device() == dev and taken.get_device() == dev
            and block_table.get_device() == dev and out.device_index == dev):
        where = "resq_kv_slots"
        _explain_devices(where, lens, new_tokens, free_pages, taken, block_table, out.lens)
        _explain_ints(where, "lens", lens)
        _explain_ints(where, "new_tokens", new_tokens, batch)
        _explain_ints(where, "free_pages", free_pages)
        _explain_ints(where, "taken", taken, 1)
        _explain_table(where, block_table, batch)
        raise ValueError(f"{where}: out holds {out.batch} requests, lens {batch}")
    st = lib().resq_kv_slots(
        lens.data_ptr(), new_tokens.data_ptr(), batch, page_size, num_pages, free_pages.data_ptr(), free_pages.shape[0],
        taken.data_ptr(), block_table.data_ptr(), ld_table, block_table.shape[1], cap, *out.pointers, _stream(stream))
    if st:
        _check(st, "resq_kv_slots")
    return out


ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}


def resq_rope_frequencies(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, low: float = 1.0,
                          high: float = 4.0, original_len: int = 8192, device="cuda"):
    """(freq fp64 [rot / 2] on `device`, mscale) for resq_rope_heads; scaling: see include/resq.h."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(ROPE_SCALINGS)}, got {scaling!r}")
    freq, mscale = torch.empty(max(rot, 0) // 2, dtype=torch.float64), C.c_float()
    _check(lib().resq_rope_frequencies(rot, base, ROPE_SCALINGS[scaling], factor, low, high, original_len,
                                       freq.data_ptr() if freq.numel() else None, C.byref(mscale)), "resq_rope_frequencies")
    return freq.to(device), mscale.value


def resq_rope_heads(x: torch.Tensor, positions: Optional[torch.Tensor], freq: Optional[torch.Tensor], heads_q: Optional[int] = None,
                    w_q: Optional[torch.Tensor] = None, w_k: Optional[torch.Tensor] = None, eps: float = 1e-6,
                    interleaved: bool = False, mscale: float = 1.0, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x: bf16 [tokens, heads, d_head], the first heads_q heads (None: all) queries, the others keys; positions int32 [tokens];
    freq fp64 [rot / 2] (None or empty: no rotation); w_q, w_k: bf16 [d_head] weights of the heads' norm (None: no norm).
    out may be x."""
    tokens, heads, d = shape = x.shape
    if heads_q is None:
        heads_q = heads
    if out is None:
        out = _empty(shape, _BF16, x.device, stream)
    rot = 0 if freq is None else 2 * freq.shape[0]
    dev = x.get_device()
    ldx, ldxh, one = x.stride()
    ldy, ldyh, one_y = out.stride()
    pos = freqs = wq = wk = None
    ok = (x.dtype == _BF16 and out.dtype == _BF16 and one == 1 and one_y == 1 and out.shape == shape and 0 <= heads_q <= heads
          and dev >= 0 and dev == _raw_device() and out.get_device() == dev)
    if rot and ok:
        ok = (positions is not None and positions.dtype == _I32 and positions.shape == (tokens,) and positions.is_contiguous()
              and freq.dtype == torch.float64 and freq.dim() == 1 and freq.is_contiguous() and positions.get_device() == dev
              and freq.get_device() == dev)
        if ok:
            pos, freqs = positions.data_ptr(), freq.data_ptr()
    if w_q is not None and ok:
        ok = w_q.dtype == _BF16 and w_q.shape == (d,) and w_q.is_contiguous() and w_q.get_device() == dev
        wq = w_q.data_ptr()
    if w_k is not None and ok:
        ok = w_k.dtype == _BF16 and w_k.shape == (d,) and w_k.is_contiguous() and w_k.get_device() == dev
        wk = w_k.data_ptr()
    if not ok:
        where = "resq_rope_heads"
        _explain_heads(where, "x", x)
        _explain_heads(where, "out", out)
        _explain_devices(where, x, positions, freq, w_q, w_k, out)
        _need(out.shape == shape and 0 <= heads_q <= heads, where,
              f"out {tuple(out.shape)}, x {tuple(shape)} or heads_q = {heads_q} do not match")
        _need(not rot or (positions is not None and freq.dtype == torch.float64 and freq.dim() == 1 and freq.is_contiguous()), where,
              "freq must be a contiguous fp64 [rot / 2] tensor, with positions")
        if rot:
            _explain_ints(where, "positions", positions, tokens)
        raise ValueError(f"{where}: w_q and w_k must be contiguous bf16 [{d}] tensors")
    st = lib().resq_rope_heads(x.data_ptr(), ldx, ldxh, tokens, heads_q, heads - heads_q, d, wq, wk, eps, pos, freqs, rot,
                               1 if interleaved else 0, mscale, out.data_ptr(), ldy, ldyh, _stream(stream))
    if st:
        _check(st, "resq_rope_heads")
    return out


def resq_append_kv_cache(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                         r: int, stream=None) -> None:
    """k, v: bf16 [tokens, heads, d_head], quantized into rows `slots` (int32 [tokens], below 0: left out) of the uint8
    [pages, heads, page_size, row bytes] pages."""
    tokens, heads, d = shape = k.shape
    dev = k.get_device()
    ldk, ldkh, one = k.stride()
    ldv, ldvh, one_v = v.stride() if v.dim() == 3 else (0, 0, 0)
    need = _page_row_bytes(d, r)
    n, h, size, width = k_pages.shape if k_pages.dim() == 4 else (0, 0, 0, 0)
    strides = k_pages.stride()
    if not (k.dtype == _BF16 and v.dtype == _BF16 and slots.dtype == _I32 and k_pages.dtype == _U8 and v_pages.dtype == _U8
            and one == 1 and one_v == 1 and v.shape == shape and slots.shape == (tokens,) and slots.is_contiguous()
            and h == heads and 0 < need <= width and strides[3] == 1 and v_pages.shape == k_pages.shape and v_pages.stride() == strides
            and dev >= 0 and dev == _raw_device() and v.get_device() == dev and slots.get_device() == dev
            and k_pages.get_device() == dev and v_pages.get_device() == dev):
        where = "resq_append_kv_cache"
        _explain_heads(where, "k", k)
        _explain_heads(where, "v", v)
        _need(v.shape == shape, where, f"k {tuple(shape)} and v {tuple(v.shape)} do not match")
        _explain_devices(where, k, v, slots, k_pages, v_pages)
        _explain_pages(where, k_pages, v_pages, heads, d, r)
        _explain_ints(where, "slots", slots, tokens)
        raise ValueError(f"{where}: invalid arguments")
    st = lib().resq_append_kv_cache(k.data_ptr(), ldk, ldkh, v.data_ptr(), ldv, ldvh, tokens, heads, d, r, slots.data_ptr(),
                                    k_pages.data_ptr(), v_pages.data_ptr(), n, size, strides[0], strides[1], strides[2],
                                    _stream(stream))
    if st:
        _check(st, "resq_append_kv_cache")


def resq_gather_kv_cache(k_pages: torch.Tensor, v_pages: torch.Tensor, slots: torch.Tensor, r: int,
                         k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None, d_head: Optional[int] = None,
                         stream=None):
    """The values of the rows in `slots` (int32 [tokens]), bf16 [tokens, heads, d_head] each for keys and values; zeros for slots
    outside the pages.  d_head is that of k where k is given."""
    _need(k_pages.dim() == 4, "resq_gather_kv_cache", "pages must be [pages, heads, page_size, row bytes] tensors")
    n, heads, size, width = k_pages.shape
    tokens = slots.shape[0]
    if k is None or v is None:
        _need(k is not None or d_head is not None, "resq_gather_kv_cache", "give k or d_head")
        shape = (tokens, heads, d_head if k is None else k.shape[-1])
        k, v = (_empty(shape, _BF16, k_pages.device, stream) if t is None else t for t in (k, v))
    shape = k.shape
    d = shape[-1]
    dev = k_pages.get_device()
    ldk, ldkh, one = k.stride() if k.dim() == 3 else (0, 0, 0)
    ldv, ldvh, one_v = v.stride() if v.dim() == 3 else (0, 0, 0)
    need = _page_row_bytes(d, r)
    strides = k_pages.stride()
    if not (k.dtype == _BF16 and v.dtype == _BF16 and slots.dtype == _I32 and k_pages.dtype == _U8 and v_pages.dtype == _U8
            and one == 1 and one_v == 1 and shape == (tokens, heads, d) and v.shape == shape and (d_head is None or d_head == d)
            and slots.dim() == 1 and slots.is_contiguous() and 0 < need <= width and strides[3] == 1 and v_pages.shape == k_pages.shape
            and v_pages.stride() == strides and dev >= 0 and dev == _raw_device() and k.get_device() == dev and v.get_device() == dev
            and slots.get_device() == dev and v_pages.get_device() == dev):
        where = "resq_gather_kv_cache"
        _explain_heads(where, "k", k)
        _explain_heads(where, "v", v)
        _need(shape == (tokens, heads, d) and v.shape == shape and (d_head is None or d_head == d), where,
              f"k {tuple(shape)} and v {tuple(v.shape)} must be [{tokens}, {heads}, {d_head or d}]")
        _explain_devices(where, k_pages, v_pages, slots, k, v)
        _explain_pages(where, k_pages, v_pages, heads, d, r)
        _explain_ints(where, "slots", slots, tokens)
        raise ValueError(f"{where}: invalid arguments")
    st = lib().resq_gather_kv_cache(k_pages.data_ptr(), v_pages.data_ptr(), n, size, strides[0], strides[1], strides[2],
                                    slots.data_ptr(), tokens, heads, d, r, k.data_ptr(), ldk, ldkh, v.data_ptr(), ldv, ldvh,
                                    _stream(stream))
    if st:
        _check(st, "resq_gather_kv_cache")
    return k, v


@functools.lru_cache(maxsize=1024, typed=True)
def resq_attend_kv_cache_workspace_bytes(batch: int, heads_q: int, heads_k: int, d_head: int) -> int:
    return int(lib().resq_attend_kv_cache_workspace_bytes(batch, heads_q, heads_k, d_head))


def resq_attend_kv_cache_workspace(batch: int, heads_q: int, heads_k: int, d_head: int, device="cuda") -> torch.Tensor:
    """A workspace for resq_attend_kv_cache calls of these sizes; calls on different streams need one each."""
    nbytes = resq_attend_kv_cache_workspace_bytes(batch, heads_q, heads_k, d_head)
    if nbytes == 0:
        raise ValueError(f"invalid (batch, heads_q, heads_k, d_head) = ({batch}, {heads_q}, {heads_k}, {d_head})")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def resq_attend_kv_cache(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, lens: torch.Tensor,
                         block_table: torch.Tensor, r: int, scale: Optional[float] = None, softcap: float = 0.0, window: int = 0,
                         out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of one new token of each sequence, q: bf16 [batch, heads, d_head], over the first lens[b] tokens of the pages that
    block_table [batch, pages] names.  scale: d_head^-0.5 when None.  lse: fp32 [batch, heads], written where given."""
    batch, heads, d = shape = q.shape
    if out is None:
        out = _empty(shape, _BF16, q.device, stream)
    if batch == 0:
        return out
    n, heads_k, size, width = k_pages.shape if k_pages.dim() == 4 else (0, 0, 0, 0)
    if workspace is None:
        nbytes = resq_attend_kv_cache_workspace_bytes(batch, heads, heads_k, d)
        workspace = _made(lambda: torch.empty(max(nbytes, 1), dtype=_U8, device=q.device), stream, q.device, handed_out=False)
    dev = q.get_device()
    ldq, ldqh, one = q.stride()
    ldo, ldoh, one_o = out.stride() if out.dim() == 3 else (0, 0, 0)
    need = _page_row_bytes(d, r)
    strides = k_pages.stride()
    ld_table, one_t = block_table.stride() if block_table.dim() == 2 else (0, 0)
    sums = None
    ok = (q.dtype == _BF16 and out.dtype == _BF16 and lens.dtype == _I32 and block_table.dtype == _I32 and k_pages.dtype == _U8
          and v_pages.dtype == _U8 and workspace.dtype == _U8 and one == 1 and one_o == 1 and one_t == 1 and out.shape == shape
          and heads_k > 0 and heads % heads_k == 0 and 0 < need <= width and strides[3] == 1 and v_pages.shape == k_pages.shape
          and v_pages.stride() == strides and lens.shape == (batch,) and lens.is_contiguous() and block_table.shape[0] == batch
          and workspace.is_contiguous() and dev >= 0 and dev == _raw_device() and out.get_device() == dev and lens.get_device() == dev
          and block_table.get_device() == dev and k_pages.get_device() == dev and v_pages.get_device() == dev
          and workspace.get_device() == dev)
    if lse is not None and ok:
        ok = lse.dtype == torch.float32 and lse.shape == (batch, heads) and lse.is_contiguous() and lse.get_device() == dev
        sums = lse.data_ptr()
    if not ok:
        where = "resq_attend_kv_cache"
        _explain_heads(where, "q", q)
        _explain_heads(where, "out", out)
        _need(out.shape == shape and heads_k > 0 and heads % heads_k == 0, where,
              f"q {tuple(shape)}, out {tuple(out.shape)} or {heads_k} K/V heads do not match")
        _need(lse is None or (lse.dtype == torch.float32 and lse.shape == (batch, heads) and lse.is_contiguous()), where,
              f"lse must be a contiguous fp32 [{batch}, {heads}] tensor")
        _need(workspace.dtype == _U8 and workspace.is_contiguous(), where, "workspace must be a contiguous uint8 tensor")
        _explain_devices(where, q, k_pages, v_pages, lens, block_table, out, lse, workspace)
        _explain_pages(where, k_pages, v_pages, heads_k, d, r)
        _explain_table(where, block_table, batch)
        _explain_ints(where, "lens", lens, batch)
        raise ValueError(f"{where}: invalid arguments")
    st = lib().resq_attend_kv_cache(
        q.data_ptr(), ldq, ldqh, batch, heads, heads_k, d, r, lens.data_ptr(), block_table.data_ptr(), ld_table, block_table.shape[1],
        k_pages.data_ptr(), v_pages.data_ptr(), n, size, strides[0], strides[1], strides[2], d ** -0.5 if scale is None else scale,
        softcap, window, out.data_ptr(), ldo, ldoh, sums, workspace.data_ptr(), workspace.numel(), _stream(stream))
    if st:
        _check(st, "resq_attend_kv_cache")
    return out


# ---- what stands around a layer's products: attention over whole prompts and behind a shared prefix, the norms between blocks ---------------------------------------

@functools.lru_cache(maxsize=1024, typed=True)
def resq_attend_prompts_workspace_bytes(tokens_q: int, tokens_k: int, batch: int, heads_q: int, heads_k: int, d_head: int) -> int:
    return int(lib().resq_attend_prompts_workspace_bytes(tokens_q, tokens_k, batch, heads_q, heads_k, d_head))


def resq_attend_prompts_workspace(tokens_q: int, tokens_k: int, batch: int, heads_q: int, heads_k: int, d_head: int,
                                  device="cuda") -> torch.Tensor:
    """A workspace for resq_attend_prompts calls of these sizes; calls on different streams need one each."""
    nbytes = resq_attend_prompts_workspace_bytes(tokens_q, tokens_k, batch, heads_q, heads_k, d_head)
    if nbytes == 0:
        raise ValueError(f"invalid (tokens_q, tokens_k, batch, heads_q, heads_k, d_head) = "
                         f"({tokens_q}, {tokens_k}, {batch}, {heads_q}, {heads_k}, {d_head})")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def resq_attend_prompts(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: Optional[torch.Tensor] = None,
                        scale: Optional[float] = None, softcap: float = 0.0, window: int = 0, out: Optional[torch.Tensor] = None,
                        lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Causal attention of packed sequences, q: bf16 [tokens, heads, d_head], k, v: bf16 [keys, K/V heads, d_head]; cu_q, cu_k (None: cu_q):
    int32 [batch + 1], where each sequence's queries and keys begin; its queries are its last tokens.  scale: d_head^-0.5 when None.
    lse: fp32 [tokens, heads], written where given.  Rows of out outside of the sequences stay as they are."""
    tokens, heads, d = shape = q.shape
    if out is None:
        out = _empty(shape, _BF16, q.device, stream)
    if cu_k is None:
        cu_k = cu_q
    keys, heads_k, _ = k.shape if k.dim() == 3 else (0, 0, 0)
    batch = cu_q.shape[0] - 1 if cu_q.dim() == 1 else 0
    if workspace is None:
        nbytes = resq_attend_prompts_workspace_bytes(tokens, keys, batch, heads, heads_k, d)
        workspace = _made(lambda: torch.empty(max(nbytes, 1), dtype=_U8, device=q.device), stream, q.device, handed_out=False)
    dev = q.get_device()
    ldq, ldqh, one = q.stride()
    ldk, ldkh, one_k = k.stride() if k.dim() == 3 else (0, 0, 0)
    ldv, ldvh, one_v = v.stride() if v.dim() == 3 else (0, 0, 0)
    ldo, ldoh, one_o = out.stride() if out.dim() == 3 else (0, 0, 0)
    sums = None
    ok = (q.dtype == _BF16 and k.dtype == _BF16 and v.dtype == _BF16 and out.dtype == _BF16 and cu_q.dtype == _I32 and cu_k.dtype == _I32
          and workspace.dtype == _U8 and one == 1 and one_k == 1 and one_v == 1 and one_o == 1 and out.shape == shape and v.shape == k.shape
          and k.shape[2] == d and heads_k > 0 and heads % heads_k == 0 and batch > 0 and cu_k.shape == cu_q.shape and cu_q.is_contiguous()
          and cu_k.is_contiguous() and workspace.is_contiguous() and dev >= 0 and dev == _raw_device() and k.get_device() == dev
          and v.get_device() == dev and out.get_device() == dev and cu_q.get_device() == dev and cu_k.get_device() == dev
          and workspace.get_device() == dev)
    if lse is not None and ok:
        ok = lse.dtype == torch.float32 and lse.shape == (tokens, heads) and lse.is_contiguous() and lse.get_device() == dev
        sums = lse.data_ptr()
    if not ok:
        where = "resq_attend_prompts"
        for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
            _explain_heads(where, name, t)
        _need(out.shape == shape and v.shape == k.shape and k.shape[2] == d and heads_k > 0 and heads % heads_k == 0, where,
              f"q {tuple(shape)}, k {tuple(k.shape)}, v {tuple(v.shape)} and out {tuple(out.shape)} do not match")
        _need(lse is None or (lse.dtype == torch.float32 and lse.shape == (tokens, heads) and lse.is_contiguous()), where,
              f"lse must be a contiguous fp32 [{tokens}, {heads}] tensor")
        _need(workspace.dtype == _U8 and workspace.is_contiguous(), where, "workspace must be a contiguous uint8 tensor")
        _explain_ints(where, "cu_q", cu_q)
        _explain_ints(where, "cu_k", cu_k, batch + 1)
        _need(batch > 0, where, "cu_q must have two entries at least")
        _explain_devices(where, q, k, v, cu_q, cu_k, out, lse, workspace)
        raise ValueError(f"{where}: invalid arguments")
    st = lib().resq_attend_prompts(
        q.data_ptr(), ldq, ldqh, tokens, k.data_ptr(), ldk, ldkh, v.data_ptr(), ldv, ldvh, keys, cu_q.data_ptr(), cu_k.data_ptr(), batch, heads,
        heads_k, d, d ** -0.5 if scale is None else scale, softcap, window, out.data_ptr(), ldo, ldoh, sums, workspace.data_ptr(),
        workspace.numel(), _stream(stream))
    if st:
        _check(st, "resq_attend_prompts")
    return out


@functools.lru_cache(maxsize=1024, typed=True)
def resq_attend_kv_prefix_workspace_bytes(batch: int, heads_q: int, heads_k: int, d_head: int) -> int:
    return int(lib().resq_attend_kv_prefix_workspace_bytes(batch, heads_q, heads_k, d_head))


def resq_attend_kv_prefix_workspace(batch: int, heads_q: int, heads_k: int, d_head: int, device="cuda") -> torch.Tensor:
    """A workspace for resq_attend_kv_prefix calls of these sizes; calls on different streams need one each."""
    nbytes = resq_attend_kv_prefix_workspace_bytes(batch, heads_q, heads_k, d_head)
    if nbytes == 0:
        raise ValueError(f"invalid (batch, heads_q, heads_k, d_head) = ({batch}, {heads_q}, {heads_k}, {d_head})")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def resq_attend_kv_prefix(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, prefix_len: torch.Tensor, prefix_table: torch.Tensor,
                          lens: torch.Tensor, block_table: torch.Tensor, r: int, scale: Optional[float] = None, softcap: float = 0.0,
                          window: int = 0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """resq_attend_kv_cache behind a prefix of prefix_len (int32 [1]) tokens in the pages of prefix_table (int32 [pages]) that all
    sequences share; lens (below 0: the sequence is not there) and block_table are their own tokens behind it."""
    batch, heads, d = shape = q.shape
    if out is None:
        out = _empty(shape, _BF16, q.device, stream)
    if batch == 0:
        return out
    n, heads_k, size, width = k_pages.shape if k_pages.dim() == 4 else (0, 0, 0, 0)
    if workspace is None:
        nbytes = resq_attend_kv_prefix_workspace_bytes(batch, heads, heads_k, d)
        workspace = _made(lambda: torch.empty(max(nbytes, 1), dtype=_U8, device=q.device), stream, q.device, handed_out=False)
    dev = q.get_device()
    ldq, ldqh, one = q.stride()
    ldo, ldoh, one_o = out.stride() if out.dim() == 3 else (0, 0, 0)
    need = _page_row_bytes(d, r)
    strides = k_pages.stride()
    ld_table, one_t = block_table.stride() if block_table.dim() == 2 else (0, 0)
    sums = None
    ok = (q.dtype == _BF16 and out.dtype == _BF16 and lens.dtype == _I32 and block_table.dtype == _I32 and prefix_len.dtype == _I32
          and prefix_table.dtype == _I32 and k_pages.dtype == _U8 and v_pages.dtype == _U8 and workspace.dtype == _U8 and one == 1
          and one_o == 1 and one_t == 1 and out.shape == shape and heads_k > 0 and heads % heads_k == 0 and 0 < need <= width
          and strides[3] == 1 and v_pages.shape == k_pages.shape and v_pages.stride() == strides and lens.shape == (batch,)
          and lens.is_contiguous() and block_table.shape[0] == batch and block_table.shape[1] > 0 and prefix_len.shape == (1,)
          and prefix_table.dim() == 1 and prefix_table.shape[0] > 0 and prefix_table.is_contiguous() and workspace.is_contiguous() and dev >= 0
          and dev == _raw_device() and out.get_device() == dev and lens.get_device() == dev and block_table.get_device() == dev
          and prefix_len.get_device() == dev and prefix_table.get_device() == dev and k_pages.get_device() == dev
          and v_pages.get_device() == dev and workspace.get_device() == dev)
    if lse is not None and ok:
        ok = lse.dtype == torch.float32 and lse.shape == (batch, heads) and lse.is_contiguous() and lse.get_device() == dev
        sums = lse.data_ptr()
    if not ok:
        where = "resq_attend_kv_prefix"
        _explain_heads(where, "q", q)
        _explain_heads(where, "out", out)
        _need(out.shape == shape and heads_k > 0 and heads % heads_k == 0, where,
              f"q {tuple(shape)}, out {tuple(out.shape)} or {heads_k} K/V heads do not match")
        _need(lse is None or (lse.dtype == torch.float32 and lse.shape == (batch, heads) and lse.is_contiguous()), where,
              f"lse must be a contiguous fp32 [{batch}, {heads}] tensor")
        _need(workspace.dtype == _U8 and workspace.is_contiguous(), where, "workspace must be a contiguous uint8 tensor")
        _explain_devices(where, q, k_pages, v_pages, prefix_len, prefix_table, lens, block_table, out, lse, workspace)
        _explain_pages(where, k_pages, v_pages, heads_k, d, r)
        _explain_table(where, block_table, batch)
        _explain_ints(where, "lens", lens, batch)
        _explain_ints(where, "prefix_len", prefix_len, 1)
        _explain_ints(where, "prefix_table", prefix_table)
        raise ValueError(f"{where}: invalid arguments")
    st = lib().resq_attend_kv_prefix(
        q.data_ptr(), ldq, ldqh, batch, heads, heads_k, d, r, prefix_len.data_ptr(), prefix_table.data_ptr(), prefix_table.shape[0],
        lens.data_ptr(), block_table.data_ptr(), ld_table, block_table.shape[1], k_pages.data_ptr(), v_pages.data_ptr(), n, size, strides[0],
        strides[1], strides[2], d ** -0.5 if scale is None else scale, softcap, window, out.data_ptr(), ldo, ldoh, sums,
        workspace.data_ptr(), workspace.numel(), _stream(stream))
    if st:
        _check(st, "resq_attend_kv_prefix")
    return out


_H_TYPES = (_BF16, torch.float32)


def resq_norm_residual(y: Optional[torch.Tensor], h: torch.Tensor, w_pre: Optional[torch.Tensor], w_post: Optional[torch.Tensor] = None,
                       gate: Optional[torch.Tensor] = None, alpha: float = 1.0, eps: float = 1e-6, w_offset: float = 0.0,
                       h_out: Optional[torch.Tensor] = None, x: Optional[torch.Tensor] = None, stream=None):
    """(h + alpha * gate * norm(y; w_post), that normed with w_pre): h bf16 or fp32 [tokens, width], y (None: no block before) bf16
    [tokens, width], gate bf16 [tokens, width] or [width], weights bf16 [width]; without w_post y is not normed, without w_pre there is
    no second output (None).  h_out may be h, x may be y.  Without y and h_out the first output is h itself."""
    tokens, width = shape = h.shape
    if h_out is None and (y is not None or w_pre is None):
        h_out = _empty(shape, h.dtype, h.device, stream)
    if x is None and w_pre is not None:
        x = _empty(shape, _BF16, h.device, stream)
    dev = h.get_device()
    ptr = {}
    ok = h.dtype in _H_TYPES and h.stride(1) == 1 and dev >= 0 and dev == _raw_device() and (y is not None or (gate is None and w_post is None)) \
        and (w_pre is not None or x is None)
    for name, t, dtype in (("y", y, _BF16), ("h_out", h_out, h.dtype), ("x", x, _BF16)):
        if t is not None:
            ok = ok and t.dtype == dtype and t.shape == shape and t.stride(1) == 1 and t.get_device() == dev
            ptr[name] = (t.data_ptr(), t.stride(0))
    if gate is not None:
        ok = ok and gate.dtype == _BF16 and (gate.shape == shape or gate.shape == shape[1:]) and gate.stride(-1) == 1 and gate.get_device() == dev
        ptr["gate"] = (gate.data_ptr(), gate.stride(0) if gate.dim() == 2 else 0)
    for w in (w_pre, w_post):
        ok = ok and (w is None or (w.dtype == _BF16 and w.shape == shape[1:] and w.is_contiguous() and w.get_device() == dev))
    if not ok:
        where = "resq_norm_residual"
        _need(h.dtype in _H_TYPES and h.stride(1) == 1, where, "h must be a row-major bf16 or fp32 [tokens, width] tensor")
        for name, t, dtype in (("y", y, _BF16), ("h_out", h_out, h.dtype), ("x", x, _BF16)):
            _need(t is None or (t.dtype == dtype and t.shape == shape and t.stride(1) == 1), where,
                  f"{name} must be a row-major {dtype} [{tokens}, {width}] tensor")
        _need(gate is None or (gate.dtype == _BF16 and gate.shape in (shape, shape[1:]) and gate.stride(-1) == 1), where,
              f"gate must be a bf16 [{tokens}, {width}] or [{width}] tensor")
        for name, w in (("w_pre", w_pre), ("w_post", w_post)):
            _need(w is None or (w.dtype == _BF16 and w.shape == shape[1:] and w.is_contiguous()), where, f"{name} must be a contiguous bf16 [{width}] tensor")
        _need(y is not None or (gate is None and w_post is None), where, "gate and w_post belong to y")
        _need(w_pre is not None or x is None, where, "x needs w_pre")
        _explain_devices(where, h, y, gate, w_pre, w_post, h_out, x)
        raise ValueError(f"{where}: invalid arguments")
    none = (None, 0)
    to = ptr.get("h_out", none)
    st = lib().resq_norm_residual(*ptr.get("y", none), *ptr.get("gate", none), h.data_ptr(), h.stride(0), int(h.dtype == torch.float32), tokens,
                                  width, None if w_pre is None else w_pre.data_ptr(), None if w_post is None else w_post.data_ptr(), w_offset,
                                  eps, alpha, *to, *ptr.get("x", none), _stream(stream))
    if st:
        _check(st, "resq_norm_residual")
    return h if h_out is None else h_out, x


def resq_online_hadamard(x: torch.Tensor, col_begin: int, col_end: int, block: int = 0,
                         out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    M, K = x.shape
    if x.stride(1) != 1:
        raise ValueError("x must be row-major")
    if out is None:
        out = _made(lambda: torch.empty_like(x), stream, x.device)
    if out.stride() != x.stride():
        raise ValueError("out must have x's layout")
    st = lib().resq_online_hadamard(_dev(x, torch.bfloat16, "x"), _dev(out, torch.bfloat16, "out"),
                                    x.stride(0), M, K, col_begin, col_end, block, _stream(stream))
    _check(st, "resq_online_hadamard")
    return out
