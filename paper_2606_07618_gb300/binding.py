"""Thin ctypes binding of libnvfp4ss.so (include/nvfp4ss.h, include/nvfp4mm.h, include/nvfp4kv.h).

Every function has the name of the C entry point it calls and only marshals
arguments: torch CUDA tensors become device pointers, the current torch CUDA
stream becomes the cudaStream_t, a non-OK status raises ``Nvfp4Error``.  All
arithmetic runs in the library's CUDA kernels; there is no CPU fallback, and a
missing library raises at load time.
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

from . import build as _build

NVFP4_IN_BF16, NVFP4_IN_F32 = 0, 1
NVFP4_OBJ_MSE, NVFP4_OBJ_WMSE = 0, 1
NVFP4_SF_LINEAR, NVFP4_SF_SWIZZLED = 1, 2
NVFP4_WINDOW_DEFAULT = -(2 ** 31)
NVFP4_WINDOW_TIGHT = -(2 ** 31) + 1

FP4_FMT_NVFP4, FP4_FMT_MXFP4 = 0, 1
FP4_ACT_SILU, FP4_ACT_GELU_TANH = 0, 1
NVFP4_ROPE_NEIGHBOURS, NVFP4_ROPE_HALVES = 0, 1
NVFP4_ROPE_PLAIN, NVFP4_ROPE_LINEAR, NVFP4_ROPE_BASE, NVFP4_ROPE_BANDS = 0, 1, 2, 3
NVFP4_KV_ABSMAX, NVFP4_KV_SWEEP = 0, 1
NVFP4_KV_STARVE_VALUES = 2

STATUS = {0: "NVFP4_OK", 1: "NVFP4_ERR_INVALID_ARG", 2: "NVFP4_ERR_UNSUPPORTED", 3: "NVFP4_ERR_ALIGNMENT",
          4: "NVFP4_ERR_RANGE", 5: "NVFP4_ERR_CUDA"}


class Nvfp4Error(RuntimeError):
    def __init__(self, fn: str, code: int, msg: str):
        super().__init__(f"{fn}: {STATUS.get(code, code)} ({msg})")
        self.code = code


_lib = None

NVFP4_GROUP_MAX = 16
NVFP4_GROUP_SCHEDULE_AUTO, NVFP4_GROUP_SCHEDULE_TWO_PHASE, NVFP4_GROUP_SCHEDULE_PIPELINED = 0, 1, 2


class RowShard(ctypes.Structure):
    """nvfp4_row_shard: one shard's rows and output offsets (nvfp4_row_shard_layout)."""
    _fields_ = [("row_begin", ctypes.c_int64), ("row_end", ctypes.c_int64), ("x_offset", ctypes.c_int64),
                ("codes_offset", ctypes.c_int64), ("sf_linear_offset", ctypes.c_int64),
                ("sf_swizzled_offset", ctypes.c_int64), ("sf_swizzled_bytes", ctypes.c_int64)]


class GroupTensor(ctypes.Structure):
    """nvfp4_group_tensor: one tensor of a scalesweep_quantize_group call."""
    _fields_ = [("x", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("w", ctypes.c_void_p),
                ("w_row_stride", ctypes.c_int64), ("codes", ctypes.c_void_p), ("sf_linear", ctypes.c_void_p),
                ("sf_swizzled", ctypes.c_void_p)]


class Fp4Operand(ctypes.Structure):
    """fp4_operand: codes, 128x4-atom scales and global scale of a quantised matrix."""
    _fields_ = [("codes", ctypes.c_void_p), ("sf", ctypes.c_void_p), ("S", ctypes.c_void_p)]


class KvCache(ctypes.Structure):
    """nvfp4_kv_cache: the pool of pages, its scales and sizes."""
    _fields_ = [("codes", ctypes.c_void_p), ("sf", ctypes.c_void_p), ("S_k", ctypes.c_void_p), ("S_v", ctypes.c_void_p),
                ("pages", ctypes.c_int64), ("page", ctypes.c_int32), ("heads", ctypes.c_int32), ("dim", ctypes.c_int32)]


def library_path() -> str:
    return _build.LIB


def lib() -> ctypes.CDLL:
    """Load libnvfp4ss.so, building it first if it is missing or stale."""
    global _lib
    if _lib is None:
        if not _build.up_to_date():
            _build.build()
        if not os.path.exists(_build.LIB):
            raise RuntimeError("libnvfp4ss.so is not built and could not be built")
        L = ctypes.CDLL(_build.LIB)
        i, i64, f, p, sz = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
        L.nvfp4_status_string.argtypes, L.nvfp4_status_string.restype = [i], ctypes.c_char_p
        L.nvfp4_global_scale_workspace.argtypes, L.nvfp4_global_scale_workspace.restype = [i64], sz
        L.nvfp4_global_scale.argtypes = [p, i, i64, f, p, p, p, sz, p]
        L.nvfp4_global_scale_noalloc.argtypes = [p, i, i64, f, p, p, p]
        L.scalesweep_quantize.argtypes = [p, i, i64, i64, i, p, i, p, i64, i, i, p, p, p, p, p]
        L.absmax_quantize.argtypes = [p, i, i64, i64, i, p, p, p, p, p, p]
        L.four_over_six_quantize.argtypes = [p, i, i64, i64, i, p, i, p, i64, p, p, p, p, p]
        L.nvfp4_dequantize.argtypes = [p, p, i, p, i64, i64, i, p, i, p]
        L.nvfp4_dynamic_workspace.argtypes, L.nvfp4_dynamic_workspace.restype = [], sz
        L.scalesweep_quantize_dynamic.argtypes = [p, i, i64, i64, i, f, i, p, i64, i, i, p, p, p, sz, p, p, p, p, p]
        L.absmax_quantize_dynamic.argtypes = [p, i, i64, i64, i, f, p, p, p, sz, p, p, p, p, p]
        L.scalesweep_quantize_group_workspace.argtypes, L.scalesweep_quantize_group_workspace.restype = [], sz
        L.scalesweep_quantize_group.argtypes = [ctypes.POINTER(GroupTensor), i, i, i, i, f, p, p, p, sz, p]
        L.scalesweep_quantize_group_scheduled.argtypes = [ctypes.POINTER(GroupTensor), i, i, i, i, f, p, p, p, sz,
                                                          i, p]
        L.absmax_quantize_group.argtypes = [ctypes.POINTER(GroupTensor), i, i, i, f, p, p, p, sz, p]
        L.nvfp4_selftest_wait_timeout.argtypes = [i, p, i64, i64, p, p, p, sz, p, p, p]
        L.nvfp4_row_shard_layout.argtypes = [i64, i64, i, i, i, ctypes.POINTER(RowShard)]
        L.nvfp4_optimal_scale.argtypes = [p, i, i64, i64, i, p, i, p, i64, p, p, p, p, p]
        L.nvfp4_ldlq_prepare_workspace.argtypes, L.nvfp4_ldlq_prepare_workspace.restype = [i64], sz
        L.nvfp4_ldlq_prepare.argtypes = [p, i64, f, p, p, p, p, p, sz, p]
        L.nvfp4_ldlq_workspace.argtypes, L.nvfp4_ldlq_workspace.restype = [i64, i64], sz
        L.ldlq_quantize.argtypes = [p, i, i64, i64, i, p, p, p, p, p, p, p, sz, p]
        op = ctypes.c_void_p                     # fp4_operand*: a Fp4Operand by reference, or its bytes
        L.mxfp4_quantize.argtypes = [p, i, i64, i64, i64, p, p, p, p, p]
        L.mxfp4_dequantize.argtypes = [p, p, i, i64, i64, p, i, p]
        L.fp4_matmul.argtypes = [i, op, op, i64, i64, i64, p, i, i64, p, p]
        L.fp4_selftest_wait_timeout.argtypes = L.fp4_matmul.argtypes
        L.fp4_matmul_backward_workspace.argtypes, L.fp4_matmul_backward_workspace.restype = [i64, i64, i64], sz
        L.fp4_matmul_backward.argtypes = [i, op, op, i64, i64, i64, p, i64, p, i64, p, i64, p, p, sz, p]
        L.fp4_gated_ff.argtypes = [i, i, op, op, op, i64, i64, i64, p, i64, p, p, p, p]
        L.fp4_gated_ff_backward_workspace.argtypes = [i64, i64, i64]
        L.fp4_gated_ff_backward_workspace.restype = sz
        L.fp4_gated_ff_backward.argtypes = [i, i, op, op, op, i64, i64, i64, p, i64, p, i64, p, p, i64, p, i64, p, p, sz,
                                            p]
        d, i32 = ctypes.c_double, ctypes.c_int32
        L.nvfp4_rope_turns.argtypes = [i, d, i, d, d, d, d, p]
        L.nvfp4_rope.argtypes = [p, i64, i64, p, i64, i64, i, i64, i32, i32, i32, p, p, f, i, i, p]
        L.nvfp4_kv_write.argtypes = [p, p, i64, i64, p, i64, i64, i, i64, p, i, p, p]
        L.nvfp4_kv_read.argtypes = [p, p, i64, i64, p, p, i64, p, i64, i64, p, i64, i64, i, i64, p, p]
        L.nvfp4_kv_attention_workspace.argtypes = [p, i64, i32, i64, i64, i64, i64]
        L.nvfp4_kv_attention_workspace.restype = sz
        L.nvfp4_kv_attention.argtypes = [p, p, i64, i64, i64, i32, p, i64, i64, p, p, i64, i64, f, i, p, i64, i64, p, p, p, sz, p]
        L.nvfp4_kv_selftest_wait_timeout.argtypes = L.nvfp4_kv_attention.argtypes
        L.nvfp4_kv_attention_prefix.argtypes = [p, p, i64, i64, i64, i32, p, i64, p, p, i64, i64, p, p, i64, i64, f, i, p, i64, i64,
                                                p, p, p, sz, p]
        for fn in ("nvfp4_rope_turns", "nvfp4_rope", "nvfp4_kv_write", "nvfp4_kv_read", "nvfp4_kv_attention",
                   "nvfp4_kv_selftest_wait_timeout", "nvfp4_kv_attention_prefix"):
            getattr(L, fn).restype = i
        for fn in ("mxfp4_quantize", "mxfp4_dequantize", "fp4_matmul", "fp4_selftest_wait_timeout", "fp4_matmul_backward",
                   "fp4_gated_ff", "fp4_gated_ff_backward"):
            getattr(L, fn).restype = i
        for fn in ("nvfp4_global_scale", "nvfp4_global_scale_noalloc", "scalesweep_quantize", "absmax_quantize",
                   "four_over_six_quantize", "nvfp4_dequantize", "scalesweep_quantize_dynamic",
                   "absmax_quantize_dynamic", "nvfp4_optimal_scale", "nvfp4_ldlq_prepare", "ldlq_quantize",
                   "scalesweep_quantize_group", "scalesweep_quantize_group_scheduled", "absmax_quantize_group",
                   "nvfp4_selftest_wait_timeout",
                   "nvfp4_row_shard_layout"):
            getattr(L, fn).restype = i
        _lib = L
    return _lib


def _ptr(t):
    # plain ints: ctypes converts them for c_void_p parameters without an object
    if t is None or isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        # torch.cuda.current_stream().cuda_stream without the Stream object
        return _current_stream(_current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _current_device() -> int:
    # torch.cuda.current_device() without its check for initialisation
    return _raw_device() if _raw_device is not None else torch.cuda.current_device()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _current_stream(device: int) -> int:
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _dtype(x) -> int:
    if x.dtype == torch.bfloat16:
        return NVFP4_IN_BF16
    if x.dtype == torch.float32:
        return NVFP4_IN_F32
    raise TypeError(f"unsupported dtype {x.dtype}")


def _check(fn: str, rc: int):
    if rc != 0:
        raise Nvfp4Error(fn, rc, lib().nvfp4_status_string(rc).decode())


def nvfp4_status_string(code: int) -> str:
    return lib().nvfp4_status_string(int(code)).decode()


def nvfp4_global_scale_workspace(n: int) -> int:
    return int(lib().nvfp4_global_scale_workspace(int(n)))


def nvfp4_global_scale(x, fp8_div: float, S_out, status=None, workspace=None, stream=None):
    ws_bytes = workspace.numel() * workspace.element_size()
    rc = lib().nvfp4_global_scale(_ptr(x), _dtype(x), x.numel(), float(fp8_div), _ptr(S_out), _ptr(status),
                                  _ptr(workspace), ws_bytes, _stream(stream))
    _check("nvfp4_global_scale", rc)


def nvfp4_global_scale_noalloc(x, fp8_div: float, S_out, status=None, stream=None):
    """Global scale for callers that cannot allocate: no workspace argument
    (the library's static device scratch is used instead)."""
    rc = lib().nvfp4_global_scale_noalloc(_ptr(x), _dtype(x), x.numel(), float(fp8_div), _ptr(S_out), _ptr(status),
                                          _stream(stream))
    _check("nvfp4_global_scale_noalloc", rc)


def scalesweep_quantize(x, block: int, S, objective: int, w, w_row_stride: int, win_lo: int, win_hi: int,
                        codes, sf_linear=None, sf_swizzled=None, block_loss=None, stream=None):
    rows, cols = x.shape
    rc = lib().scalesweep_quantize(_ptr(x), _dtype(x), rows, cols, int(block), _ptr(S), int(objective), _ptr(w),
                                   int(w_row_stride), int(win_lo), int(win_hi), _ptr(codes), _ptr(sf_linear),
                                   _ptr(sf_swizzled), _ptr(block_loss), _stream(stream))
    _check("scalesweep_quantize", rc)


def absmax_quantize(x, block: int, S, codes, sf_linear=None, sf_swizzled=None, block_loss=None, stream=None):
    rows, cols = x.shape
    rc = lib().absmax_quantize(_ptr(x), _dtype(x), rows, cols, int(block), _ptr(S), _ptr(codes), _ptr(sf_linear),
                               _ptr(sf_swizzled), _ptr(block_loss), _stream(stream))
    _check("absmax_quantize", rc)


def four_over_six_quantize(x, block: int, S, objective: int, w, w_row_stride: int, codes, sf_linear=None,
                           sf_swizzled=None, block_loss=None, stream=None):
    rows, cols = x.shape
    rc = lib().four_over_six_quantize(_ptr(x), _dtype(x), rows, cols, int(block), _ptr(S), int(objective), _ptr(w),
                                      int(w_row_stride), _ptr(codes), _ptr(sf_linear), _ptr(sf_swizzled),
                                      _ptr(block_loss), _stream(stream))
    _check("four_over_six_quantize", rc)


def nvfp4_dynamic_workspace() -> int:
    return int(lib().nvfp4_dynamic_workspace())


def scalesweep_quantize_dynamic(x, block: int, fp8_div: float, objective: int, w, w_row_stride: int, win_lo: int,
                                win_hi: int, S_out, status, workspace, codes, sf_linear=None, sf_swizzled=None,
                                block_loss=None, stream=None):
    rows, cols = x.shape
    ws_bytes = workspace.numel() * workspace.element_size()
    rc = lib().scalesweep_quantize_dynamic(_ptr(x), _dtype(x), rows, cols, int(block), float(fp8_div), int(objective),
                                           _ptr(w), int(w_row_stride), int(win_lo), int(win_hi), _ptr(S_out),
                                           _ptr(status), _ptr(workspace), ws_bytes, _ptr(codes), _ptr(sf_linear),
                                           _ptr(sf_swizzled), _ptr(block_loss), _stream(stream))
    _check("scalesweep_quantize_dynamic", rc)


def absmax_quantize_dynamic(x, block: int, fp8_div: float, S_out, status, workspace, codes, sf_linear=None,
                            sf_swizzled=None, block_loss=None, stream=None):
    rows, cols = x.shape
    ws_bytes = workspace.numel() * workspace.element_size()
    rc = lib().absmax_quantize_dynamic(_ptr(x), _dtype(x), rows, cols, int(block), float(fp8_div), _ptr(S_out),
                                       _ptr(status), _ptr(workspace), ws_bytes, _ptr(codes), _ptr(sf_linear),
                                       _ptr(sf_swizzled), _ptr(block_loss), _stream(stream))
    _check("absmax_quantize_dynamic", rc)


def scalesweep_quantize_group_workspace() -> int:
    return int(lib().scalesweep_quantize_group_workspace())


def group_descriptors(xs, ws, w_row_strides, codes, sf_linear, sf_swizzled):
    """The nvfp4_group_tensor array for tensors xs[i] with weights ws[i] (None
    for MSE) and output buffers codes[i], sf_linear[i], sf_swizzled[i] (None
    where not wanted).  Reusable across calls on the same buffers."""
    n = len(xs)
    arr = (GroupTensor * n)()
    for i, x in enumerate(xs):
        rows, cols = x.shape
        arr[i] = GroupTensor(x.data_ptr(), rows, cols, ws[i].data_ptr() if ws[i] is not None else None,
                             int(w_row_strides[i]), codes[i].data_ptr(),
                             sf_linear[i].data_ptr() if sf_linear[i] is not None else None,
                             sf_swizzled[i].data_ptr() if sf_swizzled[i] is not None else None)
    return arr


def scalesweep_quantize_group(desc, dtype: int, objective: int, fp8_div: float, S, status=None, workspace=None,
                              stream=None, block: int = 16, schedule: int | None = None):
    """desc: the array from group_descriptors.  fp8_div 0 reads S[i]; > 0
    computes and writes S[i] during the call.  schedule None calls
    scalesweep_quantize_group (the library's choice); an NVFP4_GROUP_SCHEDULE_*
    value calls scalesweep_quantize_group_scheduled with it."""
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    if schedule is None:
        rc = lib().scalesweep_quantize_group(desc, len(desc), int(dtype), int(block), int(objective), float(fp8_div),
                                             _ptr(S), _ptr(status), _ptr(workspace), ws_bytes, _stream(stream))
        _check("scalesweep_quantize_group", rc)
    else:
        rc = lib().scalesweep_quantize_group_scheduled(desc, len(desc), int(dtype), int(block), int(objective),
                                                       float(fp8_div), _ptr(S), _ptr(status), _ptr(workspace),
                                                       ws_bytes, int(schedule), _stream(stream))
        _check("scalesweep_quantize_group_scheduled", rc)


def absmax_quantize_group(desc, dtype: int, fp8_div: float, S, status=None, workspace=None, stream=None,
                          block: int = 16):
    """AbsMax over the tensors of desc in one launch (static or in-launch scales,
    as scalesweep_quantize_group)."""
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    rc = lib().absmax_quantize_group(desc, len(desc), int(dtype), int(block), float(fp8_div), _ptr(S),
                                     _ptr(status), _ptr(workspace), ws_bytes, _stream(stream))
    _check("absmax_quantize_group", rc)


def nvfp4_selftest_wait_timeout(which: int, x, S, status, workspace, codes, sf_linear, stream=None):
    """Makes a bounded device wait run out: the grouped launch's with a dynamic scale
    (which = 0 or 1; status bit 1), LDLQ's walk's (2) or trailing updates' (3; status
    bit 16; workspace: perm, U, then LDLQ's own).  See nvfp4ss.h."""
    rows, cols = x.shape
    ws_bytes = workspace.numel() * workspace.element_size()
    rc = lib().nvfp4_selftest_wait_timeout(int(which), _ptr(x), rows, cols, _ptr(S), _ptr(status), _ptr(workspace),
                                           ws_bytes, _ptr(codes), _ptr(sf_linear), _stream(stream))
    _check("nvfp4_selftest_wait_timeout", rc)


def nvfp4_optimal_scale(x, block: int, S, objective: int, w, w_row_stride: int, s_opt, loss_opt, fp8_code=None,
                        loss_fp8=None, stream=None):
    rows, cols = x.shape
    rc = lib().nvfp4_optimal_scale(_ptr(x), _dtype(x), rows, cols, int(block), _ptr(S), int(objective), _ptr(w),
                                   int(w_row_stride), _ptr(s_opt), _ptr(loss_opt), _ptr(fp8_code), _ptr(loss_fp8),
                                   _stream(stream))
    _check("nvfp4_optimal_scale", rc)


def nvfp4_dequantize(codes, sf, layout: int, S, rows: int, cols: int, block: int, out, stream=None):
    rc = lib().nvfp4_dequantize(_ptr(codes), _ptr(sf), int(layout), _ptr(S), int(rows), int(cols), int(block),
                                _ptr(out), _dtype(out), _stream(stream))
    _check("nvfp4_dequantize", rc)


# --------------------------------------------------------------------------- buffer helpers
def swizzled_bytes(rows: int, cols: int, block: int = 16) -> int:
    kb = cols // block
    return -(-rows // 128) * 128 * (-(-kb // 4)) * 4


def empty_outputs(rows: int, cols: int, block: int, device="cuda", linear=True, swizzled=False, loss=False) -> dict:
    """Allocate the output buffers of a quantise call with torch (the library
    itself never allocates)."""
    out = {"codes": torch.empty(rows, cols // 2, dtype=torch.uint8, device=device)}
    out["sf_linear"] = torch.empty(rows, cols // block, dtype=torch.uint8, device=device) if linear else None
    out["sf_swizzled"] = torch.empty(swizzled_bytes(rows, cols, block), dtype=torch.uint8, device=device) \
        if swizzled else None
    out["block_loss"] = torch.empty(rows * (cols // block), dtype=torch.float32, device=device) if loss else None
    return out


def nvfp4_ldlq_prepare_workspace(n: int) -> int:
    return int(lib().nvfp4_ldlq_prepare_workspace(int(n)))


def nvfp4_ldlq_prepare(H, damp: float, perm, U, D, status=None, workspace=None, stream=None):
    """Damped, reordered UDU^T factor of the Hessian H [n, n] float32 for LDLQ:
    perm [n] int32, U [n, n] float32, D [n] float32 (outputs)."""
    n = H.shape[0]
    ws_bytes = workspace.numel() * workspace.element_size()
    rc = lib().nvfp4_ldlq_prepare(_ptr(H), n, float(damp), _ptr(perm), _ptr(U), _ptr(D), _ptr(status),
                                  _ptr(workspace), ws_bytes, _stream(stream))
    _check("nvfp4_ldlq_prepare", rc)


def nvfp4_ldlq_workspace(rows: int, cols: int) -> int:
    return int(lib().nvfp4_ldlq_workspace(int(rows), int(cols)))


def ldlq_quantize(W, block: int, S, sf_linear, perm, U, codes, status=None, workspace=None, stream=None):
    """LDLQ (GPTQ) quantization of W [rows, cols] with the fixed scales sf_linear,
    processing order perm and factor U from nvfp4_ldlq_prepare."""
    rows, cols = W.shape
    ws_bytes = workspace.numel() * workspace.element_size()
    rc = lib().ldlq_quantize(_ptr(W), _dtype(W), rows, cols, int(block), _ptr(S), _ptr(sf_linear), _ptr(perm),
                             _ptr(U), _ptr(codes), _ptr(status), _ptr(workspace), ws_bytes, _stream(stream))
    _check("ldlq_quantize", rc)


def nvfp4_row_shard_layout(rows: int, cols: int, block: int, world: int, rank: int) -> RowShard:
    """Rows and output offsets of shard `rank` of `world` (host-only, no GPU needed)."""
    out = RowShard()
    rc = lib().nvfp4_row_shard_layout(int(rows), int(cols), int(block), int(world), int(rank), ctypes.byref(out))
    _check("nvfp4_row_shard_layout", rc)
    return out


# --------------------------------------------------------------------------- 4-bit matrices (nvfp4mm.h)
def mx_swizzled_bytes(rows: int, cols: int) -> int:
    """Bytes of the 128x4-atom scale layout of an MXFP4 matrix."""
    return swizzled_bytes(rows, cols, 32)


def _rows(t, what: str) -> int:
    """Row stride of a 2-d tensor whose rows are contiguous."""
    rows, cols = t.shape
    if t.is_contiguous():
        return cols
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{what}: a 2-d tensor with contiguous rows is wanted")
    return ld if rows > 1 else max(ld, cols)


def _buffer(t, nbytes: int, what: str):
    """Pointer of an optional buffer; a tensor's has to hold nbytes in a row."""
    if t is None or type(t) is int:
        return t
    if t.nbytes < nbytes or not t.is_contiguous():
        raise ValueError(f"{what}: {nbytes} contiguous bytes are wanted")
    return t.data_ptr()


_pack_operand = struct.Struct("3P").pack
_BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def _status(t):
    """Pointer of an optional status word, which the kernels take for an int."""
    if t is None or type(t) is int:
        return t
    if t.dtype is not _I32 or t.numel() < 1:
        raise TypeError(f"status: an int32 element is wanted, not {tuple(t.shape)} of {t.dtype}")
    return t.data_ptr()


def _operand(m, fmt: int, what: str):
    """(codes [rows, cols/2], 128x4-atom scales, S or None) as the bytes of an fp4_operand (a
    ctypes.Structure takes three times as long to fill, on a path of a few microseconds), its rows and cols.
    Which format the scales are in is the caller's word: both are bytes, in as many atoms where cols are few."""
    codes, sf, S = m
    rows, half = codes.shape
    if not codes.is_contiguous():
        raise ValueError(f"{what}: contiguous codes [rows, cols/2] are wanted")
    if not (codes.dtype is sf.dtype is _U8 or codes.itemsize == sf.itemsize == 1):
        raise TypeError(f"{what}: codes and scales in bytes are wanted, not {codes.dtype} and {sf.dtype}")
    if S is not None and (S.dtype is not _F32 or S.numel() != 1):
        raise TypeError(f"{what}: one float32 as S is wanted, not {tuple(S.shape)} of {S.dtype}")
    # atoms of 512 bytes: 128 rows by 4 scale columns
    need = (rows + 127 >> 7) * (half + 63 >> 6 if fmt == FP4_FMT_MXFP4 else half + 31 >> 5) * 512
    if sf.nbytes < need or not sf.is_contiguous():
        raise ValueError(f"{what}: scales of {need} bytes in the 128x4-atom layout are wanted")
    return _pack_operand(codes.data_ptr(), sf.data_ptr(), 0 if S is None else S.data_ptr()), rows, 2 * half


def _out(t, rows: int, cols: int, what: str):
    """Pointer and row stride of an optional bf16 tensor."""
    if t is None:
        return None, 0
    if t.dtype is not _BF16:
        raise TypeError(f"{what}: bfloat16 is wanted, not {t.dtype}")
    if t.shape != (rows, cols):
        raise ValueError(f"{what}: shape {(rows, cols)} is wanted, not {tuple(t.shape)}")
    return t.data_ptr(), cols if t.is_contiguous() else _rows(t, what)


def mxfp4_quantize(x, codes, sf_linear=None, sf_swizzled=None, status=None, stream=None):
    """MXFP4 codes and scales of x [rows, cols] (bf16 or fp32, rows contiguous, any row stride)."""
    rows, cols = x.shape
    rc = (_lib or lib()).mxfp4_quantize(x.data_ptr(), _dtype(x), rows, cols, _rows(x, "x"),
                                        _buffer(codes, rows * (cols // 2), "codes"),
                                        _buffer(sf_linear, rows * (cols // 32), "sf_linear"),
                                        _buffer(sf_swizzled, (rows + 127 >> 7) * (cols + 127 >> 7) * 512, "sf_swizzled"), _status(status),
                                        _stream(stream))
    _check("mxfp4_quantize", rc)


def mxfp4_dequantize(codes, sf, layout: int, rows: int, cols: int, out, stream=None):
    sf_bytes = mx_swizzled_bytes(rows, cols) if layout == NVFP4_SF_SWIZZLED else rows * (cols // 32)
    rc = (_lib or lib()).mxfp4_dequantize(_buffer(codes, rows * (cols // 2), "codes"), _buffer(sf, sf_bytes, "sf"), layout,
                                          rows, cols, _buffer(out, rows * cols * out.element_size(), "out"), _dtype(out),
                                          _stream(stream))
    _check("mxfp4_dequantize", rc)


def _matmul(fn: str, fmt: int, a, b, out, status, stream):
    oa, m, k = _operand(a, fmt, "a")
    ob, n, kb = _operand(b, fmt, "b")
    if k != kb:
        raise ValueError(f"{fn}: operands of {k} and {kb} columns")
    if out.shape != (m, n):
        raise ValueError(f"out: shape {(m, n)} is wanted, not {tuple(out.shape)}")
    rc = getattr(_lib or lib(), fn)(fmt, oa, ob, m, n, k, out.data_ptr(), _dtype(out),
                                    n if out.is_contiguous() else _rows(out, "out"), _status(status), _stream(stream))
    _check(fn, rc)


def fp4_matmul(fmt: int, a, b, out, status=None, stream=None):
    """out [m, n] (bf16 or fp32) = A B^T; a = (codes [m, k/2], swizzled scales, S or None), b likewise [n, k/2]."""
    _matmul("fp4_matmul", fmt, a, b, out, status, stream)


def fp4_selftest_wait_timeout(fmt: int, a, b, out, status, stream=None):
    """fp4_matmul whose waits for its operands run out (status bit 16, out not written).  See nvfp4mm.h."""
    _matmul("fp4_selftest_wait_timeout", fmt, a, b, out, status, stream)


def fp4_matmul_backward_workspace(m: int, n: int, k: int) -> int:
    return int(lib().fp4_matmul_backward_workspace(int(m), int(n), int(k)))


def fp4_matmul_backward(fmt: int, a, b, d_out, d_a=None, d_b=None, workspace=None, status=None, stream=None):
    """Gradients of fp4_matmul's operands from d_out [m, n] (bf16): d_a [m, k], d_b [n, k] (bf16, either None)."""
    oa, m, k = _operand(a, fmt, "a")
    ob, n, kb = _operand(b, fmt, "b")
    if k != kb:
        raise ValueError(f"fp4_matmul_backward: operands of {k} and {kb} columns")
    pd, ldd = _out(d_out, m, n, "d_out")
    pa, lda = _out(d_a, m, k, "d_a")
    pb, ldb = _out(d_b, n, k, "d_b")
    ws_bytes = workspace.nbytes if workspace is not None else 0
    rc = (_lib or lib()).fp4_matmul_backward(fmt, oa, ob, m, n, k, pd, ldd, pa, lda, pb, ldb, _status(status),
                                             _buffer(workspace, 0, "workspace"), ws_bytes, _stream(stream))
    _check("fp4_matmul_backward", rc)


def _gated_operands(fn: str, fmt: int, x, w_gate, w_up):
    ox, t, d = _operand(x, fmt, "x")
    og, f, dg = _operand(w_gate, fmt, "w_gate")
    ou, fu, du = _operand(w_up, fmt, "w_up")
    if dg != d or du != d or fu != f:
        raise ValueError(f"{fn}: operands [{t}, {d}], [{f}, {dg}] and [{fu}, {du}]")
    return ox, og, ou, t, f, d


def fp4_gated_ff(fmt: int, act: int, x, w_gate, w_up, h=None, h_codes=None, h_sf=None, status=None, stream=None):
    """act(x Wg^T) * (x Wu^T) of quantised operands, as h [t, f] bf16 and/or as an MXFP4 operand (h_codes [t, f/2],
    h_sf of mx_swizzled_bytes(t, f) bytes)."""
    ox, og, ou, t, f, d = _gated_operands("fp4_gated_ff", fmt, x, w_gate, w_up)
    ph, ldh = _out(h, t, f, "h")
    if h_codes is not None:
        if h_codes.shape != (t, f // 2) or not h_codes.is_contiguous():
            raise ValueError(f"h_codes: contiguous, of shape {(t, f // 2)}, is wanted")
        if h_codes.itemsize != 1:
            raise TypeError(f"h_codes: bytes are wanted, not {h_codes.dtype}")
    rc = (_lib or lib()).fp4_gated_ff(fmt, act, ox, og, ou, t, f, d, ph, ldh, _ptr(h_codes),
                                      _buffer(h_sf, mx_swizzled_bytes(t, f), "h_sf"), _status(status), _stream(stream))
    _check("fp4_gated_ff", rc)


def fp4_gated_ff_backward_workspace(t: int, f: int, d: int) -> int:
    return int(lib().fp4_gated_ff_backward_workspace(int(t), int(f), int(d)))


def fp4_gated_ff_backward(fmt: int, act: int, x, w_gate, w_up, d_h, d_x=None, d_gate=None, d_up=None, h=None,
                          workspace=None, status=None, stream=None):
    """Gradients of fp4_gated_ff's operands from d_h [t, f] (bf16): d_x [t, d], d_gate and d_up [f, d] (bf16, d_x or the
    pair may be None); h [t, f] optionally receives the forward result."""
    ox, og, ou, t, f, d = _gated_operands("fp4_gated_ff_backward", fmt, x, w_gate, w_up)
    pdh, lddh = _out(d_h, t, f, "d_h")
    px, ldx = _out(d_x, t, d, "d_x")
    pg, ldg = _out(d_gate, f, d, "d_gate")
    pu, ldu = _out(d_up, f, d, "d_up")
    if pg and pu and ldg != ldu:
        raise ValueError("d_gate and d_up: one row stride is wanted")
    ph, ldh = _out(h, t, f, "h")
    ws_bytes = workspace.nbytes if workspace is not None else 0
    rc = (_lib or lib()).fp4_gated_ff_backward(fmt, act, ox, og, ou, t, f, d, pdh, lddh, px, ldx, pg, pu, ldg, ph, ldh,
                                               _status(status), _buffer(workspace, 0, "workspace"), ws_bytes,
                                               _stream(stream))
    _check("fp4_gated_ff_backward", rc)


# --------------------------------------------------------------------------- the key/value cache (nvfp4kv.h)
_I64 = torch.int64
_pack_cache = struct.Struct("4PqiiiP").pack                      # the last word pads the structure's end


def _cache(c):
    """(codes [pages, heads, 2, page, dim/2], sf [pages, heads, 2, dim/16, page], S_k, S_v) as the bytes of an
    nvfp4_kv_cache, its heads and dim."""
    codes, sf, S_k, S_v = c
    pages, heads, two, page, half = codes.shape
    if two != 2 or sf.shape != (pages, heads, 2, half >> 3, page):
        raise ValueError(f"cache: codes {tuple(codes.shape)} and scales {tuple(sf.shape)} do not belong together")
    if not (codes.dtype is sf.dtype is _U8 or codes.itemsize == sf.itemsize == 1):
        raise TypeError(f"cache: codes and scales in bytes are wanted, not {codes.dtype} and {sf.dtype}")
    if not (codes.is_contiguous() and sf.is_contiguous()):
        raise ValueError("cache: contiguous codes and scales are wanted")
    if not (S_k.dtype is S_v.dtype is _F32 and S_k.numel() == S_v.numel() == 1):
        raise TypeError(f"cache: one float32 as S is wanted, not {tuple(S_k.shape)} of {S_k.dtype} and {tuple(S_v.shape)} of "
                        f"{S_v.dtype}")
    dim = 2 * half
    return _pack_cache(codes.data_ptr(), sf.data_ptr(), S_k.data_ptr(), S_v.data_ptr(), pages, page, heads, dim, 0), heads, dim


def _heads3(t, what: str):
    """Pointer, token and head stride of a [tokens, heads, dim] tensor whose innermost dimension is contiguous."""
    if t.dim() != 3:
        raise ValueError(f"{what}: [tokens, heads, dim] is wanted, not {tuple(t.shape)}")
    token, head, one = t.stride()
    if t.is_contiguous() and token and head:
        return t.data_ptr(), token, head
    tokens, heads, dim = t.shape
    if one != 1 and dim > 1:
        raise ValueError(f"{what}: a contiguous innermost dimension is wanted")
    if heads <= 1:
        head = max(head, dim)
    if tokens <= 1:
        token = max(token, heads * head, dim)
    return t.data_ptr(), token, head


def _list(t, n: int, dtype, what: str):
    """Pointer of n contiguous numbers of a type, on the device."""
    if t.dtype is not dtype:
        raise TypeError(f"{what}: {dtype} is wanted, not {t.dtype}")
    if t.numel() < n or t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{what}: {n} contiguous numbers are wanted, not {tuple(t.shape)}")
    return t.data_ptr()


def _pages(t, what: str):
    """Pointer, row stride, rows and width of a page table."""
    if t.dtype is not _I32:
        raise TypeError(f"{what}: {_I32} is wanted, not {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{what}: [sequences, pages] is wanted, not {tuple(t.shape)}")
    rows, width = t.shape
    if t.is_contiguous():
        return t.data_ptr(), width, rows, width
    if width > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}: contiguous rows are wanted")
    return t.data_ptr(), t.stride(0) if rows > 1 else max(t.stride(0), width), rows, width


def nvfp4_rope_turns(rot: int, base: float = 10000.0, scaling: int = NVFP4_ROPE_PLAIN, factor: float = 1.0,
                     original_len: float = 0.0, slow: float = 1.0, fast: float = 4.0, device="cuda"):
    """The frequency table [rot/2] int64 (the bits of 64-bit fractions of a turn) of nvfp4_rope, on `device`."""
    turns = torch.empty(max(int(rot) // 2, 0), dtype=_I64)
    rc = (_lib or lib()).nvfp4_rope_turns(int(rot), float(base), int(scaling), float(factor), float(original_len), float(slow),
                                          float(fast), turns.data_ptr())
    _check("nvfp4_rope_turns", rc)
    return turns.to(device)


def nvfp4_rope(x, positions, turns, out=None, magnitude: float = 1.0, layout: int = NVFP4_ROPE_HALVES, inverse: bool = False,
               stream=None):
    """Rotary positions of x [tokens, heads, dim] (bf16 or fp32): the first 2 * len(turns) elements of each head; inverse: the
    gradient of x from that of out.  out None: in place."""
    if out is None:
        out = x
    if out.dtype is not x.dtype:
        raise TypeError(f"out: {x.dtype} is wanted, not {out.dtype}")
    if out.shape != x.shape:
        raise ValueError(f"out: shape {tuple(x.shape)} is wanted, not {tuple(out.shape)}")
    tokens, heads, dim = x.shape
    pairs = turns.numel()
    rc = (_lib or lib()).nvfp4_rope(*_heads3(x, "x"), *_heads3(out, "out"), _dtype(x), tokens, heads, dim, 2 * pairs,
                                    _list(positions, tokens, _I64, "positions"), _list(turns, pairs, _I64, "turns"), magnitude,
                                    layout, 1 if inverse else 0, _stream(stream))
    _check("nvfp4_rope", rc)
    return out


def _kv_pair(k, v, heads: int, dim: int):
    """Pointers and strides of k and v (either None), their dtype code and tokens."""
    x = k if v is None else v
    if x is None:
        raise ValueError("k or v is wanted")
    shape = x.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"k, v: [tokens, {heads}, {dim}] is wanted, not {tuple(shape)}")
    if x is not k and k is not None and (k.shape != shape or k.dtype is not x.dtype):
        raise ValueError(f"k and v of one type and shape are wanted, not {tuple(k.shape)} and {tuple(shape)}")
    a = (None, 0, 0) if k is None else _heads3(k, "k")
    b = (None, 0, 0) if v is None else _heads3(v, "v")
    return a, b, _dtype(x), shape[0]


def nvfp4_kv_write(cache, k, v, slots, method: int = NVFP4_KV_SWEEP, status=None, stream=None):
    """Quantises k and v [tokens, heads, dim] (bf16 or fp32, either None) into the cache at slots [tokens] (page * size +
    offset; negative: skipped)."""
    c, heads, dim = _cache(cache)
    pk, pv, dt, tokens = _kv_pair(k, v, heads, dim)
    rc = (_lib or lib()).nvfp4_kv_write(c, *pk, *pv, dt, tokens, _list(slots, tokens, _I64, "slots"), method, _status(status),
                                        _stream(stream))
    _check("nvfp4_kv_write", rc)


def nvfp4_kv_read(cache, table, starts, offsets, k=None, v=None, status=None, stream=None):
    """Rows offsets[b] .. offsets[b+1] of k and v [tokens, heads, dim] (bf16 or fp32, either None) = tokens starts[b] .. of
    sequence b (starts None: from 0)."""
    c, heads, dim = _cache(cache)
    pk, pv, dt, tokens = _kv_pair(k, v, heads, dim)
    pt, ld, batch, width = _pages(table, "table")
    rc = (_lib or lib()).nvfp4_kv_read(c, pt, ld, width, None if starts is None else _list(starts, batch, _I32, "starts"),
                                       _list(offsets, batch + 1, _I32, "offsets"), batch, *pk, *pv, dt, tokens, _status(status),
                                       _stream(stream))
    _check("nvfp4_kv_read", rc)


def nvfp4_kv_attention_workspace(cache, q, batch: int, width: int, max_q: int, prefix_width: int = 0) -> int:
    """Bytes of workspace of attention for queries q [tokens, q_heads, dim] and page tables of these widths."""
    pages, heads, _, page, half = cache[0].shape
    tokens, q_heads, _ = q.shape
    return (_lib or lib()).nvfp4_kv_attention_workspace(_pack_cache(0, 0, 0, 0, pages, page, heads, 2 * half, 0), tokens, q_heads,
                                                        batch, width, max_q, prefix_width)


def _attention(fn: str, q, cache, prefix, table, lens, offsets, max_q, scale, out, causal, lse, workspace, status, stream):
    c, heads, dim = _cache(cache)
    if not q.dtype is out.dtype is _BF16:
        raise TypeError(f"{fn}: queries and results in bfloat16 are wanted, not {q.dtype} and {out.dtype}")
    shape = q.shape
    if len(shape) != 3 or shape[2] != dim or out.shape != shape:
        raise ValueError(f"{fn}: q and out of [tokens, heads, {dim}] are wanted, not {tuple(shape)} and {tuple(out.shape)}")
    tokens, q_heads, _ = shape
    if q_heads < 1 or q_heads % heads:
        raise ValueError(f"{fn}: a multiple of {heads} query heads is wanted, not {q_heads}")
    if lse is not None:
        if lse.dtype is not _F32:
            raise TypeError(f"lse: {_F32} is wanted, not {lse.dtype}")
        if lse.shape != (tokens, q_heads) or not lse.is_contiguous():
            raise ValueError(f"lse: contiguous, of shape {(tokens, q_heads)}, is wanted")
        lse = lse.data_ptr()
    if workspace is None:
        ws, ws_bytes = None, 0
    else:
        ws, ws_bytes = _buffer(workspace, 0, "workspace"), workspace.nbytes
    pt, ld, batch, width = _pages(table, "table")
    rc = getattr(_lib or lib(), fn)(c, *_heads3(q, "q"), tokens, q_heads, *prefix, pt, ld, width, _list(lens, batch, _I32, "lens"),
                                    _list(offsets, batch + 1, _I32, "offsets"), batch, max_q, scale, causal,
                                    *_heads3(out, "out"), lse, _status(status), ws, ws_bytes, _stream(stream))
    _check(fn, rc)


def nvfp4_kv_attention(q, cache, table, lens, offsets, max_q: int, scale: float, out, causal: bool = True, lse=None,
                       workspace=None, status=None, stream=None):
    """out = softmax(scale q K^T) V for q, out [tokens, q_heads, dim] (bf16): rows offsets[b] .. of sequence b over its
    lens[b] cached tokens.  lse [tokens, q_heads] (fp32) optional."""
    _attention("nvfp4_kv_attention", q, cache, (), table, lens, offsets, max_q, scale, out, 1 if causal else 0, lse, workspace,
               status, stream)


def nvfp4_kv_selftest_wait_timeout(q, cache, table, lens, offsets, max_q: int, scale: float, out, status, workspace=None,
                                   stream=None, values: bool = False):
    """nvfp4_kv_attention whose waits for keys, or for values, run out (status bit 4).  See nvfp4kv.h."""
    _attention("nvfp4_kv_selftest_wait_timeout", q, cache, (), table, lens, offsets, max_q, scale, out,
               1 + (NVFP4_KV_STARVE_VALUES if values else 0), None, workspace, status, stream)


def nvfp4_kv_attention_prefix(q, cache, prefix, prefix_len, table, lens, offsets, max_q: int, scale: float, out,
                              causal: bool = True, lse=None, workspace=None, status=None, stream=None):
    """The same where every query also sees the first prefix_len (int32, one element) tokens of the pages prefix [pages]."""
    pre = (_list(prefix, 0, _I32, "prefix"), prefix.numel(), _list(prefix_len.reshape(-1), 1, _I32, "prefix_len"))
    _attention("nvfp4_kv_attention_prefix", q, cache, pre, table, lens, offsets, max_q, scale, out, 1 if causal else 0, lse,
               workspace, status, stream)
