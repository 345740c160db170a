"""Thin ctypes binding of ``libhbfp.so``: same names as the C ABI, argument marshalling only.

PyTorch supplies device memory (``tensor.data_ptr()``) and the HIP stream; every
step of the path runs in the library's kernels.  There is no CPU fallback: if the
library has not been built, importing this module fails.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libhbfp.so")

OK, ERR_ARG, ERR_FORMAT, ERR_LAYOUT, ERR_RANGE, ERR_LAUNCH, ERR_WORKSPACE = 0, -1, -2, -3, -4, -5, -6
RNE, STOCHASTIC = 0, 1
HINT_HEAVY_TAILS = 1


class HbfpError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class Format(ctypes.Structure):
    """hbfp_format: how a source matrix is cut into exponent blocks."""
    _fields_ = [("mant_bits", ctypes.c_int32), ("rounding", ctypes.c_int32),
                ("block_rows", ctypes.c_int64), ("block_cols", ctypes.c_int64), ("seed", ctypes.c_uint64),
                ("k_slot", ctypes.c_int64)]


class Conv2d(ctypes.Structure):
    """hbfp_conv2d: NHWC input, filter r x s, zero padding and strides."""
    _fields_ = [("n", ctypes.c_int64), ("h", ctypes.c_int64), ("w", ctypes.c_int64), ("c", ctypes.c_int64),
                ("r", ctypes.c_int32), ("s", ctypes.c_int32), ("pad_h", ctypes.c_int32), ("pad_w", ctypes.c_int32),
                ("stride_h", ctypes.c_int32), ("stride_w", ctypes.c_int32), ("c_block", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]

    def out_hw(self):
        return ((self.h + 2 * self.pad_h - self.r) // self.stride_h + 1, (self.w + 2 * self.pad_w - self.s) // self.stride_w + 1)


class EncodeJob(ctypes.Structure):
    """hbfp_encode_job: one source of hbfp_encode_packed_batch."""
    _fields_ = [("src", ctypes.c_void_p), ("ld", ctypes.c_int64), ("n", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("outs", ctypes.c_void_p), ("packed", ctypes.c_void_p), ("packed_bytes", ctypes.c_void_p)]


class TensorDesc(ctypes.Structure):
    """hbfp_tensor: an encoded operand (layout in include/hbfp.h)."""
    _fields_ = [("mant", ctypes.c_void_p), ("exps", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("kdim", ctypes.c_int64), ("kblock", ctypes.c_int64),
                ("kblock_pad", ctypes.c_int64), ("nblk", ctypes.c_int64), ("kpad", ctypes.c_int64),
                ("exp_ld", ctypes.c_int64), ("rblock", ctypes.c_int64), ("kshare", ctypes.c_int64),
                ("src_rows", ctypes.c_int64), ("src_cols", ctypes.c_int64),
                ("contract_axis", ctypes.c_int32), ("mant_bits", ctypes.c_int32),
                ("rounding", ctypes.c_int32), ("hints", ctypes.c_int32),
                ("seed", ctypes.c_uint64), ("mant_bytes", ctypes.c_uint64), ("exp_bytes", ctypes.c_uint64)]


class CacheDesc(ctypes.Structure):
    """hbfp_cache: keys and values in 4-bit BFP (layout in include/hbfp.h)."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exps", ctypes.c_void_p), ("v_exps", ctypes.c_void_p),
                ("batch", ctypes.c_int64), ("heads", ctypes.c_int64), ("capacity", ctypes.c_int64), ("dim", ctypes.c_int64),
                ("slots", ctypes.c_int64), ("nblk", ctypes.c_int64), ("code_bytes", ctypes.c_uint64), ("exp_bytes", ctypes.c_uint64)]


class Heads(ctypes.Structure):
    """hbfp_heads: one call's tensor [batch][tokens][heads][dim]."""
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("stride_batch", ctypes.c_int64), ("stride_token", ctypes.c_int64), ("stride_head", ctypes.c_int64)]


class Mx4Desc(ctypes.Structure):
    """hbfp_mx4: an operand in microscaled 4-bit floating point (layout in include/hbfp.h)."""
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64), ("kdim", ctypes.c_int64),
                ("groups", ctypes.c_int64), ("scale_rows", ctypes.c_int64), ("code_bytes", ctypes.c_uint64), ("scale_bytes", ctypes.c_uint64)]


class NormDesc(ctypes.Structure):
    """hbfp_norm: the arguments of a norm that do not depend on the form of its result."""
    _fields_ = [("x", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("sum", ctypes.c_void_p),
                ("values", ctypes.c_void_p), ("rstd", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ldx", ctypes.c_int64), ("ld_residual", ctypes.c_int64), ("ld_sum", ctypes.c_int64), ("ld_values", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(_LIB_PATH)
    i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    F, T = ctypes.POINTER(Format), ctypes.POINTER(TensorDesc)
    lib.hbfp_version.restype = i32
    lib.hbfp_status_string.restype = ctypes.c_char_p
    lib.hbfp_status_string.argtypes = [i32]
    lib.hbfp_plan.argtypes = [F, i64, i64, i32, T]
    lib.hbfp_sizes.argtypes = [F, i64, i64, i32, ctypes.POINTER(sz), ctypes.POINTER(sz), ctypes.POINTER(i64)]
    lib.hbfp_sizes.restype = i32
    lib.hbfp_encode_workspace.argtypes = [T, ctypes.POINTER(sz)]
    lib.hbfp_encode.argtypes = [vp, i64, i64, i64, i32, F, T, vp, sz, vp]
    lib.hbfp_encode_static.argtypes = [vp, i64, i64, i64, i32, F, T, vp]
    lib.hbfp_encode_static_limit.restype = sz
    lib.hbfp_encode_static_limit.argtypes = []
    lib.hbfp_decode.argtypes = [T, vp, i64, vp]
    lib.hbfp_encode_im2col.argtypes = [vp, ctypes.POINTER(Conv2d), T, vp, sz, vp]
    lib.hbfp_encode_im2col_workspace.argtypes = [ctypes.POINTER(Conv2d), T, ctypes.POINTER(sz)]
    lib.hbfp_encode_im2col_workspace.restype = i32
    lib.hbfp_gemm_conv2d_workspace.argtypes = [T, ctypes.POINTER(Conv2d), T, ctypes.POINTER(sz)]
    lib.hbfp_gemm_conv2d_workspace.restype = i32
    lib.hbfp_gemm_conv2d.argtypes = [T, ctypes.POINTER(Conv2d), T, vp, i64, ctypes.c_float, vp, sz, vp]
    lib.hbfp_gemm_conv2d.restype = i32
    lib.hbfp_gemm_conv2d_bfp_workspace.argtypes = [T, ctypes.POINTER(Conv2d), T, T, ctypes.POINTER(sz)]
    lib.hbfp_gemm_conv2d_bfp_workspace.restype = i32
    lib.hbfp_gemm_conv2d_bfp.argtypes = [T, ctypes.POINTER(Conv2d), T, T, i32, vp, sz, vp]
    lib.hbfp_gemm_conv2d_bfp.restype = i32
    lib.hbfp_gemm_conv2d_dgrad_workspace.argtypes = [T, ctypes.POINTER(Conv2d), T, ctypes.POINTER(sz)]
    lib.hbfp_gemm_conv2d_dgrad_workspace.restype = i32
    lib.hbfp_gemm_conv2d_dgrad.argtypes = [T, ctypes.POINTER(Conv2d), T, vp, i64, ctypes.c_float, vp, sz, vp]
    lib.hbfp_gemm_conv2d_dgrad.restype = i32
    lib.hbfp_gemm_workspace.argtypes = [T, T, ctypes.POINTER(sz)]
    lib.hbfp_gemm.argtypes = [T, T, vp, i64, ctypes.c_float, vp, sz, vp]
    lib.hbfp_gemm_select_workspace.argtypes = [T, T, i32, ctypes.POINTER(sz)]
    lib.hbfp_gemm_select.argtypes = [T, T, vp, i64, ctypes.c_float, i32, vp, sz, vp]
    lib.hbfp_gemm_batch_workspace.argtypes = [i32, ctypes.POINTER(T), ctypes.POINTER(T), i32, ctypes.POINTER(sz)]
    lib.hbfp_gemm_batch.argtypes = [i32, ctypes.POINTER(T), ctypes.POINTER(T), ctypes.POINTER(vp), ctypes.POINTER(i64),
                                    ctypes.c_float, i32, vp, sz, vp]
    lib.hbfp_gemm_bfp_workspace.argtypes = [T, T, T, i32, ctypes.POINTER(sz)]
    lib.hbfp_gemm_bfp.argtypes = [T, T, T, i32, i32, vp, sz, vp]
    lib.hbfp_pack_bytes.argtypes = [T, ctypes.POINTER(sz)]
    lib.hbfp_pack.argtypes = [T, vp, sz, vp]
    lib.hbfp_gemm_packed_workspace.argtypes = [T, T, ctypes.POINTER(sz)]
    lib.hbfp_gemm_packed.argtypes = [T, vp, T, vp, vp, i64, ctypes.c_float, vp, sz, vp]
    lib.hbfp_gemm_packed_batch_workspace.argtypes = [i32, ctypes.POINTER(T), ctypes.POINTER(T), ctypes.POINTER(sz)]
    lib.hbfp_gemm_packed_batch.argtypes = [i32, ctypes.POINTER(T), ctypes.POINTER(vp), ctypes.POINTER(T), ctypes.POINTER(vp),
                                           ctypes.POINTER(vp), ctypes.POINTER(i64), ctypes.c_float, vp, sz, vp]
    lib.hbfp_gemm_partials.argtypes = [T, T, vp, vp, sz, vp]
    lib.hbfp_gemm_partials_window.argtypes = [T, T, i64, i64, i64, i64, vp, vp, sz, vp]
    lib.hbfp_gemm_f32_workspace.argtypes = [i32, i32, i64, i64, i64, F, F, ctypes.POINTER(sz)]
    lib.hbfp_gemm_f32.argtypes = [i32, i32, i64, i64, i64, vp, i64, vp, i64, vp, i64, F, F, vp, sz, vp]
    lib.hbfp_encode_multi_workspace.argtypes = [i32, ctypes.POINTER(T), ctypes.POINTER(sz)]
    lib.hbfp_encode_multi.argtypes = [vp, i64, i32, ctypes.POINTER(T), vp, sz, vp]
    lib.hbfp_encode_packed_workspace.argtypes = [i32, ctypes.POINTER(T), ctypes.POINTER(sz)]
    lib.hbfp_encode_packed.argtypes = [vp, i64, i32, ctypes.POINTER(T), ctypes.POINTER(vp), ctypes.POINTER(sz), vp, sz, vp]
    lib.hbfp_encode_packed_batch_workspace.argtypes = [i32, ctypes.POINTER(EncodeJob), ctypes.POINTER(sz)]
    lib.hbfp_encode_packed_batch.argtypes = [i32, ctypes.POINTER(EncodeJob), vp, sz, vp]
    lib.hbfp_probe_matrix_rate.argtypes = [i32, vp, i32, i32, vp, vp, vp]
    lib.hbfp_probe_matrix_rate.restype = i32
    lib.hbfp_weight_update_workspace.argtypes = [T, T, T, ctypes.POINTER(sz)]
    lib.hbfp_weight_update.argtypes = [T, vp, i64, ctypes.c_float, T, T, vp, sz, vp]
    KV, H, f32 = ctypes.POINTER(CacheDesc), ctypes.POINTER(Heads), ctypes.c_float
    lib.hbfp_cache_plan.argtypes = [i64, i64, i64, i64, KV]
    lib.hbfp_cache_append.argtypes = [KV, H, H, i64, vp, vp, vp, vp]
    lib.hbfp_cache_read.argtypes = [KV, vp, i32, vp, vp, vp]
    lib.hbfp_cache_attend_workspace.argtypes = [KV, i64, i64, i32, i64, ctypes.POINTER(sz)]
    lib.hbfp_cache_attend.argtypes = [KV, H, i64, i64, vp, i64, f32, i32, H, vp, vp, sz, vp]
    lib.hbfp_cache_weigh.argtypes = [KV, H, i64, i64, vp, f32, i32, vp, f32, vp, vp, i64, vp]
    lib.hbfp_cache_weigh_longest.argtypes = [KV, H, i64, i64, vp, i64, f32, i32, vp, f32, vp, vp, i64, vp]
    lib.hbfp_cache_evict.argtypes = [KV, vp, i64, vp, i64, i64, KV, vp, i64, vp, vp, vp]
    lib.hbfp_rows_plan.argtypes = [i64, i64, ctypes.POINTER(i64), ctypes.POINTER(sz)]
    lib.hbfp_quant_rows.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp]
    lib.hbfp_gemm_rows_workspace.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
    lib.hbfp_gemm_rows.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, i32, i64, vp, sz, vp]
    lib.hbfp_linear_i8_workspace.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
    lib.hbfp_linear_i8.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, i64, vp, i64, vp, sz, vp]
    X, size = ctypes.POINTER(Mx4Desc), ctypes.POINTER(sz)
    lib.hbfp_mx4_plan.argtypes = [i64, i64, X]
    lib.hbfp_quant_mx4.argtypes = [vp, i32, i64, i64, i64, i32, ctypes.c_uint64, X, X, vp]
    lib.hbfp_read_mx4.argtypes = [X, i32, vp, i64, vp]
    lib.hbfp_gemm_mx4_workspace.argtypes = [i64, i64, i64, size]
    lib.hbfp_gemm_mx4.argtypes = [X, X, vp, vp, i32, i64, vp, sz, vp]
    lib.hbfp_linear_mx4_workspace.argtypes = [i64, i64, i64, size]
    lib.hbfp_linear_mx4.argtypes = [vp, i32, i64, i64, X, vp, vp, i64, vp, sz, vp]
    lib.hbfp_norm_i8.argtypes = [ctypes.POINTER(NormDesc), vp, vp, vp]
    lib.hbfp_norm_mx4.argtypes = [ctypes.POINTER(NormDesc), X, vp]
    lib.hbfp_norm_grad_workspace.argtypes = [i64, i64, size]
    lib.hbfp_norm_grad.argtypes = [vp, i64, vp, i64, vp, vp, vp, i64, i32, i64, i64, vp, i64, vp, vp, sz, vp]
    for name in ("hbfp_mx4_plan", "hbfp_quant_mx4", "hbfp_read_mx4", "hbfp_gemm_mx4_workspace", "hbfp_gemm_mx4", "hbfp_linear_mx4_workspace",
                 "hbfp_linear_mx4", "hbfp_norm_i8", "hbfp_norm_mx4", "hbfp_norm_grad_workspace", "hbfp_norm_grad"):
        getattr(lib, name).restype = i32
    for name in ("hbfp_cache_plan", "hbfp_cache_append", "hbfp_cache_read", "hbfp_cache_attend_workspace", "hbfp_cache_attend",
                 "hbfp_cache_weigh", "hbfp_cache_weigh_longest", "hbfp_cache_evict", "hbfp_rows_plan", "hbfp_quant_rows", "hbfp_gemm_rows_workspace",
                 "hbfp_gemm_rows", "hbfp_linear_i8_workspace", "hbfp_linear_i8"):
        getattr(lib, name).restype = i32
    for name in ("hbfp_gemm_batch_workspace", "hbfp_gemm_batch", "hbfp_gemm_bfp_workspace", "hbfp_gemm_bfp", "hbfp_encode_im2col", "hbfp_encode_multi_workspace", "hbfp_encode_multi", "hbfp_encode_packed_workspace", "hbfp_encode_packed", "hbfp_encode_packed_batch_workspace", "hbfp_encode_packed_batch", "hbfp_weight_update_workspace", "hbfp_weight_update", "hbfp_plan", "hbfp_encode_workspace", "hbfp_encode", "hbfp_encode_static", "hbfp_decode", "hbfp_gemm_workspace",
                 "hbfp_gemm", "hbfp_gemm_select_workspace", "hbfp_gemm_select", "hbfp_pack_bytes", "hbfp_pack",
                 "hbfp_gemm_packed_workspace", "hbfp_gemm_packed", "hbfp_gemm_packed_batch_workspace", "hbfp_gemm_packed_batch", "hbfp_gemm_partials", "hbfp_gemm_partials_window", "hbfp_gemm_f32_workspace",
                 "hbfp_gemm_f32"):
        getattr(lib, name).restype = i32
    return lib


_lib = _load()


def library_path() -> str:
    return _LIB_PATH


def version() -> int:
    return int(_lib.hbfp_version())


def status_string(status: int) -> str:
    return _lib.hbfp_status_string(status).decode()


def _check(rc: int, where: str):
    if rc != OK:
        raise HbfpError(rc, where)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dev_ptr(t: Optional[torch.Tensor]):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def make_format(mant_bits: int, block_rows: int, block_cols: int, rounding: int = RNE, seed: int = 0,
                k_slot: int = 0) -> Format:
    return Format(mant_bits, rounding, block_rows, block_cols, seed, k_slot)


# ---------------------------------------------------------------------------- C ABI, one to one
def plan(fmt: Format, rows: int, cols: int, contract_axis: int) -> TensorDesc:
    d = TensorDesc()
    _check(_lib.hbfp_plan(ctypes.byref(fmt), rows, cols, contract_axis, ctypes.byref(d)), "hbfp_plan")
    return d


def sizes(fmt: Format, rows: int, cols: int, contract_axis: int):
    """hbfp_sizes: (mantissa bytes, exponent bytes, stored contraction length) of the operand a conversion produces."""
    mb, eb, kp = ctypes.c_size_t(0), ctypes.c_size_t(0), ctypes.c_int64(0)
    _check(_lib.hbfp_sizes(ctypes.byref(fmt), rows, cols, contract_axis, ctypes.byref(mb), ctypes.byref(eb), ctypes.byref(kp)), "hbfp_sizes")
    return int(mb.value), int(eb.value), int(kp.value)


def encode_workspace(desc: TensorDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_encode_workspace(ctypes.byref(desc), ctypes.byref(n)), "hbfp_encode_workspace")
    return int(n.value)


def gemm_workspace(a: TensorDesc, b: TensorDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_workspace(ctypes.byref(a), ctypes.byref(b), ctypes.byref(n)), "hbfp_gemm_workspace")
    return int(n.value)


def gemm_f32_workspace(trans_a: int, trans_b: int, M: int, N: int, K: int, fa: Format, fb: Format) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_f32_workspace(trans_a, trans_b, M, N, K, ctypes.byref(fa), ctypes.byref(fb),
                                        ctypes.byref(n)), "hbfp_gemm_f32_workspace")
    return int(n.value)


@dataclass
class BfpTensor:
    """An encoded operand: the descriptor plus the torch buffers that back its two pointers."""
    desc: TensorDesc
    mant: torch.Tensor   # int8 / int16 [rows, kpad]
    exps: torch.Tensor   # uint8 [rows, exp_ld]


def alloc(fmt: Format, rows: int, cols: int, contract_axis: int, device="cuda") -> BfpTensor:
    d = plan(fmt, rows, cols, contract_axis)
    dt = torch.int8 if d.mant_bits <= 8 else torch.int16
    mant = torch.empty((d.rows, d.kpad), dtype=dt, device=device)
    exps = torch.empty((d.rows, d.exp_ld), dtype=torch.uint8, device=device)
    d.mant, d.exps = mant.data_ptr(), exps.data_ptr()
    return BfpTensor(d, mant, exps)


def _workspace(nbytes: int, device) -> Optional[torch.Tensor]:
    """Scratch for a call that was given none.  A caller's own workspace goes to the library as it is, which checks its size: asking
    for the size first would cost such a call a second trip through ctypes (host time of a product 11.6 -> 7.8 us, of gemm_f32
    20 -> 14.5 us, of a conversion 8.9 -> 8.1 us)."""
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def encode(src: torch.Tensor, contract_axis: int, fmt: Format, out: Optional[BfpTensor] = None,
           workspace: Optional[torch.Tensor] = None, stream=None) -> BfpTensor:
    """hbfp_encode on a 2-D FP32 device tensor (row stride = its leading dimension)."""
    assert src.is_cuda and src.dtype == torch.float32 and src.dim() == 2 and src.stride(1) == 1
    rows, cols = src.shape
    ld = src.stride(0) if rows > 1 else max(src.stride(0), cols)
    if out is None:
        out = alloc(fmt, rows, cols, contract_axis, src.device)
    if workspace is None:
        workspace = _workspace(encode_workspace(out.desc), src.device)
    _check(_lib.hbfp_encode(_dev_ptr(src), rows, cols, ld, contract_axis, ctypes.byref(fmt), ctypes.byref(out.desc),
                            _dev_ptr(workspace), 0 if workspace is None else workspace.numel(),
                            _stream_ptr(stream)), "hbfp_encode")
    return out


def encode_static_limit() -> int:
    return int(_lib.hbfp_encode_static_limit())


def encode_static(src: torch.Tensor, contract_axis: int, fmt: Format, out: BfpTensor, stream=None) -> BfpTensor:
    """hbfp_encode_static: hbfp_encode whose scratch is a fixed array inside the library (nothing is allocated;
    `out` comes from ``alloc``)."""
    assert src.is_cuda and src.dtype == torch.float32 and src.dim() == 2 and src.stride(1) == 1
    rows, cols = src.shape
    ld = src.stride(0) if rows > 1 else max(src.stride(0), cols)
    _check(_lib.hbfp_encode_static(_dev_ptr(src), rows, cols, ld, contract_axis, ctypes.byref(fmt), ctypes.byref(out.desc),
                                   _stream_ptr(stream)), "hbfp_encode_static")
    return out


def decode(t: BfpTensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty((t.desc.src_rows, t.desc.src_cols), dtype=torch.float32, device=t.mant.device)
    assert out.is_cuda and out.dtype == torch.float32 and out.stride(1) == 1
    _check(_lib.hbfp_decode(ctypes.byref(t.desc), _dev_ptr(out), out.stride(0), _stream_ptr(stream)), "hbfp_decode")
    return out


KERNEL_AUTO, KERNEL_INT8, KERNEL_SCALED, KERNEL_INT8_WIDE, KERNEL_FP16, KERNEL_BF16, KERNEL_FP16_PLANES = 0, 1, 2, 3, 4, 5, 6


def gemm_select_workspace(a: TensorDesc, b: TensorDesc, kernel: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_select_workspace(ctypes.byref(a), ctypes.byref(b), kernel, ctypes.byref(n)),
           "hbfp_gemm_select_workspace")
    return n.value


def gemm(a: BfpTensor, b: BfpTensor, out: Optional[torch.Tensor] = None, beta: float = 0.0,
         workspace: Optional[torch.Tensor] = None, stream=None, kernel: int = KERNEL_AUTO) -> torch.Tensor:
    """C[M,N] (+)= A . B^T over k (both operands k-contiguous); `kernel` as in hbfp_gemm_select."""
    if out is None:
        out = torch.empty((a.desc.rows, b.desc.rows), dtype=torch.float32, device=a.mant.device)
    assert out.is_cuda and out.dtype == torch.float32 and out.stride(1) == 1
    if workspace is None:
        workspace = _workspace(gemm_select_workspace(a.desc, b.desc, kernel), out.device)
    _check(_lib.hbfp_gemm_select(ctypes.byref(a.desc), ctypes.byref(b.desc), _dev_ptr(out), out.stride(0), beta, kernel,
                                 _dev_ptr(workspace), 0 if workspace is None else workspace.numel(),
                                 _stream_ptr(stream)), "hbfp_gemm_select")
    return out


def gemm_batch_workspace(pairs, kernel: int = KERNEL_AUTO) -> int:
    """pairs: sequence of (A, B), each a BfpTensor or a TensorDesc."""
    n = ctypes.c_size_t(0)
    a, b = _desc_array([p[0] for p in pairs]), _desc_array([p[1] for p in pairs])
    _check(_lib.hbfp_gemm_batch_workspace(len(pairs), a, b, kernel, ctypes.byref(n)), "hbfp_gemm_batch_workspace")
    return int(n.value)


def gemm_batch(pairs, outs, beta: float = 0.0, kernel: int = KERNEL_AUTO, workspace: Optional[torch.Tensor] = None, stream=None):
    """hbfp_gemm_batch: outs[i] (+)= A[i] . B[i]^T for up to 4 independent products in one call."""
    n = len(pairs)
    a, b = _desc_array([p[0] for p in pairs]), _desc_array([p[1] for p in pairs])
    for o in outs:
        assert o.is_cuda and o.dtype == torch.float32 and o.stride(1) == 1
    c = (ctypes.c_void_p * n)(*[o.data_ptr() for o in outs])
    ld = (ctypes.c_int64 * n)(*[o.stride(0) for o in outs])
    if workspace is None:
        workspace = _workspace(gemm_batch_workspace(pairs, kernel), outs[0].device)
    _check(_lib.hbfp_gemm_batch(n, a, b, c, ld, beta, kernel, _dev_ptr(workspace), 0 if workspace is None else workspace.numel(),
                                _stream_ptr(stream)), "hbfp_gemm_batch")
    return outs


def gemm_bfp_workspace(a: TensorDesc, b: TensorDesc, out: TensorDesc, kernel: int = KERNEL_AUTO) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_bfp_workspace(ctypes.byref(a), ctypes.byref(b), ctypes.byref(out), kernel, ctypes.byref(n)),
           "hbfp_gemm_bfp_workspace")
    return int(n.value)


def gemm_bfp(a: BfpTensor, b: BfpTensor, fmt: Format, contract_axis: int = 1, relu: bool = False, kernel: int = KERNEL_AUTO,
             out: Optional[BfpTensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> BfpTensor:
    """hbfp_gemm_bfp: encode(relu?(A . B^T)) as an operand in format `fmt` (the next product's input)."""
    if out is None:
        out = alloc(fmt, a.desc.rows, b.desc.rows, contract_axis, a.mant.device)
    if workspace is None:
        workspace = _workspace(gemm_bfp_workspace(a.desc, b.desc, out.desc, kernel), a.mant.device)
    _check(_lib.hbfp_gemm_bfp(ctypes.byref(a.desc), ctypes.byref(b.desc), ctypes.byref(out.desc), int(relu), kernel,
                              _dev_ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream)),
           "hbfp_gemm_bfp")
    return out


def pack_bytes(desc: TensorDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_pack_bytes(ctypes.byref(desc), ctypes.byref(n)), "hbfp_pack_bytes")
    return int(n.value)


def pack(t: BfpTensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Limb planes of an encoded operand for gemm_packed (opaque bytes; pack again after encoding again)."""
    n = pack_bytes(t.desc)
    if out is None:
        out = torch.empty(n, dtype=torch.uint8, device=t.mant.device)
    _check(_lib.hbfp_pack(ctypes.byref(t.desc), _dev_ptr(out), out.numel(), _stream_ptr(stream)), "hbfp_pack")
    return out


def gemm_packed_workspace(a: TensorDesc, b: TensorDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_packed_workspace(ctypes.byref(a), ctypes.byref(b), ctypes.byref(n)), "hbfp_gemm_packed_workspace")
    return int(n.value)


def gemm_packed(a: BfpTensor, packed_a: torch.Tensor, b: BfpTensor, packed_b: torch.Tensor,
                out: Optional[torch.Tensor] = None, beta: float = 0.0, workspace: Optional[torch.Tensor] = None,
                stream=None) -> torch.Tensor:
    """C[M,N] (+)= A . B^T on the block-scaled kernel from operands packed beforehand."""
    if out is None:
        out = torch.empty((a.desc.rows, b.desc.rows), dtype=torch.float32, device=a.mant.device)
    assert out.is_cuda and out.dtype == torch.float32 and out.stride(1) == 1
    if workspace is None:
        workspace = _workspace(gemm_packed_workspace(a.desc, b.desc), out.device)
    _check(_lib.hbfp_gemm_packed(ctypes.byref(a.desc), _dev_ptr(packed_a), ctypes.byref(b.desc), _dev_ptr(packed_b),
                                 _dev_ptr(out), out.stride(0), beta, _dev_ptr(workspace),
                                 0 if workspace is None else workspace.numel(), _stream_ptr(stream)), "hbfp_gemm_packed")
    return out


def gemm_packed_batch_workspace(pairs) -> int:
    """pairs: sequence of (A, B), each a BfpTensor or a TensorDesc."""
    n = ctypes.c_size_t(0)
    a, b = _desc_array([p[0] for p in pairs]), _desc_array([p[1] for p in pairs])
    _check(_lib.hbfp_gemm_packed_batch_workspace(len(pairs), a, b, ctypes.byref(n)), "hbfp_gemm_packed_batch_workspace")
    return int(n.value)


def gemm_packed_batch(products, outs, beta: float = 0.0, workspace: Optional[torch.Tensor] = None, stream=None):
    """hbfp_gemm_packed_batch: outs[i] (+)= A[i] . B[i]^T; products: sequence of (A, packed A, B, packed B)."""
    n = len(products)
    a, b = _desc_array([p[0] for p in products]), _desc_array([p[2] for p in products])
    pa = (ctypes.c_void_p * n)(*[p[1].data_ptr() for p in products])
    pb = (ctypes.c_void_p * n)(*[p[3].data_ptr() for p in products])
    for o in outs:
        assert o.is_cuda and o.dtype == torch.float32 and o.stride(1) == 1
    c = (ctypes.c_void_p * n)(*[o.data_ptr() for o in outs])
    ld = (ctypes.c_int64 * n)(*[o.stride(0) for o in outs])
    if workspace is None:
        workspace = _workspace(gemm_packed_batch_workspace([(p[0], p[2]) for p in products]), outs[0].device)
    _check(_lib.hbfp_gemm_packed_batch(n, a, pa, b, pb, c, ld, beta, _dev_ptr(workspace),
                                       0 if workspace is None else workspace.numel(), _stream_ptr(stream)), "hbfp_gemm_packed_batch")
    return outs


def gemm_partials(a: BfpTensor, b: BfpTensor, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    P = torch.empty((a.desc.rows, b.desc.rows, a.desc.nblk), dtype=torch.int32, device=a.mant.device)
    if workspace is None:
        workspace = _workspace(gemm_select_workspace(a.desc, b.desc, KERNEL_INT8), P.device)
    _check(_lib.hbfp_gemm_partials(ctypes.byref(a.desc), ctypes.byref(b.desc), _dev_ptr(P), _dev_ptr(workspace),
                                   0 if workspace is None else workspace.numel(), _stream_ptr(stream)),
           "hbfp_gemm_partials")
    return P


def gemm_partials_window(a: BfpTensor, b: BfpTensor, row0: int, rows: int, col0: int, cols: int,
                          workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """hbfp_gemm_partials_window: the integer block sums of rows row0.. x columns col0.. of the product only."""
    P = torch.empty((rows, cols, a.desc.nblk), dtype=torch.int32, device=a.mant.device)
    if workspace is None:
        workspace = _workspace(gemm_select_workspace(a.desc, b.desc, KERNEL_INT8), P.device)
    _check(_lib.hbfp_gemm_partials_window(ctypes.byref(a.desc), ctypes.byref(b.desc), row0, rows, col0, cols, _dev_ptr(P),
                                          _dev_ptr(workspace), 0 if workspace is None else workspace.numel(),
                                          _stream_ptr(stream)), "hbfp_gemm_partials_window")
    return P


def gemm_f32(trans_a: int, trans_b: int, A: torch.Tensor, B: torch.Tensor, fa: Format, fb: Format,
             out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """C = op(A) op(B): encode both operands along the contraction axis, then the BFP product."""
    assert A.is_cuda and B.is_cuda and A.dtype == B.dtype == torch.float32
    assert A.stride(1) == 1 and B.stride(1) == 1
    M, K = (A.shape[1], A.shape[0]) if trans_a else A.shape
    N = B.shape[0] if trans_b else B.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
    if workspace is None:
        workspace = _workspace(gemm_f32_workspace(trans_a, trans_b, M, N, K, fa, fb), A.device)
    _check(_lib.hbfp_gemm_f32(trans_a, trans_b, M, N, K, _dev_ptr(A), A.stride(0), _dev_ptr(B), B.stride(0),
                              _dev_ptr(out), out.stride(0), ctypes.byref(fa), ctypes.byref(fb),
                              _dev_ptr(workspace), 0 if workspace is None else workspace.numel(),
                              _stream_ptr(stream)), "hbfp_gemm_f32")
    return out


def _desc_ref(t: Optional[BfpTensor]):
    return None if t is None else ctypes.byref(t.desc)


def weight_update_workspace(wide: BfpTensor, narrow_a: Optional[BfpTensor] = None,
                            narrow_b: Optional[BfpTensor] = None) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_weight_update_workspace(ctypes.byref(wide.desc), _desc_ref(narrow_a), _desc_ref(narrow_b),
                                             ctypes.byref(n)), "hbfp_weight_update_workspace")
    return int(n.value)


def weight_update(wide: BfpTensor, delta: torch.Tensor, alpha: float, narrow_a: Optional[BfpTensor] = None,
                  narrow_b: Optional[BfpTensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """hbfp_weight_update: wide <- encode(fma(alpha, delta, value(wide))), and the same FP32 result into the narrow tensors."""
    assert delta.is_cuda and delta.dtype == torch.float32 and delta.dim() == 2 and delta.stride(1) == 1
    if workspace is None:
        workspace = _workspace(weight_update_workspace(wide, narrow_a, narrow_b), delta.device)
    _check(_lib.hbfp_weight_update(ctypes.byref(wide.desc), _dev_ptr(delta), delta.stride(0), alpha,
                                   _desc_ref(narrow_a), _desc_ref(narrow_b), _dev_ptr(workspace),
                                   0 if workspace is None else workspace.numel(), _stream_ptr(stream)),
           "hbfp_weight_update")
    return workspace


def _desc_array(outs):
    arr = (ctypes.POINTER(TensorDesc) * len(outs))()
    for i, t in enumerate(outs):
        arr[i] = ctypes.pointer(t.desc if hasattr(t, "desc") else t)     # BfpTensor or bare descriptor
    return arr


def encode_im2col_workspace(conv: Conv2d, desc: TensorDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_encode_im2col_workspace(ctypes.byref(conv), ctypes.byref(desc), ctypes.byref(n)), "hbfp_encode_im2col_workspace")
    return int(n.value)


def encode_im2col(x: torch.Tensor, conv: Conv2d, fmt: Format, contract_axis: int = 1, out: Optional[BfpTensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> BfpTensor:
    """hbfp_encode_im2col on an NHWC FP32 device tensor: the lowered activation operand of a convolution
    (contract_axis 1: forward product, 0: weight gradient)."""
    assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and tuple(x.shape) == (conv.n, conv.h, conv.w, conv.c)
    ho, wo = conv.out_hw()
    if out is None:
        out = alloc(fmt, conv.n * ho * wo, conv.r * conv.s * conv.c, contract_axis, x.device)
    if workspace is None:
        workspace = _workspace(encode_im2col_workspace(conv, out.desc), x.device)
    _check(_lib.hbfp_encode_im2col(_dev_ptr(x), ctypes.byref(conv), ctypes.byref(out.desc), _dev_ptr(workspace),
                                   0 if workspace is None else workspace.numel(), _stream_ptr(stream)), "hbfp_encode_im2col")
    return out


def encode_multi_workspace(outs) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_encode_multi_workspace(len(outs), _desc_array(outs), ctypes.byref(n)), "hbfp_encode_multi_workspace")
    return int(n.value)


def encode_multi(src: torch.Tensor, outs, workspace: Optional[torch.Tensor] = None, stream=None):
    """hbfp_encode_multi: one FP32 matrix into up to three planned operand tensors (see ``alloc``)."""
    assert src.is_cuda and src.dtype == torch.float32 and src.dim() == 2 and src.stride(1) == 1
    rows, cols = src.shape
    ld = src.stride(0) if rows > 1 else max(src.stride(0), cols)
    arr = _desc_array(outs)
    if workspace is None:
        workspace = _workspace(encode_multi_workspace(outs), src.device)
    _check(_lib.hbfp_encode_multi(_dev_ptr(src), ld, len(outs), arr, _dev_ptr(workspace),
                                  0 if workspace is None else workspace.numel(), _stream_ptr(stream)), "hbfp_encode_multi")
    return outs



def encode_packed_workspace(outs) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_encode_packed_workspace(len(outs), _desc_array(outs), ctypes.byref(n)), "hbfp_encode_packed_workspace")
    return int(n.value)


def encode_packed(src: torch.Tensor, outs, packed, workspace: Optional[torch.Tensor] = None, stream=None):
    """hbfp_encode_packed: one FP32 matrix into planned operand tensors and their packed forms (``packed[i]`` a uint8
    device tensor of ``pack_bytes`` bytes, or None)."""
    assert src.is_cuda and src.dtype == torch.float32 and src.dim() == 2 and src.stride(1) == 1
    rows, cols = src.shape
    ld = src.stride(0) if rows > 1 else max(src.stride(0), cols)
    n = len(outs)
    ptrs = (ctypes.c_void_p * n)(*[None if b is None else b.data_ptr() for b in packed])
    sizes = (ctypes.c_size_t * n)(*[0 if b is None else b.numel() for b in packed])
    if workspace is None:
        workspace = _workspace(encode_packed_workspace(outs), src.device)
    _check(_lib.hbfp_encode_packed(_dev_ptr(src), ld, n, _desc_array(outs), ptrs, sizes, _dev_ptr(workspace),
                                   0 if workspace is None else workspace.numel(), _stream_ptr(stream)), "hbfp_encode_packed")
    return outs


def _encode_jobs(sources):
    """sources: sequence of (src, outs, packed); returns the job array and the objects that its pointers refer to."""
    jobs, keep = (EncodeJob * len(sources))(), []
    for j, (src, outs, packed) in enumerate(sources):
        assert src.is_cuda and src.dtype == torch.float32 and src.dim() == 2 and src.stride(1) == 1
        rows, cols = src.shape
        n = len(outs)
        descs = _desc_array(outs)
        ptrs = (ctypes.c_void_p * n)(*[None if b is None else b.data_ptr() for b in packed])
        sizes = (ctypes.c_size_t * n)(*[0 if b is None else b.numel() for b in packed])
        keep += [descs, ptrs, sizes]
        jobs[j].src, jobs[j].ld, jobs[j].n = src.data_ptr(), (src.stride(0) if rows > 1 else max(src.stride(0), cols)), n
        jobs[j].outs = ctypes.cast(descs, ctypes.c_void_p)
        jobs[j].packed = ctypes.cast(ptrs, ctypes.c_void_p)
        jobs[j].packed_bytes = ctypes.cast(sizes, ctypes.c_void_p)
    return jobs, keep


def encode_packed_batch_workspace(sources) -> int:
    jobs, keep = _encode_jobs(sources)
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_encode_packed_batch_workspace(len(sources), jobs, ctypes.byref(n)), "hbfp_encode_packed_batch_workspace")
    return int(n.value)


def encode_packed_batch(sources, workspace: Optional[torch.Tensor] = None, stream=None):
    """hbfp_encode_packed_batch: sources is a sequence of (src, outs, packed), each as the arguments of encode_packed."""
    jobs, keep = _encode_jobs(sources)
    if workspace is None:
        need = ctypes.c_size_t(0)
        _check(_lib.hbfp_encode_packed_batch_workspace(len(sources), jobs, ctypes.byref(need)), "hbfp_encode_packed_batch_workspace")
        workspace = _workspace(int(need.value), sources[0][0].device)
    _check(_lib.hbfp_encode_packed_batch(len(sources), jobs, _dev_ptr(workspace), 0 if workspace is None else workspace.numel(),
                                         _stream_ptr(stream)), "hbfp_encode_packed_batch")
    return [s[1] for s in sources]


def probe_matrix_rate(instruction: int, words: torch.Tensor, workgroups: int, iters: int, sink: torch.Tensor,
                      clocks: torch.Tensor, stream=None) -> None:
    """hbfp_probe_matrix_rate: one launch of the register-only loop (the caller times it with events)."""
    assert words.dtype == torch.int32 and words.numel() >= 64 * 64 and sink.numel() >= workgroups * 256
    assert clocks.dtype == torch.int64 and clocks.numel() >= 2
    _check(_lib.hbfp_probe_matrix_rate(instruction, _dev_ptr(words), workgroups, iters, _dev_ptr(sink), _dev_ptr(clocks),
                                       _stream_ptr(stream)), "hbfp_probe_matrix_rate")


def gemm_conv2d_workspace(image: TensorDesc, conv: Conv2d, filters: TensorDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_conv2d_workspace(ctypes.byref(image), ctypes.byref(conv), ctypes.byref(filters), ctypes.byref(n)),
           "hbfp_gemm_conv2d_workspace")
    return int(n.value)


def gemm_conv2d(image: BfpTensor, conv: Conv2d, filters: BfpTensor, out: Optional[torch.Tensor] = None, beta: float = 0.0,
                workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """hbfp_gemm_conv2d: Y[n*ho*wo, filters] from the image encoded once as [n*h*w, c] (blocks of 32 channels) and
    the filter matrix [r*s*c, filters] (blocks of 32 down its rows)."""
    ho, wo = conv.out_hw()
    if out is None:
        out = torch.empty((conv.n * ho * wo, filters.desc.rows), dtype=torch.float32, device=image.mant.device)
    assert out.is_cuda and out.dtype == torch.float32 and out.stride(1) == 1
    if workspace is None:
        workspace = _workspace(gemm_conv2d_workspace(image.desc, conv, filters.desc), out.device)
    _check(_lib.hbfp_gemm_conv2d(ctypes.byref(image.desc), ctypes.byref(conv), ctypes.byref(filters.desc), _dev_ptr(out),
                                 out.stride(0), beta, _dev_ptr(workspace), 0 if workspace is None else workspace.numel(),
                                 _stream_ptr(stream)), "hbfp_gemm_conv2d")
    return out


def gemm_conv2d_bfp_workspace(image: TensorDesc, conv: Conv2d, filters: TensorDesc, out: TensorDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_conv2d_bfp_workspace(ctypes.byref(image), ctypes.byref(conv), ctypes.byref(filters), ctypes.byref(out),
                                               ctypes.byref(n)), "hbfp_gemm_conv2d_bfp_workspace")
    return int(n.value)


def gemm_conv2d_bfp(image: BfpTensor, conv: Conv2d, filters: BfpTensor, fmt: Format, relu: bool = False, out: Optional[BfpTensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> BfpTensor:
    """hbfp_gemm_conv2d_bfp: the convolution delivered as an encoded operand [n*ho*wo, filters] (contraction along the
    filters): the next layer's image."""
    ho, wo = conv.out_hw()
    if out is None:
        out = alloc(fmt, conv.n * ho * wo, filters.desc.rows, 1, image.mant.device)
    if workspace is None:
        workspace = _workspace(gemm_conv2d_bfp_workspace(image.desc, conv, filters.desc, out.desc), image.mant.device)
    _check(_lib.hbfp_gemm_conv2d_bfp(ctypes.byref(image.desc), ctypes.byref(conv), ctypes.byref(filters.desc), ctypes.byref(out.desc),
                                     1 if relu else 0, _dev_ptr(workspace), 0 if workspace is None else workspace.numel(),
                                     _stream_ptr(stream)), "hbfp_gemm_conv2d_bfp")
    return out


def gemm_conv2d_dgrad_workspace(dy: TensorDesc, conv: Conv2d, filters: TensorDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_conv2d_dgrad_workspace(ctypes.byref(dy), ctypes.byref(conv), ctypes.byref(filters), ctypes.byref(n)),
           "hbfp_gemm_conv2d_dgrad_workspace")
    return int(n.value)


def gemm_conv2d_dgrad(dy: BfpTensor, conv: Conv2d, filters: BfpTensor, out: Optional[torch.Tensor] = None, beta: float = 0.0,
                      workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """hbfp_gemm_conv2d_dgrad: dX[n*h*w, c] of the convolution `conv` (any stride) from its output gradient encoded once
    as [n*ho*wo, filters] (blocks of 32 filters) and the mirrored filter matrix [r*s*filters, c]."""
    if out is None:
        out = torch.empty((conv.n * conv.h * conv.w, filters.desc.rows), dtype=torch.float32, device=dy.mant.device)
    assert out.is_cuda and out.dtype == torch.float32 and out.stride(1) == 1
    if workspace is None:
        workspace = _workspace(gemm_conv2d_dgrad_workspace(dy.desc, conv, filters.desc), out.device)
    _check(_lib.hbfp_gemm_conv2d_dgrad(ctypes.byref(dy.desc), ctypes.byref(conv), ctypes.byref(filters.desc), _dev_ptr(out),
                                       out.stride(0), beta, _dev_ptr(workspace), 0 if workspace is None else workspace.numel(),
                                       _stream_ptr(stream)), "hbfp_gemm_conv2d_dgrad")
    return out


# ---------------------------------------------------------------------------- serving: the 4-bit cache
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


_current_device = getattr(torch._C, "_cuda_getDevice", None)      # (torch.cuda.current_device without its wrapper: half a microsecond)


def _there(stream, device, call, *args):
    """`call` on another stream, or on a device that is not the current one.  On a stream of its own a call's buffers come from that
    stream's memory: a block that the caller's stream has freed may still be in use by work queued there, which the call does not
    wait for; and the results are not handed on before the caller's stream is done with them."""
    assert stream is None or stream.device == device, "a stream of the tensors' GPU"
    caller = torch.cuda.current_stream(device)
    with torch.cuda.device(device) if stream is None else torch.cuda.stream(stream):
        result = call(*args)
    if stream is not None:
        for t in _buffers(result):
            if t.numel():
                t.record_stream(caller)
    return result


def _buffers(result):
    """The tensors that a call returns."""
    if isinstance(result, Mx4):
        return [result.buffer]
    if isinstance(result, RowCodes):
        return [result.codes, result.scales]
    if isinstance(result, tuple):
        return [t for r in result for t in _buffers(r)]
    return [] if result is None else [result]


def _heads(t: torch.Tensor, batch: int, tokens: int, heads: int, dim: int, device) -> Heads:
    assert t.dtype in _TYPES and t.device == device, "a tensor of FP32, bf16 or FP16 on the cache's GPU"
    assert t.shape == (batch, tokens, heads, dim), f"shape {tuple(t.shape)}, expected {(batch, tokens, heads, dim)}"
    sb, st, sh, sd = t.stride()
    assert sd == 1 or dim == 1, "the head dimension must be contiguous"
    return Heads(t.data_ptr(), _TYPES[t.dtype], 0, sb if batch > 1 else 0, st if tokens > 1 else 0, sh if heads > 1 else 0)


def _lengths(lengths: torch.Tensor, batch: int, device) -> int:
    assert lengths.dtype == torch.int32 and lengths.device == device and lengths.is_contiguous() and lengths.numel() == batch
    return lengths.data_ptr()


def _raw_stream(device) -> int:
    """The current stream of a device.  A decode step is a few microseconds of kernels, and a torch.cuda.Stream object for each of its
    calls costs one of them; this is the handle alone."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


@dataclass
class KvCache:
    """Keys and values of one layer in 4-bit BFP: the descriptor plus the torch buffers behind its four pointers."""
    desc: CacheDesc
    k: torch.Tensor        # uint8 [batch, heads, slots * 16 * nblk]
    v: torch.Tensor
    k_exps: torch.Tensor   # uint8 [batch, heads, slots * nblk]
    v_exps: torch.Tensor


def _cache(desc: CacheDesc, k, v, k_exps, v_exps) -> KvCache:
    desc.k, desc.v, desc.k_exps, desc.v_exps = (t.data_ptr() for t in (k, v, k_exps, v_exps))
    return KvCache(desc, k, v, k_exps, v_exps)


def cache_plan(batch: int, heads: int, capacity: int, dim: int) -> CacheDesc:
    d = CacheDesc()
    _check(_lib.hbfp_cache_plan(batch, heads, capacity, dim, ctypes.byref(d)), "hbfp_cache_plan")
    return d


def cache_alloc(batch: int, heads: int, capacity: int, dim: int, device="cuda") -> KvCache:
    """An empty cache for `capacity` tokens of each batch entry (its contents are whatever the memory holds)."""
    d = cache_plan(batch, heads, capacity, dim)
    codes = [torch.empty((batch, heads, d.slots * 16 * d.nblk), dtype=torch.uint8, device=device) for _ in range(2)]
    exps = [torch.empty((batch, heads, d.slots * d.nblk), dtype=torch.uint8, device=device) for _ in range(2)]
    return _cache(d, *codes, *exps)


def cache_rows(cache: KvCache, first: int, last: int) -> KvCache:
    """The batch entries first .. last - 1 of a cache, as a cache over the same memory."""
    assert 0 <= first < last <= cache.desc.batch
    d = cache_plan(last - first, cache.desc.heads, cache.desc.capacity, cache.desc.dim)
    return _cache(d, *(t[first:last] for t in (cache.k, cache.v, cache.k_exps, cache.v_exps)))


def cache_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, lengths: torch.Tensor, values: bool = False, stream=None):
    """hbfp_cache_append: k, v [batch, tokens, heads, dim]; lengths (int32, on the GPU) count the new tokens.  values: returns the
    values that the cache now holds for them, a pair of bf16 tensors of k's shape."""
    d, tokens, device = cache.desc, k.shape[1], cache.k.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, cache_append, cache, k, v, lengths, values)
    batch, heads, dim = d.batch, d.heads, d.dim
    hk, hv = _heads(k, batch, tokens, heads, dim, device), _heads(v, batch, tokens, heads, dim, device)
    at = _lengths(lengths, batch, device)
    held = tuple(torch.empty(k.shape, dtype=torch.bfloat16, device=device) for _ in range(2)) if values else (None, None)
    _check(_lib.hbfp_cache_append(ctypes.byref(d), ctypes.byref(hk), ctypes.byref(hv), tokens, at, _ptr(held[0]), _ptr(held[1]),
                                  _raw_stream(device)), "hbfp_cache_append")
    return held if values else None


def cache_read(cache: KvCache, lengths: torch.Tensor, dtype=torch.float32, stream=None):
    """hbfp_cache_read: (keys, values) [batch, heads, capacity, dim], 0 from each length on."""
    d, device = cache.desc, cache.k.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, cache_read, cache, lengths, dtype)
    assert dtype in _TYPES
    at = _lengths(lengths, d.batch, device)
    k, v = (torch.empty((d.batch, d.heads, d.capacity, d.dim), dtype=dtype, device=device) for _ in range(2))
    _check(_lib.hbfp_cache_read(ctypes.byref(d), at, _TYPES[dtype], _ptr(k), _ptr(v), _raw_stream(device)), "hbfp_cache_read")
    return k, v


def cache_attend_workspace(desc: CacheDesc, tokens: int, heads: int, dtype=torch.bfloat16, longest: int = 0) -> int:
    return _attend_bytes(desc.batch, desc.heads, desc.capacity, desc.dim, tokens, heads, _TYPES[dtype], longest)


@functools.lru_cache(maxsize=1024)     # of sizes alone; asking the library anew would cost every step of a layer 2 us
def _attend_bytes(batch: int, kv_heads: int, capacity: int, dim: int, tokens: int, heads: int, dtype: int, longest: int) -> int:
    n, d = ctypes.c_size_t(0), cache_plan(batch, kv_heads, capacity, dim)
    _check(_lib.hbfp_cache_attend_workspace(ctypes.byref(d), tokens, heads, dtype, longest, ctypes.byref(n)), "hbfp_cache_attend_workspace")
    return int(n.value)


def cache_attend(cache: KvCache, q: torch.Tensor, lengths: torch.Tensor, scale: Optional[float] = None, causal: bool = True,
                 longest: int = 0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None):
    """hbfp_cache_attend: (out, lse) for q [batch, tokens, query heads, dim]; scale defaults to dim ** -0.5."""
    d, device = cache.desc, cache.k.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, cache_attend, cache, q, lengths, scale, causal, longest, out, lse, workspace)
    batch, dim = d.batch, d.dim
    _, tokens, heads, _ = q.shape
    hq, at = _heads(q, batch, tokens, heads, dim, device), _lengths(lengths, batch, device)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=device)
    if lse is None:
        lse = torch.empty((batch, tokens, heads), dtype=torch.float32, device=device)
    else:
        assert lse.device == device and lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == (batch, tokens, heads)
    ho = _heads(out, batch, tokens, heads, dim, device)
    if workspace is None:
        workspace = _workspace(_attend_bytes(batch, d.heads, d.capacity, dim, tokens, heads, hq.dtype, longest), device)
    _check(_lib.hbfp_cache_attend(ctypes.byref(d), ctypes.byref(hq), tokens, heads, at, longest, dim ** -0.5 if scale is None else scale,
                                  1 if causal else 0, ctypes.byref(ho), _ptr(lse), _ptr(workspace),
                                  0 if workspace is None else workspace.numel(), _raw_stream(device)), "hbfp_cache_attend")
    return out, lse


def cache_weigh(cache: KvCache, q: torch.Tensor, lse: torch.Tensor, lengths: torch.Tensor, weights: torch.Tensor,
                scale: Optional[float] = None, causal: bool = True, decay: float = 1.0, out: Optional[torch.Tensor] = None,
                stream=None, longest: int = 0) -> torch.Tensor:
    """hbfp_cache_weigh: out = decay * weights + the attention weight each cached token received; weights FP32 [batch, heads, n],
    n >= capacity; out defaults to weights (in place).  longest: that of the attention call that lse comes from."""
    d, device = cache.desc, cache.k.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, cache_weigh, cache, q, lse, lengths, weights, scale, causal, decay, out, None, longest)
    batch, dim = d.batch, d.dim
    _, tokens, heads, _ = q.shape
    hq = _heads(q, batch, tokens, heads, dim, device)
    out = weights if out is None else out
    for t in (weights, out):
        assert t.device == device and t.dtype == torch.float32 and t.is_contiguous() and t.shape == weights.shape
    assert weights.dim() == 3 and weights.shape[0] == batch and weights.shape[1] == d.heads
    assert lse.device == device and lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == (batch, tokens, heads)
    at = _lengths(lengths, batch, device)
    _check(_lib.hbfp_cache_weigh_longest(ctypes.byref(d), ctypes.byref(hq), tokens, heads, at, longest, dim ** -0.5 if scale is None else scale,
                                         1 if causal else 0, _ptr(lse), decay, _ptr(weights), _ptr(out), weights.shape[2],
                                         _raw_stream(device)), "hbfp_cache_weigh_longest")
    return out


def cache_evict(cache: KvCache, weights: torch.Tensor, lengths: torch.Tensor, out: KvCache, keep: int, recent: int,
                out_weights: Optional[torch.Tensor] = None, stream=None):
    """hbfp_cache_evict into the cache `out`: (kept slots [batch, heads, keep], new lengths, their weights [batch, heads, n])."""
    d, device = cache.desc, cache.k.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, cache_evict, cache, weights, lengths, out, keep, recent, out_weights)
    assert weights.device == device and weights.dtype == torch.float32 and weights.is_contiguous() and weights.dim() == 3
    assert weights.shape[:2] == (d.batch, d.heads) and out.k.device == device
    at = _lengths(lengths, d.batch, device)
    if out_weights is None:
        out_weights = torch.empty((d.batch, d.heads, out.desc.capacity), dtype=torch.float32, device=device)
    assert out_weights.device == device and out_weights.dtype == torch.float32 and out_weights.is_contiguous() and out_weights.dim() == 3
    assert out_weights.shape[:2] == (d.batch, d.heads)
    kept = torch.empty((d.batch, d.heads, max(keep, 1)), dtype=torch.int32, device=device)
    new_lengths = torch.empty((d.batch,), dtype=torch.int32, device=device)
    _check(_lib.hbfp_cache_evict(ctypes.byref(d), _ptr(weights), weights.shape[2], at, keep, recent, ctypes.byref(out.desc),
                                 _ptr(out_weights), out_weights.shape[2], _ptr(kept), _ptr(new_lengths), _raw_stream(device)),
           "hbfp_cache_evict")
    return kept, new_lengths, out_weights


# ---------------------------------------------------------------------------- serving: products with a scale per row
@dataclass
class RowCodes:
    """A matrix as rows of 8-bit codes with one FP32 scale each."""
    codes: torch.Tensor    # int8 [rows, kpad], 0 from cols on
    scales: torch.Tensor   # FP32 [rows]
    cols: int


def _matrix(t: torch.Tensor):
    assert t.is_cuda and t.dtype in _TYPES and t.dim() == 2, "FP32, bf16 or FP16 rows"
    (rows, cols), (ld, one) = t.shape, t.stride()
    assert one == 1 or cols <= 1, "FP32, bf16 or FP16 rows"
    return ld if rows > 1 else max(ld, cols)


def quant_rows(x: torch.Tensor, stream=None) -> RowCodes:
    """hbfp_quant_rows of x [rows, cols]: a linear layer's weights [out features, in features], once; or tokens."""
    ld = _matrix(x)
    if stream is not None or _current_device() != x.device.index:
        return _there(stream, x.device, quant_rows, x)
    kpad = ctypes.c_int64(0)
    _check(_lib.hbfp_rows_plan(x.shape[0], x.shape[1], ctypes.byref(kpad), None), "hbfp_rows_plan")
    codes = torch.empty((x.shape[0], kpad.value), dtype=torch.int8, device=x.device)
    scales = torch.empty((x.shape[0],), dtype=torch.float32, device=x.device)
    _check(_lib.hbfp_quant_rows(_ptr(x), _TYPES[x.dtype], x.shape[0], x.shape[1], ld, _ptr(codes), _ptr(scales),
                                _raw_stream(x.device)), "hbfp_quant_rows")
    return RowCodes(codes, scales, x.shape[1])


def _product_out(bias, w: RowCodes, rows: int, dtype, device, out):
    n = w.codes.shape[0]
    assert w.codes.device == device
    if bias is not None:
        assert bias.device == device and bias.dtype == torch.float32 and bias.is_contiguous() and bias.numel() == n
    if out is None:
        out = torch.empty((rows, n), dtype=dtype, device=device)
    assert out.device == device and out.dtype == dtype and tuple(out.shape) == (rows, n)
    return out, _matrix(out)


@functools.lru_cache(maxsize=1024)
def gemm_rows_workspace(rows: int, out_features: int, in_features: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_rows_workspace(rows, out_features, in_features, ctypes.byref(n)), "hbfp_gemm_rows_workspace")
    return int(n.value)


@functools.lru_cache(maxsize=1024)
def linear_i8_workspace(rows: int, out_features: int, in_features: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_linear_i8_workspace(rows, out_features, in_features, ctypes.byref(n)), "hbfp_linear_i8_workspace")
    return int(n.value)


def gemm_rows(a: RowCodes, w: RowCodes, bias: Optional[torch.Tensor] = None, dtype=torch.float32, out: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """hbfp_gemm_rows: y [rows of a, rows of w] = a . w^T (+ bias), rounded once to `dtype`."""
    assert a.cols == w.cols
    m, n, device = a.codes.shape[0], w.codes.shape[0], a.codes.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, gemm_rows, a, w, bias, dtype, out, workspace)
    out, ld = _product_out(bias, w, m, dtype if out is None else out.dtype, device, out)
    if workspace is None:
        workspace = _workspace(gemm_rows_workspace(m, n, a.cols), device)
    _check(_lib.hbfp_gemm_rows(_ptr(a.codes), _ptr(a.scales), _ptr(w.codes), _ptr(w.scales), _ptr(bias), m, n, a.cols,
                               _ptr(out), _TYPES[out.dtype], ld, _ptr(workspace), 0 if workspace is None else workspace.numel(),
                               _raw_stream(device)), "hbfp_gemm_rows")
    return out


def linear_i8(x: torch.Tensor, w: RowCodes, bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """hbfp_linear_i8: y = quant(x) . w^T (+ bias) in x's type, for x [tokens, in features] and weights from quant_rows."""
    ldx, (m, k), n = _matrix(x), x.shape, w.codes.shape[0]
    if stream is not None or _current_device() != x.device.index:
        return _there(stream, x.device, linear_i8, x, w, bias, out, workspace)
    assert k == w.cols
    out, ldy = _product_out(bias, w, m, x.dtype, x.device, out)
    if workspace is None:
        workspace = _workspace(linear_i8_workspace(m, n, k), x.device)
    _check(_lib.hbfp_linear_i8(_ptr(x), _TYPES[x.dtype], m, k, ldx, _ptr(w.codes), _ptr(w.scales), _ptr(bias), n, _ptr(out), ldy,
                               _ptr(workspace), 0 if workspace is None else workspace.numel(), _raw_stream(x.device)),
           "hbfp_linear_i8")
    return out


# ---------------------------------------------------------------------------- microscaled 4-bit floating point
# (the sizes of a new tensor are given one by one here, not as a tuple: 0.5 us less for each)
@dataclass
class Mx4:
    """An operand of products in microscaled 4-bit floating point: the descriptor plus the torch buffer that its two pointers lie in (one
    allocation instead of two is 1.6 us less for every conversion)."""
    desc: Mx4Desc
    buffer: torch.Tensor   # uint8: the codes, and the scales behind them

    @property
    def codes(self) -> torch.Tensor:
        """uint8 [groups, rows, 128]"""
        return self.buffer[:self.desc.code_bytes].view(self.desc.groups, self.desc.rows, 128)

    @property
    def scales(self) -> torch.Tensor:
        """uint8 [groups, rows rounded up to 16, 8]"""
        return self.buffer[self.desc.code_bytes:].view(self.desc.groups, self.desc.scale_rows, 8)


def mx4_plan(rows: int, kdim: int) -> Mx4Desc:
    d = Mx4Desc()
    _check(_lib.hbfp_mx4_plan(rows, kdim, ctypes.byref(d)), "hbfp_mx4_plan")
    return d


_mx4_sizes = functools.lru_cache(maxsize=1024)(mx4_plan)       # (nothing writes to what this returns; a copy of it is 1.3 us less than a new plan)


def mx4_alloc(rows: int, kdim: int, device="cuda") -> Mx4:
    """An operand of `rows` rows and a contraction of `kdim` (its contents are whatever the memory holds)."""
    d = Mx4Desc.from_buffer_copy(_mx4_sizes(rows, kdim))
    buffer = torch.empty(d.code_bytes + d.scale_bytes, dtype=torch.uint8, device=device)
    d.codes = buffer.data_ptr()
    d.scales = d.codes + d.code_bytes
    return Mx4(d, buffer)


def _quant_mx4(x, ld, along, down, rounding, seed):
    (rows, cols), device = x.shape, x.device
    a = mx4_alloc(rows, cols, device) if along else None
    d = mx4_alloc(cols, rows, device) if down else None
    _check(_lib.hbfp_quant_mx4(x.data_ptr(), _TYPES[x.dtype], rows, cols, ld, rounding, seed, ctypes.byref(a.desc) if a else None,
                               ctypes.byref(d.desc) if d else None, _raw_stream(device)), "hbfp_quant_mx4")
    return a, d


def quant_mx4(x: torch.Tensor, axis: int = 1, rounding: int = RNE, seed: int = 0, stream=None) -> Mx4:
    """hbfp_quant_mx4 of x [rows, cols] with the contraction along its rows (axis 1: weights [out features, in features], tokens) or down
    its columns (axis 0: the operand's rows are x's columns)."""
    ld = _matrix(x)
    assert axis in (0, 1)
    if stream is not None or _current_device() != x.device.index:
        return _there(stream, x.device, quant_mx4, x, axis, rounding, seed)
    return _quant_mx4(x, ld, axis == 1, axis == 0, rounding, seed)[1 - axis]


def quant_mx4_both(x: torch.Tensor, rounding: int = RNE, seed: int = 0, stream=None):
    """hbfp_quant_mx4 of x into both operands, (along its rows, down its columns), from one read: what a training step needs of a matrix."""
    ld = _matrix(x)
    if stream is not None or _current_device() != x.device.index:
        return _there(stream, x.device, quant_mx4_both, x, rounding, seed)
    return _quant_mx4(x, ld, True, True, rounding, seed)


def read_mx4(t: Mx4, dtype=torch.float32, stream=None) -> torch.Tensor:
    """hbfp_read_mx4: the values [rows, kdim] that an operand holds, in FP32 or bf16."""
    device = t.buffer.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, read_mx4, t, dtype)
    out = torch.empty(t.desc.rows, t.desc.kdim, dtype=dtype, device=device)
    _check(_lib.hbfp_read_mx4(ctypes.byref(t.desc), _TYPES[dtype], _ptr(out), t.desc.kdim, _raw_stream(device)), "hbfp_read_mx4")
    return out


@functools.lru_cache(maxsize=1024)
def gemm_mx4_workspace(rows: int, out_features: int, in_features: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_gemm_mx4_workspace(rows, out_features, in_features, ctypes.byref(n)), "hbfp_gemm_mx4_workspace")
    return int(n.value)


@functools.lru_cache(maxsize=1024)
def linear_mx4_workspace(rows: int, out_features: int, in_features: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_linear_mx4_workspace(rows, out_features, in_features, ctypes.byref(n)), "hbfp_linear_mx4_workspace")
    return int(n.value)


def _mx4_out(bias, w: Mx4, rows: int, dtype, device, out):
    n = w.desc.rows
    assert w.buffer.device == device
    if bias is not None:
        assert bias.device == device and bias.dtype == torch.float32 and bias.is_contiguous() and bias.numel() == n
    if out is None:
        return torch.empty(rows, n, dtype=dtype, device=device), n
    assert out.device == device and out.dtype == dtype and tuple(out.shape) == (rows, n)
    return out, _matrix(out)


def gemm_mx4(a: Mx4, b: Mx4, bias: Optional[torch.Tensor] = None, dtype=torch.float32, out: Optional[torch.Tensor] = None,
             workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """hbfp_gemm_mx4: y [rows of a, rows of b] = a . b^T (+ bias), rounded once to `dtype`."""
    m, n, device = a.desc.rows, b.desc.rows, a.buffer.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, gemm_mx4, a, b, bias, dtype, out, workspace)
    out, ld = _mx4_out(bias, b, m, dtype if out is None else out.dtype, device, out)
    if workspace is None:
        workspace = _workspace(gemm_mx4_workspace(m, n, a.desc.kdim), device)
    _check(_lib.hbfp_gemm_mx4(ctypes.byref(a.desc), ctypes.byref(b.desc), _ptr(bias), _ptr(out), _TYPES[out.dtype], ld, _ptr(workspace),
                              0 if workspace is None else workspace.numel(), _raw_stream(device)), "hbfp_gemm_mx4")
    return out


def linear_mx4(x: torch.Tensor, w: Mx4, bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """hbfp_linear_mx4: y = quant(x) . w^T (+ bias) in x's type, for x [tokens, in features] and weights from quant_mx4."""
    ldx, (m, k), n = _matrix(x), x.shape, w.desc.rows
    if stream is not None or _current_device() != x.device.index:
        return _there(stream, x.device, linear_mx4, x, w, bias, out, workspace)
    assert k == w.desc.kdim
    out, ldy = _mx4_out(bias, w, m, x.dtype, x.device, out)
    if workspace is None:
        workspace = _workspace(linear_mx4_workspace(m, n, k), x.device)
    _check(_lib.hbfp_linear_mx4(_ptr(x), _TYPES[x.dtype], m, ldx, ctypes.byref(w.desc), _ptr(bias), _ptr(out), ldy, _ptr(workspace),
                                0 if workspace is None else workspace.numel(), _raw_stream(x.device)), "hbfp_linear_mx4")
    return out


# ---------------------------------------------------------------------------- the norm in front of a quantised product
def _like(t: Optional[torch.Tensor], x: torch.Tensor) -> int:
    """The leading dimension of a matrix that goes with x; 0 for none."""
    if t is None:
        return 0
    assert t.device == x.device and t.dtype == x.dtype and t.shape == x.shape, "a matrix of x's shape and type on its GPU"
    return _matrix(t)


def _vector(t: Optional[torch.Tensor], n: int, device):
    if t is None:
        return None
    assert t.device == device and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == n, "a contiguous FP32 vector"
    return t.data_ptr()


def _norm(x, ldx, weight, eps, residual, total, values):
    """The arguments of a norm, and what it returns beside its codes."""
    (rows, cols), device = x.shape, x.device
    ld_sum, stored = cols, total
    if total is not None:
        ld_sum = _like(total, x)
    elif residual is not None:
        total = stored = torch.empty_like(x)            # (x's rows lie one behind the other there, whatever x is a part of)
    else:
        total = x
    held = torch.empty_like(x) if values else None
    rstd = torch.empty(rows, dtype=torch.float32, device=device)
    desc = NormDesc(x.data_ptr(), _ptr(residual), _vector(weight, cols, device), _ptr(stored), _ptr(held), rstd.data_ptr(), rows, cols, ldx,
                    _like(residual, x), ld_sum, cols, _TYPES[x.dtype], eps)
    return desc, total, rstd, held


def norm_i8(x: torch.Tensor, weight: Optional[torch.Tensor], eps: float = 1e-6, residual: Optional[torch.Tensor] = None,
            out_sum: Optional[torch.Tensor] = None, values: bool = False, stream=None):
    """hbfp_norm_i8 of x + residual: (rows for gemm_rows, the sum, 1 / rms of each row, the codes' values in x's type or None).  weight:
    FP32 [cols] or None.  out_sum: where the sum goes (x and residual are allowed); without a residual the sum is x itself."""
    ldx, device = _matrix(x), x.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, norm_i8, x, weight, eps, residual, out_sum, values)
    desc, total, rstd, held = _norm(x, ldx, weight, eps, residual, out_sum, values)
    rows, cols = x.shape
    codes = torch.empty(rows, (cols + 127) // 128 * 128, dtype=torch.int8, device=device)       # (the layout of hbfp_rows_plan)
    scales = torch.empty(rows, dtype=torch.float32, device=device)
    _check(_lib.hbfp_norm_i8(ctypes.byref(desc), codes.data_ptr(), scales.data_ptr(), _raw_stream(device)), "hbfp_norm_i8")
    return RowCodes(codes, scales, cols), total, rstd, held


def norm_mx4(x: torch.Tensor, weight: Optional[torch.Tensor], eps: float = 1e-6, residual: Optional[torch.Tensor] = None,
             out_sum: Optional[torch.Tensor] = None, values: bool = False, stream=None):
    """hbfp_norm_mx4: norm_i8 with an operand for gemm_mx4 in the place of the rows."""
    ldx, device = _matrix(x), x.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, norm_mx4, x, weight, eps, residual, out_sum, values)
    desc, total, rstd, held = _norm(x, ldx, weight, eps, residual, out_sum, values)
    out = mx4_alloc(x.shape[0], x.shape[1], device)
    _check(_lib.hbfp_norm_mx4(ctypes.byref(desc), ctypes.byref(out.desc), _raw_stream(device)), "hbfp_norm_mx4")
    return out, total, rstd, held


@functools.lru_cache(maxsize=1024)
def norm_grad_workspace(rows: int, cols: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.hbfp_norm_grad_workspace(rows, cols, ctypes.byref(n)), "hbfp_norm_grad_workspace")
    return int(n.value)


def norm_grad(g: torch.Tensor, total: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor], g_sum: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None, weight_grad: bool = True, workspace: Optional[torch.Tensor] = None, stream=None):
    """hbfp_norm_grad: (gradient of x and of the residual, gradient of the weight FP32 [cols] or None) from g, the gradient of the
    normalised rows, with the sum and rstd that the norm returned; g_sum: what reaches the sum by other ways.  out may be g or g_sum."""
    ldg, (rows, cols), device = _matrix(g), g.shape, g.device
    if stream is not None or _current_device() != device.index:
        return _there(stream, device, norm_grad, g, total, rstd, weight, g_sum, out, weight_grad, workspace)
    ldx = cols
    if out is None:
        out = torch.empty_like(g)
    else:
        ldx = _like(out, g)
    dweight = torch.empty(cols, dtype=torch.float32, device=device) if weight_grad else None
    if workspace is None and weight_grad:
        workspace = _workspace(norm_grad_workspace(rows, cols), device)
    _check(_lib.hbfp_norm_grad(_ptr(g), ldg, _ptr(total), _like(total, g), _vector(rstd, rows, device), _vector(weight, cols, device),
                               _ptr(g_sum), _like(g_sum, g), _TYPES[g.dtype], rows, cols, _ptr(out), ldx, _ptr(dweight),
                               _ptr(workspace), 0 if workspace is None else workspace.numel(), _raw_stream(device)), "hbfp_norm_grad")
    return out, dweight
