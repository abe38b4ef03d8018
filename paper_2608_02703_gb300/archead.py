"""Python binding of libarchead (ctypes).  Argument marshalling only: every
step of the forward runs in the library's CUDA kernels.  Functions carry the
C ABI's names (include/archead.h) and take torch tensors for device buffers;
torch is used for device memory and streams only.

The library must have been built (``paper_2608_02703_gb300.build.build()``);
loading fails loudly otherwise -- there is no fallback path.
"""

from __future__ import annotations

import ctypes
import os
from typing import Dict, List, Optional

import numpy as np

from .build import LIB

OK = 0
ERR_INVALID_ARG = 1
ERR_UNSUPPORTED = 2
ERR_OOM = 3
ERR_CUDA = 4
ERR_DEVICE_TIMEOUT = 5
ERR_TARGET_RANGE = 6

OUT_BF16 = 0
OUT_FP32 = 1

FORMAT_INT8 = 0
FORMAT_SC4 = 1

DTYPE_BF16 = 0
DTYPE_FP32 = 1
DTYPE_FP16 = 2

BEAM_MAX_OUT = 64
BEAM_MAX_BEAMS = 64

PATH_AUTO = 0
PATH_DECODE = 1
PATH_PREFILL = 2

COMPONENTS = {"residual": 0, "core_u": 1, "core_v": 2, "corr_a": 3, "corr_b": 4}

EXPORTED = (
    "archead_pack_create", "archead_destroy", "archead_forward", "archead_forward_path", "archead_forward_ce",
    "archead_forward_ce_path", "archead_forward_host", "archead_pack_bytes", "archead_device_bytes",
    "archead_debug_dequant", "archead_sync_status", "archead_set_wait_budget", "archead_debug_wait_timeout",
    "archead_profile_enable", "archead_profile_read", "archead_status_string", "archead_last_error",
    "archead_forward_decode_noalloc", "archead_forward_argmax", "archead_forward_argmax_path",
    "archead_forward_lse_partial", "archead_lse_combine", "archead_argmax_combine",
    "archead_quantize_symmetric", "archead_quantize_residual_sc4", "archead_pack_codes", "archead_dequant_symmetric",
    "archead_dequant_residual_sc4", "archead_pack_create_ex", "archead_abi_version",
    "archead_int8_weight_create", "archead_int8_weight_destroy", "archead_int8_device_bytes",
    "archead_int8_quantize_tokens", "archead_int8_matmul", "archead_int8_matmul_path", "archead_int8_linear",
    "archead_int8_sync_status", "archead_int8_set_wait_budget",
    "archead_beam_create", "archead_beam_destroy", "archead_beam_select", "archead_beam_reorder",
)


class ArcheadError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = f"{where}: {_status_string(status)}"
        detail = _last_error()
        if status in (ERR_CUDA, ERR_UNSUPPORTED) and detail:
            msg += f" ({detail})"
        super().__init__(msg)


class archead_desc(ctypes.Structure):  # noqa: N801 - mirrors the C struct name
    _fields_ = [
        ("vocab", ctypes.c_int64), ("hidden", ctypes.c_int64),
        ("core_rank", ctypes.c_int32), ("corr_rank", ctypes.c_int32),
        ("group_size", ctypes.c_int32), ("format", ctypes.c_int32),
        ("res_codes", ctypes.c_void_p), ("res_scales", ctypes.c_void_p),
        ("core_u", ctypes.c_void_p), ("core_u_scale", ctypes.c_void_p),
        ("core_v", ctypes.c_void_p), ("core_v_scale", ctypes.c_void_p),
        ("corr_a", ctypes.c_void_p), ("corr_a_scale", ctypes.c_void_p),
        ("corr_b", ctypes.c_void_p), ("corr_b_scale", ctypes.c_void_p),
        ("res_row_scale", ctypes.c_void_p),
    ]


class archead_kernel_stat(ctypes.Structure):  # noqa: N801
    _fields_ = [("name", ctypes.c_char_p), ("launches", ctypes.c_int64), ("total_ms", ctypes.c_double)]


class archead_beam_state_t(ctypes.Structure):  # noqa: N801 - the C struct archead_beam_state
    _fields_ = [
        ("data", ctypes.c_void_p), ("out", ctypes.c_void_p),
        ("outer", ctypes.c_int64), ("outer_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64),
        ("inner", ctypes.c_int64), ("inner_stride", ctypes.c_int64),
        ("bytes", ctypes.c_int64), ("bytes_per_position", ctypes.c_int64),
    ]


_lib: Optional[ctypes.CDLL] = None


def library_path() -> str:
    return LIB


def load() -> ctypes.CDLL:
    """Load libarchead.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB):
        raise RuntimeError(f"libarchead.so is not built ({LIB}); run paper_2608_02703_gb300.build.build()")
    lib = ctypes.CDLL(LIB)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    sig = {
        "archead_pack_create": (i32, [ctypes.POINTER(archead_desc), vp, ctypes.POINTER(vp)]),
        "archead_pack_create_ex": (i32, [ctypes.POINTER(archead_desc), ctypes.c_size_t, vp, ctypes.POINTER(vp)]),
        "archead_abi_version": (i32, []),
        "archead_destroy": (None, [vp]),
        "archead_forward": (i32, [vp, vp, i64, vp, i32, vp]),
        "archead_forward_path": (i32, [vp, vp, i64, vp, i32, i32, vp]),
        "archead_forward_ce": (i32, [vp, vp, i64, vp, vp, vp]),
        "archead_forward_ce_path": (i32, [vp, vp, i64, vp, vp, i32, vp]),
        "archead_forward_host": (i32, [vp, vp, i64, vp, i32, vp]),
        "archead_forward_decode_noalloc": (i32, [vp, vp, i64, vp, i32, vp]),
        "archead_forward_argmax": (i32, [vp, vp, i64, vp, vp, vp]),
        "archead_forward_argmax_path": (i32, [vp, vp, i64, vp, vp, i32, vp]),
        "archead_forward_lse_partial": (i32, [vp, vp, i64, vp, i64, vp, i32, vp]),
        "archead_lse_combine": (i32, [vp, i32, i64, vp, vp]),
        "archead_argmax_combine": (i32, [vp, vp, vp, i32, i64, vp, vp, vp]),
        "archead_quantize_symmetric": (i32, [vp, i64, i64, i64, i64, i32, vp, vp, vp]),
        "archead_quantize_residual_sc4": (i32, [vp, i64, i64, i32, vp, vp, vp, vp]),
        "archead_pack_codes": (i32, [vp, i64, i64, i32, vp, vp]),
        "archead_dequant_symmetric": (i32, [vp, vp, i64, i64, i64, i64, vp, vp]),
        "archead_dequant_residual_sc4": (i32, [vp, vp, vp, i64, i64, i32, vp, vp]),
        "archead_pack_bytes": (i64, [vp]),
        "archead_device_bytes": (i64, [vp]),
        "archead_debug_dequant": (i32, [vp, i32, i64, i64, vp, vp]),
        "archead_sync_status": (i32, [vp, vp]),
        "archead_set_wait_budget": (i32, [vp, i64]),
        "archead_debug_wait_timeout": (i32, [vp, vp]),
        "archead_int8_weight_create": (i32, [vp, vp, i64, i64, vp, ctypes.POINTER(vp)]),
        "archead_int8_weight_destroy": (None, [vp]),
        "archead_int8_device_bytes": (i64, [vp]),
        "archead_int8_quantize_tokens": (i32, [vp, i32, i64, i64, i64, vp, vp, vp]),
        "archead_int8_matmul": (i32, [vp, vp, vp, i64, vp, i32, i64, vp]),
        "archead_int8_matmul_path": (i32, [vp, vp, vp, i64, vp, i32, i64, i32, vp]),
        "archead_int8_linear": (i32, [vp, vp, i32, i64, i64, vp, i32, i64, vp]),
        "archead_int8_sync_status": (i32, [vp, vp]),
        "archead_int8_set_wait_budget": (i32, [vp, i64]),
        "archead_beam_create": (i32, [i64, i64, i32, ctypes.POINTER(vp)]),
        "archead_beam_destroy": (None, [vp]),
        "archead_beam_select": (i32, [vp, vp, i32, i64, i32, i64, i64, vp, vp, ctypes.c_int32, i32, vp, vp, vp, vp]),
        "archead_beam_reorder": (i32, [vp, i32, vp, i64, i32, i64, vp]),
        "archead_profile_enable": (i32, [vp, i32]),
        "archead_profile_read": (i32, [vp, ctypes.POINTER(archead_kernel_stat), i32]),
        "archead_status_string": (ctypes.c_char_p, [i32]),
        "archead_last_error": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _status_string(st: int) -> str:
    return load().archead_status_string(st).decode()


def _last_error() -> str:
    return load().archead_last_error().decode()


def _check(st: int, where: str) -> None:
    if st != OK:
        raise ArcheadError(st, where)


def _stream_ptr(stream) -> Optional[int]:
    import torch

    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


class Pack:
    """A packed head living on one CUDA device (wraps archead_pack*)."""

    def __init__(self, handle: int, shape):
        self.handle = handle
        self.shape = shape

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def close(self) -> None:
        if self.handle:
            load().archead_destroy(self.handle)
            self.handle = None


def archead_pack_create(head: Dict, shape, stream=None, desc_size=None) -> Pack:
    """Build a pack from canonical arrays (numpy host arrays or torch tensors).

    The INT8 format takes the arrays named as the struct fields; the paper's
    format (shape.fmt == "sc4") takes res_scale_codes, res_row_scale and
    core_u5 in place of res_scales and core_u.  With desc_size the call goes
    through archead_pack_create_ex with that struct size."""
    sc4 = getattr(shape, "fmt", "int8") == "sc4"
    d = archead_desc(vocab=shape.V, hidden=shape.d, core_rank=shape.core_rank, corr_rank=shape.corr_rank,
                     group_size=shape.group_size, format=FORMAT_SC4 if sc4 else FORMAT_INT8)
    source = {"res_scales": "res_scale_codes", "core_u": "core_u5"} if sc4 else {"res_row_scale": None}
    keep = []
    for name, _ in archead_desc._fields_[6:]:
        key = source.get(name, name)
        a = head.get(key) if key is not None else None
        if a is not None and hasattr(a, "flags") and not a.flags["C_CONTIGUOUS"]:
            a = np.ascontiguousarray(a)
        if a is not None and hasattr(a, "is_contiguous") and not a.is_contiguous():
            a = a.contiguous()
        keep.append(a)
        setattr(d, name, _ptr(a) if a is not None and getattr(a, "size", 1) != 0 else None)
    h = ctypes.c_void_p()
    if desc_size is None:
        _check(load().archead_pack_create(ctypes.byref(d), _stream_ptr(stream), ctypes.byref(h)), "archead_pack_create")
    else:
        _check(load().archead_pack_create_ex(ctypes.byref(d), desc_size, _stream_ptr(stream), ctypes.byref(h)),
               "archead_pack_create_ex")
    return Pack(h.value, shape)


def archead_abi_version() -> int:
    return int(load().archead_abi_version())


def archead_destroy(pack: Pack) -> None:
    pack.close()


def archead_forward(pack: Pack, x, M: int, logits, out_dtype: int = OUT_BF16, stream=None) -> None:
    _check(load().archead_forward(pack.handle, _ptr(x), M, _ptr(logits), out_dtype, _stream_ptr(stream)),
           "archead_forward")


def archead_forward_path(pack: Pack, x, M: int, logits, out_dtype: int, path: int, stream=None) -> None:
    _check(load().archead_forward_path(pack.handle, _ptr(x), M, _ptr(logits), out_dtype, path, _stream_ptr(stream)),
           "archead_forward_path")


def archead_forward_ce(pack: Pack, x, M: int, targets, ce, stream=None) -> None:
    _check(load().archead_forward_ce(pack.handle, _ptr(x), M, _ptr(targets), _ptr(ce), _stream_ptr(stream)),
           "archead_forward_ce")


def archead_forward_ce_path(pack: Pack, x, M: int, targets, ce, path: int, stream=None) -> None:
    _check(load().archead_forward_ce_path(pack.handle, _ptr(x), M, _ptr(targets), _ptr(ce), path,
                                          _stream_ptr(stream)), "archead_forward_ce_path")


def archead_forward_host(pack: Pack, x_host, M: int, logits_host, out_dtype: int = OUT_BF16, stream=None) -> None:
    _check(load().archead_forward_host(pack.handle, _ptr(x_host), M, _ptr(logits_host), out_dtype,
                                       _stream_ptr(stream)), "archead_forward_host")


def archead_forward_argmax(pack: Pack, x, M: int, index, value=None, stream=None) -> None:
    """Greedy next token per row of x: index (int32 [M]) and, optionally, its logit (fp32 [M])."""
    _check(load().archead_forward_argmax(pack.handle, _ptr(x), M, _ptr(index), _ptr(value), _stream_ptr(stream)),
           "archead_forward_argmax")


def archead_forward_argmax_path(pack: Pack, x, M: int, index, value, path: int, stream=None) -> None:
    _check(load().archead_forward_argmax_path(pack.handle, _ptr(x), M, _ptr(index), _ptr(value), path,
                                              _stream_ptr(stream)), "archead_forward_argmax_path")


def archead_forward_decode_noalloc(pack: Pack, x, M: int, logits, out_dtype: int = OUT_BF16, stream=None) -> None:
    """archead_forward for M <= 16 without any device allocation (fixed 512 KiB scratch array in the library)."""
    _check(load().archead_forward_decode_noalloc(pack.handle, _ptr(x), M, _ptr(logits), out_dtype,
                                                 _stream_ptr(stream)), "archead_forward_decode_noalloc")


def archead_forward_lse_partial(pack: Pack, x, M: int, targets, row0: int, parts, path: int = PATH_AUTO,
                                stream=None) -> None:
    """Per-token (max, sum of exp, target logit or -inf) over this shard's rows (fp32 [M][3])."""
    _check(load().archead_forward_lse_partial(pack.handle, _ptr(x), M, _ptr(targets), row0, _ptr(parts), path,
                                              _stream_ptr(stream)), "archead_forward_lse_partial")


def archead_lse_combine(parts, num_shards: int, M: int, ce, stream=None) -> None:
    """Cross entropy from the shards' partials (fp32 [num_shards][M][3], shard order)."""
    _check(load().archead_lse_combine(_ptr(parts), num_shards, M, _ptr(ce), _stream_ptr(stream)),
           "archead_lse_combine")


def archead_argmax_combine(values, indices, row0, num_shards: int, M: int, index, value=None, stream=None) -> None:
    """Greedy output from the shards' (value, local index) and their first global rows."""
    _check(load().archead_argmax_combine(_ptr(values), _ptr(indices), _ptr(row0), num_shards, M, _ptr(index),
                                         _ptr(value), _stream_ptr(stream)), "archead_argmax_combine")


def archead_quantize_symmetric(x, group_rows: int, group_cols: int, bits: int, codes, scales, stream=None) -> None:
    """Symmetric quantisation of the fp32 matrix x (rows x cols), one fp16 scale per group block."""
    rows, cols = x.shape
    _check(load().archead_quantize_symmetric(_ptr(x), rows, cols, group_rows, group_cols, bits, _ptr(codes),
                                             _ptr(scales), _stream_ptr(stream)), "archead_quantize_symmetric")


def archead_quantize_residual_sc4(r, group_size: int, codes, scale_codes, row_scale, stream=None) -> None:
    rows, cols = r.shape
    _check(load().archead_quantize_residual_sc4(_ptr(r), rows, cols, group_size, _ptr(codes), _ptr(scale_codes),
                                                _ptr(row_scale), _stream_ptr(stream)), "archead_quantize_residual_sc4")


def archead_pack_codes(codes, bits: int, packed, stream=None) -> None:
    rows, cols = codes.shape
    _check(load().archead_pack_codes(_ptr(codes), rows, cols, bits, _ptr(packed), _stream_ptr(stream)),
           "archead_pack_codes")


def archead_dequant_symmetric(codes, scales, group_rows: int, group_cols: int, out, stream=None) -> None:
    rows, cols = codes.shape
    _check(load().archead_dequant_symmetric(_ptr(codes), _ptr(scales), rows, cols, group_rows, group_cols, _ptr(out),
                                            _stream_ptr(stream)), "archead_dequant_symmetric")


def archead_dequant_residual_sc4(codes, scale_codes, row_scale, group_size: int, out, stream=None) -> None:
    rows, cols = codes.shape
    _check(load().archead_dequant_residual_sc4(_ptr(codes), _ptr(scale_codes), _ptr(row_scale), rows, cols,
                                               group_size, _ptr(out), _stream_ptr(stream)),
           "archead_dequant_residual_sc4")


_DTYPES: Dict = {}  # torch's types, filled with the first use
_raw_stream = None


def _dtype(t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        import torch

        _DTYPES.update({torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_FP32, torch.float16: DTYPE_FP16})
        code = _DTYPES.get(t.dtype)
        if code is None:
            raise ValueError(f"bf16, fp16 or fp32 is wanted, not {t.dtype}")
    return code


def _stream_at(stream, t) -> int:
    """The stream given, or the current one of the tensor's device (looked up without a Stream object, which takes
    longer than a launch)."""
    global _raw_stream
    if stream is not None:
        return _stream_ptr(stream)
    if _raw_stream is None:
        import torch

        _raw_stream = torch._C._cuda_getCurrentRawStream
    return _raw_stream(t.get_device())


def _rows(t, rows: int, cols: int, what: str) -> int:
    """Distance of the rows of a matrix of at least `rows` rows whose `cols` columns lie side by side."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[0] < rows or shape[1] != cols or (stride[1] != 1 and cols > 1):
        raise ValueError(f"{what}: {rows} rows of {cols} adjacent elements are wanted, "
                         f"not {tuple(shape)} with strides {stride}")
    if not t.is_cuda:
        raise ValueError(f"{what} is not on the GPU")
    return stride[0] if shape[0] > 1 else cols


def _flat(t, dtype, size: int, what: str, cols: Optional[int] = None):
    """Address of a contiguous tensor of at least `size` elements of the type.  A matrix that is larger has rows of
    `cols` elements: of others the wrong elements would be read or written."""
    held = t.numel()
    wider = held > size and cols is not None and t.dim() == 2 and t.shape[1] not in (1, cols)
    if t.dtype is not dtype or held < size or wider or not t.is_contiguous():
        raise ValueError(f"{what}: {size} contiguous elements of {dtype} are wanted, not {tuple(t.shape)} of {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what} is not on the GPU")
    return t.data_ptr()


class Int8Weight:
    """A weight matrix in 8-bit codes on one CUDA device (wraps archead_int8_weight*)."""

    def __init__(self, handle: int, N: int, K: int):
        self.handle = handle
        self.N = N
        self.K = K

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def close(self) -> None:
        if self.handle:
            load().archead_int8_weight_destroy(self.handle)
            self.handle = None


def archead_int8_weight_create(codes, scales, stream=None) -> Int8Weight:
    """codes int8 [N, K] and scales fp32 [N]: numpy arrays or torch tensors, on the host or the device.

    Numpy codes of another type are taken where int8 holds them all."""
    N, K = codes.shape
    if isinstance(codes, np.ndarray):
        if codes.dtype != np.int8:
            with np.errstate(invalid="ignore"):
                same = codes.astype(np.int8)
            if not np.array_equal(same, codes):
                raise ValueError(f"codes of {codes.dtype} that int8 does not hold")
            codes = same
        codes = np.ascontiguousarray(codes)
        scales = np.ascontiguousarray(scales, dtype=np.float32)
        n_scales = scales.size
    else:
        import torch

        if codes.dtype != torch.int8 or scales.dtype != torch.float32:
            raise ValueError(f"codes in int8 and scales in fp32 are wanted, not {codes.dtype} and {scales.dtype}")
        if not (codes.is_contiguous() and scales.is_contiguous()):
            # Copied in the stream that the call reads in, behind what fills them there.
            if stream is not None and (codes.is_cuda or scales.is_cuda):
                given = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream))
            else:
                given = None
            with torch.cuda.stream(given):
                codes, scales = codes.contiguous(), scales.contiguous()
        n_scales = scales.numel()
    if n_scales != N:
        raise ValueError(f"a scale for each of the {N} channels is wanted, not {n_scales}")
    h = ctypes.c_void_p()
    _check(load().archead_int8_weight_create(_ptr(codes), _ptr(scales), N, K, _stream_ptr(stream), ctypes.byref(h)),
           "archead_int8_weight_create")
    return Int8Weight(h.value, N, K)


def archead_int8_weight_destroy(weight: Int8Weight) -> None:
    weight.close()


def archead_int8_device_bytes(weight: Int8Weight) -> int:
    return int(load().archead_int8_device_bytes(weight.handle))


def archead_int8_quantize_tokens(x, codes, scales, stream=None) -> None:
    """codes int8 [M, K] and scales fp32 [M] of the rows of x (bf16, fp16 or fp32 [M, K], rows any distance apart)."""
    import torch

    M, K = x.shape
    ldx = _rows(x, M, K, "x")
    _check(load().archead_int8_quantize_tokens(x.data_ptr(), _dtype(x), M, K, ldx, _flat(codes, torch.int8, M * K, "codes", K),
                                               _flat(scales, torch.float32, M, "scales"), _stream_at(stream, x)),
           "archead_int8_quantize_tokens")


def archead_int8_matmul(weight: Int8Weight, x_codes, x_scales, M: int, y, stream=None) -> None:
    """y [M, N] (bf16, fp16 or fp32, rows any distance apart) of int8 codes [M, K] and fp32 scales [M]."""
    archead_int8_matmul_path(weight, x_codes, x_scales, M, y, PATH_AUTO, stream)


def archead_int8_matmul_path(weight: Int8Weight, x_codes, x_scales, M: int, y, path: int, stream=None) -> None:
    import torch

    ldy = _rows(y, M, weight.N, "y")
    _check(load().archead_int8_matmul_path(weight.handle, _flat(x_codes, torch.int8, M * weight.K, "x_codes", weight.K),
                                           _flat(x_scales, torch.float32, M, "x_scales"), M, y.data_ptr(), _dtype(y),
                                           ldy, path, _stream_at(stream, y)), "archead_int8_matmul")


def archead_int8_linear(weight: Int8Weight, x, M: int, y, stream=None) -> None:
    """y [M, N] of activations x [M, K], which the call quantises (each bf16, fp16 or fp32, rows any distance apart)."""
    ldx, ldy = _rows(x, M, weight.K, "x"), _rows(y, M, weight.N, "y")
    _check(load().archead_int8_linear(weight.handle, x.data_ptr(), _dtype(x), M, ldx, y.data_ptr(), _dtype(y), ldy,
                                      _stream_at(stream, y)), "archead_int8_linear")


def archead_int8_sync_status(weight: Int8Weight, stream=None) -> int:
    return int(load().archead_int8_sync_status(weight.handle, _stream_ptr(stream)))


def archead_int8_set_wait_budget(weight: Int8Weight, cycles: int) -> None:
    _check(load().archead_int8_set_wait_budget(weight.handle, cycles), "archead_int8_set_wait_budget")


class Beam:
    """Scratch of beam selections on one CUDA device (wraps archead_beam*)."""

    def __init__(self, handle: int):
        self.handle = handle

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def close(self) -> None:
        if self.handle:
            load().archead_beam_destroy(self.handle)
            self.handle = None


def archead_beam_create(max_rows: int, max_vocab: int, max_out: int) -> Beam:
    h = ctypes.c_void_p()
    _check(load().archead_beam_create(max_rows, max_vocab, max_out, ctypes.byref(h)), "archead_beam_create")
    return Beam(h.value)


def archead_beam_destroy(beam: Beam) -> None:
    beam.close()


def archead_beam_select(beam: Beam, logits, scores, out_scores, out_parents, out_tokens, ended=None,
                        end_token: int = 0, stream=None) -> None:
    """The n best (beam, token) candidates of each batch entry.

    logits [batch * beams, vocab] (bf16, fp16 or fp32, rows any distance apart), scores fp32 [batch, beams], ended
    uint8 or bool [batch, beams] or None; out_scores fp32, out_parents and out_tokens int32, all [batch, n]."""
    import torch

    batch, beams = scores.shape
    n = out_scores.shape[1]
    vocab = logits.shape[1]
    ld = _rows(logits, batch * beams, vocab, "logits")
    if ended is not None and ended.dtype == torch.bool:
        ended = ended.view(torch.uint8)
    _check(load().archead_beam_select(
        beam.handle, logits.data_ptr(), _dtype(logits), batch, beams, vocab, ld,
        _flat(scores, torch.float32, batch * beams, "scores"),
        None if ended is None else _flat(ended, torch.uint8, batch * beams, "ended", beams), end_token, n,
        _flat(out_scores, torch.float32, batch * n, "out_scores"),
        _flat(out_parents, torch.int32, batch * n, "out_parents", n),
        _flat(out_tokens, torch.int32, batch * n, "out_tokens", n), _stream_at(stream, logits)), "archead_beam_select")


def _merged(shape, strides, what: str):
    """Dimensions as one: their extent and stride."""
    dims = [(n, s) for n, s in zip(shape, strides) if n != 1]
    if any(n == 0 for n, _ in dims):
        return 0, 0
    for (_, s0), (n1, s1) in zip(dims, dims[1:]):
        if s0 != n1 * s1:
            raise ValueError(f"{what} of the state do not lie at one distance")
    extent = 1
    for n, _ in dims:
        extent *= n
    return extent, dims[-1][1] if dims else 0


class BeamState:
    """One state as archead_beam_reorder takes it: its description, its rows and the positions it has room for."""

    def __init__(self, desc, rows, room, tensors):
        self.desc = desc
        self.rows = rows
        self.room = room  # None: no positions
        self.tensors = tensors


def archead_beam_state(t, row_dim: int = 0, length_dim: Optional[int] = None, out=None) -> BeamState:
    """Describes a state [layers..., rows, heads..., positions, elements...]: rows = batch * beams in dimension
    row_dim, positions (of which a reordering moves the first `length`) in dimension length_dim, or none.  out: a
    tensor of the same shape and strides that takes the result; None: in place."""
    if out is not None and (out.shape != t.shape or out.stride() != t.stride() or out.dtype != t.dtype):
        raise ValueError("out is not laid out as the state")
    shape, strides, size = list(t.shape), list(t.stride()), t.element_size()
    for dim, what in ((row_dim, "rows"), (length_dim, "positions")):
        if dim is not None and not -t.dim() <= dim < t.dim():
            raise ValueError(f"a state of {t.dim()} dimensions has no dimension {dim} for its {what}")
    row_dim %= t.dim()
    if length_dim is None:
        # The dimensions that lie side by side at the end are one chunk.
        tail, run = t.dim(), 1
        while tail - 1 > row_dim and (shape[tail - 1] == 1 or strides[tail - 1] == run):
            tail -= 1
            run *= shape[tail]
        room, fixed, step = None, run * size, 0
    else:
        tail = length_dim % t.dim()
        if tail <= row_dim:
            raise ValueError("the positions' dimension comes after the rows'")
        run = 1
        for n, s in zip(reversed(shape[tail + 1:]), reversed(strides[tail + 1:])):
            if n != 1 and s != run:
                raise ValueError("a position's elements do not lie side by side")
            run *= n
        room, fixed, step = shape[tail], 0, run * size
        if room > 1 and strides[tail] != run:
            raise ValueError("the positions do not lie side by side")
    outer, outer_stride = _merged(shape[:row_dim], strides[:row_dim], "the dimensions before the rows")
    inner, inner_stride = _merged(shape[row_dim + 1:tail], strides[row_dim + 1:tail], "the dimensions after the rows")
    desc = archead_beam_state_t(
        data=t.data_ptr(), out=None if out is None else out.data_ptr(), outer=outer, outer_stride=outer_stride * size,
        row_stride=strides[row_dim] * size, inner=inner, inner_stride=inner_stride * size, bytes=fixed,
        bytes_per_position=step)
    return BeamState(desc, shape[row_dim], room, (t, out))


class BeamStates:
    """The states of a decoder, described once: what archead_beam_reorder takes."""

    def __init__(self, states: List[BeamState]):
        self.array = (archead_beam_state_t * max(len(states), 1))(*[s.desc for s in states])
        self.count = len(states)
        self.rows = min((s.rows for s in states), default=0)
        self.room = min((s.room for s in states if s.room is not None), default=None)
        self.tensors = [s.tensors for s in states]  # (their memory is kept)
        self.on_gpu = all(t.is_cuda for pair in self.tensors for t in pair if t is not None)


def archead_beam_states(states: List[BeamState]) -> BeamStates:
    return BeamStates(list(states))


def archead_beam_reorder(states: BeamStates, parents, length: int = 0, stream=None) -> None:
    """Row b * beams + k of every state takes what row b * beams + parents[b, k] held (parents int32 [batch, beams]),
    for the first `length` positions of states that have positions."""
    import torch

    batch, beams = parents.shape
    if states.count and (batch * beams > states.rows or (states.room is not None and length > states.room)):
        raise ValueError(f"{batch * beams} rows of {length} positions in states of {states.rows} rows and "
                         f"{states.room} positions")
    if not states.on_gpu:
        raise ValueError("a state is not on the GPU")
    _check(load().archead_beam_reorder(states.array, states.count, _flat(parents, torch.int32, batch * beams, "parents"),
                                       batch, beams, length, _stream_at(stream, parents)), "archead_beam_reorder")


def archead_pack_bytes(pack: Pack) -> int:
    return int(load().archead_pack_bytes(pack.handle))


def archead_device_bytes(pack: Pack) -> int:
    return int(load().archead_device_bytes(pack.handle))


def archead_debug_dequant(pack: Pack, component, row0: int, nrows: int, out, stream=None) -> None:
    c = COMPONENTS[component] if isinstance(component, str) else int(component)
    _check(load().archead_debug_dequant(pack.handle, c, row0, nrows, _ptr(out), _stream_ptr(stream)),
           "archead_debug_dequant")


def archead_sync_status(pack: Pack, stream=None) -> int:
    return int(load().archead_sync_status(pack.handle, _stream_ptr(stream)))


def archead_set_wait_budget(pack: Pack, cycles: int) -> None:
    _check(load().archead_set_wait_budget(pack.handle, cycles), "archead_set_wait_budget")


def archead_debug_wait_timeout(pack: Pack, stream=None) -> None:
    _check(load().archead_debug_wait_timeout(pack.handle, _stream_ptr(stream)), "archead_debug_wait_timeout")


def archead_profile_enable(pack: Pack, enable: bool = True) -> None:
    _check(load().archead_profile_enable(pack.handle, 1 if enable else 0), "archead_profile_enable")


def archead_profile_read(pack: Pack) -> List[dict]:
    buf = (archead_kernel_stat * 32)()
    n = load().archead_profile_read(pack.handle, buf, 32)
    return [{"name": buf[i].name.decode(), "launches": int(buf[i].launches), "total_ms": float(buf[i].total_ms)}
            for i in range(max(n, 0))]


def archead_status_string(status: int) -> str:
    return _status_string(status)


def archead_last_error() -> str:
    return _last_error()
