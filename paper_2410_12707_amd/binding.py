"""Python names for the C ABI of ``libadatopk.so`` (see ``include/adatopk.h``).

Argument marshalling only: every step of compress / decompress runs in the HIP kernels of
the library.  torch supplies device memory and the current stream.  There is no fallback:
if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import warnings
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# ADATOPK_LIBRARY selects another build of the same C ABI (for instance one compiled with
# different launch-shape constants); the default is the in-tree library.
LIB_PATH = os.environ.get("ADATOPK_LIBRARY") or os.path.join(_HERE, "libadatopk.so")

F32, BF16, F16 = 0, 1, 2
OK, EINVAL, EWORKSPACE, ERUNTIME, ENOTIMPL = 0, 1, 2, 3, 4
_STATUS = {OK: "ADATOPK_OK", EINVAL: "ADATOPK_EINVAL", EWORKSPACE: "ADATOPK_EWORKSPACE",
           ERUNTIME: "ADATOPK_ERUNTIME", ENOTIMPL: "ADATOPK_ENOTIMPL"}

MEASURE_LIB_PATH = os.environ.get("ADATOPK_MEASURE_LIBRARY") or os.path.join(_HERE, "libadatopk_measure.so")

_lib = None          # the product library
_measure_lib = None  # the same sources built with the benchmark's timing hooks (adatopk_measure.h)
_active = None       # what load_library() returns when set: the measuring build inside `with measuring()`


class AdaTopKError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__("%s returned %s" % (where, _STATUS.get(status, status)))
        self.status = status


def load_library() -> ctypes.CDLL:
    global _lib
    if _active is not None:
        return _active
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libadatopk.so is not built: run `python -m paper_2410_12707_amd.build` "
                          "(or __graft_entry__.build()) first; there is no CPU fallback")
    _lib = _declare(ctypes.CDLL(LIB_PATH))
    return _lib


def load_measure_library() -> ctypes.CDLL:
    """The measuring build: the whole C ABI plus the hooks of adatopk_measure.h (benchmarks only)."""
    global _measure_lib
    if _measure_lib is not None:
        return _measure_lib
    if not os.path.exists(MEASURE_LIB_PATH):
        raise ImportError("libadatopk_measure.so is not built: run `python -m paper_2410_12707_amd.build`")
    lib = _declare(ctypes.CDLL(MEASURE_LIB_PATH))
    i32, p, sz = ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
    lib.adatopk_measure_enable.argtypes = [i32]
    lib.adatopk_measure_enable.restype = i32
    lib.adatopk_measure_stage_count.restype = i32
    lib.adatopk_measure_stage_name.argtypes = [i32]
    lib.adatopk_measure_stage_name.restype = ctypes.c_char_p
    lib.adatopk_measure_read.argtypes = [p]
    lib.adatopk_measure_read.restype = i32
    lib.adatopk_measure_judge.argtypes = [i32, i32]
    lib.adatopk_measure_judge.restype = None
    lib.adatopk_measure_workspace_offset.argtypes = [i32, ctypes.c_int64, i32, i32]
    lib.adatopk_measure_workspace_offset.restype = sz
    lib.adatopk_measure_weight_grad_cut.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, i32, ctypes.c_int64, p]
    lib.adatopk_measure_weight_grad_cut.restype = i32
    lib.adatopk_measure_layernorm_cut.argtypes = [ctypes.c_int64, ctypes.c_int64, i32, p]
    lib.adatopk_measure_layernorm_cut.restype = i32
    lib.adatopk_measure_fp8_product_cut.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, i32, p]
    lib.adatopk_measure_fp8_product_cut.restype = i32
    lib.adatopk_measure_muon_update_cut.argtypes = [ctypes.c_int64, ctypes.c_int64, p]
    lib.adatopk_measure_muon_update_cut.restype = i32
    lib.adatopk_measure_muon_update_next_cut.argtypes = [ctypes.c_int64, ctypes.c_int64, p]
    lib.adatopk_measure_muon_update_next_cut.restype = i32
    lib.adatopk_measure_copy.argtypes = [p, p, sz, p]
    lib.adatopk_measure_copy.restype = i32
    lib.adatopk_measure_read_only.argtypes = [p, sz, p, p]
    lib.adatopk_measure_read_only.restype = i32
    lib.adatopk_measure_fill.argtypes = [p, sz, p]
    lib.adatopk_measure_fill.restype = i32
    _measure_lib = lib
    return lib


class measuring:
    """``with measuring():`` routes every call of this module through the measuring build and times each
    kernel launch with events of its own; ``measure_read()`` inside the block returns the durations."""

    def __enter__(self):
        global _active
        lib = load_measure_library()
        _check(lib.adatopk_measure_enable(1), "adatopk_measure_enable")
        _active = lib
        return self

    def __exit__(self, *exc):
        global _active
        _active = None
        _check(load_measure_library().adatopk_measure_enable(0), "adatopk_measure_enable")
        return False


def _declare(lib: ctypes.CDLL) -> ctypes.CDLL:
    i64, i32, p, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
    lib.adatopk_workspace_bytes.argtypes = [i64, i32, i32]
    lib.adatopk_workspace_bytes.restype = sz
    lib.adatopk_compress.argtypes = [p, i64, i32, i64, p, p, p, p, sz, p]
    lib.adatopk_compress.restype = i32
    lib.adatopk_decompress.argtypes = [p, p, i64, i32, p, i64, p]
    lib.adatopk_decompress.restype = i32
    lib.adatopk_decompress_sorted.argtypes = [p, p, i64, i32, p, i64, p]
    lib.adatopk_decompress_sorted.restype = i32
    lib.adatopk_decompress_accumulate.argtypes = [p, p, i64, i32, p, i64, p]
    lib.adatopk_decompress_accumulate.restype = i32
    lib.adatopk_decompress_segmented.argtypes = [p, p, p, i32, i32, p, p, p]
    lib.adatopk_decompress_segmented.restype = i32
    lib.adatopk_wire_bytes.argtypes = [i64, i32, i32]
    lib.adatopk_wire_bytes.restype = sz
    lib.adatopk_wire_keep_count.argtypes = [sz, i32, i32]
    lib.adatopk_wire_keep_count.restype = i64
    lib.adatopk_wire_parse_header.argtypes = [p, sz, p]
    lib.adatopk_wire_parse_header.restype = i32
    lib.adatopk_compress_wire.argtypes = [p, i64, i32, i64, i32, ctypes.c_double, p, sz, p, sz, p]
    lib.adatopk_compress_wire.restype = i32
    lib.adatopk_compress_wire_segmented.argtypes = [p, p, p, i32, i32, i32, p, p, p, sz, p, sz, p]
    lib.adatopk_compress_wire_segmented.restype = i32
    lib.adatopk_decompress_wire.argtypes = [p, sz, i32, i32, i64, i32, p, p]
    lib.adatopk_decompress_wire.restype = i32
    lib.adatopk_compress_segmented.argtypes = [p, p, p, i32, i32, p, p, p, p, p, sz, p]
    lib.adatopk_compress_segmented.restype = i32
    lib.adatopk_adaptive_ratios.argtypes = [p, i32, ctypes.c_double, ctypes.c_double, p]
    lib.adatopk_adaptive_ratios.restype = i32
    lib.adatopk_k_for_ratio.argtypes = [i64, ctypes.c_double]
    lib.adatopk_k_for_ratio.restype = i64
    dbl = ctypes.c_double
    lib.adatopk_link_time.argtypes = [dbl, dbl, dbl]
    lib.adatopk_link_time.restype = dbl
    lib.adatopk_pipeline_time.argtypes = [p, p, i32, i32]
    lib.adatopk_pipeline_time.restype = dbl
    lib.adatopk_pipeline_time_compressed.argtypes = [p, p, i32, i32, dbl, dbl, i32]
    lib.adatopk_pipeline_time_compressed.restype = dbl
    lib.adatopk_plan_keep_counts.argtypes = [p, p, p, i32, i32, dbl, dbl, p, p]
    lib.adatopk_plan_keep_counts.restype = i32
    lib.adatopk_compress_noalloc.argtypes = [p, i64, i32, i64, p, p, p, p]
    lib.adatopk_compress_noalloc.restype = i32
    f32 = ctypes.c_float
    lib.adatopk_act8_bytes.argtypes = [i64, i64]
    lib.adatopk_act8_bytes.restype = sz
    lib.adatopk_act8_store.argtypes = [p, i64, i64, i64, i32, p, p]
    lib.adatopk_act8_store.restype = i32
    lib.adatopk_act8_load.argtypes = [p, i64, i64, i32, p, i64, p]
    lib.adatopk_act8_load.restype = i32
    lib.adatopk_gelu_forward.argtypes = [p, i64, i64, i64, i32, i32, p, i64, p, p, p]
    lib.adatopk_gelu_forward.restype = i32
    lib.adatopk_gelu_backward.argtypes = [p, i64, p, i64, i64, i32, i32, p, i64, p]
    lib.adatopk_gelu_backward.restype = i32
    lib.adatopk_layernorm_forward.argtypes = [p, i64, p, i64, p, p, i32, i64, i64, i32, f32, p, i64, p, i64, p, p, p, p]
    lib.adatopk_layernorm_forward.restype = i32
    lib.adatopk_layernorm_backward_workspace_bytes.argtypes = [i64, i64]
    lib.adatopk_layernorm_backward_workspace_bytes.restype = sz
    lib.adatopk_layernorm_backward.argtypes = [p, i64, p, i64, p, p, p, p, i32, p, i64, i64, i64, i32, p, i64, p, p, i32, p, sz, p]
    lib.adatopk_layernorm_backward.restype = i32
    lib.adatopk_weight_grad_workspace_bytes.argtypes = [i64, i64, i64, i32]
    lib.adatopk_weight_grad_workspace_bytes.restype = sz
    lib.adatopk_weight_grad.argtypes = [p, i64, p, i64, i64, i64, i32, p, p, i32, p, p, i32, p, sz, p]
    lib.adatopk_weight_grad.restype = i32
    lib.adatopk_fp8_bytes.argtypes = [i64, i64]
    lib.adatopk_fp8_bytes.restype = sz
    lib.adatopk_fp8_store.argtypes = [p, i64, i64, i64, i32, p, p]
    lib.adatopk_fp8_store.restype = i32
    lib.adatopk_fp8_load.argtypes = [p, i64, i64, i32, p, i64, p]
    lib.adatopk_fp8_load.restype = i32
    lib.adatopk_fp8_store_weight.argtypes = [p, i64, i64, i64, i32, p, p, p]
    lib.adatopk_fp8_store_weight.restype = i32
    lib.adatopk_fp8_product_workspace_bytes.argtypes = [i64, i64, i64]
    lib.adatopk_fp8_product_workspace_bytes.restype = sz
    lib.adatopk_fp8_product.argtypes = [p, p, i64, i64, i64, p, i32, p, i64, p, i64, i32, p, sz, p]
    lib.adatopk_fp8_product.restype = i32
    lib.adatopk_rmsnorm_forward.argtypes = [p, i64, p, i64, p, i32, i64, i64, i32, f32, p, i64, p, i64, p, p, p, p]
    lib.adatopk_rmsnorm_forward.restype = i32
    lib.adatopk_rmsnorm_backward_workspace_bytes.argtypes = [i64, i64]
    lib.adatopk_rmsnorm_backward_workspace_bytes.restype = sz
    lib.adatopk_rmsnorm_backward.argtypes = [p, i64, p, i64, p, p, p, i32, p, i64, i64, i64, i32, p, i64, p, i32, p, sz, p]
    lib.adatopk_rmsnorm_backward.restype = i32
    lib.adatopk_muon_update_workspace_bytes.argtypes = [i64, i64]
    lib.adatopk_muon_update_workspace_bytes.restype = sz
    lib.adatopk_muon_update.argtypes = [p, i64, i32, p, f32, i32, i64, i64, i32, f32, p, i64, i32, f32, f32, p, sz, p]
    lib.adatopk_muon_update.restype = i32
    lib.adatopk_muon_update_coarse.argtypes = lib.adatopk_muon_update.argtypes
    lib.adatopk_muon_update_coarse.restype = i32
    lib.address = _Addresses(lib)
    return lib


class _Addresses:
    """Where the functions are that the _marshal extension calls for itself."""

    def __init__(self, lib: ctypes.CDLL):
        for name in ("compress", "decompress", "decompress_sorted", "decompress_accumulate", "decompress_segmented", "compress_wire",
                     "compress_wire_segmented", "decompress_wire", "compress_segmented", "act8_store", "act8_load", "gelu_forward", "gelu_backward",
                     "layernorm_forward", "layernorm_backward", "weight_grad", "fp8_store", "fp8_load", "fp8_store_weight", "fp8_product", "rmsnorm_forward",
                     "rmsnorm_backward", "muon_update", "muon_update_coarse"):
            setattr(self, name, ctypes.cast(getattr(lib, "adatopk_" + name), ctypes.c_void_p).value)


def _check(status: int, where: str) -> None:
    if status != OK:
        raise AdaTopKError(status, where)


def _dtype_code(t: torch.dtype) -> int:
    if t == torch.float32:
        return F32
    if t == torch.bfloat16:
        return BF16
    if t == torch.float16:
        return F16
    raise TypeError("adatopk supports float32, bfloat16 and float16 tensors, got %s" % t)


# The handle alone: a Stream object around it costs a microsecond and a half per call.  (Not a public name of torch.)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dev(t: torch.Tensor) -> int:
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError("adatopk needs contiguous device tensors")
    return t.data_ptr()


def _dev_or_pinned(t: torch.Tensor) -> int:
    """Device tensor, or pinned host memory (which the device addresses directly: the kernels then write over the bus)."""
    if t.is_contiguous() and (t.is_cuda or t.is_pinned()):
        return t.data_ptr()
    raise ValueError("adatopk needs a contiguous device tensor or pinned host tensor here")


def _check_outputs(dtype: torch.dtype, k_total: int, idx_out: torch.Tensor, val_out: torch.Tensor,
                   err_norm_out: Optional[torch.Tensor], num_tensors: int) -> None:
    """Output buffers of a compress call: the library gets raw pointers and cannot see their sizes or
    types, so a buffer that is too small or of another type is refused here."""
    if idx_out.dtype != torch.int32 or idx_out.numel() < k_total:
        raise ValueError("idx_out must be int32 with at least %d entries" % k_total)
    if val_out.dtype != dtype or val_out.numel() < k_total:
        raise ValueError("val_out must have the dense tensor's dtype (%s) and at least %d entries" % (dtype, k_total))
    if err_norm_out is not None and (err_norm_out.dtype != torch.float32 or err_norm_out.numel() < num_tensors):
        raise ValueError("err_norm_out must be float32 with one entry per tensor (%d)" % num_tensors)


def _check_pairs(dtype: torch.dtype, k_total: int, idx: torch.Tensor, val: torch.Tensor) -> None:
    if idx.dtype != torch.int32 or idx.numel() < k_total:
        raise ValueError("idx must be int32 with at least %d entries" % k_total)
    if val.dtype != dtype or val.numel() < k_total:
        raise ValueError("val must have the dense tensor's dtype (%s) and at least %d entries" % (dtype, k_total))


_marshal = None  # the extension that reads the arguments and makes the calls; False: there is none
_MARSHAL_NAMES = ("tensors", "int64s", "streams", "compress", "decompress", "compress_wire", "decompress_wire", "compress_segmented",
                  "decompress_segmented", "compress_wire_segmented", "act8_store", "act8_load", "gelu_forward", "gelu_backward", "layernorm_forward",
                  "layernorm_backward", "weight_grad", "fp8_store", "fp8_load", "fp8_store_weight", "fp8_product", "rmsnorm_forward", "rmsnorm_backward",
                  "muon_update")


def _load_marshal():
    """The extension, or None where it is not built (for this Python, or from an older source): Python then reads the arguments itself, with the
    same result, microseconds per call and half a microsecond per tensor slower."""
    global _marshal
    if _marshal is None:
        try:
            from . import _marshal as m
            missing = [name for name in _MARSHAL_NAMES if not hasattr(m, name)]
            if missing:
                raise ImportError("built from an older source, without %s" % ", ".join(missing))
            if _raw_stream is not None:
                m.streams(torch.cuda.current_device, _raw_stream)
        except ImportError as e:
            warnings.warn("calls go without the _marshal extension (%s): run `python -m paper_2410_12707_amd.build`" % e,
                          RuntimeWarning, stacklevel=3)
            m = False
        _marshal = m
    return _marshal or None


def _done(status: Optional[int], where: str) -> bool:
    """Whether the extension has made the call (None: its arguments are left to Python)."""
    if status is None:
        return False
    if status != OK:
        raise AdaTopKError(status, where)
    return True


def _segments(tensors: Sequence[torch.Tensor]):
    """(addresses, lengths, dtype) of the tensors of a segmented call, or None if they want a closer look in Python."""
    m = _load_marshal()
    return m.tensors(tensors) if m else None


def _counts(values: Sequence[int], count: int):
    """(int64 array, sum) of `count` numbers of a segmented call."""
    m = _load_marshal()
    packed = m.int64s(values, count) if m else None
    if packed is None:
        ints = [int(v) for v in values]
        packed = (ctypes.c_int64 * max(count, 1))(*ints), sum(ints)
    return packed


def _segment_arrays(tensors: Sequence[torch.Tensor]):
    S = max(len(tensors), 1)
    return (ctypes.c_void_p * S)(*[_dev(t) for t in tensors]), (ctypes.c_int64 * S)(*[t.numel() for t in tensors])


def _one_dtype(tensors: Sequence[torch.Tensor]) -> None:
    if any(t.dtype != tensors[0].dtype for t in tensors):
        raise ValueError("all tensors of a segmented call must share one dtype")


def adatopk_workspace_bytes(n_total: int, num_segments: int, dtype: torch.dtype) -> int:
    return int(load_library().adatopk_workspace_bytes(int(n_total), int(num_segments), _dtype_code(dtype)))


def new_workspace(n_total: int, num_segments: int, dtype: torch.dtype, device="cuda") -> torch.Tensor:
    nbytes = adatopk_workspace_bytes(n_total, num_segments, dtype)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def adatopk_compress(dense: torch.Tensor, k: int, idx_out: torch.Tensor, val_out: torch.Tensor,
                     err_norm_out: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    """Enqueues compress of one tensor on the current stream; outputs are written in place."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.compress(lib.address.compress, dense, k, idx_out, val_out, err_norm_out, workspace), "adatopk_compress"):
        return
    _check_outputs(dense.dtype, int(k), idx_out, val_out, err_norm_out, 1)
    err_ptr = _dev(err_norm_out) if err_norm_out is not None else None
    _check(lib.adatopk_compress(_dev(dense), dense.numel(), _dtype_code(dense.dtype), int(k), _dev(idx_out),
                                _dev(val_out), err_ptr, _dev(workspace), workspace.numel(), _stream()),
           "adatopk_compress")


def adatopk_compress_noalloc(dense: torch.Tensor, k: int, idx_out: torch.Tensor, val_out: torch.Tensor,
                             err_norm_out: Optional[torch.Tensor]) -> None:
    """adatopk_compress on the library's own resident scratch (no workspace argument, nothing allocated)."""
    lib = load_library()
    _check_outputs(dense.dtype, int(k), idx_out, val_out, err_norm_out, 1)
    err_ptr = _dev(err_norm_out) if err_norm_out is not None else None
    _check(lib.adatopk_compress_noalloc(_dev(dense), dense.numel(), _dtype_code(dense.dtype), int(k), _dev(idx_out),
                                        _dev(val_out), err_ptr, _stream()), "adatopk_compress_noalloc")


def adatopk_decompress(idx: torch.Tensor, val: torch.Tensor, k: int, dense_out: torch.Tensor) -> None:
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.decompress(lib.address.decompress, idx, val, k, dense_out), "adatopk_decompress"):
        return
    _check_pairs(dense_out.dtype, int(k), idx, val)
    _check(lib.adatopk_decompress(_dev(idx), _dev(val), int(k), _dtype_code(dense_out.dtype), _dev(dense_out),
                                  dense_out.numel(), _stream()), "adatopk_decompress")


def adatopk_decompress_sorted(idx: torch.Tensor, val: torch.Tensor, k: int, dense_out: torch.Tensor) -> None:
    """Decompress for strictly ascending idx (what adatopk_compress produces)."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.decompress(lib.address.decompress_sorted, idx, val, k, dense_out), "adatopk_decompress_sorted"):
        return
    _check_pairs(dense_out.dtype, int(k), idx, val)
    _check(lib.adatopk_decompress_sorted(_dev(idx), _dev(val), int(k), _dtype_code(dense_out.dtype),
                                         _dev(dense_out), dense_out.numel(), _stream()), "adatopk_decompress_sorted")


def adatopk_decompress_accumulate(idx: torch.Tensor, val: torch.Tensor, k: int, dense_inout: torch.Tensor) -> None:
    """dense_inout[idx[j]] += val[j] for unique indices; every other entry is left alone."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.decompress(lib.address.decompress_accumulate, idx, val, k, dense_inout), "adatopk_decompress_accumulate"):
        return
    _check_pairs(dense_inout.dtype, int(k), idx, val)
    _check(lib.adatopk_decompress_accumulate(_dev(idx), _dev(val), int(k), _dtype_code(dense_inout.dtype),
                                             _dev(dense_inout), dense_inout.numel(), _stream()),
           "adatopk_decompress_accumulate")


def adatopk_decompress_segmented(idx: torch.Tensor, val: torch.Tensor, out_offset: Sequence[int],
                                 dense_out: Sequence[torch.Tensor]) -> None:
    """Decompress of S tensors from the concatenated, per-tensor ascending pairs in few launches."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.decompress_segmented(lib.address.decompress_segmented, idx, val, out_offset, dense_out), "adatopk_decompress_segmented"):
        return
    S = len(dense_out)
    segments = _segments(dense_out)
    dtype = segments[2] if segments else dense_out[0].dtype if S else torch.float32
    dt = _dtype_code(dtype)
    if S:
        if not segments:
            _one_dtype(dense_out)
        _check_pairs(dtype, int(out_offset[S]), idx, val)
    ptrs, ns = segments[:2] if segments else _segment_arrays(dense_out)
    off, _ = _counts(out_offset, S + 1)
    _check(lib.adatopk_decompress_segmented(_dev(idx), _dev(val), off, S, dt, ptrs, ns, _stream()),
           "adatopk_decompress_segmented")


class WireHeader(ctypes.Structure):
    """Mirror of adatopk_wire_header (64 bytes)."""
    _fields_ = [("magic", ctypes.c_uint32), ("version", ctypes.c_uint16), ("algorithm", ctypes.c_uint8),
                ("dtype", ctypes.c_uint8), ("index_bytes", ctypes.c_uint8), ("reserved0", ctypes.c_uint8 * 3),
                ("err_norm", ctypes.c_float), ("n", ctypes.c_int64), ("k", ctypes.c_int64),
                ("ratio", ctypes.c_double), ("idx_offset", ctypes.c_int64), ("val_offset", ctypes.c_int64),
                ("reserved1", ctypes.c_uint8 * 8)]


def adatopk_wire_bytes(k: int, dtype_code: int, index_bytes: int) -> int:
    return int(load_library().adatopk_wire_bytes(int(k), int(dtype_code), int(index_bytes)))


def adatopk_wire_keep_count(wire_bytes: int, dtype_code: int, index_bytes: int) -> int:
    return int(load_library().adatopk_wire_keep_count(int(wire_bytes), int(dtype_code), int(index_bytes)))


def adatopk_wire_parse_header(host_bytes: bytes, wire_bytes: int) -> WireHeader:
    """Checks the first 64 bytes of a message held in host memory; raises AdaTopKError if they do not fit."""
    h = WireHeader()
    buf = ctypes.create_string_buffer(bytes(host_bytes[:64]), 64) if len(host_bytes) >= 64 else None
    _check(load_library().adatopk_wire_parse_header(buf, int(wire_bytes), ctypes.byref(h)), "adatopk_wire_parse_header")
    return h


def adatopk_compress_wire(dense: torch.Tensor, k: int, index_bytes: int, ratio: float, wire_out: torch.Tensor,
                          workspace: torch.Tensor) -> None:
    """adatopk_compress writing one wire message into the uint8 tensor wire_out (device memory, or pinned
    host memory: the message then needs no copy before the host can send it)."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.compress_wire(lib.address.compress_wire, dense, k, index_bytes, ratio, wire_out, workspace), "adatopk_compress_wire"):
        return
    _check(lib.adatopk_compress_wire(_dev(dense), dense.numel(), _dtype_code(dense.dtype), int(k), int(index_bytes),
                                     float(ratio), _dev_or_pinned(wire_out), wire_out.numel() * wire_out.element_size(),
                                     _dev(workspace), workspace.numel(), _stream()), "adatopk_compress_wire")


def adatopk_compress_wire_segmented(dense: Sequence[torch.Tensor], ks: Sequence[int], index_bytes: int,
                                    ratios: Optional[Sequence[float]], wire_out: torch.Tensor,
                                    wire_offset: Sequence[int], workspace: torch.Tensor) -> None:
    """One wire message per tensor, message s at byte wire_offset[s] of the uint8 tensor wire_out."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.compress_wire_segmented(lib.address.compress_wire_segmented, dense, ks, index_bytes, ratios, wire_out, wire_offset, workspace), "adatopk_compress_wire_segmented"):
        return
    S = len(dense)
    segments = _segments(dense)
    dt = _dtype_code(segments[2] if segments else dense[0].dtype) if S else F32
    if S and not segments:
        _one_dtype(dense)
    ptrs, ns = segments[:2] if segments else _segment_arrays(dense)
    kk, _ = _counts(ks, S)
    off, _ = _counts(wire_offset, S)
    rr = _dbl_array(ratios) if ratios is not None else None
    _check(lib.adatopk_compress_wire_segmented(ptrs, ns, kk, S, dt, int(index_bytes), rr, _dev_or_pinned(wire_out), off,
                                               wire_out.numel() * wire_out.element_size(), _dev(workspace),
                                               workspace.numel(), _stream()), "adatopk_compress_wire_segmented")


def adatopk_decompress_wire(wire: torch.Tensor, wire_bytes: int, index_bytes: int, dense: torch.Tensor,
                            accumulate: bool = False) -> None:
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.decompress_wire(lib.address.decompress_wire, wire, wire_bytes, index_bytes, dense, accumulate), "adatopk_decompress_wire"):
        return
    _check(lib.adatopk_decompress_wire(_dev(wire), int(wire_bytes), _dtype_code(dense.dtype), int(index_bytes),
                                       dense.numel(), 1 if accumulate else 0, _dev(dense), _stream()),
           "adatopk_decompress_wire")


def adatopk_compress_segmented(dense: Sequence[torch.Tensor], ks: Sequence[int], idx_out: torch.Tensor,
                               val_out: torch.Tensor, out_offset: Sequence[int],
                               err_norm_out: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.compress_segmented(lib.address.compress_segmented, dense, ks, idx_out, val_out, out_offset, err_norm_out, workspace), "adatopk_compress_segmented"):
        return
    S = len(dense)
    segments = _segments(dense)
    dtype = segments[2] if segments else dense[0].dtype if S else torch.float32
    dt = _dtype_code(dtype)
    if S and not segments:
        _one_dtype(dense)
    kk, k_total = _counts(ks, S)
    if S:
        _check_outputs(dtype, k_total, idx_out, val_out, err_norm_out, S)
    ptrs, ns = segments[:2] if segments else _segment_arrays(dense)
    off, _ = _counts(out_offset, S + 1)
    err_ptr = _dev(err_norm_out) if err_norm_out is not None else None
    _check(lib.adatopk_compress_segmented(ptrs, ns, kk, S, dt, _dev(idx_out), _dev(val_out), off, err_ptr,
                                          _dev(workspace), workspace.numel(), _stream()),
           "adatopk_compress_segmented")


def adatopk_adaptive_ratios(R: Sequence[float], r_user: float, coeff: float = 3.0):
    lib = load_library()
    m = len(R)
    arr = (ctypes.c_double * max(m, 1))(*[float(v) for v in R])
    out = (ctypes.c_double * max(m, 1))()
    _check(lib.adatopk_adaptive_ratios(arr, m, float(r_user), float(coeff), out), "adatopk_adaptive_ratios")
    return [out[i] for i in range(m)]


def adatopk_k_for_ratio(n: int, r_i: float) -> int:
    return int(load_library().adatopk_k_for_ratio(int(n), float(r_i)))


def _dbl_array(v):
    return (ctypes.c_double * max(len(v), 1))(*[float(x) for x in v])


def adatopk_link_time(alpha: float, beta: float, message_bytes: float) -> float:
    return float(load_library().adatopk_link_time(float(alpha), float(beta), float(message_bytes)))


def adatopk_pipeline_time(C: Sequence[float], R: Sequence[float], n_b: int) -> float:
    return float(load_library().adatopk_pipeline_time(_dbl_array(C), _dbl_array(R), len(C), int(n_b)))


def adatopk_pipeline_time_compressed(C: Sequence[float], R: Sequence[float], n_b: int, r_user: float,
                                     coeff: float = 3.0, variant: int = 0) -> float:
    return float(load_library().adatopk_pipeline_time_compressed(_dbl_array(C), _dbl_array(R), len(C), int(n_b),
                                                                 float(r_user), float(coeff), int(variant)))


def adatopk_plan_keep_counts(alpha: Sequence[float], beta: Sequence[float], n: Sequence[int], dtype_code: int,
                             r_user: float, coeff: float = 3.0):
    """(ratios, keep counts) for tensors of n[s] values crossing links (alpha[s], beta[s])."""
    m = len(n)
    ns = (ctypes.c_int64 * max(m, 1))(*[int(v) for v in n])
    r_out = (ctypes.c_double * max(m, 1))()
    k_out = (ctypes.c_int64 * max(m, 1))()
    _check(load_library().adatopk_plan_keep_counts(_dbl_array(alpha), _dbl_array(beta), ns, m, int(dtype_code),
                                                   float(r_user), float(coeff), r_out, k_out),
           "adatopk_plan_keep_counts")
    return [r_out[i] for i in range(m)], [int(k_out[i]) for i in range(m)]


# ------------------------------------------------------------------ the training step of a stage around the link
# A matrix is a tensor whose last dimension is contiguous and whose other dimensions are rows at one distance from the next: contiguous tensors of any
# number of dimensions, and views that cut columns out of one.  A tensor without elements is one whatever its strides.
def _matrix(t: torch.Tensor, what: str):
    """(address, stride, rows, cols) of a tensor seen as rows of its last dimension."""
    if not t.is_cuda:
        raise ValueError("%s: adatopk needs device tensors" % what)
    shape = t.shape
    if not shape:
        raise ValueError("%s needs at least one dimension" % what)
    cols, strides = shape[-1], t.stride()
    if 0 in shape:
        return t.data_ptr(), cols, math.prod(shape[:-1]), cols
    if cols > 1 and strides[-1] != 1:
        raise ValueError("%s must be contiguous in its last dimension" % what)
    rows, stride = 1, cols
    for size, step in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if size != 1:
            if rows == 1:
                stride = step
            elif step != rows * stride:
                raise ValueError("%s must have its rows at one distance from the next" % what)
        rows *= size
    return t.data_ptr(), stride, rows, cols


def _like(t: Optional[torch.Tensor], dtype: torch.dtype, rows: int, cols: int, what: str):
    """(address, stride) of another matrix of the call, (None, 0) for None."""
    if t is None:
        return None, 0
    address, stride, r, c = _matrix(t, what)
    if t.dtype != dtype or r != rows or c != cols:
        raise ValueError("%s must be %s with %d rows of %d" % (what, dtype, rows, cols))
    return address, stride


def _floats(t: Optional[torch.Tensor], count: int, what: str):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != count:
        raise ValueError("%s must be float32 with %d entries" % (what, count))
    return _dev(t)


def _act8(t: torch.Tensor, rows: int, cols: int, what: str):
    if t is None:
        return None
    if t.dtype != torch.uint8 or t.numel() < adatopk_act8_bytes(rows, cols):
        raise ValueError("%s must be uint8 with adatopk_act8_bytes(%d, %d) entries" % (what, rows, cols))
    return _dev(t)


def _weights(weight: Optional[torch.Tensor], bias: Optional[torch.Tensor], dtype: torch.dtype, cols: int):
    """(address of the weight, of the bias, code of their type)."""
    kind = weight.dtype if weight is not None else bias.dtype if bias is not None else dtype
    for t, what in ((weight, "weight"), (bias, "bias")):
        if t is not None and (t.dtype != kind or t.numel() != cols or kind not in (dtype, torch.float32)):
            raise ValueError("%s must have %d entries of the activations' type or, like the other, of float32" % (what, cols))
    return None if weight is None else _dev(weight), None if bias is None else _dev(bias), _dtype_code(kind)


def adatopk_act8_bytes(rows: int, cols: int) -> int:
    return int(load_library().adatopk_act8_bytes(int(rows), int(cols)))


def new_act8(rows: int, cols: int, device="cuda") -> torch.Tensor:
    """Buffer of a rows x cols activation in 8 bits."""
    return torch.empty(max(adatopk_act8_bytes(rows, cols), 16), dtype=torch.uint8, device=device)


def adatopk_act8_store(x: torch.Tensor, act8: torch.Tensor) -> None:
    """Puts a matrix away in 8 bits."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.act8_store(lib.address.act8_store, x, act8), "adatopk_act8_store"):
        return
    address, stride, rows, cols = _matrix(x, "x")
    _check(lib.adatopk_act8_store(address, stride, rows, cols, _dtype_code(x.dtype), _act8(act8, rows, cols, "act8"), _stream()),
           "adatopk_act8_store")


def adatopk_act8_load(act8: torch.Tensor, y: torch.Tensor) -> None:
    """Reads a matrix of y's shape back."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.act8_load(lib.address.act8_load, act8, y), "adatopk_act8_load"):
        return
    address, stride, rows, cols = _matrix(y, "y")
    _check(lib.adatopk_act8_load(_act8(act8, rows, cols, "act8"), rows, cols, _dtype_code(y.dtype), address, stride, _stream()),
           "adatopk_act8_load")


def adatopk_gelu_forward(x: torch.Tensor, y: torch.Tensor, act8_x: Optional[torch.Tensor] = None, act8_y: Optional[torch.Tensor] = None,
                         tanh: bool = False) -> None:
    """y = GELU(x); x and y put away in 8 bits where buffers are given."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.gelu_forward(lib.address.gelu_forward, x, y, act8_x, act8_y, tanh), "adatopk_gelu_forward"):
        return
    address, stride, rows, cols = _matrix(x, "x")
    _check(lib.adatopk_gelu_forward(address, stride, rows, cols, _dtype_code(x.dtype), 1 if tanh else 0, *_like(y, x.dtype, rows, cols, "y"),
                                               _act8(act8_x, rows, cols, "act8_x"), _act8(act8_y, rows, cols, "act8_y"), _stream()),
           "adatopk_gelu_forward")


def adatopk_gelu_backward(dy: torch.Tensor, act8_x: torch.Tensor, dx: torch.Tensor, tanh: bool = False) -> None:
    """dx = dy * GELU'(x), x from its 8 bits."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.gelu_backward(lib.address.gelu_backward, dy, act8_x, dx, tanh), "adatopk_gelu_backward"):
        return
    address, stride, rows, cols = _matrix(dy, "dy")
    _check(lib.adatopk_gelu_backward(address, stride, _act8(act8_x, rows, cols, "act8_x"), rows, cols, _dtype_code(dy.dtype), 1 if tanh else 0,
                                                *_like(dx, dy.dtype, rows, cols, "dx"), _stream()), "adatopk_gelu_backward")


def adatopk_layernorm_forward(x: torch.Tensor, weight: Optional[torch.Tensor], bias: Optional[torch.Tensor], eps: float, y: torch.Tensor,
                              mean: Optional[torch.Tensor], rstd: Optional[torch.Tensor], residual: Optional[torch.Tensor] = None,
                              sum_out: Optional[torch.Tensor] = None, act8: Optional[torch.Tensor] = None) -> None:
    """y = layer norm of x + residual; the sum, the statistics and the normalised rows in 8 bits where buffers are given."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.layernorm_forward(lib.address.layernorm_forward, x, weight, bias, eps, y, mean, rstd, residual, sum_out, act8), "adatopk_layernorm_forward"):
        return
    address, stride, rows, cols = _matrix(x, "x")
    _check(lib.adatopk_layernorm_forward(
        address, stride, *_like(residual, x.dtype, rows, cols, "residual"), *_weights(weight, bias, x.dtype, cols), rows, cols, _dtype_code(x.dtype),
        float(eps), *_like(sum_out, x.dtype, rows, cols, "sum_out"), *_like(y, x.dtype, rows, cols, "y"), _floats(mean, rows, "mean"),
        _floats(rstd, rows, "rstd"), _act8(act8, rows, cols, "act8"), _stream()), "adatopk_layernorm_forward")


def adatopk_layernorm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return int(load_library().adatopk_layernorm_backward_workspace_bytes(int(rows), int(cols)))


def adatopk_layernorm_backward(dy: torch.Tensor, x: Optional[torch.Tensor], act8: Optional[torch.Tensor], mean: Optional[torch.Tensor],
                               rstd: torch.Tensor, weight: Optional[torch.Tensor], dx: torch.Tensor, dweight: Optional[torch.Tensor],
                               dbias: Optional[torch.Tensor], workspace: Optional[torch.Tensor], dsum: Optional[torch.Tensor] = None,
                               accumulate: bool = False) -> None:
    """Gradients of a layer norm from its input x (with mean) or from its normalised rows in 8 bits; dsum is added to dx."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.layernorm_backward(lib.address.layernorm_backward, dy, x, act8, mean, rstd, weight, dx, dweight, dbias, workspace, dsum, accumulate), "adatopk_layernorm_backward"):
        return
    address, stride, rows, cols = _matrix(dy, "dy")
    weight_address, _, weight_code = _weights(weight, None, dy.dtype, cols)
    _check(lib.adatopk_layernorm_backward(
        address, stride, *_like(x, dy.dtype, rows, cols, "x"), _act8(act8, rows, cols, "act8"), _floats(mean, rows, "mean"), _floats(rstd, rows, "rstd"),
        weight_address, weight_code, *_like(dsum, dy.dtype, rows, cols, "dsum"), rows, cols, _dtype_code(dy.dtype), *_like(dx, dy.dtype, rows, cols, "dx"),
        _floats(dweight, cols, "dweight"), _floats(dbias, cols, "dbias"), 1 if accumulate else 0, None if workspace is None else _dev(workspace),
        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()), "adatopk_layernorm_backward")


def adatopk_weight_grad_workspace_bytes(rows: int, n_out: int, n_in: int, dtype: torch.dtype) -> int:
    return int(load_library().adatopk_weight_grad_workspace_bytes(int(rows), int(n_out), int(n_in), _dtype_code(dtype)))


def adatopk_weight_grad(dy: torch.Tensor, act8_x: torch.Tensor, dw: torch.Tensor, db: Optional[torch.Tensor], workspace: torch.Tensor,
                        weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, accumulate: bool = False) -> None:
    """dw = dy^T x and db, x from its 8 bits (behind a layer norm: weight * rows + bias)."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.weight_grad(lib.address.weight_grad, dy, act8_x, dw, db, workspace, weight, bias, accumulate), "adatopk_weight_grad"):
        return
    address, stride, rows, n_out = _matrix(dy, "dy")
    if dw.dim() != 2 or dw.dtype != torch.float32 or dw.shape[0] != n_out:
        raise ValueError("dw must be float32 with %d rows, one for each of dy's columns" % n_out)
    n_in = dw.shape[1]
    _check(lib.adatopk_weight_grad(
        address, stride, _act8(act8_x, rows, n_in, "act8_x"), rows, n_out, n_in, _dtype_code(dy.dtype), *_weights(weight, bias, dy.dtype, n_in), _dev(dw),
        _floats(db, n_out, "db"), 1 if accumulate else 0, _dev(workspace), workspace.numel() * workspace.element_size(), _stream()),
        "adatopk_weight_grad")


# ------------------------------------------------------------------ projections in 8-bit floating point, the norm before them, the update of their weights
def _fp8(t: torch.Tensor, rows: int, cols: int, what: str):
    if t is None:
        return None
    if t.dtype != torch.uint8 or t.numel() < adatopk_fp8_bytes(rows, cols):
        raise ValueError("%s must be uint8 with adatopk_fp8_bytes(%d, %d) entries" % (what, rows, cols))
    return _dev(t)


def adatopk_fp8_bytes(rows: int, cols: int) -> int:
    return int(load_library().adatopk_fp8_bytes(int(rows), int(cols)))


def new_fp8(rows: int, cols: int, device="cuda") -> torch.Tensor:
    """Buffer of a rows x cols matrix in 8-bit floating point."""
    return torch.empty(max(adatopk_fp8_bytes(rows, cols), 16), dtype=torch.uint8, device=device)


def adatopk_fp8_store(x: torch.Tensor, fp8: torch.Tensor) -> None:
    """Puts a matrix away in 8-bit floating point, a scale for 128 elements of a row."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.fp8_store(lib.address.fp8_store, x, fp8), "adatopk_fp8_store"):
        return
    address, stride, rows, cols = _matrix(x, "x")
    _check(lib.adatopk_fp8_store(address, stride, rows, cols, _dtype_code(x.dtype), _fp8(fp8, rows, cols, "fp8"), _stream()), "adatopk_fp8_store")


def adatopk_fp8_load(fp8: torch.Tensor, y: torch.Tensor) -> None:
    """Reads a matrix of y's shape back."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.fp8_load(lib.address.fp8_load, fp8, y), "adatopk_fp8_load"):
        return
    address, stride, rows, cols = _matrix(y, "y")
    _check(lib.adatopk_fp8_load(_fp8(fp8, rows, cols, "fp8"), rows, cols, _dtype_code(y.dtype), address, stride, _stream()), "adatopk_fp8_load")


def adatopk_fp8_store_weight(w: torch.Tensor, fp8: Optional[torch.Tensor], fp8_transposed: Optional[torch.Tensor] = None) -> None:
    """Puts a weight matrix away with a scale for each tile of 128 x 128, as it is and transposed."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.fp8_store_weight(lib.address.fp8_store_weight, w, fp8, fp8_transposed), "adatopk_fp8_store_weight"):
        return
    address, stride, rows, cols = _matrix(w, "w")
    _check(lib.adatopk_fp8_store_weight(address, stride, rows, cols, _dtype_code(w.dtype), _fp8(fp8, rows, cols, "fp8"),
                                        _fp8(fp8_transposed, cols, rows, "fp8_transposed"), _stream()), "adatopk_fp8_store_weight")


def adatopk_fp8_product_workspace_bytes(rows: int, n_out: int, n_in: int) -> int:
    return int(load_library().adatopk_fp8_product_workspace_bytes(int(rows), int(n_out), int(n_in)))


def adatopk_fp8_product(fp8_x: torch.Tensor, fp8_w: torch.Tensor, n_in: int, y: torch.Tensor, workspace: Optional[torch.Tensor],
                        bias: Optional[torch.Tensor] = None, add: Optional[torch.Tensor] = None) -> None:
    """y = x W^T + bias + add, x and W from their 8 bits; n_in: the features of a row of either."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.fp8_product(lib.address.fp8_product, fp8_x, fp8_w, n_in, y, workspace, bias, add), "adatopk_fp8_product"):
        return
    n_in = int(n_in)
    address, stride, rows, n_out = _matrix(y, "y")
    _, bias_address, bias_code = _weights(None, bias, y.dtype, n_out)
    _check(lib.adatopk_fp8_product(
        _fp8(fp8_x, rows, n_in, "fp8_x"), _fp8(fp8_w, n_out, n_in, "fp8_w"), rows, n_out, n_in, bias_address, bias_code, *_like(add, y.dtype, rows, n_out, "add"),
        address, stride, _dtype_code(y.dtype), None if workspace is None else _dev(workspace),
        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()), "adatopk_fp8_product")


def adatopk_rmsnorm_forward(x: torch.Tensor, weight: Optional[torch.Tensor], eps: float, y: Optional[torch.Tensor], rstd: Optional[torch.Tensor],
                            residual: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None, act8: Optional[torch.Tensor] = None,
                            fp8: Optional[torch.Tensor] = None) -> None:
    """y = root-mean-square norm of x + residual; the sum, the statistic, the divided rows and the weighted ones in 8 bits where buffers are given."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.rmsnorm_forward(lib.address.rmsnorm_forward, x, weight, eps, y, rstd, residual, sum_out, act8, fp8), "adatopk_rmsnorm_forward"):
        return
    address, stride, rows, cols = _matrix(x, "x")
    weight_address, _, weight_code = _weights(weight, None, x.dtype, cols)
    _check(lib.adatopk_rmsnorm_forward(
        address, stride, *_like(residual, x.dtype, rows, cols, "residual"), weight_address, weight_code, rows, cols, _dtype_code(x.dtype), float(eps),
        *_like(sum_out, x.dtype, rows, cols, "sum_out"), *_like(y, x.dtype, rows, cols, "y"), _floats(rstd, rows, "rstd"), _act8(act8, rows, cols, "act8"),
        _fp8(fp8, rows, cols, "fp8"), _stream()), "adatopk_rmsnorm_forward")


def adatopk_rmsnorm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return int(load_library().adatopk_rmsnorm_backward_workspace_bytes(int(rows), int(cols)))


def adatopk_rmsnorm_backward(dy: torch.Tensor, x: Optional[torch.Tensor], act8: Optional[torch.Tensor], rstd: torch.Tensor, weight: Optional[torch.Tensor],
                             dx: torch.Tensor, dweight: Optional[torch.Tensor], workspace: Optional[torch.Tensor], dsum: Optional[torch.Tensor] = None,
                             accumulate: bool = False) -> None:
    """Gradients of a root-mean-square norm from its input x or from its divided rows in 8 bits; dsum is added to dx."""
    lib = load_library()
    m = _marshal or _load_marshal()
    if m and _done(m.rmsnorm_backward(lib.address.rmsnorm_backward, dy, x, act8, rstd, weight, dx, dweight, workspace, dsum, accumulate), "adatopk_rmsnorm_backward"):
        return
    address, stride, rows, cols = _matrix(dy, "dy")
    weight_address, _, weight_code = _weights(weight, None, dy.dtype, cols)
    _check(lib.adatopk_rmsnorm_backward(
        address, stride, *_like(x, dy.dtype, rows, cols, "x"), _act8(act8, rows, cols, "act8"), _floats(rstd, rows, "rstd"), weight_address, weight_code,
        *_like(dsum, dy.dtype, rows, cols, "dsum"), rows, cols, _dtype_code(dy.dtype), *_like(dx, dy.dtype, rows, cols, "dx"), _floats(dweight, cols, "dweight"),
        1 if accumulate else 0, None if workspace is None else _dev(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
        _stream()), "adatopk_rmsnorm_backward")


def adatopk_muon_update_workspace_bytes(rows: int, cols: int) -> int:
    return int(load_library().adatopk_muon_update_workspace_bytes(int(rows), int(cols)))


def _momentum(t: Optional[torch.Tensor], rows: int, cols: int):
    if t is None:
        return None
    shape = t.shape
    if t.dtype != torch.float32 or t.numel() != rows * cols or (len(shape) > 1 and shape[-1] != cols):
        raise ValueError("momentum must be float32 with %d rows of %d" % (rows, cols))
    return _dev(t)


def adatopk_muon_update(grad: torch.Tensor, momentum: Optional[torch.Tensor], mu: float, nesterov: bool, w: torch.Tensor, scale: float, decay: float,
                        workspace: torch.Tensor, steps: int = 5, eps: float = 1e-7, coarse: bool = False) -> None:
    """w = decay * w + scale * (the orthogonalised gradient, or momentum, which takes its step first); coarse: 16-bit weights with products of 11 bits in some steps."""
    lib = load_library()
    m = _marshal or _load_marshal()
    where = "adatopk_muon_update_coarse" if coarse else "adatopk_muon_update"
    if m and _done(m.muon_update(lib.address.muon_update_coarse if coarse else lib.address.muon_update, grad, momentum, mu, nesterov, w, scale, decay, workspace, steps, eps),
                   where):
        return
    address, stride, rows, cols = _matrix(w, "w")
    grad_address, grad_stride, grad_rows, grad_cols = _matrix(grad, "grad")
    if (grad_rows, grad_cols) != (rows, cols):
        raise ValueError("grad must have %d rows of %d" % (rows, cols))
    _check((lib.adatopk_muon_update_coarse if coarse else lib.adatopk_muon_update)(
        grad_address, grad_stride, _dtype_code(grad.dtype), _momentum(momentum, rows, cols), float(mu), 1 if nesterov else 0, rows, cols, int(steps),
        float(eps), address, stride, _dtype_code(w.dtype), float(scale), float(decay), _dev(workspace), workspace.numel() * workspace.element_size(), _stream()),
        where)


# ------------------------------------------------------------------ measurement hooks (measuring build only)
def measure_stage_names():
    lib = load_measure_library()
    return [lib.adatopk_measure_stage_name(i).decode() for i in range(lib.adatopk_measure_stage_count())]


def measure_read():
    lib = load_measure_library()
    n = lib.adatopk_measure_stage_count()
    buf = (ctypes.c_float * n)()
    _check(lib.adatopk_measure_read(buf), "adatopk_measure_read")
    return [buf[i] for i in range(n)]


def measure_judge(missing_workgroups: int = 0, wait_rounds: int = -1) -> None:
    load_measure_library().adatopk_measure_judge(int(missing_workgroups), int(wait_rounds))


MEASURE_CLAIMS, MEASURE_CHUNK_COUNTS, MEASURE_PART_COUNTS = 0, 1, 2


def measure_workspace_offset(what: int, n_total: int, num_segments: int, dtype: torch.dtype) -> int:
    return int(load_measure_library().adatopk_measure_workspace_offset(int(what), int(n_total), int(num_segments), _dtype_code(dtype)))


def measure_weight_grad_cut(rows: int, n_out: int, n_in: int, dtype: torch.dtype, dy_stride: int):
    """(sides of a tile, whether each load is bounded for itself, shares of the tokens) of a weight gradient."""
    out = (ctypes.c_int32 * 4)()
    _check(load_measure_library().adatopk_measure_weight_grad_cut(int(rows), int(n_out), int(n_in), _dtype_code(dtype), int(dy_stride), out),
           "adatopk_measure_weight_grad_cut")
    return (out[0], out[1]), bool(out[2]), out[3]


def measure_layernorm_cut(rows: int, cols: int, backward: bool):
    """(lanes to a row, octets to a lane, rows under way at a time, shares of the rows whose columns are added up apart or 0) of a layer norm."""
    out = (ctypes.c_int32 * 4)()
    _check(load_measure_library().adatopk_measure_layernorm_cut(int(rows), int(cols), 1 if backward else 0, out), "adatopk_measure_layernorm_cut")
    return tuple(out)


def measure_fp8_product_cut(rows: int, n_out: int, n_in: int, dtype: torch.dtype):
    """(side of a tile or 0 for a few tokens, whether its wavefronts take turns along the sum, shares of the sum, whether the last tiles are in quarters) of a product."""
    out = (ctypes.c_int32 * 4)()
    _check(load_measure_library().adatopk_measure_fp8_product_cut(int(rows), int(n_out), int(n_in), _dtype_code(dtype), out), "adatopk_measure_fp8_product_cut")
    return out[0], bool(out[1]), out[2], bool(out[3])


def measure_muon_update_cut(rows: int, cols: int):
    """((sides of a tile, whether its wavefronts take turns along the sum, shares of the sum)) of an update's eight products: X X^T, the
    polynomial, X's next step and the change of w, from pairs and from the coarse steps' halves."""
    out = (ctypes.c_int32 * 24)()
    _check(load_measure_library().adatopk_measure_muon_update_cut(int(rows), int(cols), out), "adatopk_measure_muon_update_cut")
    return tuple(((out[3 * i], out[3 * i + 1]), out[3 * i + 2] >= 64, out[3 * i + 2] % 64) for i in range(8))


def measure_muon_update_next_cut(rows: int, cols: int):
    """((sides of a tile, whether its wavefronts take turns along the sum, whether its operands change places)) of X's next step: from pairs, from the halves with
    another such step behind it, and with one from pairs behind it."""
    out = (ctypes.c_int32 * 12)()
    _check(load_measure_library().adatopk_measure_muon_update_next_cut(int(rows), int(cols), out), "adatopk_measure_muon_update_next_cut")
    return tuple(((out[4 * i], out[4 * i + 1]), bool(out[4 * i + 2]), bool(out[4 * i + 3])) for i in range(3))


def measure_copy(dst: torch.Tensor, src: torch.Tensor) -> None:
    nbytes = src.numel() * src.element_size()
    _check(load_measure_library().adatopk_measure_copy(_dev(dst), _dev(src), nbytes, _stream()), "adatopk_measure_copy")


def measure_read_only(src: torch.Tensor, sink: torch.Tensor) -> None:
    nbytes = src.numel() * src.element_size()
    _check(load_measure_library().adatopk_measure_read_only(_dev(src), nbytes, _dev(sink), _stream()),
           "adatopk_measure_read_only")


def measure_fill(dst: torch.Tensor) -> None:
    nbytes = dst.numel() * dst.element_size()
    _check(load_measure_library().adatopk_measure_fill(_dev(dst), nbytes, _stream()), "adatopk_measure_fill")
