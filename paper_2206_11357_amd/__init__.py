"""MI355X-native GACT activation compressor / decompressor (arXiv 2206.11357).

Thin ctypes binding over ``libgact.so`` (hand-written HIP for gfx950 behind the
C ABI of ``include/gact.h``).  The functions carry the C names and only marshal
arguments: torch supplies device memory and the current stream, every step of
the path runs in the library's kernels.  There is no CPU fallback: if the
shared library cannot be loaded the import fails.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
from typing import Optional, Sequence, Tuple

import numpy as np
import torch   # imported before the library so that both share one HIP runtime

from . import build as _build

GACT_F32 = 0
GACT_BF16 = 1

GACT_OK = 0
GACT_E_ARG = -1
GACT_E_BITS = -2
GACT_E_GROUP = -3
GACT_E_BUDGET = -4
GACT_E_HIP = -5
GACT_E_CAPTURE = -6
GACT_E_SCRATCH = -7
GACT_NOALLOC_SCRATCH_BYTES = 2 << 20
GACT_NORM_2 = 0
GACT_NORM_INF = 1

EXPORTS = (
    "gact_num_groups", "gact_packed_bytes", "gact_error_string", "gact_compress",
    "gact_decompress", "gact_multi_workspace_bytes", "gact_compress_multi",
    "gact_decompress_multi", "gact_allocate_bits", "gact_reduce_workspace_bytes",
    "gact_sensitivity", "gact_grad_stats_update", "gact_variance_alert",
    "gact_allocate_bits_levels", "gact_footprint", "gact_compress_footprint",
    "gact_compress_footprint_workspace_bytes", "gact_compress_footprint_noalloc", "gact_copy_bounded",
    "gact_grad_norm_workspace_bytes", "gact_grad_norm", "gact_grad_clip", "gact_grad_clip_by",
    "gact_head_norm_rotate_workspace_bytes", "gact_head_norm_rotate", "gact_head_norm_rotate_backward",
)
GACT_BITS_UNCOMPRESSED = 32


class GactError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (code %d)" % (where, error_string(code), code))


class TensorDesc(ctypes.Structure):
    """Mirror of gact_tensor_desc."""
    _fields_ = [("x", ctypes.c_void_p), ("packed", ctypes.c_void_p), ("gmin", ctypes.c_void_p),
                ("gscale", ctypes.c_void_p), ("y", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("seed", ctypes.c_uint64), ("bits", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("index_base", ctypes.c_int64)]


class GradPair(ctypes.Structure):
    """Mirror of gact_grad_pair."""
    _fields_ = [("g0", ctypes.c_void_p), ("g1", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class GradStat(ctypes.Structure):
    """Mirror of gact_grad_stat."""
    _fields_ = [("g", ctypes.c_void_p), ("mean", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class GradBuf(ctypes.Structure):
    """Mirror of gact_grad_buf."""
    _fields_ = [("g", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class Heads(ctypes.Structure):
    """Mirror of gact_heads."""
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("dy", ctypes.c_void_p), ("dx", ctypes.c_void_p),
                ("w", ctypes.c_void_p), ("dw", ctypes.c_void_p), ("rstd", ctypes.c_void_p), ("packed", ctypes.c_void_p),
                ("gmin", ctypes.c_void_p), ("gscale", ctypes.c_void_p), ("x_stride", ctypes.c_int64 * 3),
                ("y_stride", ctypes.c_int64 * 3), ("dy_stride", ctypes.c_int64 * 3), ("dx_stride", ctypes.c_int64 * 3),
                ("seed", ctypes.c_uint64), ("heads", ctypes.c_int32), ("bits", ctypes.c_int32)]


class Rotation(ctypes.Structure):
    """Mirror of gact_rotation."""
    _fields_ = [("batch", ctypes.c_int64), ("tokens", ctypes.c_int64), ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p),
                ("positions", ctypes.c_void_p), ("n_positions", ctypes.c_int64), ("head_dim", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("w_dtype", ctypes.c_int32), ("group_size", ctypes.c_int32), ("eps", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


def _load() -> ctypes.CDLL:
    path = _build.LIB
    if not os.path.exists(path):
        _build.build()
    lib = ctypes.CDLL(path)
    vp, i64, u64, i32, sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_uint64, ctypes.c_int,
                             ctypes.c_size_t)
    lib.gact_num_groups.argtypes = [i64, i32]
    lib.gact_num_groups.restype = sz
    lib.gact_packed_bytes.argtypes = [i64, i32]
    lib.gact_packed_bytes.restype = sz
    lib.gact_error_string.argtypes = [i32]
    lib.gact_error_string.restype = ctypes.c_char_p
    lib.gact_compress.argtypes = [vp, i32, i64, i32, i32, u64, vp, vp, vp, vp]
    lib.gact_compress.restype = i32
    lib.gact_decompress.argtypes = [vp, vp, vp, i64, i32, i32, vp, i32, vp]
    lib.gact_decompress.restype = i32
    lib.gact_multi_workspace_bytes.argtypes = [i32]
    lib.gact_multi_workspace_bytes.restype = sz
    lib.gact_compress_multi.argtypes = [vp, i32, i32, vp, sz, vp]
    lib.gact_compress_multi.restype = i32
    lib.gact_decompress_multi.argtypes = [vp, i32, i32, vp, sz, vp]
    lib.gact_decompress_multi.restype = i32
    lib.gact_allocate_bits.argtypes = [vp, vp, i32, ctypes.c_double, vp]
    lib.gact_allocate_bits.restype = i32
    lib.gact_allocate_bits_levels.argtypes = [vp, vp, i32, ctypes.c_double, vp, i32, vp]
    lib.gact_allocate_bits_levels.restype = i32
    lib.gact_reduce_workspace_bytes.argtypes = [i32, i64]
    lib.gact_reduce_workspace_bytes.restype = sz
    lib.gact_sensitivity.argtypes = [vp, i32, i32, vp, vp, sz, vp]
    lib.gact_sensitivity.restype = i32
    lib.gact_grad_stats_update.argtypes = [vp, i32, i64, vp, vp, sz, vp]
    lib.gact_grad_stats_update.restype = i32
    lib.gact_footprint.argtypes = [vp, i32, i64, i32, vp, vp, sz, vp]
    lib.gact_footprint.restype = i32
    lib.gact_compress_footprint_workspace_bytes.argtypes = [i64, i32]
    lib.gact_compress_footprint_workspace_bytes.restype = sz
    lib.gact_compress_footprint.argtypes = [vp, i32, i64, i32, i32, ctypes.c_uint64, vp, vp, vp, i32, vp,
                                            vp, sz, vp]
    lib.gact_compress_footprint.restype = i32
    lib.gact_compress_footprint_noalloc.argtypes = [vp, i32, i64, i32, i32, ctypes.c_uint64, vp, vp, vp, i32, vp, vp]
    lib.gact_compress_footprint_noalloc.restype = i32
    lib.gact_copy_bounded.argtypes = [vp, vp, sz, i32, vp]
    lib.gact_copy_bounded.restype = i32
    lib.gact_variance_alert.argtypes = [vp, vp, i32, ctypes.c_double, ctypes.c_double, vp]
    lib.gact_variance_alert.restype = i32
    lib.gact_grad_norm_workspace_bytes.argtypes = [i32]
    lib.gact_grad_norm_workspace_bytes.restype = sz
    lib.gact_grad_norm.argtypes = [vp, i32, i32, vp, vp, sz, vp]
    lib.gact_grad_norm.restype = i32
    lib.gact_grad_clip.argtypes = [vp, i32, i32, ctypes.c_double, vp, vp, sz, vp]
    lib.gact_grad_clip.restype = i32
    lib.gact_grad_clip_by.argtypes = [vp, i32, ctypes.c_double, vp, vp, sz, vp]
    lib.gact_grad_clip_by.restype = i32
    lib.gact_head_norm_rotate_workspace_bytes.argtypes = [i32]
    lib.gact_head_norm_rotate_workspace_bytes.restype = sz
    lib.gact_head_norm_rotate.argtypes = [vp, i32, vp, vp]
    lib.gact_head_norm_rotate.restype = i32
    lib.gact_head_norm_rotate_backward.argtypes = [vp, i32, vp, vp, sz, vp]
    lib.gact_head_norm_rotate_backward.restype = i32
    return lib


lib = _load()


# ------------------------------------------------------------------ helpers
def error_string(code: int) -> str:
    return lib.gact_error_string(code).decode()


def gact_num_groups(n: int, group_size: int) -> int:
    return int(lib.gact_num_groups(n, group_size))


def gact_packed_bytes(n: int, bits: int) -> int:
    return int(lib.gact_packed_bytes(n, bits))


def gact_multi_workspace_bytes(L: int) -> int:
    return int(lib.gact_multi_workspace_bytes(L))


_DTYPE_CODES = {torch.float32: GACT_F32, torch.bfloat16: GACT_BF16}


def dtype_code(dtype: torch.dtype) -> int:
    try:
        return _DTYPE_CODES[dtype]
    except KeyError:
        raise TypeError("gact handles float32 and bfloat16 tensors, got %s" % dtype) from None


# The current stream's handle without a Stream object around it: 0.4 us a call instead of 2.7 us, on calls
# of which the launch itself takes the host 3 us.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    """hipStream_t as an integer: None = torch's current stream; a torch stream; or the integer itself
    (a call site that issues many calls resolves the stream once and passes the handle)."""
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if type(stream) is int:
        return stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(x: torch.Tensor) -> torch.Tensor:
    if not x.is_cuda:
        raise ValueError("gact needs device tensors")
    if not x.is_contiguous():
        raise ValueError("gact needs contiguous tensors")
    return x


def _flat(x: torch.Tensor) -> torch.Tensor:
    return _check(x).view(-1)


def alloc_compressed(n: int, group_size: int, bits: int, device) -> Tuple[torch.Tensor, ...]:
    """(packed uint8, gmin f32, gscale f32) buffers of the sizes the C ABI asks for."""
    packed = torch.empty(gact_packed_bytes(n, bits), dtype=torch.uint8, device=device)
    ng = gact_num_groups(n, group_size)
    gmin = torch.empty(ng, dtype=torch.float32, device=device)
    gscale = torch.empty(ng, dtype=torch.float32, device=device)
    return packed, gmin, gscale


# --------------------------------------------------------------- single tensor
def gact_compress(x: torch.Tensor, group_size: int, bits: int, seed: int,
                  packed: Optional[torch.Tensor] = None, gmin: Optional[torch.Tensor] = None,
                  gscale: Optional[torch.Tensor] = None, stream=None):
    """Compress one tensor; returns (packed, gmin, gscale) device tensors."""
    n = _check(x).numel()
    if packed is None:
        packed, gmin, gscale = alloc_compressed(n, max(group_size, 1), bits if bits > 0 else 1,
                                                x.device)
    rc = lib.gact_compress(x.data_ptr(), dtype_code(x.dtype), n, group_size, bits,
                           seed & (2**64 - 1), packed.data_ptr(), gmin.data_ptr(),
                           gscale.data_ptr(), _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_compress")
    return packed, gmin, gscale


def gact_decompress(packed: torch.Tensor, gmin: torch.Tensor, gscale: torch.Tensor, n: int,
                    group_size: int, bits: int, dtype: torch.dtype = torch.float32,
                    y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Decompress into y (allocated when not given); returns y."""
    if y is None:
        y = torch.empty(n, dtype=dtype, device=packed.device)
    rc = lib.gact_decompress(packed.data_ptr(), gmin.data_ptr(), gscale.data_ptr(), n,
                             group_size, bits, _check(y).data_ptr(), dtype_code(y.dtype),
                             _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_decompress")
    return y


class PreparedCall:
    """One single-tensor call with its arguments marshalled once: ``call(stream_handle)`` enqueues it
    on that stream (an integer hipStream_t, e.g. ``torch.cuda.current_stream().cuda_stream``).  For
    loops that issue the same call many times (a serving loop, one call per saved tensor and step):
    nothing is looked up or converted per call.  The object keeps the tensors alive."""
    __slots__ = ("_fn", "_args", "_name", "_keep")

    def __init__(self, fn, name, args, keep):
        self._fn, self._name, self._args, self._keep = fn, name, args, keep

    def __call__(self, stream_handle: int = 0) -> None:
        rc = self._fn(*self._args, stream_handle)
        if rc != GACT_OK:
            raise GactError(rc, self._name)


def prepare_compress(x: torch.Tensor, group_size: int, bits: int, seed: int, packed: torch.Tensor,
                     gmin: torch.Tensor, gscale: torch.Tensor) -> PreparedCall:
    """gact_compress(x, ...) into the given buffers, as a PreparedCall."""
    vp = ctypes.c_void_p
    args = (vp(_check(x).data_ptr()), dtype_code(x.dtype), ctypes.c_int64(x.numel()), group_size, bits,
            ctypes.c_uint64(seed & (2**64 - 1)), vp(packed.data_ptr()), vp(gmin.data_ptr()), vp(gscale.data_ptr()))
    return PreparedCall(lib.gact_compress, "gact_compress", args, (x, packed, gmin, gscale))


def prepare_decompress(packed: torch.Tensor, gmin: torch.Tensor, gscale: torch.Tensor, n: int,
                       group_size: int, bits: int, y: torch.Tensor) -> PreparedCall:
    """gact_decompress(...) into y, as a PreparedCall."""
    vp = ctypes.c_void_p
    args = (vp(packed.data_ptr()), vp(gmin.data_ptr()), vp(gscale.data_ptr()), ctypes.c_int64(n), group_size, bits,
            vp(_check(y).data_ptr()), dtype_code(y.dtype))
    return PreparedCall(lib.gact_decompress, "gact_decompress", args, (packed, gmin, gscale, y))


# ---------------------------------------------------------------- multi tensor
def make_descs(xs: Sequence[Optional[torch.Tensor]], packed: Sequence[torch.Tensor],
               gmin: Sequence[torch.Tensor], gscale: Sequence[torch.Tensor],
               ys: Sequence[Optional[torch.Tensor]], ns: Sequence[int], bits: Sequence[int],
               seeds: Sequence[int], dtypes: Sequence[torch.dtype],
               index_bases: Optional[Sequence[int]] = None):
    """ctypes array of gact_tensor_desc from per-tensor buffers; index_bases gives each
    entry's offset in its tensor's noise stream when the entries are shards (default 0)."""
    L = len(ns)
    arr = (TensorDesc * max(L, 1))()
    for l in range(L):
        d = arr[l]
        d.x = xs[l].data_ptr() if xs[l] is not None else None
        d.y = ys[l].data_ptr() if ys[l] is not None else None
        d.packed = packed[l].data_ptr()
        d.gmin = gmin[l].data_ptr()
        d.gscale = gscale[l].data_ptr()
        d.n = int(ns[l])
        d.seed = int(seeds[l]) & (2**64 - 1)
        d.bits = int(bits[l])
        d.dtype = dtype_code(dtypes[l])
        d.index_base = int(index_bases[l]) if index_bases is not None else 0
    return arr


def gact_compress_multi(descs, L: int, group_size: int, workspace: torch.Tensor, stream=None):
    rc = lib.gact_compress_multi(ctypes.addressof(descs), L, group_size, workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_compress_multi")


def gact_decompress_multi(descs, L: int, group_size: int, workspace: torch.Tensor, stream=None):
    rc = lib.gact_decompress_multi(ctypes.addressof(descs), L, group_size, workspace.data_ptr(),
                                   workspace.numel() * workspace.element_size(), _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_decompress_multi")


# ------------------------------------------------------------------- allocator
def gact_allocate_bits(sensitivity, numel, avg_bit_budget: float) -> np.ndarray:
    c = np.ascontiguousarray(sensitivity, dtype=np.float32)
    d = np.ascontiguousarray(numel, dtype=np.int64)
    if c.shape != d.shape or c.ndim != 1:
        raise ValueError("sensitivity and numel must be 1-D and of equal length")
    out = np.empty(c.size, dtype=np.int32)
    rc = lib.gact_allocate_bits(c.ctypes.data, d.ctypes.data, c.size, float(avg_bit_budget),
                                out.ctypes.data)
    if rc != GACT_OK:
        raise GactError(rc, "gact_allocate_bits")
    return out


def gact_allocate_bits_levels(sensitivity, numel, avg_bit_budget: float, levels) -> np.ndarray:
    """Allocator over a level set drawn from {1, 2, 4, 8, 32}; 32 = leave uncompressed."""
    c = np.ascontiguousarray(sensitivity, dtype=np.float32)
    d = np.ascontiguousarray(numel, dtype=np.int64)
    lv = np.ascontiguousarray(levels, dtype=np.int32)
    if c.shape != d.shape or c.ndim != 1 or lv.ndim != 1:
        raise ValueError("sensitivity and numel must be 1-D and of equal length")
    out = np.empty(c.size, dtype=np.int32)
    rc = lib.gact_allocate_bits_levels(c.ctypes.data, d.ctypes.data, c.size, float(avg_bit_budget),
                                       lv.ctypes.data, lv.size, out.ctypes.data)
    if rc != GACT_OK:
        raise GactError(rc, "gact_allocate_bits_levels")
    return out


# ------------------------------------------------- sensitivity and the alert
def gact_reduce_workspace_bytes(K: int, total_elems: int) -> int:
    return int(lib.gact_reduce_workspace_bytes(K, total_elems))


def _reduce_workspace(tensors, workspace):
    """The caller's workspace, or one of the size that the buffers need (the library checks either)."""
    if workspace is not None:
        return workspace
    tensors = list(tensors)              # a stacked tensor and a dict's values as well
    need = gact_reduce_workspace_bytes(len(tensors), sum(int(t.numel()) for t in tensors))
    dev = tensors[0].device if tensors else torch.device("cuda")
    return torch.empty(max(need, 16), dtype=torch.uint8, device=dev)


def make_grad_pairs(g0: Sequence[torch.Tensor], g1: Sequence[torch.Tensor]):
    """ctypes array of gact_grad_pair (reusable across calls while the buffers live)."""
    K = len(g0)
    if len(g1) != K:
        raise ValueError("g0 and g1 must list the same buffers")
    arr = (GradPair * max(K, 1))()
    for k in range(K):
        a, b = _flat(g0[k]), _flat(g1[k])
        if a.numel() != b.numel() or a.dtype != b.dtype:
            raise ValueError("buffer %d: g0 and g1 differ in size or dtype" % k)
        arr[k].g0, arr[k].g1, arr[k].n, arr[k].dtype = a.data_ptr(), b.data_ptr(), a.numel(), dtype_code(a.dtype)
    return arr


def make_grad_stats(g: Sequence[torch.Tensor], mean: Sequence[torch.Tensor]):
    """ctypes array of gact_grad_stat."""
    K = len(g)
    if len(mean) != K:
        raise ValueError("g and mean must list the same buffers")
    arr = (GradStat * max(K, 1))()
    for k in range(K):
        a, m = _flat(g[k]), _flat(mean[k])
        if a.numel() != m.numel() or m.dtype != torch.float32:
            raise ValueError("buffer %d: mean must be float32 of the gradient's size" % k)
        arr[k].g, arr[k].mean, arr[k].n, arr[k].dtype = a.data_ptr(), m.data_ptr(), a.numel(), dtype_code(a.dtype)
    return arr


def gact_sensitivity(g0: Sequence[torch.Tensor], g1: Sequence[torch.Tensor], bits: int,
                     out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None, pairs=None) -> torch.Tensor:
    """1/2 ||g0 - g1||^2 / S(bits) over lists of gradient buffers -> device float64[1].
    `pairs` (from make_grad_pairs) skips re-marshalling the buffer list."""
    K = len(g0)
    arr = pairs if pairs is not None else make_grad_pairs(g0, g1)
    workspace = _reduce_workspace(g0, workspace)
    if out is None:
        out = torch.empty(1, dtype=torch.float64, device=workspace.device)
    rc = lib.gact_sensitivity(ctypes.addressof(arr), K, bits, out.data_ptr(), workspace.data_ptr(),
                              workspace.numel(), _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_sensitivity")
    return out


def gact_grad_stats_update(g: Sequence[torch.Tensor], mean: Sequence[torch.Tensor], t: int,
                           out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                           stream=None, stats=None) -> torch.Tensor:
    """Running-mean step t over gradient buffers -> device float64[2] = (sum g^2, sum mean^2)."""
    K = len(g)
    arr = stats if stats is not None else make_grad_stats(g, mean)
    workspace = _reduce_workspace(g, workspace)
    if out is None:
        out = torch.empty(2, dtype=torch.float64, device=workspace.device)
    rc = lib.gact_grad_stats_update(ctypes.addressof(arr), K, t, out.data_ptr(), workspace.data_ptr(),
                                    workspace.numel(), _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_grad_stats_update")
    return out


def gact_footprint(x: torch.Tensor, n_samples: int = 8, out: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """-> device float64[1 + n_samples]: sum of x, then n_samples evenly spaced elements."""
    x = _flat(x)
    workspace = _reduce_workspace([x], workspace)
    if out is None:
        out = torch.empty(1 + n_samples, dtype=torch.float64, device=x.device)
    rc = lib.gact_footprint(x.data_ptr(), dtype_code(x.dtype), x.numel(), n_samples, out.data_ptr(),
                            workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_footprint")
    return out


def gact_compress_footprint_workspace_bytes(n: int, group_size: int) -> int:
    return int(lib.gact_compress_footprint_workspace_bytes(int(n), int(group_size)))


def gact_compress_footprint(x: torch.Tensor, group_size: int, bits: int, seed: int, n_samples: int = 8,
                            packed: Optional[torch.Tensor] = None, gmin: Optional[torch.Tensor] = None,
                            gscale: Optional[torch.Tensor] = None, footprint: Optional[torch.Tensor] = None,
                            workspace: Optional[torch.Tensor] = None, stream=None):
    """Compress one tensor and take its footprint in the same read;
    returns (packed, gmin, gscale, footprint float64[1 + n_samples])."""
    x = _flat(x)
    n = x.numel()
    if packed is None:
        packed, gmin, gscale = alloc_compressed(n, max(group_size, 1), bits if bits > 0 else 1, x.device)
    if footprint is None:
        footprint = torch.empty(1 + n_samples, dtype=torch.float64, device=x.device)
    if workspace is None:
        workspace = torch.empty(max(gact_compress_footprint_workspace_bytes(n, group_size), 16),
                                dtype=torch.uint8, device=x.device)
    rc = lib.gact_compress_footprint(x.data_ptr(), dtype_code(x.dtype), n, group_size, bits,
                                     seed & (2**64 - 1), packed.data_ptr(), gmin.data_ptr(),
                                     gscale.data_ptr(), n_samples, footprint.data_ptr(),
                                     workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_compress_footprint")
    return packed, gmin, gscale, footprint


def gact_compress_footprint_noalloc(x: torch.Tensor, group_size: int, bits: int, seed: int, n_samples: int,
                                    packed: torch.Tensor, gmin: torch.Tensor, gscale: torch.Tensor,
                                    footprint: torch.Tensor, stream=None) -> None:
    """gact_compress_footprint on the library's own scratch area: every buffer comes from the
    caller and neither the call nor this wrapper allocates."""
    rc = lib.gact_compress_footprint_noalloc(x.data_ptr(), dtype_code(x.dtype), x.numel(), group_size, bits,
                                             seed & (2**64 - 1), packed.data_ptr(), gmin.data_ptr(),
                                             gscale.data_ptr(), n_samples, footprint.data_ptr(),
                                             _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_compress_footprint_noalloc")


def gact_copy_bounded(dst: torch.Tensor, src: torch.Tensor, workgroups: int = 16, stream=None) -> None:
    """dst <- src (same byte size; device tensors or pinned host tensors) by a kernel of `workgroups` workgroups."""
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("dst and src differ in size")
    rc = lib.gact_copy_bounded(dst.data_ptr(), src.data_ptr(), nbytes, workgroups, _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, "gact_copy_bounded")


def gact_variance_alert(sensitivity, bits, grad_var: float, threshold: float):
    """-> (alert: bool, V(b) / grad_var)"""
    c = np.ascontiguousarray(sensitivity, dtype=np.float32)
    b = np.ascontiguousarray(bits, dtype=np.int32)
    if c.shape != b.shape or c.ndim != 1:
        raise ValueError("sensitivity and bits must be 1-D and of equal length")
    ratio = ctypes.c_double(0.0)
    rc = lib.gact_variance_alert(c.ctypes.data, b.ctypes.data, c.size, float(grad_var),
                                 float(threshold), ctypes.addressof(ratio))
    if rc < 0:
        raise GactError(rc, "gact_variance_alert")
    return bool(rc), ratio.value


# ------------------------------------------------- gradient norm and clipping
def _enqueue(fn, name: str, device: torch.device, stream, *args) -> None:
    """fn(*args, stream) on the tensors' device, whichever is current."""
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            rc = fn(*args, _stream(stream))
    else:
        rc = fn(*args, _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, name)


def _allocating_for(stream, device: torch.device):
    """Where a call on `stream` allocates its outputs and scratch: under that stream, so that the allocator hands their
    memory out again only behind the call."""
    if stream is None:
        return contextlib.nullcontext()
    if type(stream) is int:
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


def _same_device(tensors) -> torch.device:
    device = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("gact needs device tensors")
        if device is None:
            device = t.device
        elif t.device != device:
            raise ValueError("the tensors of a call lie on different devices")
    return device if device is not None else torch.device("cuda", torch.cuda.current_device())


def _dense(t: torch.Tensor) -> bool:
    return (t.is_contiguous() or (t.dim() == 4 and t.is_contiguous(memory_format=torch.channels_last))
            or (t.dim() == 5 and t.is_contiguous(memory_format=torch.channels_last_3d)))


def gact_grad_norm_workspace_bytes(K: int) -> int:
    return int(lib.gact_grad_norm_workspace_bytes(K))


def make_grad_bufs(g: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None):
    """ctypes array of gact_grad_buf (reusable across calls while the buffers live); without `outs` in place."""
    g = list(g)
    outs = g if outs is None else list(outs)
    if len(outs) != len(g):
        raise ValueError("g and outs must list the same buffers")
    _same_device(g + outs if outs is not g else g)
    arr = (GradBuf * max(len(g), 1))()
    for k, (a, o) in enumerate(zip(g, outs)):
        if not _dense(a):
            raise ValueError("buffer %d: gact needs contiguous tensors" % k)
        if o is not a and (o.dtype != a.dtype or o.shape != a.shape or o.stride() != a.stride()):
            raise ValueError("buffer %d: g and its output differ in size, dtype or strides" % k)
        arr[k].g, arr[k].out, arr[k].n, arr[k].dtype = a.data_ptr(), o.data_ptr(), a.numel(), dtype_code(a.dtype)
    return arr


def _norm_kind(norm_type: float) -> int:
    if norm_type == 2:
        return GACT_NORM_2
    if norm_type == math.inf:
        return GACT_NORM_INF
    raise ValueError("norm_type must be 2 or inf, got %r" % (norm_type,))


def _norm_call(g, outs, norm, workspace, stream, bufs):
    """What the three calls share: (K, table, device, norm, workspace)."""
    g = list(g)
    arr = bufs if bufs is not None else make_grad_bufs(g, outs)
    if len(arr) < len(g):
        raise ValueError("bufs lists fewer buffers than g")
    device = _same_device(g[:1])
    if norm is None or workspace is None:
        with _allocating_for(stream, device):
            if norm is None:
                norm = torch.empty(1, dtype=torch.float64, device=device)
            if workspace is None:
                workspace = torch.empty(gact_grad_norm_workspace_bytes(len(g)), dtype=torch.uint8, device=device)
    if norm.dtype != torch.float64 or norm.numel() != 1:
        raise ValueError("the norm is one float64 element")
    if _same_device([norm, workspace]) != device:
        raise ValueError("the tensors of a call lie on different devices")
    return len(g), arr, device, norm, workspace


def gact_grad_norm(g: Sequence[torch.Tensor], norm_type: float = 2.0, out: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None, bufs=None) -> torch.Tensor:
    """Norm over all buffers together, 2 or inf -> device float64[1].  `bufs` (from make_grad_bufs) skips
    re-marshalling the list."""
    kind = _norm_kind(norm_type)
    K, arr, device, out, workspace = _norm_call(g, None, out, workspace, stream, bufs)
    _enqueue(lib.gact_grad_norm, "gact_grad_norm", device, stream, ctypes.addressof(arr), K, kind, out.data_ptr(),
             workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return out


def gact_grad_clip(g: Sequence[torch.Tensor], max_norm: float, norm_type: float = 2.0,
                   outs: Optional[Sequence[torch.Tensor]] = None, norm: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None, bufs=None) -> torch.Tensor:
    """Scales the buffers by min(1, max_norm / (norm + 1e-6)), in place or into `outs`; returns their norm before,
    device float64[1]."""
    kind = _norm_kind(norm_type)
    K, arr, device, norm, workspace = _norm_call(g, outs, norm, workspace, stream, bufs)
    _enqueue(lib.gact_grad_clip, "gact_grad_clip", device, stream, ctypes.addressof(arr), K, kind, float(max_norm),
             norm.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return norm


def gact_grad_clip_by(g: Sequence[torch.Tensor], max_norm: float, norm: torch.Tensor,
                      outs: Optional[Sequence[torch.Tensor]] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None, bufs=None) -> None:
    """gact_grad_clip by a norm that is known already (device float64[1])."""
    K, arr, device, norm, workspace = _norm_call(g, outs, norm, workspace, stream, bufs)
    _enqueue(lib.gact_grad_clip_by, "gact_grad_clip_by", device, stream, ctypes.addressof(arr), K, float(max_norm),
             norm.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size())


# ---------------------------------------------- norms of heads and rotation
class HeadContext:
    """What the forward pass keeps of one tensor (queries or keys) for its gradient: rstd, and the compressed
    context where bits is not GACT_BITS_UNCOMPRESSED."""
    __slots__ = ("bits", "group_size", "seed", "rstd", "packed", "gmin", "gscale")

    def __init__(self, bits, group_size, seed, rstd, packed=None, gmin=None, gscale=None):
        self.bits, self.group_size, self.seed, self.rstd = bits, group_size, seed, rstd
        self.packed, self.gmin, self.gscale = packed, gmin, gscale


def make_head_context(x: torch.Tensor, bits: int = GACT_BITS_UNCOMPRESSED, group_size: int = 0, seed: int = 0,
                      stream=None) -> HeadContext:
    """Buffers for the context of x, [batch, tokens, heads, head_dim] or [tokens, heads, head_dim]."""
    with _allocating_for(stream, x.device):
        rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        if bits == GACT_BITS_UNCOMPRESSED:
            return HeadContext(bits, group_size, seed, rstd)
        return HeadContext(bits, group_size, seed, rstd, *alloc_compressed(x.numel(), max(group_size, 1), bits, x.device))


def head_context_fits(group_size: int, head_dim: int, *heads: int) -> bool:
    """Whether the forward pass can compress the context of heads of this size in groups of group_size (gact.h)."""
    if group_size < 32 or group_size % 32 or head_dim % 8 or not 8 <= head_dim <= 512:
        return False
    lanes = 1 << (head_dim // 8 - 1).bit_length()
    n = group_size // head_dim
    fits = (head_dim % group_size == 0 and group_size & (group_size - 1) == 0 if group_size < head_dim
            else group_size % head_dim == 0 and n & (n - 1) == 0 and n * lanes <= 64)
    return fits and all(h * head_dim % group_size == 0 for h in heads)


def gact_head_norm_rotate_workspace_bytes(head_dim: int) -> int:
    return int(lib.gact_head_norm_rotate_workspace_bytes(head_dim))


def _head_shape(x: torch.Tensor):
    if x.dim() not in (3, 4):
        raise ValueError("gact needs [batch, tokens, heads, head_dim] or [tokens, heads, head_dim]")
    return tuple(x.shape) if x.dim() == 4 else (1,) + tuple(x.shape)


def _head_strides(x: torch.Tensor):
    if x.shape[-1] > 1 and x.stride(-1) != 1:
        raise ValueError("a head's elements must be consecutive")
    return x.stride()[:3] if x.dim() == 4 else (0,) + x.stride()[:2]


def _rotation(x: torch.Tensor, cos, sin, positions, interleaved: bool, weights) -> Rotation:
    """The record that queries and keys share, from one of them."""
    B, S, _, D = _head_shape(x)
    r = Rotation()
    r.batch, r.tokens, r.head_dim, r.dtype, r.interleaved = B, S, D, dtype_code(x.dtype), int(bool(interleaved))
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin belong together")
    if cos is not None:
        if cos.dim() != 2 or cos.shape != sin.shape or cos.dtype != torch.float32 or sin.dtype != torch.float32 \
                or not cos.is_contiguous() or not sin.is_contiguous():
            raise ValueError("cos and sin must be contiguous float32 tables [positions, rot_dim / 2]")
        r.n_positions, r.rot_dim = cos.shape[0], 2 * cos.shape[1]
        r.cos, r.sin = cos.data_ptr(), sin.data_ptr()
        if positions is not None:
            if positions.dtype != torch.int64 or positions.numel() != B * S or not positions.is_contiguous():
                raise ValueError("positions must be contiguous int64, one per token")
            r.positions = positions.data_ptr()
        elif S > r.n_positions:
            raise ValueError("the tables hold fewer positions than a sequence has tokens")
    types = {w.dtype for w in weights if w is not None}
    if len(types) > 1:
        raise ValueError("the weights must have one type")
    r.w_dtype = dtype_code(types.pop()) if types else GACT_F32
    return r


def _head_part(h: Heads, field: str, t: torch.Tensor, like: torch.Tensor) -> None:
    if _head_shape(t) != _head_shape(like) or t.dtype != like.dtype:
        raise ValueError("%s: shape or dtype differ" % field)
    setattr(h, field, t.data_ptr())
    setattr(h, field + "_stride", (ctypes.c_int64 * 3)(*_head_strides(t)))


def _head_weights(h: Heads, w, D: int) -> None:
    if w is not None:
        if w.numel() != D or not w.is_contiguous():
            raise ValueError("the weights must be contiguous, one per element of a head")
        h.w = w.data_ptr()


def _head_context(h: Heads, c: Optional[HeadContext], shape, r: Rotation) -> None:
    h.heads, h.bits = shape[2], GACT_BITS_UNCOMPRESSED
    if c is None:
        return
    n = shape[0] * shape[1] * shape[2]
    if c.rstd.numel() != n or c.rstd.dtype != torch.float32 or not c.rstd.is_contiguous():
        raise ValueError("the context was made for another shape")
    h.rstd, h.bits, h.seed = c.rstd.data_ptr(), c.bits, c.seed & (2**64 - 1)
    if c.bits != GACT_BITS_UNCOMPRESSED:
        n *= shape[3]
        groups = gact_num_groups(n, c.group_size)
        if c.packed.numel() < gact_packed_bytes(n, c.bits) or c.gmin.numel() < groups or c.gscale.numel() < groups:
            raise ValueError("the context was made for another shape")
        if r.group_size not in (0, c.group_size):
            raise ValueError("the contexts of a call must have one group size")
        r.group_size = c.group_size
        h.packed, h.gmin, h.gscale = c.packed.data_ptr(), c.gmin.data_ptr(), c.gscale.data_ptr()


def _forward_record(q, k, cos, sin, wq, wk, positions, eps, interleaved, out, context):
    """(parts, number of parts, rotation) of a forward call into `out`."""
    xs = [q] if k is None else [q, k]
    ws, ctxs = (wq, wk), context if context is not None else (None, None)
    _same_device(xs + [cos, sin, wq, wk, positions] + list(out))
    if k is not None and (_head_shape(k)[:2] != _head_shape(q)[:2] or k.shape[-1] != q.shape[-1] or k.dtype != q.dtype):
        raise ValueError("queries and keys differ in batch, tokens, head_dim or dtype")
    r = _rotation(q, cos, sin, positions, interleaved, ws[:len(xs)])
    r.eps = eps
    parts = (Heads * 2)()
    for h, x, y, w, c in zip(parts, xs, out, ws, ctxs):
        _head_part(h, "x", x, x)
        _head_part(h, "y", y, x)
        _head_weights(h, w, x.shape[-1])
        _head_context(h, c, _head_shape(x), r)
    return parts, len(xs), r


def gact_head_norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor], cos: Optional[torch.Tensor],
                          sin: Optional[torch.Tensor], wq: Optional[torch.Tensor] = None,
                          wk: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                          eps: float = 1e-6, interleaved: bool = False, out=None, context=None, stream=None):
    """RMS norm of every head of q and k ([batch, tokens, heads, head_dim], any strides but the last) with its weights,
    then the position rotation; returns (yq, yk).  cos, sin: float32 tables [positions, rot_dim / 2], or None for no
    rotation; positions: int64 per token, or None for a token's place in its sequence; out: tensors of the same shapes
    (a transposed view lets the result lie head by head); context: two HeadContexts that the pass fills."""
    device = _same_device([q, k])
    if out is None:
        with _allocating_for(stream, device):
            out = tuple(None if x is None else torch.empty(x.shape, dtype=x.dtype, device=device) for x in (q, k))
    parts, n, r = _forward_record(q, k, cos, sin, wq, wk, positions, eps, interleaved, out, context)
    _enqueue(lib.gact_head_norm_rotate, "gact_head_norm_rotate", device, stream, ctypes.addressof(parts), n,
             ctypes.addressof(r))
    return out


def prepare_head_norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor], cos, sin, wq=None, wk=None, positions=None,
                             eps: float = 1e-6, interleaved: bool = False, *, out, context=None) -> PreparedCall:
    """gact_head_norm_rotate(...) into `out`, as a PreparedCall."""
    parts, n, r = _forward_record(q, k, cos, sin, wq, wk, positions, eps, interleaved, out, context)
    vp = ctypes.c_void_p
    args = (vp(ctypes.addressof(parts)), n, vp(ctypes.addressof(r)))
    return PreparedCall(lib.gact_head_norm_rotate, "gact_head_norm_rotate", args,
                        (parts, r, q, k, cos, sin, wq, wk, positions, out, context))


def gact_head_norm_rotate_backward(dyq: Optional[torch.Tensor], dyk: Optional[torch.Tensor], cos, sin, wq=None, wk=None,
                                   positions=None, *, context, x=None, interleaved: bool = False, out=None,
                                   weight_grads=(True, True), workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradients of gact_head_norm_rotate from dyq, dyk (any strides but the last) and the contexts it has filled; x =
    (q, k) where these are not compressed.  Returns (dq, dk, dwq, dwk); None for a part without dy, without weights or
    whose weight gradient is not wanted."""
    dys, ws = (dyq, dyk), (wq, wk)
    live = [i for i in (0, 1) if dys[i] is not None]
    if not live:
        return None, None, None, None
    xs = x if x is not None else (None, None)
    device = _same_device([dyq, dyk, cos, sin, wq, wk, positions] + list(xs) + [context[i].rstd for i in live])
    first = dys[live[0]]
    D = first.shape[-1]
    if len(live) == 2 and (_head_shape(dyk)[:2] != _head_shape(dyq)[:2] or dyk.shape[-1] != D or dyk.dtype != dyq.dtype):
        raise ValueError("queries and keys differ in batch, tokens, head_dim or dtype")
    r = _rotation(first, cos, sin, positions, interleaved, [ws[i] for i in live])
    wanted = [ws[i] is not None and bool(weight_grads[i]) for i in (0, 1)]
    dxs, dws = [None, None], [None, None]
    with _allocating_for(stream, device):
        for i in live:
            dxs[i] = out[i] if out is not None else torch.empty(dys[i].shape, dtype=dys[i].dtype, device=device)
            if wanted[i]:
                dws[i] = torch.empty(ws[i].shape, dtype=ws[i].dtype, device=device)
        if any(wanted[i] for i in live) and workspace is None:
            workspace = torch.empty(gact_head_norm_rotate_workspace_bytes(D), dtype=torch.uint8, device=device)
    _same_device([first, workspace] + dxs)
    parts = (Heads * 2)()
    for h, i in zip(parts, live):
        _head_part(h, "dy", dys[i], dys[i])
        _head_part(h, "dx", dxs[i], dys[i])
        _head_weights(h, ws[i], D)
        if dws[i] is not None:
            h.dw = dws[i].data_ptr()
        _head_context(h, context[i], _head_shape(dys[i]), r)
        if context[i].bits == GACT_BITS_UNCOMPRESSED:
            if xs[i] is None:
                raise ValueError("the context is not compressed: x is needed")
            _head_part(h, "x", xs[i], dys[i])
    _enqueue(lib.gact_head_norm_rotate_backward, "gact_head_norm_rotate_backward", device, stream, ctypes.addressof(parts),
             len(live), ctypes.addressof(r), workspace.data_ptr() if workspace is not None else None,
             workspace.numel() * workspace.element_size() if workspace is not None else 0)
    return dxs[0], dxs[1], dws[0], dws[1]
