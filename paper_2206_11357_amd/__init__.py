"""MI355X-native GACT activation compressor / decompressor (arXiv 2206.11357).

Thin ctypes binding over ``libgact.so`` (hand-written HIP for gfx950 behind the
C ABI of ``include/gact.h``).  The functions carry the C names and only marshal
arguments: torch supplies device memory and the current stream, every step of
the path runs in the library's kernels.  There is no CPU fallback: if the
shared library cannot be loaded the import fails.
"""
from __future__ import annotations

import ctypes
import functools
import math
import operator
import os
import struct
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


# gact_heads: x, y, dy, dx, w, dw, rstd, packed, gmin, gscale; strides of x, y, dy, dx; seed; heads, bits.
_HEADS = struct.Struct("10P12qQ2i")
# gact_rotation: batch, tokens; cos, sin, positions; n_positions; head_dim, rot_dim, interleaved, dtype, w_dtype,
# group_size; eps, reserved.
_ROTATION = struct.Struct("2q3Pq6ifi")


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
# The current device's index without torch's check whether a device has been set up: a tensor on one is at hand.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _enqueue(fn, name: str, device: int, stream, *args) -> None:
    """fn(*args, stream) on the tensors' device, whichever is current."""
    if device != _current_device():
        with torch.cuda.device(device):
            rc = fn(*args, _stream(stream))
    elif stream is None and _raw_stream is not None:
        rc = fn(*args, _raw_stream(device))
    else:
        rc = fn(*args, _stream(stream))
    if rc != GACT_OK:
        raise GactError(rc, name)


def _allocating_for(stream, device: int):
    """Where a call on `stream` allocates its outputs and scratch: under that stream, so that the allocator hands their
    memory out again only behind the call."""
    if type(stream) is int:
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


def _same_device(*tensors) -> int:
    """Index of the device that all of them (None aside) lie on; -2 without tensors."""
    device = -2                          # get_device() of host memory is -1
    for t in tensors:
        if t is not None:
            d = t.get_device()
            if d != device:
                if d < 0:
                    raise ValueError("gact needs device tensors")
                if device >= 0:
                    raise ValueError("the tensors of a call lie on different devices")
                device = d
    return device


def _dense(t: torch.Tensor) -> bool:
    """Whether t's elements are numel() consecutive ones, in whatever order of its axes."""
    if t.is_contiguous():
        return True
    extent = 1
    for stride, size in sorted(zip(t.stride(), t.shape)):
        if size != 1:
            if stride != extent:
                return False
            extent *= size
    return True


@functools.lru_cache(maxsize=64)
def gact_grad_norm_workspace_bytes(K: int) -> int:
    return int(lib.gact_grad_norm_workspace_bytes(K))


class _GradTable(ctypes.Array):
    """gact_grad_buf entries, the tensors that they describe (kept alive) and where these were."""
    _type_, _length_ = GradBuf, 0

    def describes(self, g: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]]) -> bool:
        """Whether the first len(g) entries are those of g and, if given, outs."""
        K = len(g)
        if K > len(self.g):
            return False
        whole, copies = K == len(self.g), outs is not None and not (outs is g and self.outs is self.g)
        # addresses first: a tensor can have been given other memory
        if list(map(_address, g)) != (self.g_at if whole else self.g_at[:K]):
            return False
        if copies and list(map(_address, outs)) != (self.outs_at if whole else self.outs_at[:K]):
            return False
        if all(map(operator.is_, g, self.g)) and not (copies and not all(map(operator.is_, outs, self.outs))):
            return True
        return all(_dense(a) and a.numel() == b.numel() and a.dtype == b.dtype for a, b in zip(g, self.g)) and \
            (outs is None or all(map(_alike, outs, g)))


_address = torch.Tensor.data_ptr


def _alike(o: torch.Tensor, a: torch.Tensor) -> bool:
    return o is a or (o.dtype == a.dtype and o.shape == a.shape and o.stride() == a.stride())


@functools.lru_cache(maxsize=64)
def _grad_table_type(K: int):
    return type("_GradTable%d" % K, (_GradTable,), {"_type_": GradBuf, "_length_": K})


def make_grad_bufs(g: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None):
    """ctypes array of gact_grad_buf; without `outs` in place.  It can be used for any number of calls with the same buffers
    and keeps the tensors alive."""
    in_place = outs is None or outs is g
    g = list(g)
    outs = g if in_place else list(outs)
    if len(outs) != len(g):
        raise ValueError("g and outs must list the same buffers")
    if _same_device(*g) != _same_device(*outs):
        raise ValueError("the tensors of a call lie on different devices")
    arr = _grad_table_type(len(g))()
    arr.g, arr.outs = g, outs
    arr.g_at = list(map(_address, g))
    arr.outs_at = arr.g_at if outs is g else list(map(_address, outs))
    for b, a, o, at, out_at in zip(arr, g, outs, arr.g_at, arr.outs_at):
        if not _dense(a):
            raise ValueError("gact needs contiguous tensors")
        if not _alike(o, a):
            raise ValueError("a buffer and its output differ in size, dtype or strides")
        b.g, b.out, b.n, b.dtype = at, out_at, a.numel(), dtype_code(a.dtype)
    return arr


def _norm_kind(norm_type: float) -> int:
    if norm_type == 2:
        return GACT_NORM_2
    if norm_type == math.inf:
        return GACT_NORM_INF
    raise ValueError("norm_type must be 2 or inf, got %r" % (norm_type,))


def _norm_scratch(K: int, norm, workspace, device: int):
    if norm is None:
        norm = torch.empty(1, dtype=torch.float64, device=device)
    if workspace is None:
        workspace = torch.empty(gact_grad_norm_workspace_bytes(K), dtype=torch.uint8, device=device)
    return norm, workspace


def _norm_call(g, outs, norm, workspace, stream, bufs):
    """What the three calls share: (number of buffers, table, device, norm, workspace).  outs: None if the call writes no
    buffers.  The table lives as long as the caller holds it."""
    K = len(g)
    if bufs is None:
        arr = make_grad_bufs(g, outs)
    else:
        arr = bufs
        if not arr.describes(g, outs):
            raise ValueError("bufs was made for other buffers")
    device = g[0].get_device() if K else _current_device()
    if norm is not None:
        if norm.dtype != torch.float64 or norm.numel() != 1:
            raise ValueError("the norm is one float64 element")
        if norm.get_device() != device:
            raise ValueError("the tensors of a call lie on different devices")
    if workspace is not None:
        if workspace.get_device() != device:
            raise ValueError("the tensors of a call lie on different devices")
        if not workspace.is_contiguous():
            raise ValueError("the workspace must be contiguous")
    if norm is None or workspace is None:
        if stream is None:
            norm, workspace = _norm_scratch(K, norm, workspace, device)
        else:
            with _allocating_for(stream, device):
                norm, workspace = _norm_scratch(K, norm, workspace, device)
    return K, arr, device, norm, workspace


def gact_grad_norm(g: Sequence[torch.Tensor], norm_type: float = 2.0, out: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None, bufs=None) -> torch.Tensor:
    """Norm over all buffers together, 2 or inf -> device float64[1].  `bufs` (from make_grad_bufs) skips
    re-marshalling the list."""
    K, table, device, out, workspace = _norm_call(g, None, out, workspace, stream, bufs)
    _enqueue(lib.gact_grad_norm, "gact_grad_norm", device, stream, table, K, _norm_kind(norm_type), out.data_ptr(),
             workspace.data_ptr(), workspace.nbytes)
    return out


def gact_grad_clip(g: Sequence[torch.Tensor], max_norm: float, norm_type: float = 2.0,
                   outs: Optional[Sequence[torch.Tensor]] = None, norm: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None, bufs=None) -> torch.Tensor:
    """Scales the buffers by min(1, max_norm / (norm + 1e-6)), in place or into `outs`; returns their norm before,
    device float64[1].  `bufs` (from make_grad_bufs with the same g and outs) skips re-marshalling the list."""
    K, table, device, norm, workspace = _norm_call(g, g if outs is None else outs, norm, workspace, stream, bufs)
    _enqueue(lib.gact_grad_clip, "gact_grad_clip", device, stream, table, K, _norm_kind(norm_type), float(max_norm),
             norm.data_ptr(), workspace.data_ptr(), workspace.nbytes)
    return norm


def gact_grad_clip_by(g: Sequence[torch.Tensor], max_norm: float, norm: torch.Tensor,
                      outs: Optional[Sequence[torch.Tensor]] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None, bufs=None) -> None:
    """gact_grad_clip by a norm that is known already (device float64[1])."""
    if norm is None:
        raise ValueError("the norm to clip by is missing")
    K, table, device, norm, workspace = _norm_call(g, g if outs is None else outs, norm, workspace, stream, bufs)
    _enqueue(lib.gact_grad_clip_by, "gact_grad_clip_by", device, stream, table, K, float(max_norm), norm.data_ptr(),
             workspace.data_ptr(), workspace.nbytes)


# ---------------------------------------------- norms of heads and rotation
class HeadContext:
    """What the forward pass keeps of one tensor (queries or keys) for its gradient, in one buffer: rstd, float32 of x's
    shape without head_dim, and, where bits is not GACT_BITS_UNCOMPRESSED, packed, gmin and gscale as gact_compress
    lays them out."""
    __slots__ = ("bits", "group_size", "seed", "shape", "device", "blob", "groups", "off")

    def __init__(self, x: torch.Tensor, bits: int, group_size: int, seed: int):
        self.bits, self.group_size, self.seed, self.device = bits, group_size, seed & (2**64 - 1), x.get_device()
        self.shape = shape = x.shape
        n = x.numel()
        packed = self.groups = meta = 0
        if bits != GACT_BITS_UNCOMPRESSED:
            packed = (n * bits + 127 >> 7) * 16
            self.groups = -(-n // group_size) if group_size > 0 else 0
            meta = (self.groups + 3 >> 2) * 16
        self.off = (0, packed, packed + meta, packed + 2 * meta)           # of packed, gmin, gscale, rstd
        rows = n // shape[-1] if n else 0
        self.blob = x.new_empty(packed + 2 * meta + 4 * rows, dtype=torch.uint8)

    def filled(self, blob: torch.Tensor) -> "HeadContext":
        """The same layout over a buffer that the forward pass has filled (and that was kept apart from it: what keeps it may
        hand back another, made again with other widths)."""
        rows = math.prod(self.shape[:-1])
        if blob.dtype != torch.uint8 or blob.numel() != self.off[3] + 4 * rows or not blob.is_contiguous() \
                or blob.get_device() != self.device:
            raise ValueError("the buffer is not this context's")
        c = HeadContext.__new__(HeadContext)
        c.bits, c.group_size, c.seed, c.shape, c.device, c.groups, c.off = \
            self.bits, self.group_size, self.seed, self.shape, self.device, self.groups, self.off
        c.blob = blob
        return c

    @property
    def packed(self) -> torch.Tensor:
        return self.blob[:self.off[1]]

    def _floats(self, k: int, count: int) -> torch.Tensor:
        return self.blob[self.off[k]:self.off[k] + 4 * count].view(torch.float32)

    @property
    def gmin(self) -> torch.Tensor:
        return self._floats(1, self.groups)

    @property
    def gscale(self) -> torch.Tensor:
        return self._floats(2, self.groups)

    @property
    def rstd(self) -> torch.Tensor:
        return self.blob[self.off[3]:].view(torch.float32).view(self.shape[:-1])

    def addresses(self):
        """Addresses of rstd, packed, gmin, gscale; seed; bits."""
        a = self.blob.data_ptr()
        if self.bits == GACT_BITS_UNCOMPRESSED:
            return a, 0, 0, 0, 0, GACT_BITS_UNCOMPRESSED
        off = self.off
        return a + off[3], a, a + off[1], a + off[2], self.seed, self.bits


_NO_CONTEXT = (0, 0, 0, 0, 0, GACT_BITS_UNCOMPRESSED)


def make_head_context(x: torch.Tensor, bits: int = GACT_BITS_UNCOMPRESSED, group_size: int = 0, seed: int = 0,
                      stream=None) -> HeadContext:
    """Buffers for the context of x, [batch, tokens, heads, head_dim] or [tokens, heads, head_dim]."""
    if stream is None:
        return HeadContext(x, bits, group_size, seed)
    with _allocating_for(stream, x.get_device()):
        return HeadContext(x, bits, group_size, seed)


def head_context_fits(group_size: int, head_dim: int, *heads: int) -> bool:
    """Whether the forward pass can compress the context of heads of this size in groups of group_size (gact.h)."""
    if group_size < 32 or group_size % 32 or head_dim % 8 or not 8 <= head_dim <= 512:
        return False
    lanes = 1 << (head_dim // 8 - 1).bit_length()
    n = group_size // head_dim
    fits = (head_dim % group_size == 0 and group_size & (group_size - 1) == 0 if group_size < head_dim
            else group_size % head_dim == 0 and n & (n - 1) == 0 and n * lanes <= 64)
    return fits and all(h * head_dim % group_size == 0 for h in heads)


@functools.lru_cache(maxsize=64)
def gact_head_norm_rotate_workspace_bytes(head_dim: int) -> int:
    return int(lib.gact_head_norm_rotate_workspace_bytes(head_dim))


_NO_STRIDES = (0, 0, 0)


def _head_strides(x: torch.Tensor) -> tuple:
    """Of batch, token and head, in elements."""
    st = x.stride()
    if len(st) == 4:
        a, b, c, last = st
    elif len(st) == 3:
        a, (b, c, last) = 0, st
    else:
        raise ValueError("gact needs [batch, tokens, heads, head_dim] or [tokens, heads, head_dim]")
    if last != 1 and x.shape[-1] > 1:
        raise ValueError("a head's elements must be consecutive")
    return a, b, c


def _head_shape(x: torch.Tensor) -> tuple:
    """(batch, tokens, heads, head_dim)"""
    shape = x.shape
    if len(shape) == 4:
        return shape
    if len(shape) == 3:
        return (1, *shape)
    raise ValueError("gact needs [batch, tokens, heads, head_dim] or [tokens, heads, head_dim]")


def _rotation(B: int, S: int, D: int, dtype, cos, sin, positions, interleaved, w_dtype, group_size: int, eps: float) -> bytes:
    """gact_rotation of queries and keys."""
    a_cos = a_sin = a_pos = n_positions = rot = 0
    if cos is not None and sin is not None:
        shape = cos.shape
        if len(shape) != 2 or sin.shape != shape or cos.dtype is not torch.float32 or sin.dtype is not torch.float32 \
                or not cos.is_contiguous() or not sin.is_contiguous():
            raise ValueError("cos and sin must be contiguous float32 tables [positions, rot_dim / 2]")
        n_positions = shape[0]
        rot, a_cos, a_sin = 2 * shape[1], cos.data_ptr(), sin.data_ptr()
        if positions is not None:
            if positions.dtype is not torch.int64 or positions.numel() != B * S or not positions.is_contiguous():
                raise ValueError("positions must be contiguous int64, one per token")
            a_pos = positions.data_ptr()
        elif S > n_positions:
            raise ValueError("the tables hold fewer positions than a sequence has tokens")
    elif cos is not None or sin is not None:
        raise ValueError("cos and sin belong together")
    return _ROTATION.pack(B, S, a_cos, a_sin, a_pos, n_positions, D, rot, 1 if interleaved else 0, dtype_code(dtype),
                          GACT_F32 if w_dtype is None else dtype_code(w_dtype), group_size, eps, 0)


def _weights_dtype(wq, wk, D: int):
    """The one type of those that are given; None if none is."""
    dtype = None
    for w in (wq, wk):
        if w is not None:
            if w.numel() != D or not w.is_contiguous():
                raise ValueError("the weights must be contiguous, one per element of a head")
            if dtype is None:
                dtype = w.dtype
            elif w.dtype is not dtype:
                raise ValueError("the weights must have one type")
    return dtype


def _check_like(y: torch.Tensor, x: torch.Tensor) -> None:
    if y.shape != x.shape or y.dtype is not x.dtype:
        raise ValueError("shape or dtype differ: %s %s, %s %s" % (tuple(y.shape), y.dtype, tuple(x.shape), x.dtype))


def _check_context(c: HeadContext, x: torch.Tensor, device: int, group_size: int) -> int:
    """The group size of the contexts looked at so far, and this one; 0 while none is compressed."""
    if c.shape != x.shape or c.device != device:
        raise ValueError("the context was made for another shape or device")
    if c.bits == GACT_BITS_UNCOMPRESSED:
        return group_size
    if group_size and c.group_size != group_size:
        raise ValueError("the contexts of a call must have one group size")
    return c.group_size


_NONE = (None, None)


def _forward_record(q, k, cos, sin, wq, wk, positions, eps, interleaved, out, context):
    """(device, parts, number of parts, rotation) of a forward call into `out`."""
    yq, yk = out
    cq, ck = context if context is not None else _NONE
    B, S, H, D = _head_shape(q)
    dtype, G = q.dtype, 0
    if k is None:
        yk = wk = ck = None
    device = _same_device(q, k, yq, yk, wq, wk, cos, sin, positions)
    w_dtype = _weights_dtype(wq, wk, D)
    if yq is not q:
        _check_like(yq, q)
    a_q = _NO_CONTEXT
    if cq is not None:
        G, a_q = _check_context(cq, q, device, G), cq.addresses()
    parts = _HEADS.pack(q.data_ptr(), yq.data_ptr(), 0, 0, 0 if wq is None else wq.data_ptr(), 0, *a_q[:4], *_head_strides(q),
                        *_head_strides(yq), 0, 0, 0, 0, 0, 0, a_q[4], H, a_q[5])
    if k is not None:
        Bk, Sk, Hk, Dk = _head_shape(k)
        if Bk != B or Sk != S or Dk != D or k.dtype is not dtype:
            raise ValueError("queries and keys differ in batch, tokens, head_dim or dtype")
        if yk is not k:
            _check_like(yk, k)
        a_k = _NO_CONTEXT
        if ck is not None:
            G, a_k = _check_context(ck, k, device, G), ck.addresses()
        parts += _HEADS.pack(k.data_ptr(), yk.data_ptr(), 0, 0, 0 if wk is None else wk.data_ptr(), 0, *a_k[:4], *_head_strides(k),
                             *_head_strides(yk), 0, 0, 0, 0, 0, 0, a_k[4], Hk, a_k[5])
    return device, parts, 1 if k is None else 2, _rotation(B, S, D, dtype, cos, sin, positions, interleaved, w_dtype, G, eps)


def _empty_heads(q: Optional[torch.Tensor], k: Optional[torch.Tensor]) -> tuple:
    return None if q is None else q.new_empty(q.shape), None if k is None else k.new_empty(k.shape)


def gact_head_norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor], cos: Optional[torch.Tensor],
                          sin: Optional[torch.Tensor], wq: Optional[torch.Tensor] = None,
                          wk: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                          eps: float = 1e-6, interleaved: bool = False, out=None, context=None, stream=None):
    """RMS norm of every head of q and k ([batch, tokens, heads, head_dim], any strides but the last) with its weights,
    then the position rotation; returns (yq, yk).  cos, sin: float32 tables [positions, rot_dim / 2], or None for no
    rotation; positions: int64 per token, or None for a token's place in its sequence; out: tensors of the same shapes
    (a transposed view lets the result lie head by head); context: two HeadContexts that the pass fills."""
    if out is None:
        if stream is None:
            out = _empty_heads(q, k)
        else:
            with _allocating_for(stream, q.get_device()):
                out = _empty_heads(q, k)
    device, parts, n, rotation = _forward_record(q, k, cos, sin, wq, wk, positions, eps, interleaved, out, context)
    _enqueue(lib.gact_head_norm_rotate, "gact_head_norm_rotate", device, stream, parts, n, rotation)
    return out


def prepare_head_norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor], cos, sin, wq=None, wk=None, positions=None,
                             eps: float = 1e-6, interleaved: bool = False, *, out, context=None) -> PreparedCall:
    """gact_head_norm_rotate(...) into `out`, as a PreparedCall."""
    _, parts, n, rotation = _forward_record(q, k, cos, sin, wq, wk, positions, eps, interleaved, out, context)
    vp = ctypes.c_void_p
    keep = (ctypes.create_string_buffer(parts, len(parts)), ctypes.create_string_buffer(rotation, len(rotation)))
    args = (vp(ctypes.addressof(keep[0])), n, vp(ctypes.addressof(keep[1])))
    return PreparedCall(lib.gact_head_norm_rotate, "gact_head_norm_rotate", args,
                        (keep, q, k, cos, sin, wq, wk, positions, out, context))


def gact_head_norm_rotate_backward(dyq: Optional[torch.Tensor], dyk: Optional[torch.Tensor], cos, sin, wq=None, wk=None,
                                   positions=None, *, context, x=None, interleaved: bool = False, out=None,
                                   weight_grads=(True, True), workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradients of gact_head_norm_rotate from dyq, dyk (any strides but the last) and the contexts it has filled; x =
    (q, k) where these are not compressed.  Returns (dq, dk, dwq, dwk); None for a part without dy, without weights or
    whose weight gradient is not wanted."""
    if dyq is None or dyk is None:
        return _backward_of_one(dyq, dyk, cos, sin, wq, wk, positions, context, x, interleaved, out, weight_grads, workspace, stream)
    xq, xk = x if x is not None else _NONE
    device = _same_device(dyq, dyk, cos, sin, wq, wk, positions, xq, xk, workspace)
    B, S, H, D = _head_shape(dyq)
    Bk, Sk, Hk, Dk = _head_shape(dyk)
    dtype = dyq.dtype
    if Bk != B or Sk != S or Dk != D or dyk.dtype is not dtype:
        raise ValueError("queries and keys differ in batch, tokens, head_dim or dtype")
    w_dtype = _weights_dtype(wq, wk, D)
    want = (wq is not None and weight_grads[0], wk is not None and weight_grads[1])
    if stream is None:
        dq, dk, dwq, dwk, workspace = _backward_buffers(dyq, dyk, wq, wk, want, out, workspace, D)
    else:
        with _allocating_for(stream, device):
            dq, dk, dwq, dwk, workspace = _backward_buffers(dyq, dyk, wq, wk, want, out, workspace, D)
    if out is not None:
        _same_device(dyq, dq, dk)
        _check_like(dq, dyq)
        _check_like(dk, dyk)
    G = _check_context(context[1], dyk, device, _check_context(context[0], dyq, device, 0))
    parts = _backward_part(dyq, xq, dq, wq, dwq, context[0], H) + _backward_part(dyk, xk, dk, wk, dwk, context[1], Hk)
    rotation = _rotation(B, S, D, dtype, cos, sin, positions, interleaved, w_dtype, G, 0.0)
    if workspace is None:
        _enqueue(lib.gact_head_norm_rotate_backward, "gact_head_norm_rotate_backward", device, stream, parts, 2, rotation, None, 0)
    else:
        _enqueue(lib.gact_head_norm_rotate_backward, "gact_head_norm_rotate_backward", device, stream, parts, 2, rotation,
                 workspace.data_ptr(), workspace.nbytes)
    return dq, dk, dwq, dwk


def _backward_of_one(dyq, dyk, cos, sin, wq, wk, positions, context, x, interleaved, out, weight_grads, workspace, stream):
    """Where only one of the two has a gradient to pass on."""
    if dyq is None and dyk is None:
        return None, None, None, None
    i = 0 if dyq is not None else 1
    dy, w, c, xi = (dyq, dyk)[i], (wq, wk)[i], context[i], x[i] if x is not None else None
    device = _same_device(dy, cos, sin, w, positions, xi, workspace)
    B, S, H, D = _head_shape(dy)
    w_dtype = _weights_dtype(w, None, D)
    want = (w is not None and weight_grads[i], False)
    one = None if out is None else (out[i], None)
    if stream is None:
        dx, _, dw, _, workspace = _backward_buffers(dy, None, w, None, want, one, workspace, D)
    else:
        with _allocating_for(stream, device):
            dx, _, dw, _, workspace = _backward_buffers(dy, None, w, None, want, one, workspace, D)
    _same_device(dy, dx)
    _check_like(dx, dy)
    parts = _backward_part(dy, xi, dx, w, dw, c, H)
    rotation = _rotation(B, S, D, dy.dtype, cos, sin, positions, interleaved, w_dtype, _check_context(c, dy, device, 0), 0.0)
    _enqueue(lib.gact_head_norm_rotate_backward, "gact_head_norm_rotate_backward", device, stream, parts, 1, rotation,
             *(workspace.data_ptr(), workspace.nbytes) if workspace is not None else (None, 0))
    return (dx, None, dw, None) if i == 0 else (None, dx, None, dw)


def _backward_buffers(dyq, dyk, wq, wk, want, out, workspace, D: int):
    """(dq, dk, dwq, dwk, workspace): those that are wanted and not given."""
    dq, dk = out if out is not None else _empty_heads(dyq, dyk)
    dwq = wq.new_empty(wq.shape) if want[0] else None
    dwk = wk.new_empty(wk.shape) if want[1] else None
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("the workspace must be contiguous")
    elif want[0] or want[1]:
        workspace = dyq.new_empty(gact_head_norm_rotate_workspace_bytes(D), dtype=torch.uint8)
    return dq, dk, dwq, dwk, workspace


def _backward_part(dy, x, dx, w, dw, c: HeadContext, H: int) -> bytes:
    a_x, strides = 0, _NO_STRIDES
    rstd, packed, gmin, gscale, seed, bits = c.addresses()
    if bits == GACT_BITS_UNCOMPRESSED:
        if x is None:
            raise ValueError("the context is not compressed: x is needed")
        _check_like(x, dy)
        a_x, strides = x.data_ptr(), _head_strides(x)
    return _HEADS.pack(a_x, 0, dy.data_ptr(), dx.data_ptr(), 0 if w is None else w.data_ptr(), 0 if dw is None else dw.data_ptr(),
                       rstd, packed, gmin, gscale, *strides, 0, 0, 0, *_head_strides(dy), *_head_strides(dx), seed, H, bits)
