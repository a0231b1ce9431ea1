"""Thin ctypes binding of libgnnfd.so: argument marshalling only.

PyTorch supplies device memory and streams; every step of the aggregation runs inside the library's
CUDA kernels.  There is no fallback: if the shared library is missing or fails to load, importing
the entry points raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

from . import build as _build

F32, BF16 = 0, 1
I32, I64 = 0, 1
CSR_ADD_SELF_LOOPS, CSR_DEDUP, CSR_SYMMETRIZE, CSR_INPUT_ORDER = 1, 2, 4, 8
OK, INVALID_ARG, BAD_INDEX, TOO_LARGE, WORKSPACE_TOO_SMALL, UNSUPPORTED, CUDA_ERROR = 0, -1, -2, -3, -4, -5, -6
STATIC_SCRATCH_EXCEEDED = -7
COMBINE_TF32, COMBINE_FP32 = 0, 1
ACTIVATIONS = {"none": 0, "relu": 1, "elu": 2, "silu": 3, "gelu": 4}
ROTARY_SCALINGS = {"none": 0, "position": 1, "base": 2, "ramp": 3}
GATES = {"factor": 0, "sigmoid": 1}
STATE_ROWS, RECURRENCE_FEW_ROWS, RECURRENCE_FEW_VALUES = 8, 4096, 524288
STATIC_SCRATCH_BYTES = 32 << 20
HUB_DEGREE, HUB_SEGMENT, HUB_RANGE_ROWS = 2048, 1024, 524288
EMBEDDING_FEW_IDS, EMBEDDING_FEW_ROWS = 16384, 3629056

_lib = None


class GnnfdError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().gnnfd_status_string(status).decode()
        if status == CUDA_ERROR:
            msg += " (cudaError %d)" % lib().gnnfd_last_cuda_error()
        super().__init__("%s: %s" % (where, msg))


def lib() -> ctypes.CDLL:
    """Loads libgnnfd.so from the package directory (never builds, never falls back)."""
    global _lib
    if _lib is None:
        path = _build.LIB_PATH
        if not os.path.exists(path):
            raise ImportError("libgnnfd.so is not built: run paper_2104_03058_b200.build.build_library()")
        L = ctypes.CDLL(path)
        i64, i32, u32, vp, sz, fl = (ctypes.c_int64, ctypes.c_int32, ctypes.c_uint32, ctypes.c_void_p,
                                     ctypes.c_size_t, ctypes.c_float)
        pp = ctypes.POINTER
        L.gnnfd_csr_workspace_bytes.argtypes = [i64, i64, u32, pp(sz), pp(sz)]
        L.gnnfd_build_csr.argtypes = [i64, i64, vp, vp, i32, u32, vp, sz, vp, sz, vp, pp(vp)]
        L.gnnfd_csr_info.argtypes = [vp] * 10             # all results are read out of one array: see Csr
        L.gnnfd_csr_schedule.argtypes = [vp] * 9
        L.gnnfd_csr_destroy.argtypes = [vp]
        L.gnnfd_csr_destroy.restype = None
        L.gnnfd_aggregate_workspace_bytes.argtypes = [vp, i32, pp(sz)]
        L.gnnfd_aggregate_best_workspace_bytes.argtypes = [vp, vp, i64, i32, i32, i32, pp(sz)]
        agg = [vp, vp, i64, i32, vp, i64, i32, i32, i32, vp, sz, vp]
        L.gnnfd_aggregate_gcn.argtypes = agg
        L.gnnfd_aggregate_sage.argtypes = agg
        L.gnnfd_aggregate_gcn_static.argtypes = [vp, vp, i64, i32, vp, i64, i32, i32, i32, vp]
        L.gnnfd_oneshot_workspace_bytes.argtypes = [i64, i64, u32, i32, pp(sz)]
        one = [i64, i64, vp, vp, i32, u32, vp, i64, i32, vp, i64, i32, i32, i32, vp, sz, vp]
        L.gnnfd_oneshot_gcn.argtypes = one
        L.gnnfd_oneshot_sage.argtypes = one
        L.gnnfd_oneshot_gat_workspace_bytes.argtypes = [i64, i64, u32, i32, i32, pp(sz)]
        L.gnnfd_oneshot_gat.argtypes = [i64, i64, vp, vp, i32, u32, vp, i64, i32, vp, vp, i32, i32, fl, vp, i64, i32, i32,
                                        vp, sz, vp]
        L.gnnfd_default_chunk_candidates.argtypes = [i32, i32, pp(i32), ctypes.c_int]
        L.gnnfd_tune_chunk_width.argtypes = [vp, ctypes.c_int, vp, i64, i32, vp, i64, i32, i32, pp(i32), ctypes.c_int,
                                             vp, sz, vp, pp(i32), pp(fl)]
        L.gnnfd_gat_scores.argtypes = [i64, vp, i64, i32, vp, vp, i32, i32, vp, vp, vp]
        L.gnnfd_gat_workspace_bytes.argtypes = [vp, i32, i32, pp(sz)]
        L.gnnfd_gat_best_workspace_bytes.argtypes = [vp, vp, i64, i32, i32, i32, i32, pp(sz)]
        L.gnnfd_aggregate_gat.argtypes = [vp, vp, i64, i32, vp, vp, i32, i32, fl, vp, i64, i32, i32, vp, sz, vp]
        L.gnnfd_edge_softmax_workspace_bytes.argtypes = [vp, i32, pp(sz)]
        L.gnnfd_edge_softmax.argtypes = [vp, vp, vp, i32, fl, vp, vp, sz, vp]
        L.gnnfd_combine.argtypes = [i64, vp, i64, i32, i32, vp, i64, i32, vp, i64, i32, vp, vp]
        L.gnnfd_combine_ex.argtypes = [i64, vp, i64, i32, i32, vp, i64, i32, vp, i64, i32, ctypes.c_int, vp, vp, i32, i32,
                                       vp, vp, vp, vp]
        L.gnnfd_layer_workspace_bytes.argtypes = [vp, ctypes.c_int, i32, i32, i32, i32, pp(sz)]
        L.gnnfd_layer_best_workspace_bytes.argtypes = [vp, ctypes.c_int, i32, i32, i32, i32, i32, pp(sz)]
        layer = [vp, vp, i64, i32, i32, vp, i64, i32, ctypes.c_int, vp, i64, i32, i32, vp, sz, vp, vp]
        L.gnnfd_layer_gcn.argtypes = layer
        L.gnnfd_layer_sage.argtypes = layer
        L.gnnfd_layer_gat.argtypes = [vp, vp, i64, i32, i32, vp, i64, i32, i32, vp, vp, fl, ctypes.c_int, vp, i64, i32, i32,
                                      vp, sz, vp, vp]
        L.gnnfd_attention_workspace_bytes.argtypes = [vp, i32, i32, pp(sz)]
        L.gnnfd_aggregate_attention.argtypes = [vp, vp, i64, vp, i64, vp, i64, i32, i32, i32, fl, fl, vp, vp, i32, vp, i64, i32, vp, i32,
                                                vp, sz, vp]
        L.gnnfd_attention_backward_workspace_bytes.argtypes = [vp, vp, i32, i32, i32, pp(sz)]
        L.gnnfd_aggregate_attention_backward.argtypes = [vp, vp, vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, i32, i32, fl, fl, vp, vp, vp,
                                                         i32, vp, i64, vp, i64, vp, i64, i32, vp, i32, vp, sz, vp]
        L.gnnfd_group_norm_workspace_bytes.argtypes = [i64, i32, i32, i64, ctypes.c_int, pp(sz)]
        L.gnnfd_group_norm.argtypes = [i64, vp, i64, i32, i32, i32, i64, vp, i32, vp, vp, fl, ctypes.c_int, vp, i64, i32, vp, vp, vp, sz, vp]
        L.gnnfd_group_norm_backward.argtypes = [i64, vp, i64, vp, i64, i32, i32, i32, i64, vp, i32, vp, vp, vp, vp, ctypes.c_int, vp, i64,
                                                i32, vp, vp, vp, sz, vp]
        L.gnnfd_layer_norm.argtypes = [i64, vp, i64, i32, i32, vp, vp, fl, vp, i64, i32, vp, vp, vp]
        L.gnnfd_layer_norm_backward_workspace_bytes.argtypes = [i64, i32, pp(sz)]
        L.gnnfd_layer_norm_backward.argtypes = [i64, vp, i64, vp, i64, i32, i32, vp, vp, vp, vp, i64, i32, vp, vp, vp, sz, vp]
        L.gnnfd_rotary_frequencies.argtypes = [i32, ctypes.c_double, ctypes.c_int, ctypes.c_double, i64, ctypes.c_double, ctypes.c_double, vp]
        L.gnnfd_rotary.argtypes = [i64, vp, i64, i32, i32, i32, i32, ctypes.c_int, vp, i32, vp, fl, ctypes.c_int, vp, i64, i32, vp]
        L.gnnfd_linear_recurrence_workspace_bytes.argtypes = [i64, i32, i64, ctypes.c_int, ctypes.c_int, pp(sz)]
        L.gnnfd_linear_recurrence.argtypes = [i64, vp, i64, vp, i64, i32, i32, ctypes.c_int, i64, vp, i32, vp, vp, i64, i32, vp, vp, vp, sz, vp]
        L.gnnfd_linear_recurrence_backward.argtypes = [i64, vp, i64, vp, i64, vp, i64, i32, i32, ctypes.c_int, i64, vp, i32, vp, vp, vp, vp, i64,
                                                       vp, i64, i32, vp, vp, sz, vp]
        L.gnnfd_embedding.argtypes = [i64, vp, i32, i64, vp, i64, i32, i32, fl, vp, i64, i32, vp, vp]
        L.gnnfd_embedding_backward_workspace_bytes.argtypes = [i64, i64, i32, pp(sz)]
        L.gnnfd_embedding_backward.argtypes = [i64, vp, i32, vp, i64, i32, i64, i32, fl, i64, ctypes.c_int, vp, i64, i32, vp, sz, vp, vp]
        L.gnnfd_debug_combine_fault.argtypes = [i64, i32]
        L.gnnfd_debug_build_fault.argtypes = [i32, i32]
        L.gnnfd_status_string.argtypes = [ctypes.c_int]
        L.gnnfd_status_string.restype = ctypes.c_char_p
        L.gnnfd_last_cuda_error.restype = ctypes.c_int
        L.gnnfd_launch_count.restype = i64
        L.gnnfd_kernel_timing_enable.argtypes = [ctypes.c_int]
        L.gnnfd_kernel_timing_read.argtypes = [pp(ctypes.c_char_p), pp(ctypes.c_double), pp(i64), ctypes.c_int]
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != OK:
        raise GnnfdError(status, where)


# The calls on small graphs take the GPU a few microseconds, so what Python does per call counts: raw stream handles
# instead of Stream objects, plain integers for pointer arguments (the declared argtypes convert them), and no
# overlap test against an output that the call itself has just allocated.
def _stream_ptr(stream=None) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("features must be float32 or bfloat16, got %s" % t.dtype)


def _matrix(t: torch.Tensor, cols: int, name: str):
    """(pointer, leading dimension) of a row-major device matrix with at least `cols` columns."""
    if t.is_cuda and t.dim() == 2:
        (rows, width), (pitch, step) = t.shape, t.stride()
        if width >= cols and (width <= 1 or step == 1):
            if cols > 0x7fffffff:
                raise ValueError("%s has more than 2^31 - 1 columns" % name)          # (the library's counters of columns are 32 bits)
            return t.data_ptr(), pitch if rows > 1 else max(pitch, width)
    raise ValueError("%s must be a 2-D CUDA tensor with unit column stride and >= %d columns" % (name, cols))


def _alloc_bytes(nbytes: int, device, stream=None) -> torch.Tensor:
    """Scratch of at least `nbytes` (torch's caching allocator returns 512-byte aligned blocks).  The
    block is taken under the stream the work will run on, so that the allocator does not hand it to
    another stream's tensor while the kernels that use it are still queued."""
    if stream is None:
        return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _alloc_best(best: int, least, device, stream=None):
    """`best` bytes of scratch or, where the device has no room for them, the `least()` bytes that the call needs (the library then
    does without its aligned copy).  None for no bytes at all."""
    if best == 0:
        return None
    try:
        return _alloc_bytes(best, device, stream)
    except torch.OutOfMemoryError:
        return _alloc_less(best, least(), device, stream)


def _alloc_less(best: int, need: int, device, stream=None):
    """The rest of _alloc_best, called while its allocation error is handled."""
    if need >= best:
        raise
    return _alloc_bytes(need, device, stream) if need else None


def _same_device(csr_device, **tensors):
    """Every operand must live on the device the CSR was built on (the library never migrates data)."""
    for name, t in tensors.items():
        if t is not None and t.device != csr_device:
            raise ValueError("%s is on %s but the CSR is on %s" % (name, t.device, csr_device))


def _need_rows(t, rows: int, name: str):
    if t.shape[0] < rows:
        raise ValueError("%s has %d rows, the graph needs %d" % (name, t.shape[0], rows))


def _extent(t):
    """[first byte, one past the last byte) of the storage a strided 2-D / 1-D tensor touches."""
    begin, count = t.data_ptr(), t.numel()
    if count == 0:
        return (begin, begin)
    if t.is_contiguous():
        return (begin, begin + count * t.element_size())
    last = sum((n - 1) * st for n, st in zip(t.shape, t.stride()))
    return (begin, begin + (last + 1) * t.element_size())


def _pitch_and_width(t):
    """Bytes from row to row (0: a single stretch) and of a row."""
    if t.is_contiguous() or t.shape[0] == 1:
        return 0, t.numel() * t.element_size()
    return t.stride(0) * t.element_size(), (t.shape[1] if t.dim() == 2 else 1) * t.element_size()


def _no_overlap(a, b, name_a: str, name_b: str):
    """The kernels read features through the read-only data path, so an output that overlaps an input
    is undefined behaviour the header forbids: refuse it here."""
    a0, a1 = _extent(a)
    b0, b1 = _extent(b)
    if not (a0 < b1 and b0 < a1):
        return
    # Two column ranges of one row-major buffer interleave row by row without sharing an element: same row
    # pitch (a contiguous tensor is one row, which goes with any), and the column intervals (taken modulo the pitch) apart.
    if a.dim() <= 2 and b.dim() <= 2:
        (pitch_a, width_a), (pitch_b, width_b) = _pitch_and_width(a), _pitch_and_width(b)
        pitch = max(pitch_a, pitch_b)
        if pitch > 0 and min(pitch_a, pitch_b) in (0, pitch):
            w_first, w_second = (width_a, width_b) if a0 <= b0 else (width_b, width_a)
            off = (max(a0, b0) - min(a0, b0)) % pitch
            if w_first <= off and off + w_second <= pitch:
                return
    raise ValueError("%s and %s overlap in memory" % (name_a, name_b))


def _check_aggregate_operands(csr, x, out, f: int, name_x: str = "x", fresh: bool = False):
    """Shape, device and aliasing rules of the aggregation entry points, checked before any launch; `fresh`: the call
    itself allocated `out` beside x, with the right shape."""
    if x.device != csr.device or out.device != csr.device:
        _same_device(csr.device, **{name_x: x, "out": out})
    _need_rows(x, csr.n, name_x)
    if not fresh:
        _need_rows(out, csr.n, "out")
        _no_overlap(x, out, name_x, "out")


def _scratch_args(scratch, device):
    """(pointer, bytes) of an optional scratch tensor."""
    if scratch is None:
        return None, 0
    if scratch.device != device:
        _same_device(device, scratch=scratch)
    return scratch.data_ptr(), scratch.numel() * scratch.element_size()


class Csr:
    """Handle of a built CSR; keeps the persistent device buffer alive."""

    def __init__(self, handle, persistent: torch.Tensor, device, e: int | None = None):
        self._h = handle
        self._persistent = persistent
        self.device = device
        self.e = e                                 # edges of the list that the graph was built from
        # one array of 64-bit words takes every result: n, nnz, max degree, segments, five bin counts, twelve pointers
        r = (ctypes.c_int64 * 21)()
        at = [ctypes.addressof(r) + 8 * i for i in range(21)]
        _check(lib().gnnfd_csr_info(self._h, at[0], at[1], *at[9:15], at[2]), "gnnfd_csr_info")
        _check(lib().gnnfd_csr_schedule(self._h, at[4], at[15], at[3], *at[16:21]), "gnnfd_csr_schedule")
        self.n, self.nnz, self.n_segments = r[0], r[1], r[3]
        self.max_degree = r[2]                     # an int32 in a zeroed little-endian word, never negative
        self.bin_count = r[4:9]
        self._ptrs = dict(zip(("row_ptr", "col_idx", "perm", "dinv_sqrt", "rdeg", "edge_weight", "row_order", "seg_row",
                               "seg_begin", "seg_end", "seg_slot", "hub_seg_ptr"), r[9:21]))

    @property
    def handle(self):
        if self._h is None:
            raise RuntimeError("CSR handle was destroyed")
        return self._h

    def _view(self, name: str, count: int, dtype) -> torch.Tensor:
        """A tensor view (no copy) of one of the arrays inside the persistent buffer."""
        off = self._ptrs[name] - self._persistent.data_ptr()
        size = torch.empty(0, dtype=dtype).element_size()
        return self._persistent[off:off + count * size].view(dtype)

    row_ptr = property(lambda self: self._view("row_ptr", self.n + 1, torch.int32))
    col_idx = property(lambda self: self._view("col_idx", self.nnz, torch.int32))
    perm = property(lambda self: self._view("perm", self.nnz, torch.int32))
    dinv_sqrt = property(lambda self: self._view("dinv_sqrt", self.n, torch.float32))
    rdeg = property(lambda self: self._view("rdeg", self.n, torch.float32))
    edge_weight = property(lambda self: self._view("edge_weight", self.nnz, torch.float32))
    row_order = property(lambda self: self._view("row_order", self.n, torch.int32))
    seg_row = property(lambda self: self._view("seg_row", self.n_segments, torch.int32))
    seg_begin = property(lambda self: self._view("seg_begin", self.n_segments, torch.int32))
    seg_end = property(lambda self: self._view("seg_end", self.n_segments, torch.int32))
    seg_slot = property(lambda self: self._view("seg_slot", self.n_segments, torch.int32))
    hub_seg_ptr = property(lambda self: self._view("hub_seg_ptr", self.bin_count[4] + 1, torch.int32))

    def destroy(self):
        if self._h is not None:
            lib().gnnfd_csr_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def csr_workspace_bytes(n: int, e: int, flags: int):
    p, s = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().gnnfd_csr_workspace_bytes(n, e, flags, ctypes.byref(p), ctypes.byref(s)), "gnnfd_csr_workspace_bytes")
    return p.value, s.value


def build_csr(n: int, src: torch.Tensor, dst: torch.Tensor, flags: int = 0, stream=None,
              persistent: torch.Tensor | None = None, scratch: torch.Tensor | None = None) -> Csr:
    """gnnfd_build_csr on device tensors src/dst (int32 or int64, same dtype and length)."""
    if not (src.is_cuda and dst.is_cuda) or src.dtype != dst.dtype or src.shape != dst.shape or src.dim() != 1:
        raise ValueError("src and dst must be 1-D CUDA tensors of the same dtype and length")
    if src.dtype not in (torch.int32, torch.int64):
        raise TypeError("edge ids must be int32 or int64")
    src, dst = src.contiguous(), dst.contiguous()
    e = src.numel()
    pb, sb = csr_workspace_bytes(n, e, flags)
    if persistent is None:
        persistent = _alloc_bytes(pb, src.device)
    if scratch is None:
        scratch = _alloc_bytes(sb, src.device)
    handle = ctypes.c_void_p()
    st = lib().gnnfd_build_csr(n, e, src.data_ptr(), dst.data_ptr(), I32 if src.dtype == torch.int32 else I64, flags,
                               persistent.data_ptr(), persistent.numel(), scratch.data_ptr(), scratch.numel(),
                               _stream_ptr(stream), ctypes.byref(handle))
    _check(st, "gnnfd_build_csr")
    return Csr(handle, persistent, src.device, e)


def aggregate_workspace_bytes(csr: Csr, f: int) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_aggregate_workspace_bytes(csr.handle, f, ctypes.byref(s)), "gnnfd_aggregate_workspace_bytes")
    return s.value


def aggregate_best_workspace_bytes(csr: Csr, x: torch.Tensor, f: int | None = None, chunk_width: int | None = None) -> int:
    """Scratch with which an aggregation of these features is fastest (at least aggregate_workspace_bytes)."""
    f = x.shape[1] if f is None else f
    xp, ldx = _matrix(x, f, "x")
    s = ctypes.c_size_t()
    _check(lib().gnnfd_aggregate_best_workspace_bytes(csr.handle, xp, ldx, _dtype_code(x), f, f if chunk_width is None else chunk_width,
                                                      ctypes.byref(s)), "gnnfd_aggregate_best_workspace_bytes")
    return s.value


def _aggregate(fn, name, csr: Csr, x, f, chunk_width, out, out_dtype, scratch, stream):
    f = x.shape[1] if f is None else f
    chunk_width = f if chunk_width is None else chunk_width
    fresh = out is None
    if fresh:
        out = torch.empty((csr.n, f), dtype=out_dtype or torch.float32, device=x.device)
    xp, ldx = _matrix(x, f, "x")
    op, ldo = _matrix(out, f, "out")
    _check_aggregate_operands(csr, x, out, f, fresh=fresh)
    xdt = _dtype_code(x)
    if scratch is None:
        need = ctypes.c_size_t()
        _check(lib().gnnfd_aggregate_best_workspace_bytes(csr.handle, xp, ldx, xdt, f, chunk_width, ctypes.byref(need)), name)
        if need.value:
            try:
                scratch = _alloc_bytes(need.value, x.device, stream)
            except torch.OutOfMemoryError:
                scratch = _alloc_less(need.value, aggregate_workspace_bytes(csr, f), x.device, stream)
    sp, sn = _scratch_args(scratch, csr.device)
    _check(fn(csr.handle, xp, ldx, xdt, op, ldo, _dtype_code(out), f, chunk_width, sp, sn, _stream_ptr(stream)), name)
    return out


def aggregate_gcn(csr: Csr, x: torch.Tensor, f: int | None = None, chunk_width: int | None = None,
                  out: torch.Tensor | None = None, out_dtype=None, scratch=None, stream=None) -> torch.Tensor:
    return _aggregate(lib().gnnfd_aggregate_gcn, "gnnfd_aggregate_gcn", csr, x, f, chunk_width, out, out_dtype,
                      scratch, stream)


def aggregate_sage(csr: Csr, x: torch.Tensor, f: int | None = None, chunk_width: int | None = None,
                   out: torch.Tensor | None = None, out_dtype=None, scratch=None, stream=None) -> torch.Tensor:
    return _aggregate(lib().gnnfd_aggregate_sage, "gnnfd_aggregate_sage", csr, x, f, chunk_width, out, out_dtype,
                      scratch, stream)


def oneshot_workspace_bytes(n: int, e: int, flags: int, f: int) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_oneshot_workspace_bytes(n, e, flags, f, ctypes.byref(s)), "gnnfd_oneshot_workspace_bytes")
    return s.value


def oneshot(model: str, n: int, src: torch.Tensor, dst: torch.Tensor, x: torch.Tensor, flags: int = 0, f: int | None = None,
            chunk_width: int | None = None, out: torch.Tensor | None = None, out_dtype=None, scratch=None, stream=None):
    """gnnfd_oneshot_gcn / gnnfd_oneshot_sage: light build + aggregation of a COO edge list in one call."""
    if not (src.is_cuda and dst.is_cuda) or src.dtype != dst.dtype or src.shape != dst.shape or src.dim() != 1:
        raise ValueError("src and dst must be 1-D CUDA tensors of the same dtype and length")
    if src.dtype not in (torch.int32, torch.int64):
        raise TypeError("edge ids must be int32 or int64")
    src, dst = src.contiguous(), dst.contiguous()
    f = x.shape[1] if f is None else f
    chunk_width = f if chunk_width is None else chunk_width
    if out is None:
        out = torch.empty((n, f), dtype=out_dtype or torch.float32, device=x.device)
    xp, ldx = _matrix(x, f, "x")
    op, ldo = _matrix(out, f, "out")
    _same_device(src.device, dst=dst, x=x, out=out)
    _need_rows(x, n, "x")
    _need_rows(out, n, "out")
    _no_overlap(x, out, "x", "out")
    if scratch is None:
        scratch = _alloc_bytes(oneshot_workspace_bytes(n, src.numel(), flags, f), x.device, stream)
    _same_device(src.device, scratch=scratch)
    fn = {"gcn": lib().gnnfd_oneshot_gcn, "sage": lib().gnnfd_oneshot_sage}[model]
    _check(fn(n, src.numel(), src.data_ptr(), dst.data_ptr(),
              I32 if src.dtype == torch.int32 else I64, flags, xp, ldx, _dtype_code(x), op, ldo, _dtype_code(out), f,
              chunk_width, scratch.data_ptr(), scratch.numel() * scratch.element_size(),
              _stream_ptr(stream)), "gnnfd_oneshot_" + model)
    return out


def oneshot_gat(n: int, src: torch.Tensor, dst: torch.Tensor, z: torch.Tensor, a_src: torch.Tensor, a_dst: torch.Tensor,
                heads: int, dim: int, negative_slope: float = 0.2, flags: int = 0, chunk_width: int | None = None,
                out: torch.Tensor | None = None, out_dtype=None, scratch=None, stream=None):
    """gnnfd_oneshot_gat: light build + GAT aggregation of a COO edge list in one call."""
    if not (src.is_cuda and dst.is_cuda) or src.dtype != dst.dtype or src.shape != dst.shape or src.dim() != 1:
        raise ValueError("src and dst must be 1-D CUDA tensors of the same dtype and length")
    if src.dtype not in (torch.int32, torch.int64):
        raise TypeError("edge ids must be int32 or int64")
    src, dst = src.contiguous(), dst.contiguous()
    f = heads * dim
    chunk_width = f if chunk_width is None else chunk_width
    if out is None:
        out = torch.empty((n, f), dtype=out_dtype or torch.float32, device=z.device)
    zp, ldz = _matrix(z, f, "z")
    op, ldo = _matrix(out, f, "out")
    _same_device(src.device, dst=dst, z=z, out=out)
    _need_rows(z, n, "z")
    _need_rows(out, n, "out")
    _no_overlap(z, out, "z", "out")
    a_src, a_dst = _attention_vectors(a_src, a_dst, heads, dim, z.device, stream)
    if scratch is None:
        need = ctypes.c_size_t()
        _check(lib().gnnfd_oneshot_gat_workspace_bytes(n, src.numel(), flags, heads, dim, ctypes.byref(need)),
               "gnnfd_oneshot_gat_workspace_bytes")
        scratch = _alloc_bytes(need.value, z.device, stream)
    _same_device(src.device, scratch=scratch)
    _check(lib().gnnfd_oneshot_gat(n, src.numel(), src.data_ptr(), dst.data_ptr(),
                                   I32 if src.dtype == torch.int32 else I64, flags, zp, ldz, _dtype_code(z),
                                   a_src.data_ptr(), a_dst.data_ptr(), heads, dim,
                                   negative_slope, op, ldo, _dtype_code(out), chunk_width,
                                   scratch.data_ptr(), scratch.numel() * scratch.element_size(),
                                   _stream_ptr(stream)), "gnnfd_oneshot_gat")
    return out


def default_chunk_candidates(f: int, dtype=torch.float32) -> list:
    buf = (ctypes.c_int32 * 16)()
    k = lib().gnnfd_default_chunk_candidates(f, F32 if dtype == torch.float32 else BF16, buf, 16)
    if k < 0:
        raise GnnfdError(k, "gnnfd_default_chunk_candidates")
    return list(buf[:k])


def tune_chunk_width(csr: Csr, x: torch.Tensor, model: str = "gcn", f: int | None = None, candidates=None,
                     out: torch.Tensor | None = None, scratch=None, stream=None):
    """gnnfd_tune_chunk_width: times the candidates on this graph and these features; -> (width, ms)."""
    f = x.shape[1] if f is None else f
    candidates = default_chunk_candidates(f, x.dtype) if candidates is None else list(candidates)
    if out is None:
        out = torch.empty((csr.n, f), dtype=torch.float32, device=x.device)
    xp, ldx = _matrix(x, f, "x")
    op, ldo = _matrix(out, f, "out")
    _check_aggregate_operands(csr, x, out, f)
    if scratch is None:
        need = max([aggregate_best_workspace_bytes(csr, x, f, w) for w in candidates if w > 0], default=0)
        scratch = _alloc_best(need, lambda: aggregate_workspace_bytes(csr, f), x.device, stream)
    _same_device(csr.device, scratch=scratch)
    sp = scratch.data_ptr() if scratch is not None else None
    sn = scratch.numel() * scratch.element_size() if scratch is not None else 0
    arr = (ctypes.c_int32 * len(candidates))(*candidates)
    best, ms = ctypes.c_int32(), ctypes.c_float()
    _check(lib().gnnfd_tune_chunk_width(csr.handle, {"gcn": 0, "sage": 1}[model], xp, ldx, _dtype_code(x), op, ldo,
                                        _dtype_code(out), f, arr, len(candidates), sp, sn, _stream_ptr(stream),
                                        ctypes.byref(best), ctypes.byref(ms)), "gnnfd_tune_chunk_width")
    return best.value, ms.value


def aggregate_gcn_static(csr: Csr, x: torch.Tensor, f: int | None = None, chunk_width: int | None = None,
                         out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """gnnfd_aggregate_gcn_static: GCN aggregation whose hub-row workspace is the library's built-in
    array, for callers that can neither allocate device memory nor spare a buffer.  ``out`` should be
    passed by such callers (when it is None this wrapper allocates it with torch, which the C entry
    point itself never does).  Raises GnnfdError(STATIC_SCRATCH_EXCEEDED) beyond the built-in size."""
    f = x.shape[1] if f is None else f
    chunk_width = f if chunk_width is None else chunk_width
    if out is None:
        out = torch.empty((csr.n, f), dtype=torch.float32, device=x.device)
    xp, ldx = _matrix(x, f, "x")
    op, ldo = _matrix(out, f, "out")
    _check_aggregate_operands(csr, x, out, f)
    _check(lib().gnnfd_aggregate_gcn_static(csr.handle, xp, ldx, _dtype_code(x), op, ldo, _dtype_code(out), f,
                                            chunk_width, _stream_ptr(stream)), "gnnfd_aggregate_gcn_static")
    return out


def _attention_vectors(a_src, a_dst, heads: int, dim: int, device, stream):
    """The two [heads, dim] fp32 attention vectors, contiguous and on `device`.  A conversion makes a
    temporary; it is created under the launch stream for the same reason as the scratch buffers."""
    for name, a in (("a_src", a_src), ("a_dst", a_dst)):
        if a.numel() != heads * dim:
            raise ValueError("%s must hold heads*dim = %d values" % (name, heads * dim))
        if a.device != device:
            raise ValueError("%s is on %s, the features are on %s" % (name, a.device, device))
    if a_src.dtype == a_dst.dtype == torch.float32 and a_src.is_contiguous() and a_dst.is_contiguous():
        return a_src, a_dst
    if stream is None:
        return a_src.contiguous().float(), a_dst.contiguous().float()
    with torch.cuda.stream(stream):
        return a_src.contiguous().float(), a_dst.contiguous().float()


def gat_scores(z: torch.Tensor, a_src: torch.Tensor, a_dst: torch.Tensor, heads: int, dim: int, stream=None):
    n = z.shape[0]
    zp, ldz = _matrix(z, heads * dim, "z")
    a_src, a_dst = _attention_vectors(a_src, a_dst, heads, dim, z.device, stream)
    s_src = torch.empty((n, heads), dtype=torch.float32, device=z.device)
    s_dst = torch.empty((n, heads), dtype=torch.float32, device=z.device)
    _check(lib().gnnfd_gat_scores(n, zp, ldz, _dtype_code(z), a_src.data_ptr(),
                                  a_dst.data_ptr(), heads, dim, s_src.data_ptr(),
                                  s_dst.data_ptr(), _stream_ptr(stream)), "gnnfd_gat_scores")
    return s_src, s_dst


def gat_workspace_bytes(csr: Csr, heads: int, dim: int) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_gat_workspace_bytes(csr.handle, heads, dim, ctypes.byref(s)), "gnnfd_gat_workspace_bytes")
    return s.value


def gat_best_workspace_bytes(csr: Csr, z: torch.Tensor, heads: int, dim: int, chunk_width: int | None = None) -> int:
    """Scratch with which the attention aggregation of these features is fastest (at least gat_workspace_bytes)."""
    f = heads * dim
    zp, ldz = _matrix(z, f, "z")
    s = ctypes.c_size_t()
    _check(lib().gnnfd_gat_best_workspace_bytes(csr.handle, zp, ldz, _dtype_code(z), heads, dim, f if chunk_width is None else chunk_width,
                                                ctypes.byref(s)), "gnnfd_gat_best_workspace_bytes")
    return s.value


def aggregate_gat(csr: Csr, z: torch.Tensor, a_src: torch.Tensor, a_dst: torch.Tensor, heads: int, dim: int,
                  negative_slope: float = 0.2, chunk_width: int | None = None, out: torch.Tensor | None = None,
                  out_dtype=None, scratch=None, stream=None) -> torch.Tensor:
    f = heads * dim
    chunk_width = f if chunk_width is None else chunk_width
    fresh = out is None
    if fresh:
        out = torch.empty((csr.n, f), dtype=out_dtype or torch.float32, device=z.device)
    zp, ldz = _matrix(z, f, "z")
    op, ldo = _matrix(out, f, "out")
    _check_aggregate_operands(csr, z, out, f, "z", fresh)
    a_src, a_dst = _attention_vectors(a_src, a_dst, heads, dim, z.device, stream)
    if scratch is None:
        need = ctypes.c_size_t()
        _check(lib().gnnfd_gat_best_workspace_bytes(csr.handle, zp, ldz, _dtype_code(z), heads, dim, chunk_width,
                                                    ctypes.byref(need)), "gnnfd_aggregate_gat")
        try:
            scratch = _alloc_bytes(need.value, z.device, stream)
        except torch.OutOfMemoryError:
            scratch = _alloc_less(need.value, gat_workspace_bytes(csr, heads, dim), z.device, stream)
    _same_device(csr.device, scratch=scratch)
    _check(lib().gnnfd_aggregate_gat(csr.handle, zp, ldz, _dtype_code(z), a_src.data_ptr(),
                                     a_dst.data_ptr(), heads, dim, negative_slope, op, ldo,
                                     _dtype_code(out), chunk_width, scratch.data_ptr(),
                                     scratch.numel() * scratch.element_size(), _stream_ptr(stream)),
           "gnnfd_aggregate_gat")
    return out


def edge_softmax_workspace_bytes(csr: Csr, heads: int) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_edge_softmax_workspace_bytes(csr.handle, heads, ctypes.byref(s)),
           "gnnfd_edge_softmax_workspace_bytes")
    return s.value


def edge_softmax(csr: Csr, s_src: torch.Tensor, s_dst: torch.Tensor, negative_slope: float = 0.2,
                 out: torch.Tensor | None = None, scratch=None, stream=None) -> torch.Tensor:
    heads = s_src.shape[1]
    if not (s_src.is_contiguous() and s_dst.is_contiguous()):
        raise ValueError("scores must be contiguous")
    if s_src.dtype != torch.float32 or s_dst.dtype != torch.float32 or s_src.shape != s_dst.shape:
        raise TypeError("scores must be float32 [n, heads]")
    if s_src.dim() != 2 or s_src.shape[0] != csr.n:
        raise ValueError("scores must be [n, heads] with n = %d rows, got %s" % (csr.n, tuple(s_src.shape)))
    fresh = out is None
    if fresh:
        out = torch.empty((csr.nnz, heads), dtype=torch.float32, device=s_src.device)
    if out.dtype != torch.float32 or out.dim() != 2 or not out.is_contiguous() or out.shape[1] != heads \
            or out.shape[0] < csr.nnz:
        raise ValueError("alpha must be a contiguous float32 [nnz >= %d, heads = %d] tensor" % (csr.nnz, heads))
    _same_device(csr.device, s_src=s_src, s_dst=s_dst, alpha=out)
    if not fresh:
        _no_overlap(s_src, out, "s_src", "alpha")
        _no_overlap(s_dst, out, "s_dst", "alpha")
    if scratch is None:
        scratch = _alloc_bytes(edge_softmax_workspace_bytes(csr, heads), s_src.device, stream)
    _same_device(csr.device, scratch=scratch)
    _check(lib().gnnfd_edge_softmax(csr.handle, s_src.data_ptr(), s_dst.data_ptr(),
                                    heads, negative_slope, out.data_ptr(),
                                    scratch.data_ptr(), scratch.numel() * scratch.element_size(),
                                    _stream_ptr(stream)),
           "gnnfd_edge_softmax")
    return out


def _combine_mode(mode) -> int:
    if mode in (COMBINE_TF32, "tf32"):
        return COMBINE_TF32
    if mode in (COMBINE_FP32, "fp32"):
        return COMBINE_FP32
    raise ValueError("mode must be 'tf32' or 'fp32'")


def combine(x: torch.Tensor, w_t: torch.Tensor, f_in: int | None = None, out: torch.Tensor | None = None,
            out_dtype=None, status: torch.Tensor | None = None, stream=None, mode="tf32", a_src=None, a_dst=None,
            heads: int = 0, dim: int = 0):
    """gnnfd_combine_ex: z = x[:, :f_in] @ w_t[:, :f_in].T on the tensor cores with fp32 sums.  float32 inputs
    are multiplied as tf32 (``mode="tf32"``) or fp32-faithfully as tf32 pairs (``mode="fp32"``); bfloat16 inputs
    as they are.  ``status`` is an int32 tensor of one element that the kernel sets to 1 if a block gave up
    waiting.  With ``a_src`` / ``a_dst`` ([heads, dim], heads * dim == f_out) the GAT scores of z are formed in
    the same pass and the call returns (z, s_src, s_dst) instead of z."""
    f_in = w_t.shape[1] if f_in is None else f_in
    f_out = w_t.shape[0]
    if x.dtype != w_t.dtype:
        raise TypeError("x and w_t must have the same dtype")
    fresh = out is None
    if fresh:
        out = torch.empty((x.shape[0], f_out), dtype=out_dtype or torch.float32, device=x.device)
    xp, ldx = _matrix(x, f_in, "x")
    wp, ldw = _matrix(w_t, f_in, "w_t")
    op, ldo = _matrix(out, f_out, "out")
    _same_device(x.device, w_t=w_t, out=out, status=status)
    _need_rows(out, x.shape[0], "out")
    if not fresh:
        _no_overlap(x, out, "x", "out")
        _no_overlap(w_t, out, "w_t", "out")
    sp = status.data_ptr() if status is not None else None
    scores = a_src is not None or a_dst is not None
    s_src = s_dst = None
    asp = adp = ssp = sdp = None
    if scores:
        a_src, a_dst = _attention_vectors(a_src, a_dst, heads, dim, x.device, stream)
        s_src = torch.empty((x.shape[0], heads), dtype=torch.float32, device=x.device)
        s_dst = torch.empty((x.shape[0], heads), dtype=torch.float32, device=x.device)
        asp, adp = a_src.data_ptr(), a_dst.data_ptr()
        ssp, sdp = s_src.data_ptr(), s_dst.data_ptr()
    _check(lib().gnnfd_combine_ex(x.shape[0], xp, ldx, _dtype_code(x), f_in, wp, ldw, f_out, op, ldo, _dtype_code(out),
                                  _combine_mode(mode), asp, adp, heads, dim, ssp, sdp, sp, _stream_ptr(stream)),
           "gnnfd_combine_ex")
    return (out, s_src, s_dst) if scores else out


def layer_workspace_bytes(csr: Csr, model: str, f_out: int, heads: int = 0, dim: int = 0, dtype=torch.float32) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_layer_workspace_bytes(csr.handle, {"gcn": 0, "sage": 1, "gat": 2}[model], f_out, heads, dim,
                                             F32 if dtype == torch.float32 else BF16, ctypes.byref(s)),
           "gnnfd_layer_workspace_bytes")
    return s.value


def layer_best_workspace_bytes(csr: Csr, model: str, f_out: int, heads: int = 0, dim: int = 0, dtype=torch.float32,
                               chunk_width: int | None = None) -> int:
    """Scratch with which a layer is fastest (at least layer_workspace_bytes)."""
    s = ctypes.c_size_t()
    _check(lib().gnnfd_layer_best_workspace_bytes(csr.handle, {"gcn": 0, "sage": 1, "gat": 2}[model], f_out, heads, dim,
                                                  F32 if dtype == torch.float32 else BF16, f_out if chunk_width is None else chunk_width,
                                                  ctypes.byref(s)), "gnnfd_layer_best_workspace_bytes")
    return s.value


def layer(csr: Csr, model: str, x: torch.Tensor, w_t: torch.Tensor, f_in: int | None = None, mode="tf32",
          chunk_width: int | None = None, out: torch.Tensor | None = None, out_dtype=None, a_src=None, a_dst=None,
          heads: int = 0, dim: int = 0, negative_slope: float = 0.2, scratch=None, status=None, stream=None):
    """gnnfd_layer_gcn / _sage / _gat: out = Aggregate(x[:, :f_in] @ w_t[:, :f_in].T) on a built CSR; the
    transformed features stay in the scratch buffer."""
    f_in = w_t.shape[1] if f_in is None else f_in
    f_out = w_t.shape[0]
    if x.dtype != w_t.dtype:
        raise TypeError("x and w_t must have the same dtype")
    if model == "gat" and heads * dim != f_out:
        raise ValueError("heads * dim must equal the number of rows of w_t")
    chunk_width = f_out if chunk_width is None else chunk_width
    fresh = out is None
    if fresh:
        out = torch.empty((csr.n, f_out), dtype=out_dtype or torch.float32, device=x.device)
    xp, ldx = _matrix(x, f_in, "x")
    wp, ldw = _matrix(w_t, f_in, "w_t")
    op, ldo = _matrix(out, f_out, "out")
    _same_device(csr.device, x=x, w_t=w_t, out=out, status=status)
    _need_rows(x, csr.n, "x")
    _need_rows(out, csr.n, "out")
    if not fresh:
        _no_overlap(x, out, "x", "out")
        _no_overlap(w_t, out, "w_t", "out")
    if scratch is None:
        scratch = _alloc_best(layer_best_workspace_bytes(csr, model, f_out, heads, dim, x.dtype, chunk_width),
                              lambda: layer_workspace_bytes(csr, model, f_out, heads, dim, x.dtype), x.device, stream)
    _same_device(csr.device, scratch=scratch)
    sp = status.data_ptr() if status is not None else None
    scr, scr_n = scratch.data_ptr(), scratch.numel() * scratch.element_size()
    if model == "gat":
        a_src, a_dst = _attention_vectors(a_src, a_dst, heads, dim, x.device, stream)
        _check(lib().gnnfd_layer_gat(csr.handle, xp, ldx, _dtype_code(x), f_in, wp, ldw, heads, dim,
                                     a_src.data_ptr(), a_dst.data_ptr(), negative_slope,
                                     _combine_mode(mode), op, ldo, _dtype_code(out), chunk_width, scr, scr_n, sp,
                                     _stream_ptr(stream)), "gnnfd_layer_gat")
    else:
        fn = lib().gnnfd_layer_gcn if model == "gcn" else lib().gnnfd_layer_sage
        _check(fn(csr.handle, xp, ldx, _dtype_code(x), f_in, wp, ldw, f_out, _combine_mode(mode), op, ldo,
                  _dtype_code(out), chunk_width, scr, scr_n, sp, _stream_ptr(stream)), "gnnfd_layer_" + model)
    return out


# Kernels are launched on the current device, so the entry points below make that of their tensors current where it is another one: they call
# themselves once more inside _elsewhere.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)      # (a torch without CUDA lacks it)


def _elsewhere(device, stream, again, *args, **kwargs):
    with torch.cuda.device(device):
        return again(*args, stream=stream, **kwargs)


def _stream_handle(index: int, stream) -> int:
    """Raw handle of the stream named, or of the current one of device `index`, which is the current device."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(index)
    if stream.device.index != index:
        raise ValueError("the stream is on %s, the tensors are on cuda:%d" % (stream.device, index))
    return stream.cuda_stream


def _new(like: torch.Tensor, shape, dtype, stream):
    """Memory that a call allocates beside a tensor: taken under the stream the work runs on (see _alloc_bytes)."""
    if stream is None:
        if like.shape == shape:                    # (the quicker of the two)
            return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _index_list(ids: torch.Tensor, name: str):
    """(contiguous ids, count, type code) of a 1-D device tensor of ids."""
    if not ids.is_cuda or ids.dim() != 1:
        raise ValueError("%s must be a 1-D CUDA tensor" % name)
    if ids.dtype == torch.int32:
        code = I32
    elif ids.dtype == torch.int64:
        code = I64
    else:
        raise TypeError("%s must be int32 or int64" % name)
    if not ids.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return ids.data_ptr(), ids.shape[0], code


def _status_ptr(status, device):
    if status is None:
        return None
    if status.dtype != torch.int32 or status.numel() < 1 or status.device != device:
        raise ValueError("status must be an int32 tensor on %s" % device)
    return status.data_ptr()


def edge_values(csr: Csr, values: torch.Tensor, loop=0) -> torch.Tensor:
    """The values [e] of the input edges, one for each edge of the list that the graph was built from, in CSR slot order: a reverse edge
    that the build added has its edge's value, an added self-loop the value ``loop``."""
    if values.dim() != 1 or values.device != csr.device:
        raise ValueError("values must be a 1-D tensor on %s" % csr.device)
    if values.shape[0] != csr.e:
        raise ValueError("values has %d entries, the graph was built from %d edges" % (values.shape[0], csr.e))
    perm, e = csr.perm.long(), csr.e
    if e == 0:
        return torch.full((csr.nnz,), loop, dtype=values.dtype, device=csr.device)
    return torch.where(perm < 0, torch.full((), loop, dtype=values.dtype, device=csr.device), values[perm.clamp_min(0) % e])


def _attention_operands(csr: Csr, f: int, heads: int, dist, bias, **tensors):
    """(pointer, leading dimension) of each [n, >= f] operand, the inputs of one type, then (dist pointer, bias pointer, buckets)."""
    first = next(iter(tensors.values()))
    got = []
    for name, t in tensors.items():
        got.append(_matrix(t, f, name))
        if t.device != csr.device:
            _same_device(csr.device, **{name: t})
        if t.dtype != first.dtype:
            raise TypeError("%s must have one dtype" % ", ".join(tensors))
        _need_rows(t, csr.n, name)
    if (dist is None) != (bias is None):
        raise ValueError("dist and bias come together")
    if bias is None:
        return got, None, None, 0
    if bias.dtype != torch.float32 or bias.dim() != 2 or bias.shape[1] != heads or bias.shape[0] < 1 or not bias.is_contiguous():
        raise ValueError("bias must be a contiguous float32 [buckets, heads = %d] tensor" % heads)
    _check_dist(csr, dist, "dist")
    _same_device(csr.device, bias=bias)
    return got, dist.data_ptr(), bias.data_ptr(), bias.shape[0]


def _check_dist(csr: Csr, dist, name: str):
    if dist.dtype != torch.int32 or dist.dim() != 1 or dist.shape[0] < csr.nnz or not dist.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of nnz = %d values" % (name, csr.nnz))
    _same_device(csr.device, **{name: dist})


def attention_workspace_bytes(csr: Csr, heads: int, dim: int) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_attention_workspace_bytes(csr.handle, heads, dim, ctypes.byref(s)), "gnnfd_attention_workspace_bytes")
    return s.value


def aggregate_attention(csr: Csr, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, heads: int, dim: int, scale: float | None = None,
                        softcap: float = 0.0, dist: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                        chunk_width: int | None = None, out: torch.Tensor | None = None, out_dtype=None, with_lse: bool = False,
                        scratch=None, stream=None):
    """gnnfd_aggregate_attention: softmax attention of every vertex over the sources of its edges.  ``scale`` defaults to dim ** -0.5;
    ``dist`` holds a bucket of ``bias`` ([buckets, heads]) per CSR slot (see edge_values).  With ``with_lse`` the call returns
    (out, lse [n, heads, 2]), which aggregate_attention_backward takes."""
    index = csr.device.index
    if index != _current_device():
        return _elsewhere(csr.device, stream, aggregate_attention, csr, q, k, v, heads, dim, scale, softcap, dist, bias, chunk_width, out,
                          out_dtype, with_lse, scratch)
    f = heads * dim
    scale = dim ** -0.5 if scale is None else scale
    chunk_width = f if chunk_width is None else chunk_width
    ((qp, ldq), (kp, ldk), (vp_, ldv)), dp, bp, buckets = _attention_operands(csr, f, heads, dist, bias, q=q, k=k, v=v)
    fresh = out is None
    if fresh:
        out = _new(q, (csr.n, f), out_dtype or torch.float32, stream)
    op, ldo = _matrix(out, f, "out")
    if not fresh:
        _same_device(csr.device, out=out)
        _need_rows(out, csr.n, "out")
        for name, t in (("q", q), ("k", k), ("v", v)):
            _no_overlap(t, out, name, "out")
    lse = _new(q, (csr.n, heads, 2), torch.float32, stream) if with_lse else None
    if scratch is None and csr.n_segments:
        scratch = _new(q, attention_workspace_bytes(csr, heads, dim), torch.uint8, stream)
    scr, scr_n = _scratch_args(scratch, csr.device)
    dt, odt, lp = _dtype_code(q), _dtype_code(out), lse.data_ptr() if with_lse else None
    _check(lib().gnnfd_aggregate_attention(csr.handle, qp, ldq, kp, ldk, vp_, ldv, dt, heads, dim, scale, softcap, dp, bp, buckets, op, ldo, odt, lp,
                                           chunk_width, scr, scr_n, _stream_handle(index, stream)), "gnnfd_aggregate_attention")
    return (out, lse) if with_lse else out


def attention_backward_workspace_bytes(csr: Csr, csr_t: Csr, heads: int, dim: int, buckets: int = 0) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_attention_backward_workspace_bytes(csr.handle, csr_t.handle, heads, dim, buckets, ctypes.byref(s)),
           "gnnfd_attention_backward_workspace_bytes")
    return s.value


def aggregate_attention_backward(csr: Csr, csr_t: Csr, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, dout: torch.Tensor,
                                 lse: torch.Tensor, heads: int, dim: int, scale: float | None = None, softcap: float = 0.0,
                                 dist: torch.Tensor | None = None, dist_t: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                                 chunk_width: int | None = None, out_dtype=None, scratch=None, stream=None):
    """gnnfd_aggregate_attention_backward: (dq, dk, dv, dbias) for the gradient ``dout`` of aggregate_attention's result; dbias is None
    without a bias.  ``csr_t`` is the CSR of the reversed edges (build_csr with src and dst exchanged and the same flags), ``dist_t`` the
    buckets in its slot order, ``lse`` what the forward call returned."""
    index = csr.device.index
    if index != _current_device():
        return _elsewhere(csr.device, stream, aggregate_attention_backward, csr, csr_t, q, k, v, dout, lse, heads, dim, scale, softcap, dist,
                          dist_t, bias, chunk_width, out_dtype, scratch)
    f = heads * dim
    scale = dim ** -0.5 if scale is None else scale
    chunk_width = f if chunk_width is None else chunk_width
    if csr_t.device != csr.device or csr_t.n != csr.n or csr_t.nnz != csr.nnz:
        raise ValueError("csr_t must be the reverse of csr: as many vertices and entries, on the same device")
    operands, dp, bp, buckets = _attention_operands(csr, f, heads, dist, bias, q=q, k=k, v=v, dout=dout)
    (qp, ldq), (kp, ldk), (vp_, ldv), (gp, ldg) = operands
    if (dist_t is None) != (bias is None):
        raise ValueError("dist_t and bias come together")
    dtp = None
    if dist_t is not None:
        _check_dist(csr_t, dist_t, "dist_t")
        dtp = dist_t.data_ptr()
    if lse.dtype != torch.float32 or lse.dim() != 3 or lse.shape[0] < csr.n or tuple(lse.shape[1:]) != (heads, 2) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 [n, heads, 2] tensor")
    _same_device(csr.device, lse=lse)
    odt = out_dtype or torch.float32

    dq, dk, dv = (_new(q, (csr.n, f), odt, stream) for _ in range(3))
    dbias = _new(q, (buckets, heads), torch.float32, stream) if buckets else None
    if scratch is None:
        scratch = _new(q, max(256, attention_backward_workspace_bytes(csr, csr_t, heads, dim, buckets)), torch.uint8, stream)
    scr, scr_n = _scratch_args(scratch, csr.device)
    dt, code, bgp = _dtype_code(q), _dtype_code(dq), dbias.data_ptr() if buckets else None
    _check(lib().gnnfd_aggregate_attention_backward(
        csr.handle, csr_t.handle, qp, ldq, kp, ldk, vp_, ldv, gp, ldg, dt, lse.data_ptr(), heads, dim, scale, softcap, dp, dtp, bp, buckets,
        dq.data_ptr(), f, dk.data_ptr(), f, dv.data_ptr(), f, code, bgp, chunk_width, scr, scr_n, _stream_handle(index, stream)),
        "gnnfd_aggregate_attention_backward")
    return dq, dk, dv, dbias


def group_norm_workspace_bytes(n: int, f: int, groups: int, graphs: int = 1, backward: bool = False) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_group_norm_workspace_bytes(n, f, groups, graphs, int(backward), ctypes.byref(s)), "gnnfd_group_norm_workspace_bytes")
    return s.value


def _norm_operands(x, groups: int, weight, bias, graph_ptr, activation: str, f: int):
    """(weight pointer, bias pointer, graphs, offsets pointer, offsets type, activation code)"""
    for name, t in (("weight", weight), ("bias", bias)):
        if t is not None and (t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != f or not t.is_contiguous() or t.device != x.device):
            raise ValueError("%s must be a contiguous float32 tensor of %d values on %s" % (name, f, x.device))
    if activation not in ACTIVATIONS:
        raise ValueError("activation must be one of %s" % ", ".join(ACTIVATIONS))
    if groups < 1 or f % groups:
        raise ValueError("%d columns do not make %d groups" % (f, groups))
    graphs, pp, itype = 1, None, I32
    if graph_ptr is not None:
        pp, count, itype = _index_list(graph_ptr, "graph_ptr")
        if count < 2 or graph_ptr.device != x.device:
            raise ValueError("graph_ptr must hold graphs + 1 >= 2 offsets on %s" % x.device)
        graphs = count - 1
    return (None if weight is None else weight.data_ptr(), None if bias is None else bias.data_ptr(), graphs, pp, itype,
            ACTIVATIONS[activation])


def _same_place(a, b) -> bool:
    return a.data_ptr() == b.data_ptr() and a.stride() == b.stride() and a.dtype == b.dtype


def group_norm(x: torch.Tensor, groups: int, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
               graph_ptr: torch.Tensor | None = None, eps: float = 1e-5, activation: str = "none", f: int | None = None,
               out: torch.Tensor | None = None, out_dtype=None, with_stats: bool = False, scratch=None, stream=None):
    """gnnfd_group_norm: rows of x are vertices, ``graph_ptr`` [graphs + 1] the row offsets of the graphs of a batch (None: one graph), and
    each of ``groups`` groups of columns is normalised over the rows of its graph, scaled, shifted and passed through the activation
    ("none", "relu", "elu", "silu", "gelu").  ``out`` may be x itself.  Rows behind the last offset keep what ``out`` holds (undefined
    where the call allocates it).  With ``with_stats`` the call returns (out, mean, rstd), each [graphs, groups], for group_norm_backward."""
    index = x.get_device()
    if index >= 0 and index != _current_device():
        return _elsewhere(x.device, stream, group_norm, x, groups, weight, bias, graph_ptr, eps, activation, f, out, out_dtype, with_stats, scratch)
    n, width = x.shape
    f = width if f is None else f
    xp, ldx = _matrix(x, f, "x")
    wp, bp, graphs, pp, itype, act = _norm_operands(x, groups, weight, bias, graph_ptr, activation, f)
    if out is None:
        out = _new(x, (n, f), out_dtype or torch.float32, stream)
    else:
        _same_device(x.device, out=out)
        _need_rows_of(out, n, "out")
        if not _same_place(x, out):
            _no_overlap(x, out, "x", "out")
    op, ldo = _matrix(out, f, "out")
    mean = rstd = None
    if with_stats:
        mean, rstd = _new(x, (2, graphs, groups), torch.float32, stream)
    if scratch is None:
        scratch = _new(x, group_norm_workspace_bytes(n, f, groups, graphs), torch.uint8, stream)
    scr, scr_n = _scratch_args(scratch, x.device)
    xdt, odt = _dtype_code(x), _dtype_code(out)
    mp, rp = (mean.data_ptr(), rstd.data_ptr()) if with_stats else (None, None)
    _check(lib().gnnfd_group_norm(n, xp, ldx, xdt, f, groups, graphs, pp, itype, wp, bp, eps, act, op, ldo, odt, mp, rp, scr, scr_n,
                                  _stream_handle(index, stream)), "gnnfd_group_norm")
    return (out, mean, rstd) if with_stats else out


def _need_rows_of(t, rows: int, name: str):
    if t.shape[0] < rows:
        raise ValueError("%s has %d rows, x has %d" % (name, t.shape[0], rows))


def group_norm_backward(dout: torch.Tensor, x: torch.Tensor, groups: int, mean: torch.Tensor, rstd: torch.Tensor,
                        weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, graph_ptr: torch.Tensor | None = None,
                        activation: str = "none", f: int | None = None, out: torch.Tensor | None = None, out_dtype=None,
                        with_params: bool = True, scratch=None, stream=None):
    """gnnfd_group_norm_backward: (dx, dweight, dbias) for the gradient ``dout`` of group_norm's result, of the type of x; dweight and dbias are
    None where ``with_params`` is false.  ``mean`` and ``rstd`` are what the forward call returned; ``out`` receives dx and may be dout itself."""
    index = x.get_device()
    if index >= 0 and index != _current_device():
        return _elsewhere(x.device, stream, group_norm_backward, dout, x, groups, mean, rstd, weight, bias, graph_ptr, activation, f, out,
                          out_dtype, with_params, scratch)
    n, width = x.shape
    f = width if f is None else f
    xp, ldx = _matrix(x, f, "x")
    wp, bp, graphs, pp, itype, act = _norm_operands(x, groups, weight, bias, graph_ptr, activation, f)
    dp, ldd = _matrix(dout, f, "dout")
    if dout.dtype != x.dtype:
        raise TypeError("dout must have the dtype of x")
    _need_rows_of(dout, n, "dout")
    _same_device(x.device, dout=dout)
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t.dtype != torch.float32 or tuple(t.shape) != (graphs, groups) or not t.is_contiguous() or t.device != x.device:
            raise ValueError("%s must be a contiguous float32 [graphs = %d, groups = %d] tensor on %s" % (name, graphs, groups, x.device))
    if out is None:
        out = _new(x, (n, f), out_dtype or torch.float32, stream)
    else:
        _same_device(x.device, out=out)
        _need_rows_of(out, n, "out")
        _no_overlap(x, out, "x", "out")
        if not _same_place(dout, out):
            _no_overlap(dout, out, "dout", "out")
    op, ldo = _matrix(out, f, "out")
    dweight = dbias = None
    if with_params:
        dweight, dbias = _new(x, (2, f), torch.float32, stream)
    if scratch is None:
        scratch = _new(x, group_norm_workspace_bytes(n, f, groups, graphs, True), torch.uint8, stream)
    scr, scr_n = _scratch_args(scratch, x.device)
    xdt, odt = _dtype_code(x), _dtype_code(out)
    dwp, dbp = (dweight.data_ptr(), dbias.data_ptr()) if with_params else (None, None)
    _check(lib().gnnfd_group_norm_backward(n, dp, ldd, xp, ldx, xdt, f, groups, graphs, pp, itype, wp, bp, mean.data_ptr(), rstd.data_ptr(), act,
                                           op, ldo, odt, dwp, dbp, scr, scr_n, _stream_handle(index, stream)), "gnnfd_group_norm_backward")
    return out, dweight, dbias


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, eps: float = 1e-5, f: int | None = None,
               out: torch.Tensor | None = None, out_dtype=None, with_stats: bool = False, stream=None):
    """gnnfd_layer_norm: every row of x by itself normalised over its columns, scaled and shifted.  ``out`` may be x itself.  With
    ``with_stats`` the call returns (out, mean, rstd), each [n], for layer_norm_backward."""
    index = x.get_device()
    if index >= 0 and index != _current_device():
        return _elsewhere(x.device, stream, layer_norm, x, weight, bias, eps, f, out, out_dtype, with_stats)
    n, width = x.shape
    f = width if f is None else f
    xp, ldx = _matrix(x, f, "x")
    wp, bp = _column_values(x, f, "weight", weight), _column_values(x, f, "bias", bias)
    if out is None:
        out = _new(x, (n, f), out_dtype or torch.float32, stream)
        op, ldo = out.data_ptr(), f
    else:
        _same_device(x.device, out=out)
        _need_rows_of(out, n, "out")
        if not _same_place(x, out):
            _no_overlap(x, out, "x", "out")
        op, ldo = _matrix(out, f, "out")
    mean = rstd = mp = rp = None
    if with_stats:
        mean, rstd = _new(x, (2, n), torch.float32, stream)
        mp, rp = mean.data_ptr(), rstd.data_ptr()
    _check(lib().gnnfd_layer_norm(n, xp, ldx, _dtype_code(x), f, wp, bp, eps, op, ldo, _dtype_code(out), mp, rp, _stream_handle(index, stream)),
           "gnnfd_layer_norm")
    return (out, mean, rstd) if with_stats else out


def _column_values(x, f: int, name: str, t):
    """Pointer of a row of f fp32 values beside x, or None."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != f or not t.is_contiguous() or t.device != x.device:
        raise ValueError("%s must be a contiguous float32 tensor of %d values on %s" % (name, f, x.device))
    return t.data_ptr()


@functools.lru_cache(maxsize=256)
def layer_norm_backward_workspace_bytes(n: int, f: int) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_layer_norm_backward_workspace_bytes(n, f, ctypes.byref(s)), "gnnfd_layer_norm_backward_workspace_bytes")
    return s.value


def layer_norm_backward(dout: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: torch.Tensor | None = None,
                        f: int | None = None, out: torch.Tensor | None = None, out_dtype=None, with_params: bool = True, scratch=None, stream=None):
    """gnnfd_layer_norm_backward: (dx, dweight, dbias) for the gradient ``dout`` of layer_norm's result, of the type of x; dweight and dbias
    are None where ``with_params`` is false.  ``mean`` and ``rstd`` are what the forward call returned; ``out`` receives dx and may be dout itself."""
    index = x.get_device()
    if index >= 0 and index != _current_device():
        return _elsewhere(x.device, stream, layer_norm_backward, dout, x, mean, rstd, weight, f, out, out_dtype, with_params, scratch)
    n, width = x.shape
    f = width if f is None else f
    xp, ldx = _matrix(x, f, "x")
    dp, ldd = _matrix(dout, f, "dout")
    if dout.dtype != x.dtype:
        raise TypeError("dout must have the dtype of x")
    _need_rows_of(dout, n, "dout")
    _same_device(x.device, dout=dout)
    wp = _column_values(x, f, "weight", weight)
    mp, rp = _column_values(x, n, "mean", mean), _column_values(x, n, "rstd", rstd)
    if out is None:
        out = _new(x, (n, f), out_dtype or torch.float32, stream)
        op, ldo = out.data_ptr(), f
    else:
        _same_device(x.device, out=out)
        _need_rows_of(out, n, "out")
        _no_overlap(x, out, "x", "out")
        if not _same_place(dout, out):
            _no_overlap(dout, out, "dout", "out")
        op, ldo = _matrix(out, f, "out")
    dweight = dbias = dwp = dbp = None
    if with_params:
        dweight, dbias = _new(x, (2, f), torch.float32, stream)
        dwp, dbp = dweight.data_ptr(), dbias.data_ptr()
        if scratch is None and n:
            scratch = _new(x, layer_norm_backward_workspace_bytes(n, f), torch.uint8, stream)
    scr, scr_n = _scratch_args(scratch, x.device)
    _check(lib().gnnfd_layer_norm_backward(n, dp, ldd, xp, ldx, _dtype_code(x), f, wp, mp, rp, op, ldo, _dtype_code(out), dwp, dbp, scr, scr_n,
                                           _stream_handle(index, stream)), "gnnfd_layer_norm_backward")
    return out, dweight, dbias


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, length: int = 0, turns=(1.0, 32.0),
                       device="cuda") -> torch.Tensor:
    """gnnfd_rotary_frequencies: float64 [rotary_dim / 2] radians per position for rotary, made once.  ``scaling`` ("none", "position", "base",
    "ramp") stretches contexts beyond ``length`` positions by ``factor``; "ramp" keeps frequencies of more than turns[1] turns over ``length``
    and divides those of fewer than turns[0]."""
    if scaling not in ROTARY_SCALINGS:
        raise ValueError("scaling must be one of %s" % ", ".join(ROTARY_SCALINGS))
    freq = torch.empty(max(0, rotary_dim) // 2, dtype=torch.float64)
    _check(lib().gnnfd_rotary_frequencies(rotary_dim, base, ROTARY_SCALINGS[scaling], factor, length, turns[0], turns[1], freq.data_ptr()),
           "gnnfd_rotary_frequencies")
    return freq.to(device)


def rotary(x: torch.Tensor, freq: torch.Tensor, heads: int, dim: int, positions: torch.Tensor | None = None, interleaved: bool = False,
           scale: float = 1.0, inverse: bool = False, out: torch.Tensor | None = None, out_dtype=None, stream=None) -> torch.Tensor:
    """gnnfd_rotary: the first 2 * len(freq) columns of each of ``heads`` heads of ``dim`` columns turned in pairs by positions[row] * freq
    (``positions`` None: the row's number), halves of the head against each other or ``interleaved`` neighbours.  ``inverse`` turns back: the
    gradient of x for that of the result.  ``out`` may be x itself; other columns than those of the heads then stay as they are."""
    index = x.get_device()
    if index >= 0 and index != _current_device():
        return _elsewhere(x.device, stream, rotary, x, freq, heads, dim, positions, interleaved, scale, inverse, out, out_dtype)
    f = heads * dim
    xp, ldx = _matrix(x, f, "x")
    n = x.shape[0]
    if freq.dtype != torch.float64 or freq.dim() != 1 or freq.device != x.device or not freq.is_contiguous():
        raise ValueError("freq must be a contiguous float64 tensor on %s" % x.device)
    if not 0 < 2 * freq.shape[0] <= dim:
        raise ValueError("%d frequencies do not fit heads of %d columns" % (freq.shape[0], dim))
    pp, itype = None, I32
    if positions is not None:
        pp, count, itype = _index_list(positions, "positions")
        if count != n or positions.device != x.device:
            raise ValueError("positions must hold a position for each of the %d rows, on %s" % (n, x.device))
    if out is None:
        out = _new(x, (n, f), out_dtype or torch.float32, stream)
        op, ldo = out.data_ptr(), f
    else:
        _same_device(x.device, out=out)
        _need_rows_of(out, n, "out")
        if not _same_place(x, out):
            _no_overlap(x, out, "x", "out")
        op, ldo = _matrix(out, f, "out")
    _check(lib().gnnfd_rotary(n, xp, ldx, _dtype_code(x), heads, dim, 2 * freq.shape[0], int(interleaved), pp, itype, freq.data_ptr(), scale,
                              int(inverse), op, ldo, _dtype_code(out), _stream_handle(index, stream)), "gnnfd_rotary")
    return out


@functools.lru_cache(maxsize=256)
def linear_recurrence_workspace_bytes(n: int, f: int, graphs: int = 1, equal_lengths: bool = False, backward: bool = False) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_linear_recurrence_workspace_bytes(n, f, graphs, int(equal_lengths), int(backward), ctypes.byref(s)),
           "gnnfd_linear_recurrence_workspace_bytes")
    return s.value


def _recurrence_operands(x, gate, form: str, graph_ptr, graphs, f: int):
    """(pointer of x, pitch, pointer of the gates, pitch, form, graphs, offsets pointer, offsets type)"""
    xp, ldx = _matrix(x, f, "x")
    gp, ldg = _matrix(gate, f, "gate")
    if gate.dtype != x.dtype:
        raise TypeError("gate must have the dtype of x")
    if gate.device != x.device:
        _same_device(x.device, gate=gate)
    n = x.shape[0]
    if gate.shape[0] < n:
        _need_rows_of(gate, n, "gate")
    if form not in GATES:
        raise ValueError("form must be one of %s" % ", ".join(GATES))
    if graph_ptr is None:
        graphs = 1 if graphs is None else graphs
        if graphs < 1 or n % graphs:
            raise ValueError("%d rows do not make %d graphs of one length" % (n, graphs))
        return xp, ldx, gp, ldg, GATES[form], graphs, None, I32
    pp, count, itype = _index_list(graph_ptr, "graph_ptr")
    if count < 2 or graph_ptr.device != x.device:
        raise ValueError("graph_ptr must hold graphs + 1 >= 2 offsets on %s" % x.device)
    if graphs is not None and graphs != count - 1:
        raise ValueError("graph_ptr holds the offsets of %d graphs, not of %d" % (count - 1, graphs))
    return xp, ldx, gp, ldg, GATES[form], count - 1, pp, itype


def _graph_states(t, x, graphs: int, f: int, name: str):
    """Pointer of fp32 states [graphs, f] beside x, or None."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != (graphs, f) or not t.is_contiguous() or t.device != x.device:
        raise ValueError("%s must be a contiguous float32 [graphs = %d, %d] tensor on %s" % (name, graphs, f, x.device))
    return t.data_ptr()


def linear_recurrence(x: torch.Tensor, gate: torch.Tensor, form: str = "sigmoid", graph_ptr: torch.Tensor | None = None, graphs: int | None = None,
                      initial: torch.Tensor | None = None, f: int | None = None, out: torch.Tensor | None = None, out_dtype=None,
                      final: torch.Tensor | None = None, with_final: bool = False, with_states: bool = False, scratch=None, stream=None):
    """gnnfd_linear_recurrence: h[t] = a[t] h[t - 1] + b[t] down the rows of each graph of a batch, per column; ``form`` "factor": a = gate,
    b = x, "sigmoid": a = 1 / (1 + exp(-gate)), b = (1 - a) x.  ``graph_ptr`` [graphs + 1] holds the graphs' row offsets; without it the rows are
    ``graphs`` (1) graphs of one length, so graphs = n is a single token for each of n sequences.  ``initial`` [graphs, f]: states ahead of the
    first rows; it does not lie in ``out`` (for single tokens it may be ``out``).  Rows behind the last offset keep what ``out`` holds (undefined where the call allocates it).  Returns out, with ``with_final`` or
    ``final`` (filled; for single tokens it may be ``initial``) also the last states, with ``with_states`` also what linear_recurrence_backward takes."""
    index = x.get_device()
    if index >= 0 and index != _current_device():
        return _elsewhere(x.device, stream, linear_recurrence, x, gate, form, graph_ptr, graphs, initial, f, out, out_dtype, final, with_final,
                          with_states, scratch)
    n, width = x.shape
    f = width if f is None else f
    xp, ldx, gp, ldg, code, graphs, pp, itype = _recurrence_operands(x, gate, form, graph_ptr, graphs, f)
    ip, fp = _graph_states(initial, x, graphs, f, "initial"), _graph_states(final, x, graphs, f, "final")
    fresh = out is None
    if fresh:
        out = _new(x, (n, f), out_dtype or torch.float32, stream)
        op, ldo = out.data_ptr(), f
    else:
        op, ldo = _matrix(out, f, "out")
        _same_device(x.device, out=out)
        _need_rows_of(out, n, "out")
        _no_overlap(x, out, "x", "out")
        _no_overlap(gate, out, "gate", "out")
        # (a single token's state is read by the thread that then writes its result to the same place)
        if initial is not None and not (graph_ptr is None and graphs == n and ip == op and out.dtype == initial.dtype and (n == 1 or ldo == f)):
            _no_overlap(initial, out, "initial", "out")
    if final is not None:
        if initial is not None and not (ip == fp and graph_ptr is None and graphs == n):
            _no_overlap(initial, final, "initial", "final")
        _no_overlap(x, final, "x", "final")
        _no_overlap(gate, final, "gate", "final")
        if not fresh:
            _no_overlap(final, out, "final", "out")
    elif with_final:
        final = _new(x, (graphs, f), torch.float32, stream)
        fp = final.data_ptr()
    states = _new(x, (-(-n // STATE_ROWS), f), torch.float32, stream) if with_states else None
    if scratch is None and n > RECURRENCE_FEW_ROWS:
        need = linear_recurrence_workspace_bytes(n, f, graphs, graph_ptr is None)
        scratch = _new(x, need, torch.uint8, stream) if need else None
    scr, scr_n = _scratch_args(scratch, x.device)
    _check(lib().gnnfd_linear_recurrence(n, xp, ldx, gp, ldg, _dtype_code(x), f, code, graphs, pp, itype, ip, op, ldo, _dtype_code(out), fp,
                                         states.data_ptr() if with_states else None, scr, scr_n, _stream_handle(index, stream)),
           "gnnfd_linear_recurrence")
    got = [out] + ([final] if final is not None else []) + ([states] if with_states else [])
    return tuple(got) if len(got) > 1 else out


def linear_recurrence_backward(dout: torch.Tensor, x: torch.Tensor, gate: torch.Tensor, states: torch.Tensor, form: str = "sigmoid",
                               graph_ptr: torch.Tensor | None = None, graphs: int | None = None, initial: torch.Tensor | None = None,
                               dfinal: torch.Tensor | None = None, f: int | None = None, out_dtype=None, scratch=None, stream=None):
    """gnnfd_linear_recurrence_backward: (dx, dgate, dinitial) for the gradients ``dout`` of linear_recurrence's result, of the type of x, and
    ``dfinal`` of its last states; dinitial is None where there was no ``initial``.  ``states`` is what the forward call with the same arguments returned."""
    index = x.get_device()
    if index >= 0 and index != _current_device():
        return _elsewhere(x.device, stream, linear_recurrence_backward, dout, x, gate, states, form, graph_ptr, graphs, initial, dfinal, f,
                          out_dtype, scratch)
    n, width = x.shape
    f = width if f is None else f
    xp, ldx, gp, ldg, code, graphs, pp, itype = _recurrence_operands(x, gate, form, graph_ptr, graphs, f)
    ip, dfp = _graph_states(initial, x, graphs, f, "initial"), _graph_states(dfinal, x, graphs, f, "dfinal")
    dp, ldd = _matrix(dout, f, "dout")
    if dout.dtype != x.dtype:
        raise TypeError("dout must have the dtype of x")
    if dout.device != x.device:
        _same_device(x.device, dout=dout)
    _need_rows_of(dout, n, "dout")
    if states.dtype != torch.float32 or states.shape != (-(-n // STATE_ROWS), f) or not states.is_contiguous() or states.device != x.device:
        raise ValueError("states must be the contiguous float32 [%d, %d] tensor of the forward call, on %s" % (-(-n // STATE_ROWS), f, x.device))
    odt = out_dtype or torch.float32
    dx, dgate = _new(x, (n, f), odt, stream), _new(x, (n, f), odt, stream)
    dinitial = _new(x, (graphs, f), torch.float32, stream) if initial is not None else None
    if scratch is None and (n > RECURRENCE_FEW_ROWS // 2 or n * f > RECURRENCE_FEW_VALUES):
        need = linear_recurrence_workspace_bytes(n, f, graphs, graph_ptr is None, True)
        scratch = _new(x, need, torch.uint8, stream) if need else None
    scr, scr_n = _scratch_args(scratch, x.device)
    _check(lib().gnnfd_linear_recurrence_backward(
        n, dp, ldd, xp, ldx, gp, ldg, _dtype_code(x), f, code, graphs, pp, itype, ip, states.data_ptr(), dfp, dx.data_ptr(), f, dgate.data_ptr(), f,
        _dtype_code(dx), None if dinitial is None else dinitial.data_ptr(), scr, scr_n, _stream_handle(index, stream)),
        "gnnfd_linear_recurrence_backward")
    return dx, dgate, dinitial


def embedding(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, f: int | None = None, out: torch.Tensor | None = None,
              out_dtype=None, status: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """gnnfd_embedding: out[i] = scale * table[ids[i], :f].  ``status`` is an int32 tensor of one element whose bit 0 the kernel sets
    where an id lies outside the table (its output row is zero)."""
    index = table.get_device()
    if index >= 0 and index != _current_device():
        return _elsewhere(table.device, stream, embedding, table, ids, scale, f, out, out_dtype, status)
    vocab, width = table.shape
    f = width if f is None else f
    ip, n, itype = _index_list(ids, "ids")
    tp, ldt = _matrix(table, f, "table")
    fresh = out is None
    if fresh:
        out = _new(table, (n, f), out_dtype or torch.float32, stream)
    op, ldo = _matrix(out, f, "out")
    if ids.get_device() != index or out.get_device() != index:
        raise ValueError("table, ids and out must be on one device")
    if not fresh:
        _need_ids(out, n, "out")
        _no_overlap(table, out, "table", "out")
        _no_overlap(ids, out, "ids", "out")
    sp = _status_ptr(status, table.device)
    tdt, odt = _dtype_code(table), _dtype_code(out)
    _check(lib().gnnfd_embedding(n, ip, itype, vocab, tp, ldt, tdt, f, scale, op, ldo, odt, sp, _stream_handle(index, stream)), "gnnfd_embedding")
    return out


def _need_ids(t, n: int, name: str):
    if t.shape[0] < n:
        raise ValueError("%s has %d rows for %d ids" % (name, t.shape[0], n))


def embedding_backward_workspace_bytes(n: int, vocab: int, f: int) -> int:
    s = ctypes.c_size_t()
    _check(lib().gnnfd_embedding_backward_workspace_bytes(n, vocab, f, ctypes.byref(s)), "gnnfd_embedding_backward_workspace_bytes")
    return s.value


def embedding_backward(ids: torch.Tensor, dout: torch.Tensor, vocab: int, scale: float = 1.0, padding_idx: int | None = None,
                       accumulate: bool = False, f: int | None = None, out: torch.Tensor | None = None, out_dtype=None, scratch=None,
                       status: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """gnnfd_embedding_backward: the gradient [vocab, f] of a table from the gradients of the rows looked up.  ``accumulate`` adds to
    ``out`` (which must then be given); ids equal to ``padding_idx`` take no part (a negative one is no row of the table: none, not one
    counted from the end); ``status``: see the header."""
    index = dout.get_device()
    if index >= 0 and index != _current_device():
        return _elsewhere(dout.device, stream, embedding_backward, ids, dout, vocab, scale, padding_idx, accumulate, f, out, out_dtype, scratch,
                          status)
    f = dout.shape[1] if f is None else f
    ip, n, itype = _index_list(ids, "ids")
    dp, ldd = _matrix(dout, f, "dout")
    _need_ids(dout, n, "dout")
    fresh = out is None
    if fresh:
        if accumulate:
            raise ValueError("accumulate needs the gradient to add to (out)")
        out = _new(dout, (vocab, f), out_dtype or torch.float32, stream)
    op, ldo = _matrix(out, f, "out")
    if ids.get_device() != index or out.get_device() != index:
        raise ValueError("ids, dout and out must be on one device")
    if not fresh:
        if out.shape[0] < vocab:
            raise ValueError("out has %d rows, the table has %d" % (out.shape[0], vocab))
        _no_overlap(dout, out, "dout", "out")
        _no_overlap(ids, out, "ids", "out")
    if scratch is None and (n > EMBEDDING_FEW_IDS or vocab > EMBEDDING_FEW_ROWS):
        scratch = _new(dout, embedding_backward_workspace_bytes(n, vocab, f), torch.uint8, stream)
    scr, scr_n = _scratch_args(scratch, dout.device)
    sp = _status_ptr(status, dout.device)
    padding = -1 if padding_idx is None else padding_idx
    ddt, odt = _dtype_code(dout), _dtype_code(out)
    _check(lib().gnnfd_embedding_backward(n, ip, itype, dp, ldd, ddt, vocab, f, scale, padding, int(accumulate), op, ldo, odt, scr, scr_n, sp,
                                          _stream_handle(index, stream)), "gnnfd_embedding_backward")
    return out


def debug_combine_fault(wait_ns: int, skip_k_block: int):
    """gnnfd_debug_combine_fault: arms the give-up drill for this thread's next transform launch."""
    _check(lib().gnnfd_debug_combine_fault(wait_ns, skip_k_block), "gnnfd_debug_combine_fault")


def debug_build_fault(max_polls: int, sweep: int):
    """gnnfd_debug_build_fault: arms the give-up drill for this thread's next build."""
    _check(lib().gnnfd_debug_build_fault(max_polls, sweep), "gnnfd_debug_build_fault")


def launch_count() -> int:
    return int(lib().gnnfd_launch_count())


def kernel_timing_enable(on: bool = True):
    _check(lib().gnnfd_kernel_timing_enable(int(on)), "gnnfd_kernel_timing_enable")


def kernel_timing_read() -> dict:
    """{kernel name: (total ms, launches)} since the last read."""
    cap = 64
    names = (ctypes.c_char_p * cap)()
    ms = (ctypes.c_double * cap)()
    cnt = (ctypes.c_int64 * cap)()
    k = lib().gnnfd_kernel_timing_read(names, ms, cnt, cap)
    if k < 0:
        raise GnnfdError(k, "gnnfd_kernel_timing_read")
    return {names[i].decode(): (ms[i], cnt[i]) for i in range(min(k, cap))}
