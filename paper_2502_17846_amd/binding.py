"""Thin ctypes binding of libgrem.so (see include/grem.h).  Argument marshalling only: torch is
used for device memory and streams, every step of the computation runs in the library's kernels.

The functions carry the library's names.  Device arrays are torch tensors on a ROCm device;
there is no CPU path: a missing library or a CPU tensor is an error."""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Union

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgrem.so")

OK, ERR_ARG, ERR_NOMEM, ERR_HIP, ERR_RANGE, ERR_SEED, ERR_LIMIT = 0, -1, -2, -3, -4, -5, -6
HIST_AUTO, HIST_LDS, HIST_GLOBAL, HIST_SWEEP = 0, 1, 2, 3
MAX_K = 4096
KERNEL_CLASSES = 11
KERNEL_SCORE = 1

EXPORTS = [
    "grem_partition", "grem_partition_seeded", "grem_partition_r32", "grem_partition_seeded_r32",
    "grem_partition_state", "grem_partition_opt", "grem_plan_create", "grem_plan_destroy",
    "grem_plan_device_bytes", "grem_plan_max_k", "grem_plan_call_bytes", "grem_partition_planned", "grem_edge_cut", "grem_edge_cut_r32", "grem_capacity",
    "grem_workspace_bytes", "grem_workspace_bytes_two_phase", "grem_set_workspace", "grem_profile_enable",
    "grem_profile_reset", "grem_profile_read", "grem_profile_read_marks", "grem_status_string", "grem_kernel_name",
    "grem_edge_stream_bipartition", "grem_edge_list_cut", "grem_edge_stream_profile_enable",
    "grem_edge_stream_profile_read", "grem_recursive_bisection", "grem_edge_buckets", "grem_expected_cut",
    "grem_expected_cut_noalloc", "grem_expected_cut_noalloc_max_n",
    "grem_neighbour_mean_bytes", "grem_neighbour_mean", "grem_neighbour_mean_backward", "grem_linear",
    "grem_linear_backward_bytes", "grem_linear_backward", "grem_layer_norm", "grem_layer_norm_backward_bytes",
    "grem_layer_norm_backward", "grem_checkpoint_pack", "grem_checkpoint_unpack",
    "grem_plan_n", "grem_plan_neighbour_counts", "grem_plan_edge_cut", "grem_plan_expected_cut",
]
EDGE_REFINE, EDGE_FIXED = 0, 1
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
CHECKPOINT_GROUP = 32        # columns that share an exponent byte


class Options(ctypes.Structure):
    """grem_options of include/grem.h: how a run is carried out, never what it computes."""
    _fields_ = [("histogram_mode", ctypes.c_int32), ("col_bits", ctypes.c_int32), ("hub_degree", ctypes.c_int32),
                ("long_row_degree", ctypes.c_int32), ("plan_max_k", ctypes.c_int32), ("reserved", ctypes.c_int32 * 3)]


def options(histogram_mode: int = 0, col_bits: int = 0, hub_degree: int = 0, long_row_degree: int = 0,
            plan_max_k: int = 0) -> Options:
    o = Options()
    o.histogram_mode, o.col_bits, o.hub_degree, o.long_row_degree = histogram_mode, col_bits, hub_degree, long_row_degree
    o.plan_max_k = plan_max_k
    return o


def _opt(o):
    return None if o is None else ctypes.byref(o)


class Rows(ctypes.Structure):
    """grem_rows of include/grem.h: rows of values, or of a checkpoint's codes and exponent bytes."""
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64), ("exponents", ctypes.c_void_p),
                ("exponent_stride", ctypes.c_int64)]


class Checkpoint(NamedTuple):
    """Rows kept in 8 bits: codes int8 (n, d), exponents uint8 (n, ceil(d / 32)), and the type they are read back as."""
    codes: torch.Tensor
    exponents: torch.Tensor
    dtype: torch.dtype


class GremError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {code} ({status_string(code)})")
        self.code = code


_lib = None


def load():
    """Loads libgrem.so; raises if it has not been built (python -m paper_2502_17846_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                           "or `python paper_2502_17846_amd/build.py`; there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
    part = [vp, vp, i64, i32, dbl, i64, i32, vp, vp]
    seeded = [vp, vp, i64, i32, dbl, i64, i32, vp, vp, vp]
    for name, args in (("grem_partition", part), ("grem_partition_r32", part),
                       ("grem_partition_seeded", seeded), ("grem_partition_seeded_r32", seeded)):
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = args
    lib.grem_partition_state.restype = ctypes.c_int
    lib.grem_partition_state.argtypes = [vp, i32, vp, i64, i32, dbl, i64, i32, vp, vp, vp, vp, vp]
    for name in ("grem_edge_cut", "grem_edge_cut_r32"):
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = [vp, vp, i64, vp, vp, vp]
    lib.grem_capacity.restype = i64
    lib.grem_capacity.argtypes = [i64, i32, dbl]
    optp = ctypes.POINTER(Options)
    lib.grem_partition_opt.restype = ctypes.c_int
    lib.grem_partition_opt.argtypes = [vp, i32, vp, i64, i32, dbl, i64, i32, vp, vp, vp, vp, optp, vp]
    lib.grem_plan_create.restype = ctypes.c_int
    lib.grem_plan_create.argtypes = [vp, i32, vp, i64, i64, optp, vp, ctypes.POINTER(vp)]
    lib.grem_plan_destroy.restype = ctypes.c_int
    lib.grem_plan_destroy.argtypes = [vp]
    lib.grem_plan_device_bytes.restype = ctypes.c_size_t
    lib.grem_plan_device_bytes.argtypes = [vp]
    lib.grem_plan_max_k.restype = ctypes.c_int32
    lib.grem_plan_max_k.argtypes = [vp]
    lib.grem_plan_call_bytes.restype = ctypes.c_size_t
    lib.grem_plan_call_bytes.argtypes = [vp, i32, i32, i32, i32]
    lib.grem_plan_n.restype = ctypes.c_int64
    lib.grem_plan_n.argtypes = [vp]
    lib.grem_plan_neighbour_counts.restype = ctypes.c_int
    lib.grem_plan_neighbour_counts.argtypes = [vp, i32, vp, vp, vp]
    lib.grem_plan_edge_cut.restype = ctypes.c_int
    lib.grem_plan_edge_cut.argtypes = [vp, i32, vp, vp, vp]
    lib.grem_plan_expected_cut.restype = ctypes.c_int
    lib.grem_plan_expected_cut.argtypes = [vp, vp, dbl, vp, vp]
    lib.grem_partition_planned.restype = ctypes.c_int
    lib.grem_partition_planned.argtypes = [vp, i32, dbl, i32, vp, vp, vp, vp, vp]
    lib.grem_workspace_bytes.restype = ctypes.c_size_t
    lib.grem_workspace_bytes.argtypes = [i64, i32, i64]
    lib.grem_workspace_bytes_two_phase.restype = ctypes.c_size_t
    lib.grem_workspace_bytes_two_phase.argtypes = [i64, i64, i32, i64, optp]
    lib.grem_set_workspace.restype = ctypes.c_int
    lib.grem_set_workspace.argtypes = [vp, ctypes.c_size_t]
    lib.grem_profile_read_marks.restype = ctypes.c_int
    lib.grem_profile_read_marks.argtypes = [ctypes.POINTER(dbl), i32]
    lib.grem_profile_enable.restype = ctypes.c_int
    lib.grem_profile_enable.argtypes = [i32]
    lib.grem_profile_reset.restype = ctypes.c_int
    lib.grem_profile_reset.argtypes = []
    lib.grem_profile_read.restype = ctypes.c_int
    lib.grem_profile_read.argtypes = [i32, ctypes.POINTER(dbl), ctypes.POINTER(i64)]
    lib.grem_status_string.restype = ctypes.c_char_p
    lib.grem_status_string.argtypes = [ctypes.c_int]
    lib.grem_kernel_name.restype = ctypes.c_char_p
    lib.grem_kernel_name.argtypes = [i32]
    lib.grem_edge_stream_bipartition.restype = ctypes.c_int
    lib.grem_edge_stream_bipartition.argtypes = [vp, vp, i64, i64, i64, i64, vp, i32, vp, vp, vp, vp]
    lib.grem_recursive_bisection.restype = ctypes.c_int
    lib.grem_recursive_bisection.argtypes = [vp, vp, i64, i64, i32, i64, dbl, vp, i32, vp, vp]
    lib.grem_edge_buckets.restype = ctypes.c_int
    lib.grem_edge_buckets.argtypes = [vp, vp, i64, i64, vp, i32, vp, vp, vp, vp]
    lib.grem_expected_cut.restype = ctypes.c_int
    lib.grem_expected_cut.argtypes = [vp, i32, vp, i64, vp, dbl, vp, vp]
    lib.grem_expected_cut_noalloc.restype = ctypes.c_int
    lib.grem_expected_cut_noalloc.argtypes = [vp, i32, vp, i64, vp, dbl, vp, vp]
    lib.grem_expected_cut_noalloc_max_n.restype = i64
    lib.grem_expected_cut_noalloc_max_n.argtypes = []
    lib.grem_edge_list_cut.restype = ctypes.c_int
    lib.grem_edge_list_cut.argtypes = [vp, vp, i64, vp, vp, vp]
    lib.grem_edge_stream_profile_enable.restype = ctypes.c_int
    lib.grem_edge_stream_profile_enable.argtypes = [i32]
    lib.grem_edge_stream_profile_read.restype = ctypes.c_int
    lib.grem_edge_stream_profile_read.argtypes = [ctypes.POINTER(dbl), ctypes.POINTER(i64), ctypes.POINTER(i64)]
    size = ctypes.c_size_t
    rows = ctypes.POINTER(Rows)
    for name, res, args in (
            ("grem_neighbour_mean_bytes", size, [i32, i64, i64, i64, i32]),
            ("grem_neighbour_mean", ctypes.c_int, [vp, i32, vp, i64, i64, vp, i32, i64, vp, i64, vp, i64, vp, vp, size, vp]),
            ("grem_neighbour_mean_backward", ctypes.c_int,
             [vp, i32, vp, i64, i64, vp, vp, i32, i64, vp, i64, vp, i64, vp, size, vp]),
            ("grem_linear", ctypes.c_int,
             [i32, i64, i64, vp, i64, i64, vp, i64, i64, vp, i64, vp, i32, vp, i64, vp, i64, vp, i64, vp]),
            ("grem_linear_backward_bytes", size, [i32, i64, i64, i64, i64, i32]),
            ("grem_linear_backward", ctypes.c_int,
             [i32, i64, i64, vp, i64, i32, vp, i64, rows, i64, rows, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, size, vp]),
            ("grem_layer_norm", ctypes.c_int, [i32, i64, i64, vp, i64, vp, vp, dbl, vp, i64, vp, vp, vp]),
            ("grem_layer_norm_backward_bytes", size, [i64, i64]),
            ("grem_layer_norm_backward", ctypes.c_int,
             [i32, i64, i64, vp, i64, rows, vp, vp, vp, vp, i64, vp, vp, vp, size, vp]),
            ("grem_checkpoint_pack", ctypes.c_int, [i32, i64, i64, vp, i64, vp, i64, vp, i64, vp]),
            ("grem_checkpoint_unpack", ctypes.c_int, [i32, i64, i64, rows, vp, i64, vp])):
        getattr(lib, name).restype = res
        getattr(lib, name).argtypes = args
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load().grem_status_string(code).decode()


def kernel_name(kernel_class: int) -> str:
    return load().grem_kernel_name(kernel_class).decode()


def _dev(t: torch.Tensor, dtype, what: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a tensor on the GPU")
    if t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{what} must be contiguous {dtype}, got {t.dtype}")
    return t.data_ptr()


_dummy_colidx = {}


def _colidx(colidx: torch.Tensor) -> int:
    """colidx pointer; an edgeless graph gets a one-element stand-in so the pointer is not null."""
    if colidx.numel() == 0:
        key = str(colidx.device)
        if key not in _dummy_colidx:
            _dummy_colidx[key] = torch.zeros(1, dtype=torch.int32, device=colidx.device)
        colidx = _dummy_colidx[key]
    return _dev(colidx, torch.int32, "colidx")


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _check(rc: int, what: str):
    if rc != OK:
        raise GremError(rc, what)


def grem_capacity(n: int, k: int, balance_slack: float) -> int:
    return int(load().grem_capacity(n, k, float(balance_slack)))


def grem_workspace_bytes(n: int, k: int, chunk: int) -> int:
    return int(load().grem_workspace_bytes(n, k, chunk))


def grem_workspace_bytes_two_phase(n: int, nnz: int, k: int, chunk: int, options: Optional[Options] = None) -> int:
    return int(load().grem_workspace_bytes_two_phase(n, nnz, k, chunk, _opt(options)))


def grem_set_workspace(buf: Optional[torch.Tensor]):
    """`buf`: a uint8 tensor on the GPU that the caller keeps alive, or None to remove it."""
    if buf is None:
        _check(load().grem_set_workspace(None, 0), "grem_set_workspace")
    else:
        _check(load().grem_set_workspace(_dev(buf, torch.uint8, "workspace"), buf.numel()),
               "grem_set_workspace")


def _rowptr_bits(rowptr: torch.Tensor) -> int:
    if rowptr.dtype == torch.int64:
        return 64
    if rowptr.dtype == torch.int32:
        return 32
    raise TypeError("rowptr must be int32 or int64")


def grem_partition_seeded(rowptr, colidx, n, k, balance_slack, chunk, refine_passes, seed_labels,
                          labels_out=None, stream=None, options: Optional[Options] = None) -> torch.Tensor:
    lib = load()
    bits = _rowptr_bits(rowptr)
    if labels_out is None:
        labels_out = torch.empty(n, dtype=torch.int32, device=colidx.device)
    if options is not None:
        rc = lib.grem_partition_opt(_dev(rowptr, rowptr.dtype, "rowptr"), bits, _colidx(colidx), n, k,
                                    float(balance_slack), chunk, refine_passes,
                                    None if seed_labels is None else _dev(seed_labels, torch.int32, "seed_labels"),
                                    _dev(labels_out, torch.int32, "labels_out"), None, None, _opt(options),
                                    _stream(stream))
        _check(rc, "grem_partition_opt")
        return labels_out
    fn = lib.grem_partition_seeded if bits == 64 else lib.grem_partition_seeded_r32
    rc = fn(_dev(rowptr, rowptr.dtype, "rowptr"), _colidx(colidx), n, k,
            float(balance_slack), chunk, refine_passes,
            None if seed_labels is None else _dev(seed_labels, torch.int32, "seed_labels"),
            _dev(labels_out, torch.int32, "labels_out"), _stream(stream))
    _check(rc, "grem_partition_seeded")
    return labels_out


def grem_partition(rowptr, colidx, n, k, balance_slack, chunk, refine_passes, labels_out=None,
                   stream=None, options: Optional[Options] = None) -> torch.Tensor:
    if options is not None:
        return grem_partition_seeded(rowptr, colidx, n, k, balance_slack, chunk, refine_passes, None, labels_out,
                                     stream, options)
    lib = load()
    bits = _rowptr_bits(rowptr)
    if labels_out is None:
        labels_out = torch.empty(n, dtype=torch.int32, device=colidx.device)
    fn = lib.grem_partition if bits == 64 else lib.grem_partition_r32
    rc = fn(_dev(rowptr, rowptr.dtype, "rowptr"), _colidx(colidx), n, k,
            float(balance_slack), chunk, refine_passes, _dev(labels_out, torch.int32, "labels_out"),
            _stream(stream))
    _check(rc, "grem_partition")
    return labels_out


def grem_partition_state(rowptr, colidx, n, k, balance_slack, chunk, refine_passes, seed_labels=None,
                         want_sizes=True, want_estimates=True, stream=None, options: Optional[Options] = None):
    """Returns (labels int32[n], sizes int64[k] or None, estimates uint32-as-int32 view [n,k] or
    None).  With `options` the call goes through grem_partition_opt."""
    lib = load()
    bits = _rowptr_bits(rowptr)
    dev = colidx.device
    labels = torch.empty(n, dtype=torch.int32, device=dev)
    sizes = torch.empty(k, dtype=torch.int64, device=dev) if want_sizes else None
    est = torch.empty((n, k), dtype=torch.int32, device=dev) if want_estimates else None
    args = [_dev(rowptr, rowptr.dtype, "rowptr"), bits, _colidx(colidx), n, k,
            float(balance_slack), chunk, refine_passes,
            None if seed_labels is None else _dev(seed_labels, torch.int32, "seed_labels"),
            _dev(labels, torch.int32, "labels_out"),
            None if sizes is None else _dev(sizes, torch.int64, "sizes_out"),
            None if est is None else _dev(est, torch.int32, "estimates_out")]
    if options is None:
        _check(lib.grem_partition_state(*args, _stream(stream)), "grem_partition_state")
    else:
        _check(lib.grem_partition_opt(*args, _opt(options), _stream(stream)), "grem_partition_opt")
    return labels, sizes, est


class Plan:
    """A grem_plan: the re-laid-out copy of one graph's entries for the two-phase route.  Keeps the
    rowptr tensor alive (the plan reads it in every run); close() (or the context manager) frees the
    plan's device memory."""

    def __init__(self, rowptr, colidx, n, chunk, options: Optional[Options] = None, stream=None):
        lib = load()
        self._rowptr = rowptr
        self.n = n
        h = ctypes.c_void_p()
        rc = lib.grem_plan_create(_dev(rowptr, rowptr.dtype, "rowptr"), _rowptr_bits(rowptr), _colidx(colidx), n,
                                  chunk, _opt(options), _stream(stream), ctypes.byref(h))
        _check(rc, "grem_plan_create")
        self._h = h

    @property
    def device_bytes(self) -> int:
        return int(load().grem_plan_device_bytes(self._h))

    @property
    def max_k(self) -> int:
        return int(load().grem_plan_max_k(self._h))

    def call_bytes(self, k: int, refine_passes: int, seeded: bool = False, with_estimates_out: bool = False) -> int:
        return int(load().grem_plan_call_bytes(self._h, k, refine_passes, int(seeded), int(with_estimates_out)))

    def close(self):
        if self._h:
            _check(load().grem_plan_destroy(self._h), "grem_plan_destroy")
            self._h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def grem_partition_planned(plan: Plan, k, balance_slack, refine_passes, seed_labels=None, labels_out=None,
                           want_sizes=False, want_estimates=False, stream=None):
    """Returns labels, or (labels, sizes, estimates) when either of the two is asked for."""
    lib = load()
    dev = plan._rowptr.device
    if labels_out is None:
        labels_out = torch.empty(plan.n, dtype=torch.int32, device=dev)
    sizes = torch.empty(k, dtype=torch.int64, device=dev) if want_sizes else None
    est = torch.empty((plan.n, k), dtype=torch.int32, device=dev) if want_estimates else None
    rc = lib.grem_partition_planned(plan._h, k, float(balance_slack), refine_passes,
                                    None if seed_labels is None else _dev(seed_labels, torch.int32, "seed_labels"),
                                    _dev(labels_out, torch.int32, "labels_out"),
                                    None if sizes is None else _dev(sizes, torch.int64, "sizes_out"),
                                    None if est is None else _dev(est, torch.int32, "estimates_out"), _stream(stream))
    _check(rc, "grem_partition_planned")
    if want_sizes or want_estimates:
        return labels_out, sizes, est
    return labels_out


def grem_plan_neighbour_counts(plan: Plan, k, labels, counts_out=None, stream=None) -> torch.Tensor:
    """Device int32 tensor (n, k): per vertex, its CSR entries by the label of their column."""
    if counts_out is None:
        counts_out = torch.empty((plan.n, k), dtype=torch.int32, device=plan._rowptr.device)
    rc = load().grem_plan_neighbour_counts(plan._h, k, _dev(labels, torch.int32, "labels"),
                                           _dev(counts_out, torch.int32, "counts_out"), _stream(stream))
    _check(rc, "grem_plan_neighbour_counts")
    return counts_out


def grem_plan_edge_cut(plan: Plan, k, labels, stream=None) -> torch.Tensor:
    """Device int64 tensor with one element: the number of cut CSR entries of the plan's graph."""
    out = torch.empty(1, dtype=torch.int64, device=plan._rowptr.device)
    rc = load().grem_plan_edge_cut(plan._h, k, _dev(labels, torch.int32, "labels"),
                                   _dev(out, torch.int64, "cut_entries_out"), _stream(stream))
    _check(rc, "grem_plan_edge_cut")
    return out


def grem_plan_expected_cut(plan: Plan, labels, x, stream=None) -> torch.Tensor:
    """Device float64 tensor [E[C](x), sum_i (k_i - k0_i)] of Eq. (1) for the plan's graph."""
    out = torch.empty(2, dtype=torch.float64, device=plan._rowptr.device)
    rc = load().grem_plan_expected_cut(plan._h, _dev(labels, torch.int32, "labels"), float(x),
                                       _dev(out, torch.float64, "out"), _stream(stream))
    _check(rc, "grem_plan_expected_cut")
    return out


def grem_edge_cut(rowptr, colidx, n, labels, stream=None) -> torch.Tensor:
    """Device int64 tensor with one element: the number of cut CSR entries."""
    lib = load()
    bits = _rowptr_bits(rowptr)
    out = torch.empty(1, dtype=torch.int64, device=colidx.device)
    fn = lib.grem_edge_cut if bits == 64 else lib.grem_edge_cut_r32
    rc = fn(_dev(rowptr, rowptr.dtype, "rowptr"), _colidx(colidx), n,
            _dev(labels, torch.int32, "labels"), _dev(out, torch.int64, "cut_entries_out"),
            _stream(stream))
    _check(rc, "grem_edge_cut")
    return out


def grem_profile_enable(level: int):
    """0: off; 1: marks at the passes' boundaries; 2: also a pair of events around every launch."""
    _check(load().grem_profile_enable(int(level)), "grem_profile_enable")


def grem_profile_read_marks(capacity: int = 64):
    """Milliseconds between consecutive marks: [before the first pass, pass 0, pass 1, ..., output expansion]."""
    buf = (ctypes.c_double * capacity)()
    cnt = load().grem_profile_read_marks(buf, capacity)
    if cnt < 0:
        raise GremError(cnt, "grem_profile_read_marks")
    return [buf[i] for i in range(cnt)]


def grem_profile_reset():
    _check(load().grem_profile_reset(), "grem_profile_reset")


def grem_profile_read(kernel_class: int):
    ms = ctypes.c_double(0.0)
    cnt = ctypes.c_int64(0)
    _check(load().grem_profile_read(kernel_class, ctypes.byref(ms), ctypes.byref(cnt)),
           "grem_profile_read")
    return ms.value, cnt.value


def grem_edge_stream_bipartition(src, dst, n, c_size, P, seed_parts, mode=EDGE_REFINE, want_sizes=True,
                                 want_nbr_counts=True, stream=None):
    """Returns (parts int32[n], sizes int64[2] or None, nbr_counts float64[n,2] or None)."""
    lib = load()
    dev = src.device
    m = src.numel()
    if dst.numel() != m:
        raise ValueError("src and dst differ in length")
    if seed_parts.numel() != n:
        raise ValueError("seed_parts must have n entries")
    parts = torch.empty(n, dtype=torch.int32, device=dev)
    sizes = torch.empty(2, dtype=torch.int64, device=dev) if want_sizes else None
    est = torch.empty((n, 2), dtype=torch.float64, device=dev) if want_nbr_counts else None
    rc = lib.grem_edge_stream_bipartition(
        _dev(src, torch.int32, "src"), _dev(dst, torch.int32, "dst"), m, n, c_size, P,
        _dev(seed_parts, torch.int32, "seed_parts"), mode, _dev(parts, torch.int32, "parts_out"),
        None if sizes is None else _dev(sizes, torch.int64, "sizes_out"),
        None if est is None else _dev(est, torch.float64, "nbr_counts_out"), _stream(stream))
    _check(rc, "grem_edge_stream_bipartition")
    return parts, sizes, est


def grem_edge_list_cut(src, dst, parts, stream=None) -> torch.Tensor:
    """Device int64 tensor with one element: the number of listed edges that are cut."""
    lib = load()
    out = torch.empty(1, dtype=torch.int64, device=src.device)
    rc = lib.grem_edge_list_cut(_dev(src, torch.int32, "src"), _dev(dst, torch.int32, "dst"), src.numel(),
                                _dev(parts, torch.int32, "parts"), _dev(out, torch.int64, "cut_out"),
                                _stream(stream))
    _check(rc, "grem_edge_list_cut")
    return out


def grem_edge_stream_profile_enable(on: bool):
    _check(load().grem_edge_stream_profile_enable(1 if on else 0), "grem_edge_stream_profile_enable")


def grem_edge_stream_profile_read():
    ms = ctypes.c_double(0.0)
    cnt = ctypes.c_int64(0)
    edges = ctypes.c_int64(0)
    _check(load().grem_edge_stream_profile_read(ctypes.byref(ms), ctypes.byref(cnt), ctypes.byref(edges)),
           "grem_edge_stream_profile_read")
    return ms.value, cnt.value, edges.value


def grem_recursive_bisection(src, dst, n, levels, chunks, balance_slack, seed_bits, mode=EDGE_REFINE, stream=None):
    """Labels int32[n] in [0, 2^levels); seed_bits: int32 tensor of levels*n entries (levels x n)."""
    lib = load()
    if seed_bits.numel() != levels * n:
        raise ValueError("seed_bits must have levels*n entries")
    labels = torch.empty(n, dtype=torch.int32, device=src.device)
    rc = lib.grem_recursive_bisection(_dev(src, torch.int32, "src"), _dev(dst, torch.int32, "dst"), src.numel(), n,
                                      levels, chunks, float(balance_slack), _dev(seed_bits, torch.int32, "seed_bits"),
                                      mode, _dev(labels, torch.int32, "labels_out"), _stream(stream))
    _check(rc, "grem_recursive_bisection")
    return labels


def grem_edge_buckets(src, dst, n, labels, k, stream=None):
    """Returns (out_src int32[m], out_dst int32[m], bucket_offsets int64[k*k+1])."""
    lib = load()
    m = src.numel()
    out_s, out_d = torch.empty_like(src), torch.empty_like(dst)
    offsets = torch.empty(k * k + 1, dtype=torch.int64, device=src.device)
    rc = lib.grem_edge_buckets(_dev(src, torch.int32, "src"), _dev(dst, torch.int32, "dst"), m, n,
                               _dev(labels, torch.int32, "labels"), k, _dev(out_s, torch.int32, "out_src"),
                               _dev(out_d, torch.int32, "out_dst"), _dev(offsets, torch.int64, "bucket_offsets"),
                               _stream(stream))
    _check(rc, "grem_edge_buckets")
    return out_s, out_d, offsets


def grem_expected_cut(rowptr, colidx, n, labels, x, stream=None) -> torch.Tensor:
    """Device float64 tensor [E[C](x), sum_i (k_i - k0_i)] of Eq. (1) for a two-way labelling."""
    lib = load()
    out = torch.empty(2, dtype=torch.float64, device=colidx.device)
    rc = lib.grem_expected_cut(_dev(rowptr, rowptr.dtype, "rowptr"), _rowptr_bits(rowptr), _colidx(colidx), n,
                               _dev(labels, torch.int32, "labels"), float(x), _dev(out, torch.float64, "out"),
                               _stream(stream))
    _check(rc, "grem_expected_cut")
    return out


def grem_expected_cut_noalloc(rowptr, colidx, n, labels, x, out, stream=None) -> torch.Tensor:
    """grem_expected_cut through the entry point that allocates nothing; `out`: the caller's float64[2]."""
    rc = load().grem_expected_cut_noalloc(_dev(rowptr, rowptr.dtype, "rowptr"), _rowptr_bits(rowptr), _colidx(colidx),
                                          n, _dev(labels, torch.int32, "labels"), float(x),
                                          _dev(out, torch.float64, "out"), _stream(stream))
    _check(rc, "grem_expected_cut_noalloc")
    return out


def grem_expected_cut_noalloc_max_n() -> int:
    return int(load().grem_expected_cut_noalloc_max_n())


# ---- layers on a partitioned graph ------------------------------------------------------------------------------
#
# Torch's automatic differentiation does not see these calls (each has a backward call of its own), so tensors that require gradients are
# refused while it records.

# the current stream's handle without a Stream object around it (2.7 us of a call's 14)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _run(fn, here: int, stream, *args):
    """The library's call, launched on GPU `here`, on `stream` or on that GPU's current one; raises where it fails."""
    if stream is not None:
        handle = stream.cuda_stream
    else:
        handle = _raw_stream(here) if _raw_stream else torch.cuda.current_stream(here).cuda_stream
    if torch._C._cuda_getDevice() == here:
        rc = fn(*args, handle)
    else:
        with torch.cuda.device(here):
            rc = fn(*args, handle)
    if rc != OK:
        raise GremError(rc, fn.__name__)


def _new(stream, like: torch.Tensor, shape, dtype=None) -> torch.Tensor:
    """What a call allocates (outputs, workspace) belongs to the stream that it runs on; the current one is the allocator's own
    choice, and switching to it would cost a small call a fifth of its time."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return like.new_empty(shape, dtype=dtype)
    return like.new_empty(shape) if dtype is None else torch.empty(shape, dtype=dtype, device=like.device)


def _into(stream, out: Optional[torch.Tensor], like: torch.Tensor, here: int, n: int, d: int, what: str):
    """`out` checked, or a new matrix of `like`'s type; with its pointer and the values between its rows."""
    if out is None:
        out = _new(stream, like, (n, d))
        return out, out.data_ptr(), d
    return (out, *_matrix(out, here, like.dtype, n, d, what))


def _space(stream, like: torch.Tensor, nbytes: int):
    """A workspace and its pointer."""
    if nbytes == 0:
        return None, None
    buf = _new(stream, like, nbytes, torch.uint8)
    return buf, buf.data_ptr()


def _home(t: torch.Tensor, stream, what: str) -> int:
    """The GPU of the call's first tensor: where the others and the stream have to be."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a tensor on the GPU")
    here = t.get_device()
    if stream is not None and stream.device_index != here:
        raise ValueError(f"the stream is one of cuda:{stream.device_index}, {what} is on cuda:{here}")
    return here


def _at(t: torch.Tensor, here: int, what: str):
    """Returns if t is on GPU `here` and no gradient of it is lost.  (Called only where one of the two is in doubt: a call has half a dozen
    tensors; with the looks at each that is 0.4 us of its 11.)"""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a tensor on the GPU")
    if t.get_device() != here:
        raise ValueError(f"{what} is on cuda:{t.get_device()}, the call's first tensor on cuda:{here}")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, and this call would not be recorded: detach it or call inside torch.no_grad(), and take "
                         "the gradient from the operator's backward call")


def _first(t: torch.Tensor, stream, what: str):
    """(GPU, type, rows, columns) of the matrix whose type is the call's."""
    here = _home(t, stream, what)
    if t.dtype not in TYPES:
        raise TypeError(f"{what} must be float32, bfloat16 or float16, got {t.dtype}")
    n, d = _sides(t, what)
    return here, TYPES[t.dtype], n, d


def _sides(t: torch.Tensor, what: str):
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{what} must be a matrix, got shape {tuple(shape)}")
    return shape


def _matrix(t: torch.Tensor, here: int, dtype, n: int, d: int, what: str):
    """(pointer, values between rows) of a matrix whose rows' values lie side by side; rows may be any distance apart."""
    if not isinstance(t, torch.Tensor) or t.requires_grad or t.get_device() != here:
        _at(t, here, what)
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if t.shape != (n, d):
        raise ValueError(f"{what} must have shape {(n, d)}, got {tuple(t.shape)}")
    if t.is_contiguous():
        return t.data_ptr(), d
    between, beside = t.stride()
    if d > 1 and n > 0 and beside != 1:
        raise ValueError(f"the values of a row of {what} must lie side by side (strides {t.stride()})")
    if n < 2:
        between = d
    elif between < d:
        raise ValueError(f"the rows of {what} overlap (strides {t.stride()})")
    return t.data_ptr(), between


def _vector(t: Optional[torch.Tensor], here: int, dtype, count: int, what: str):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.requires_grad or t.get_device() != here:
        _at(t, here, what)
    if t.shape != (count,):
        raise ValueError(f"{what} must have {count} entries, got shape {tuple(t.shape)}")
    if t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{what} must be contiguous {dtype}, got {t.dtype}")
    return t.data_ptr()


def _width(t: Union[torch.Tensor, Checkpoint], what: str) -> int:
    return _sides(t.codes if isinstance(t, Checkpoint) else t, what)[1]


def _source(t: Union[torch.Tensor, Checkpoint], here: int, dtype, n: int, d: int, what: str) -> Rows:
    """grem_rows of a matrix or of a checkpoint of that shape and type."""
    if not isinstance(t, Checkpoint):
        p, ld = _matrix(t, here, dtype, n, d, what)
        return Rows(p, ld, None, 0)
    if t.dtype != dtype:
        raise TypeError(f"{what} is a checkpoint of {t.dtype}, not of {dtype}")
    p, ld = _matrix(t.codes, here, torch.int8, n, d, what + ".codes")
    e, lde = _matrix(t.exponents, here, torch.uint8, n, -(-d // CHECKPOINT_GROUP), what + ".exponents")
    return Rows(p, ld, e, lde)


def _graph(rowptr: torch.Tensor, colidx: torch.Tensor, here: int, n: int, what: str):
    """(rowptr's pointer, its bits, colidx's pointer, its length)"""
    for t, name in ((rowptr, what), (colidx, "colidx")):
        if not isinstance(t, torch.Tensor) or t.get_device() != here:
            _at(t, here, name)
    if rowptr.numel() != n + 1:
        raise ValueError(f"{what} must have {n + 1} entries, got {rowptr.numel()}")
    return _dev(rowptr, rowptr.dtype, what), _rowptr_bits(rowptr), _colidx(colidx), colidx.numel()


def grem_neighbour_mean(rowptr, colidx, n, x, labels=None, out=None, stream=None):
    """Returns (out (n, d), counts int32[n]): the mean over every vertex's neighbours of its own partition, and how many
    they are; without labels over all neighbours."""
    here, t, _, d = _first(x, stream, "x")
    lib = load()
    px, ldx = _matrix(x, here, x.dtype, n, d, "x")
    rp, bits, ci, nnz = _graph(rowptr, colidx, here, n, "rowptr")
    out, po, ldo = _into(stream, out, x, here, n, d, "out")
    counts = _new(stream, x, n, torch.int32)
    nbytes = lib.grem_neighbour_mean_bytes(t, n, nnz, d, labels is not None)
    keep, ws = _space(stream, x, nbytes)
    _run(lib.grem_neighbour_mean, here, stream, rp, bits, ci, nnz, n, _vector(labels, here, torch.int32, n, "labels"), t, d, px, ldx, po, ldo,
         counts.data_ptr(), ws, nbytes)
    return out, counts


def grem_neighbour_mean_backward(rowptr_t, colidx_t, n, dout, counts, labels=None, dx=None, stream=None) -> torch.Tensor:
    """dx (n, d) from dout and the forward call's counts; rowptr_t, colidx_t: the transposed graph (a symmetric one is its own)."""
    here, t, _, d = _first(dout, stream, "dout")
    lib = load()
    pd, ldd = _matrix(dout, here, dout.dtype, n, d, "dout")
    rp, bits, ci, nnz = _graph(rowptr_t, colidx_t, here, n, "rowptr_t")
    dx, px, ldx = _into(stream, dx, dout, here, n, d, "dx")
    nbytes = lib.grem_neighbour_mean_bytes(t, n, nnz, d, labels is not None)
    keep, ws = _space(stream, dout, nbytes)
    _run(lib.grem_neighbour_mean_backward, here, stream, rp, bits, ci, nnz, n, _vector(labels, here, torch.int32, n, "labels"),
         _vector(counts, here, torch.int32, n, "counts"), t, d, pd, ldd, px, ldx, ws, nbytes)
    return dx


def grem_linear(a, w, bias=None, b=None, act=ACT_NONE, residual=None, out=None, want_pre=False, stream=None):
    """act([a | b] w^T + bias) + residual, (n, m); with want_pre also z = [a | b] w^T + bias, as (out, z)."""
    here, t, n, ka = _first(a, stream, "a")
    dtype, m, kb = a.dtype, _sides(w, "w")[0], 0
    pb, ldb, pr, ldr, z, pz, ldz = None, 0, None, 0, None, None, 0
    pa, lda = _matrix(a, here, dtype, n, ka, "a")
    if b is not None:
        kb = _sides(b, "b")[1]
        pb, ldb = _matrix(b, here, dtype, n, kb, "b")
    pw, ldw = _matrix(w, here, dtype, m, ka + kb, "w")
    if residual is not None:
        pr, ldr = _matrix(residual, here, dtype, n, m, "residual")
    out, po, ldo = _into(stream, out, a, here, n, m, "out")
    if want_pre:
        z, pz, ldz = _into(stream, None, a, here, n, m, "pre")
    _run(load().grem_linear, here, stream, t, n, m, pa, lda, ka, pb, ldb, kb, pw, ldw, _vector(bias, here, dtype, m, "bias"), act, pr, ldr,
         po, ldo, pz, ldz)
    return (out, z) if want_pre else out


def grem_linear_backward(dout, a, w, b=None, act=ACT_NONE, pre=None, want_inputs=True, want_params=True, stream=None):
    """Returns (da, db, dw, dbias); db is None without b, and so are the inputs' or the parameters' gradients that are not
    wanted.  a, b: the forward call's inputs, or checkpoints of them; pre: its z (not used without an activation)."""
    here, t, n, m = _first(dout, stream, "dout")
    dtype, lib = dout.dtype, load()
    _sides(w, "w")
    ka, kb = _width(a, "a"), 0 if b is None else _width(b, "b")
    pd, ldd = _matrix(dout, here, dtype, n, m, "dout")
    pw, ldw = _matrix(w, here, dtype, m, ka + kb, "w")
    ra, rb = _source(a, here, dtype, n, ka, "a"), None if b is None else _source(b, here, dtype, n, kb, "b")
    pz, ldz = None, 0
    if act != ACT_NONE:
        if pre is None:
            raise ValueError("an activation's backward pass needs pre")
        pz, ldz = _matrix(pre, here, dtype, n, m, "pre")
    da, pda, ldda = _into(stream, None, dout, here, n, ka, "da") if want_inputs else (None, None, 0)
    db, pdb, lddb = _into(stream, None, dout, here, n, kb, "db") if want_inputs and kb else (None, None, 0)
    dw, pdw, lddw = _into(stream, None, dout, here, m, ka + kb, "dw") if want_params else (None, None, 0)
    dbias = _new(stream, dout, m) if want_params else None
    nbytes = lib.grem_linear_backward_bytes(t, n, m, ka, kb, act)
    keep, ws = _space(stream, dout, nbytes)
    _run(lib.grem_linear_backward, here, stream, t, n, m, pd, ldd, act, pz, ldz, ctypes.byref(ra), ka, None if rb is None else ctypes.byref(rb),
         kb, pw, ldw, pda, ldda, pdb, lddb, pdw, lddw, None if dbias is None else dbias.data_ptr(), ws, nbytes)
    return da, db, dw, dbias


def grem_layer_norm(x, gamma=None, beta=None, eps=1e-5, out=None, stream=None):
    """Returns (y (n, d), mean float32[n], rstd float32[n])."""
    here, t, n, d = _first(x, stream, "x")
    dtype = x.dtype
    px, ldx = _matrix(x, here, dtype, n, d, "x")
    out, po, ldo = _into(stream, out, x, here, n, d, "out")
    mean, rstd = _new(stream, x, n, torch.float32), _new(stream, x, n, torch.float32)
    _run(load().grem_layer_norm, here, stream, t, n, d, px, ldx, _vector(gamma, here, dtype, d, "gamma"), _vector(beta, here, dtype, d, "beta"),
         float(eps), po, ldo, mean.data_ptr(), rstd.data_ptr())
    return out, mean, rstd


def grem_layer_norm_backward(dy, x, mean, rstd, gamma=None, dx=None, want_params=True, stream=None):
    """Returns (dx, dgamma, dbeta) (the last two None unless wanted); x: the forward call's input, or a checkpoint of it."""
    here, t, n, d = _first(dy, stream, "dy")
    dtype, lib = dy.dtype, load()
    pd, ldd = _matrix(dy, here, dtype, n, d, "dy")
    rx = _source(x, here, dtype, n, d, "x")
    dx, px, ldx = _into(stream, dx, dy, here, n, d, "dx")
    dgamma = dbeta = pg = pb = keep = ws = None
    nbytes = 0
    if want_params:
        dgamma, dbeta = _new(stream, dy, d), _new(stream, dy, d)
        pg, pb = dgamma.data_ptr(), dbeta.data_ptr()
        nbytes = lib.grem_layer_norm_backward_bytes(n, d)
        keep, ws = _space(stream, dy, nbytes)
    _run(lib.grem_layer_norm_backward, here, stream, t, n, d, pd, ldd, ctypes.byref(rx), _vector(mean, here, torch.float32, n, "mean"),
         _vector(rstd, here, torch.float32, n, "rstd"), _vector(gamma, here, dtype, d, "gamma"), px, ldx, pg, pb, ws, nbytes)
    return dx, dgamma, dbeta


def grem_checkpoint_pack(x, stream=None) -> Checkpoint:
    """x's rows in 8 bits: groups of 32 columns, int8 codes and one exponent byte each."""
    here, t, n, d = _first(x, stream, "x")
    px, ldx = _matrix(x, here, x.dtype, n, d, "x")
    groups = -(-d // CHECKPOINT_GROUP)
    codes, exponents = _new(stream, x, (n, d), torch.int8), _new(stream, x, (n, groups), torch.uint8)
    _run(load().grem_checkpoint_pack, here, stream, t, n, d, px, ldx, codes.data_ptr(), d, exponents.data_ptr(), groups)
    return Checkpoint(codes, exponents, x.dtype)


def grem_checkpoint_unpack(checkpoint: Checkpoint, out=None, stream=None) -> torch.Tensor:
    """The values that a checkpoint's codes stand for, in its type."""
    codes, exponents, dtype = checkpoint
    here = _home(codes, stream, "checkpoint.codes")
    n, d = _sides(codes, "checkpoint.codes")
    if dtype not in TYPES:
        raise TypeError(f"a checkpoint is read back as float32, bfloat16 or float16, not {dtype}")
    rx = _source(checkpoint, here, dtype, n, d, "checkpoint")
    if out is None:
        out = _new(stream, codes, (n, d), dtype)
        po, ldo = out.data_ptr(), d
    else:
        po, ldo = _matrix(out, here, dtype, n, d, "out")
    _run(load().grem_checkpoint_unpack, here, stream, TYPES[dtype], n, d, ctypes.byref(rx), po, ldo)
    return out
