"""ctypes binding of libsagnn.so: same names as the C ABI, argument marshalling only."""
from __future__ import annotations

import ctypes
import functools
import importlib
import os
import types
from dataclasses import dataclass

import numpy as np
import torch

from . import build as _build

ACT_IDENTITY, ACT_RELU, ACT_SILU = 0, 1, 2
F32, BF16, E4M3 = 0, 1, 2
GEMM_FP32, GEMM_BF16, GEMM_FP32_BF16X3 = 0, 1, 2
PLAN_VALIDATE, PLAN_OBLIVIOUS, PLAN_MULTIPASS = 1, 2, 4

EXPORTS = [
    "sagnn_strerror", "sagnn_last_hip_error", "sagnn_version",
    "spmm_plan_workspace_bytes", "spmm_plan_needed_rows", "spmm_plan_needed_rows_noalloc", "spmm_pack_rows",
    "spmm_csr_workspace_bytes", "spmm_csr_workspace_bytes_opt", "spmm_csr_tile_info", "spmm_csr_prepare", "spmm_csr_prepare_opt", "spmm_csr_prepare_tuned", "spmm_csr_schedule_info", "spmm_csr_launch_info",
    "spmm_csr_release", "spmm_csr_tallskinny",
    "dense_gemm_act", "gcn_layer_fwd", "gcn_layer_fwd_fused", "gcn_layer_fwd_form", "gcn_bwd_workspace_bytes", "gcn_layer_bwd",
    "spmm_split_workspace_bytes", "spmm_split_colblocks", "spmm_stage_loop", "spmm_volume_stats",
    "spmm_transpose_workspace_bytes", "spmm_csr_transpose",
    "spmm_permute_workspace_bytes", "spmm_perm_from_labels", "spmm_csr_permute_symmetric",
    "grouped_gemm_act", "grouped_gemm_bwd_workspace_bytes", "grouped_gemm_bwd",
    "group_norm_workspace_bytes", "group_norm_act_fwd", "group_norm_act_bwd",
    "grad_norm_workspace_bytes", "grad_global_norm", "grad_clip_norm", "grad_scale_to_norm",
    "dropout_add", "rms_norm_fwd", "rms_norm_bwd_workspace_bytes", "rms_norm_bwd", "spmm_pack_rows_e4m3",
    "softmax_xent_workspace_bytes", "softmax_xent_bwd_workspace_bytes", "softmax_xent_fwd", "softmax_xent_bwd",
]


class _Stage(ctypes.Structure):
    """struct sagnn_stage of the C header."""
    _fields_ = [("d_rowptr", ctypes.c_void_p), ("d_colidx", ctypes.c_void_p),
                ("d_val", ctypes.c_void_p), ("nnz", ctypes.c_int64), ("d_rows", ctypes.c_void_p),
                ("N", ctypes.c_int64), ("d_ws", ctypes.c_void_p), ("ws_bytes", ctypes.c_size_t)]


class SpmmOptions(ctypes.Structure):
    """struct sagnn_spmm_options of the C header (zero = let the library decide)."""
    _fields_ = [(n, ctypes.c_int32) for n in
                ("schedule", "min_long", "piece", "slab_kb", "min_waves", "window_pct", "snake", "groups",
                 "sync_slabs", "pace_ps_per_step", "barriers", "sync_timeout_us", "sync_test_extra",
                 "narrow_slots", "slab_width", "short_rows", "dense_tiles", "tile_reuse_x10")]


# The library itself reads no environment variables.  For experiments and for tests that force a
# code path on small inputs, the binding translates these variables into the options struct:
#   SAGNN_SWEEP=0|1 (never / whenever possible), SAGNN_SWEEP_MINDEG, SAGNN_SWEEP_PIECE,
#   SAGNN_SWEEP_SLAB_MB (0 = as many slabs as possible), SAGNN_SWEEP_MIN_WAVES,
#   SAGNN_SWEEP_WINDOW_PCT (0 = one window), SAGNN_SWEEP_LPT=0 (snake dealing),
#   SAGNN_SWEEP_GROUPS=1|2, SAGNN_SWEEP_SYNC (slabs per interval, 0 = one interval),
#   SAGNN_SWEEP_PACE_PS (picoseconds per stream step, -1 = never pace), SAGNN_SWEEP_BARRIERS=1,
#   SAGNN_SWEEP_SYNC_US, SAGNN_SWEEP_SYNC_TEST_EXTRA, SAGNN_SWEEP_NARROW_SLOTS=1, SAGNN_SWEEP_SLAB_WIDTH=128,
#   SAGNN_SWEEP_SHORT_ROWS=1 (short rows swept as whole rows),
#   SAGNN_TILES=1|-1 (dense tiles out of LDS: always / never), SAGNN_TILE_REUSE_X10
def options_from_env() -> SpmmOptions:
    o = SpmmOptions()
    env = os.environ.get

    def num(name):
        v = env(name)
        return None if v is None or v == "" else int(v)

    v = num("SAGNN_SWEEP")
    if v is not None:
        o.schedule = 1 if v == 0 else (2 if v == 1 else 0)
    for name, field in (("SAGNN_SWEEP_MINDEG", "min_long"), ("SAGNN_SWEEP_PIECE", "piece"),
                        ("SAGNN_SWEEP_MIN_WAVES", "min_waves"), ("SAGNN_SWEEP_GROUPS", "groups"),
                        ("SAGNN_SWEEP_SYNC_US", "sync_timeout_us"), ("SAGNN_SWEEP_PACE_PS", "pace_ps_per_step"),
                        ("SAGNN_SWEEP_BARRIERS", "barriers"), ("SAGNN_SWEEP_NARROW_SLOTS", "narrow_slots"),
                        ("SAGNN_SWEEP_SYNC_TEST_EXTRA", "sync_test_extra"), ("SAGNN_SWEEP_SLAB_WIDTH", "slab_width"),
                        ("SAGNN_SWEEP_SHORT_ROWS", "short_rows"), ("SAGNN_TILES", "dense_tiles"),
                        ("SAGNN_TILE_REUSE_X10", "tile_reuse_x10")):
        v = num(name)
        if v is not None:
            setattr(o, field, v)
    v = num("SAGNN_SWEEP_SLAB_MB")
    if v is not None:
        o.slab_kb = -1 if v <= 0 else v * 1024
    v = num("SAGNN_SWEEP_WINDOW_PCT")
    if v is not None:
        o.window_pct = -1 if v <= 0 else v
    v = num("SAGNN_SWEEP_LPT")
    if v is not None:
        o.snake = 1 if v == 0 else 0
    v = num("SAGNN_SWEEP_SYNC")
    if v is not None:
        o.sync_slabs = -1 if v <= 0 else v
    return o


class SagnnError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().sagnn_strerror(code).decode()
        extra = f" (hipError {lib().sagnn_last_hip_error()})" if code == -4 else ""
        super().__init__(f"{where}: {msg}{extra} [{code}]")


_lib = None


def lib_path() -> str:
    return _build.LIB


def lib():
    """Load libsagnn.so (building it first only if it does not exist)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.LIB):
            _build.build_all()
        L = ctypes.CDLL(_build.LIB)
        i64, i32, u32, vp, sz = (ctypes.c_int64, ctypes.c_int32, ctypes.c_uint32, ctypes.c_void_p,
                                 ctypes.c_size_t)
        psz = ctypes.POINTER(ctypes.c_size_t)
        L.sagnn_strerror.restype = ctypes.c_char_p
        L.sagnn_strerror.argtypes = [ctypes.c_int]
        L.sagnn_last_hip_error.restype = ctypes.c_int
        L.sagnn_version.restype = ctypes.c_int
        L.spmm_plan_workspace_bytes.argtypes = [i64, i64, i64, i32, psz]
        L.spmm_plan_needed_rows.argtypes = [vp, vp, i64, i64, i64, vp, i32, vp, i64, vp, vp, vp, sz,
                                            u32, vp]
        L.spmm_plan_needed_rows_noalloc.argtypes = [vp, vp, i64, i64, i64, vp, i32, vp, i64, vp, vp, u32, vp]
        L.spmm_pack_rows.argtypes = [vp, i64, i64, i32, vp, i64, vp, i64, vp]
        L.spmm_csr_workspace_bytes.argtypes = [i64, i64, i32, psz]
        L.spmm_csr_workspace_bytes_opt.argtypes = [i64, i64, i64, i32, vp, psz]
        L.spmm_csr_tile_info.argtypes = [vp, vp]
        L.spmm_csr_prepare.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp, sz, vp]
        L.spmm_csr_prepare_opt.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp, sz, vp, vp]
        L.spmm_csr_prepare_tuned.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp, sz, vp, i64, vp, i64, vp, vp, vp]
        L.spmm_csr_schedule_info.argtypes = [vp, vp]
        L.spmm_csr_launch_info.argtypes = [vp, vp]
        L.spmm_csr_release.argtypes = [vp]
        L.spmm_csr_tallskinny.argtypes = [vp, vp, vp, i64, i64, i64, vp, i64, i32, vp, i64, i32, vp,
                                          sz, vp]
        L.dense_gemm_act.argtypes = [vp, i64, vp, i64, i32, i64, i32, i32, i32, i32, vp, i64, vp, i64,
                                     vp, i64, vp]
        L.gcn_layer_fwd.argtypes = [vp, vp, vp, i64, i64, i64, vp, i64, i32, vp, i32, i32, i32, vp,
                                    vp, vp, vp, sz, vp]
        L.gcn_layer_fwd_fused.argtypes = [vp, vp, vp, i64, i64, i64, vp, i64, i32, vp, i32, i32, i32, vp,
                                          vp, vp, vp]
        L.gcn_layer_fwd_form.argtypes = [vp, i32, i32, i32, ctypes.POINTER(ctypes.c_int32)]
        L.gcn_bwd_workspace_bytes.argtypes = [i64, i32, i32, psz]
        L.gcn_layer_bwd.argtypes = [vp, vp, vp, i64, i64, vp, i32, vp, i32, vp, vp, i32, vp, vp, vp,
                                    vp, sz, vp, sz, vp]
        L.spmm_split_workspace_bytes.argtypes = [i64, i32, psz]
        L.spmm_split_colblocks.argtypes = [vp, vp, vp, i64, i64, vp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.spmm_stage_loop.argtypes = [vp, i32, i64, vp, i64, i64, i32, vp, vp, i64, vp, i64, i32, vp,
                                      vp]
        L.spmm_volume_stats.argtypes = [vp, i32, i32, i32, vp]
        L.spmm_transpose_workspace_bytes.argtypes = [i64, psz]
        L.spmm_csr_transpose.argtypes = [vp, vp, vp, i64, i64, i64, vp, vp, vp, vp, sz, vp]
        L.spmm_permute_workspace_bytes.argtypes = [i64, i64, psz]
        L.spmm_perm_from_labels.argtypes = [vp, i64, i32, vp, vp, vp, vp, sz, vp]
        L.spmm_csr_permute_symmetric.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp, vp, vp, sz, vp]
        f64 = ctypes.c_double
        L.grouped_gemm_act.argtypes = [i32, vp, i64, vp, i64, i64, i32, vp, i32, i64, i32, i32, i32, i32, vp, i64, vp, i64, vp]
        L.grouped_gemm_bwd_workspace_bytes.argtypes = [i64, i32, i32, i32, psz]
        L.grouped_gemm_bwd.argtypes = [i32, vp, i64, vp, i64, i64, vp, i32, i64, i32, i32, i32, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]
        L.group_norm_workspace_bytes.argtypes = [i32, i64, i32, i64, i32, i32, i64, i32, psz]
        L.group_norm_act_fwd.argtypes = [i32, vp, i64, vp, i32, i64, i64, i32, i32, vp, vp, f64, i32, vp, i64, vp, vp, vp, sz, vp]
        L.group_norm_act_bwd.argtypes = [i32, vp, i64, vp, i64, vp, i32, i64, i64, i32, i32, vp, vp, i32, vp, vp, vp, i64, vp, vp, vp,
                                         sz, vp]
        L.grad_norm_workspace_bytes.argtypes = [i32, psz]
        L.grad_global_norm.argtypes = [vp, i32, vp, vp, sz, vp]
        L.grad_clip_norm.argtypes = [vp, i32, f64, vp, vp, sz, vp]
        L.grad_scale_to_norm.argtypes = [vp, i32, f64, vp, vp]
        u64 = ctypes.c_uint64
        L.dropout_add.argtypes = [i32, vp, i64, vp, i64, i64, i32, i32, u64, u64, vp, i64, vp, i64, vp]
        L.rms_norm_fwd.argtypes = [i32, vp, i64, vp, i64, i64, i32, vp, f64, i32, u64, u64, vp, i64, i32, vp, i64, vp, vp, i64, vp, vp]
        L.rms_norm_bwd_workspace_bytes.argtypes = [i64, i32, psz]
        L.rms_norm_bwd.argtypes = [i32, vp, i64, vp, i64, vp, i64, i64, i32, vp, vp, i32, u64, u64, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]
        L.spmm_pack_rows_e4m3.argtypes = [vp, i64, vp, i64, i32, vp, i64, i32, vp, i64, vp]
        L.softmax_xent_workspace_bytes.argtypes = [i32, i64, i32, i32, i32, i32, psz]
        L.softmax_xent_bwd_workspace_bytes.argtypes = [i32, i64, i32, i32, i32, i32, psz]
        L.softmax_xent_fwd.argtypes = [i32, vp, i64, vp, i64, i32, vp, vp, i64, i32, i32, i32, vp, vp, vp, sz, vp]
        L.softmax_xent_bwd.argtypes = [i32, vp, i64, vp, i64, i32, vp, vp, vp, vp, f64, i64, i32, i32, i32, vp, i64, vp, vp, vp, sz, vp]
        for name in EXPORTS[3:]:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


class ArgumentError(ctypes.ArgumentError, TypeError):
    """An argument of a call that is none, as ctypes refuses it."""


_bound = None
# the calls of a step: integers and pointers, and one double at most
STEP_CALLS = ("spmm_plan_needed_rows", "spmm_pack_rows", "spmm_csr_tallskinny", "dense_gemm_act", "gcn_layer_fwd", "gcn_layer_bwd",
              "grouped_gemm_act", "grouped_gemm_bwd", "group_norm_act_fwd", "group_norm_act_bwd", "grad_global_norm", "grad_clip_norm",
              "grad_scale_to_norm", "dropout_add", "rms_norm_fwd", "rms_norm_bwd", "spmm_pack_rows_e4m3",
              "softmax_xent_fwd", "softmax_xent_bwd")
_KIND = {ctypes.c_void_p: "p", ctypes.c_double: "d"}


def _extension(name="_marshal", path=None):
    """csrc/marshal.c (or another) as built for this interpreter; None where it is not."""
    try:
        return importlib.import_module(f"{__package__}.{name}") if os.path.exists(path or _build.MARSHAL) else None
    except ImportError:
        return None


def _by_ctypes(function):
    """A declared function that takes host arrays for pointers, as the bound ones do."""
    return lambda *args: function(*[_host(a) if isinstance(a, np.ndarray) and a.ndim else a for a in args])


def _calls():
    """The calls of a step, with the parameters that lib() declares: by address (csrc/marshal.c), or through ctypes."""
    global _bound
    if _bound is None:
        L, ext = lib(), _extension()
        _bound = types.SimpleNamespace(**{
            name: ext.bind(ctypes.cast(getattr(L, name), ctypes.c_void_p).value,
                           "".join(_KIND.get(t, "i") for t in getattr(L, name).argtypes), ArgumentError)
            if ext else _by_ctypes(getattr(L, name)) for name in STEP_CALLS})
    return _bound


def _check(rc: int, where: str):
    if rc != 0:
        raise SagnnError(rc, where)


# Marshalling is on the path of every call and a launch is only a few microseconds: pointers travel as plain
# integers (the argument types convert them), the stream comes from the runtime without a Stream object.
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _host(a: np.ndarray) -> int:
    """Address of a host array."""
    return a.__array_interface__["data"][0]


def _dev(t: torch.Tensor, dtype, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA/HIP tensor (there is no CPU path)")
    if t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype}")
    return t


def _mat(t: torch.Tensor, name: str):
    """A row-major fp32 matrix, possibly a column slice of a wider one: unit stride along a row,
    the row stride is passed to the library as the leading dimension."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA/HIP tensor (there is no CPU path)")
    if t.dtype is not torch.float32 or t.dim() != 2:
        raise ValueError(f"{name}: expected a 2-D float32 tensor")
    if not t.is_contiguous() and not _rows_apart(t):
        raise ValueError(f"{name}: rows must be contiguous (unit stride inside a row) and must not overlap")
    return t


def _rows_apart(t: torch.Tensor) -> bool:
    """Whether a matrix (with elements) lies row by row.  A row's own stride is asked for however many rows there are, a
    single one too; what lies between rows only where there are two."""
    n, f = t.shape
    return (f == 1 or t.stride(1) == 1) and (n == 1 or t.stride(0) >= f)


def _ld(t: torch.Tensor) -> int:
    n, f = t.shape
    ld = t.stride(0)
    return ld if n > 1 or ld > f else f


def _ws(nbytes: int, device) -> torch.Tensor:
    # torch's caching allocator returns 512-byte aligned blocks
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


@dataclass
class Plan:
    needed: torch.Tensor          # int32 [N], ascending global column ids
    blk_off: np.ndarray           # int64 [nb+1] (host)
    colidx_compact: torch.Tensor  # int32 [nnz] or None

    @property
    def N(self) -> int:
        return int(self.blk_off[-1])


def _plan_flags(validate, oblivious, multipass):
    if multipass is None:
        multipass = os.environ.get("SAGNN_PLAN_MULTIPASS", "0") not in ("", "0")
    return ((PLAN_VALIDATE if validate else 0) | (PLAN_OBLIVIOUS if oblivious else 0) |
            (PLAN_MULTIPASS if multipass else 0))


def spmm_plan_needed_rows(rowptr, colidx, n: int, colblk, want_compact=True, validate=False,
                          needed_cap=None, bufs=None, oblivious=False, multipass=None) -> Plan:
    """NnzCols of every column block (Sec. 4.1).  Outputs are torch tensors; `needed` is sized
    min(n, nnz) unless needed_cap is given.  `bufs` = (ws, needed, compact) reuses buffers of an
    earlier call (see plan_buffers) so that a repeated call allocates nothing.  `multipass=True`
    (default: the environment variable SAGNN_PLAN_MULTIPASS) keeps small blocks off the one-launch
    path."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    m, nnz = rowptr.numel() - 1, colidx.numel()
    colblk = np.ascontiguousarray(colblk, dtype=np.int64)
    nb = colblk.size - 1
    cap = int((n if oblivious else min(n, nnz)) if needed_cap is None else needed_cap)
    if bufs is None:
        bufs = plan_buffers(m, n, nnz, nb, rowptr.device, cap, want_compact)
    ws, needed, compact = bufs
    blk_off = np.zeros(nb + 1, dtype=np.int64)
    rc = _calls().spmm_plan_needed_rows(_ptr(rowptr), _ptr(colidx), m, n, nnz, colblk, nb, _ptr(needed), cap,
                                        blk_off, _ptr(compact), _ptr(ws), ws.numel(),
                                        _plan_flags(validate, oblivious, multipass), _stream())
    _check(rc, "spmm_plan_needed_rows")
    N = int(blk_off[-1])
    if compact is not None and compact.numel() != nnz:
        compact = compact[:nnz]
    return Plan(needed if N == needed.numel() else needed[:N], blk_off, compact)


def spmm_plan_needed_rows_noalloc(rowptr, colidx, n: int, colblk, needed, compact=None, validate=False,
                                  oblivious=False, multipass=None) -> Plan:
    """spmm_plan_needed_rows without a workspace: the library's fixed per-GPU scratch array is
    used and nothing is allocated, here or in the library.  `needed` (int32, capacity = its
    length) and `compact` (int32, nnz entries, or None) are the caller's output buffers."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    needed = _dev(needed, torch.int32, "needed")
    if compact is not None:
        compact = _dev(compact, torch.int32, "compact")
    m, nnz = rowptr.numel() - 1, colidx.numel()
    colblk = np.ascontiguousarray(colblk, dtype=np.int64)
    nb = colblk.size - 1
    blk_off = np.zeros(nb + 1, dtype=np.int64)
    rc = lib().spmm_plan_needed_rows_noalloc(
        _ptr(rowptr), _ptr(colidx), m, n, nnz, _host(colblk), nb, _ptr(needed),
        needed.numel(), _host(blk_off), _ptr(compact),
        _plan_flags(validate, oblivious, multipass), _stream())
    _check(rc, "spmm_plan_needed_rows_noalloc")
    N = int(blk_off[-1])
    return Plan(needed[:N], blk_off, compact[:nnz] if compact is not None else None)


def plan_buffers(m, n, nnz, nb, device, cap=None, want_compact=True):
    """Workspace and output buffers of spmm_plan_needed_rows."""
    wsb = ctypes.c_size_t(0)
    _check(lib().spmm_plan_workspace_bytes(m, n, nnz, nb, ctypes.byref(wsb)), "spmm_plan_workspace_bytes")
    cap = int(min(n, nnz) if cap is None else cap)
    ws = _ws(wsb.value, device)
    needed = torch.empty(max(cap, 1), dtype=torch.int32, device=device)
    compact = torch.empty(max(nnz, 1), dtype=torch.int32, device=device) if want_compact else None
    return ws, needed, compact


def spmm_pack_rows(H, rows, out=None):
    """out[r,:] = H[rows[r],:] (Alg. 1, packed buffer)."""
    H = _mat(H, "H")
    rows = _dev(rows, torch.int32, "rows")
    n, f = H.shape
    N = rows.numel()
    if out is None:
        out = torch.empty((N, f), dtype=torch.float32, device=H.device)
    _mat(out, "out")
    _check(_calls().spmm_pack_rows(_ptr(H), n, _ld(H), f, _ptr(rows), N, _ptr(out), _ld(out),
                                _stream()), "spmm_pack_rows")
    return out


@dataclass
class SpmmWorkspace:
    buf: torch.Tensor
    m: int
    nnz: int
    f: int
    choice: dict = None           # filled in by spmm_csr_prepare_tuned
    k: int = 0                    # rows of B the schedule was prepared for

    def release(self):
        """Drop the library's host descriptor of this workspace (spmm_csr_release)."""
        if self.buf is not None:
            lib().spmm_csr_release(_ptr(self.buf))
            self.buf = None

    def __del__(self):
        try:
            self.release()
        except Exception:
            pass

    def info(self) -> dict:
        """Schedule chosen by spmm_csr_prepare (see spmm_csr_schedule_info)."""
        a = np.zeros(16, dtype=np.int64)
        _check(lib().spmm_csr_schedule_info(_ptr(self.buf), _host(a)),
               "spmm_csr_schedule_info")
        keys = ("mode", "sweep_waves", "sweep_entries", "chunk_rows", "chunk_entries", "chunks",
                "split_rows", "has_empty_rows", "intervals", "sync_slabs", "gave_up_offset", "groups",
                "pace_ps_per_step", "barriers", "slots", "longest_stream_steps")
        return dict(zip(keys, (int(x) for x in a)))

    def launch_info(self) -> dict:
        """How the product and the layer are launched (see spmm_csr_launch_info)."""
        a = np.zeros(4, dtype=np.int64)
        _check(lib().spmm_csr_launch_info(_ptr(self.buf), _host(a)), "spmm_csr_launch_info")
        return dict(zip(("columns", "waves", "layer_waves", "slabs"), (int(x) for x in a)))

    def tile_info(self) -> dict:
        """What a preparation with dense tiles decided (see spmm_csr_tile_info)."""
        a = np.zeros(6, dtype=np.int64)
        _check(lib().spmm_csr_tile_info(_ptr(self.buf), _host(a)), "spmm_csr_tile_info")
        keys = ("tiles", "tile_entries", "kept_tiles", "items", "ranked_rows", "rest_entries")
        return dict(zip(keys, (int(x) for x in a)))

    def barriers_gave_up(self) -> bool:
        """True if a barrier wait of the most recent product hit its time limit (synchronises)."""
        off = self.info()["gave_up_offset"]
        return bool(self.buf[off:off + 4].view(torch.int32).item() != 0)


def spmm_csr_prepare(rowptr, colidx, val, k: int, f: int, options: SpmmOptions = None) -> SpmmWorkspace:
    """One-time schedule for C = A*B with A = (rowptr, colidx, val), B of k rows and width f.
    `options` defaults to options_from_env() (all zero unless SAGNN_SWEEP* variables are set)."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    val = _dev(val, torch.float32, "val")
    m, nnz = rowptr.numel() - 1, colidx.numel()
    L = lib()
    wsb = ctypes.c_size_t(0)
    opt = options if options is not None else options_from_env()
    _check(L.spmm_csr_workspace_bytes_opt(m, k, nnz, f, ctypes.byref(opt), ctypes.byref(wsb)),
           "spmm_csr_workspace_bytes_opt")
    buf = _ws(wsb.value, rowptr.device)
    _check(L.spmm_csr_prepare_opt(_ptr(rowptr), _ptr(colidx), _ptr(val), m, k, nnz, f, _ptr(buf),
                                  buf.numel(), ctypes.byref(opt), _stream()), "spmm_csr_prepare_opt")
    return SpmmWorkspace(buf, m, nnz, f, None, int(k))


def spmm_csr_prepare_tuned(rowptr, colidx, val, B, C=None, options: SpmmOptions = None) -> SpmmWorkspace:
    """spmm_csr_prepare with a measured choice between a few plan variants, timed on B (k x f).
    C (m x f) is overwritten with the product; allocated here when not given."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    val = _dev(val, torch.float32, "val")
    B = _dev(B, torch.float32, "B")
    m, nnz = rowptr.numel() - 1, colidx.numel()
    k, f = B.shape
    if C is None:
        C = torch.empty((m, f), dtype=torch.float32, device=B.device)
    _dev(C, torch.float32, "C")
    L = lib()
    wsb = ctypes.c_size_t(0)
    opt = options if options is not None else options_from_env()
    _check(L.spmm_csr_workspace_bytes_opt(m, k, nnz, f, ctypes.byref(opt), ctypes.byref(wsb)),
           "spmm_csr_workspace_bytes_opt")
    buf = _ws(wsb.value, rowptr.device)
    choice = np.zeros(4, dtype=np.int32)
    _check(L.spmm_csr_prepare_tuned(_ptr(rowptr), _ptr(colidx), _ptr(val), m, k, nnz, f, _ptr(buf),
                                    buf.numel(), _ptr(B), B.stride(0), _ptr(C), C.stride(0),
                                    _host(choice), ctypes.byref(opt), _stream()),
           "spmm_csr_prepare_tuned")
    return SpmmWorkspace(buf, m, nnz, f, {"piece": int(choice[0]), "min_long": int(choice[1]),
                                         "best_us": int(choice[2]), "variant": int(choice[3])}, int(k))


def spmm_csr_tallskinny(rowptr, colidx, val, B, C=None, accumulate=False, ws: SpmmWorkspace = None):
    """C (+)= A * B (Alg. 1/2 local SpMM)."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    val = _dev(val, torch.float32, "val")
    B = _mat(B, "B")
    m, nnz = rowptr.numel() - 1, colidx.numel()
    k, f = B.shape
    if C is None:
        if accumulate:
            raise ValueError("accumulate needs C")
        C = torch.empty((m, f), dtype=torch.float32, device=B.device)
    _mat(C, "C")
    if ws is not None and (ws.m != m or ws.nnz != nnz or ws.f < f or k < ws.k):
        raise ValueError("workspace was prepared for another matrix or a taller operand")
    rc = _calls().spmm_csr_tallskinny(_ptr(rowptr), _ptr(colidx), _ptr(val), m, k, nnz, _ptr(B),
                                   _ld(B), f, _ptr(C), _ld(C), int(accumulate),
                                   _ptr(ws.buf) if ws else None, ws.buf.numel() if ws else 0,
                                   _stream())
    _check(rc, "spmm_csr_tallskinny")
    return C


def dense_gemm_act(X, W, transW=False, prec=GEMM_FP32, act=ACT_IDENTITY, mask=None, want_z=True,
                   want_act=False, out=None):
    X = _mat(X, "X")
    W = _mat(W, "W")
    m, kdim = X.shape
    nout = W.shape[0] if transW else W.shape[1]
    if out is not None:
        Z, A = out
    else:
        Z = torch.empty((m, nout), dtype=torch.float32, device=X.device) if want_z else None
        A = torch.empty((m, nout), dtype=torch.float32, device=X.device) if want_act else None
    rc = _calls().dense_gemm_act(_ptr(X), _ld(X), _ptr(W), _ld(W), int(transW), m, kdim, nout,
                              prec, act, _ptr(mask), _ld(mask) if mask is not None else 0,
                              _ptr(Z), nout, _ptr(A), nout, _stream())
    _check(rc, "dense_gemm_act")
    return Z, A


def gcn_layer_fwd(rowptr, colidx, val, H, W, act=ACT_RELU, prec=GEMM_FP32, ws: SpmmWorkspace = None,
                  want_z=True, want_h=True, out=None, want_t=True, fused=False):
    """T = A H, Z = T W, Hout = sigma(Z).  Returns (T, Z, Hout).  want_t=False: T is not stored
    (returned as None) and the layer runs as one fused kernel; fused=True calls that kernel
    directly and still returns T."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    val = _dev(val, torch.float32, "val")
    H = _mat(H, "H")
    W = _dev(W, torch.float32, "W")
    m, nnz = rowptr.numel() - 1, colidx.numel()
    k, f_in = H.shape
    f_out = W.shape[1]
    if out is None:
        T = torch.empty((m, f_in), dtype=torch.float32, device=H.device) if want_t else None
        Z = torch.empty((m, f_out), dtype=torch.float32, device=H.device) if want_z else None
        Ho = torch.empty((m, f_out), dtype=torch.float32, device=H.device) if want_h else None
    else:
        T, Z, Ho = out
    if fused:
        rc = lib().gcn_layer_fwd_fused(_ptr(rowptr), _ptr(colidx), _ptr(val), m, k, nnz, _ptr(H), _ld(H),
                                       f_in, _ptr(W), f_out, act, prec, _ptr(T), _ptr(Z), _ptr(Ho), _stream())
        _check(rc, "gcn_layer_fwd_fused")
        return T, Z, Ho
    rc = _calls().gcn_layer_fwd(_ptr(rowptr), _ptr(colidx), _ptr(val), m, k, nnz, _ptr(H), _ld(H),
                             f_in, _ptr(W), f_out, act, prec, _ptr(T), _ptr(Z), _ptr(Ho),
                             _ptr(ws.buf) if ws else None, ws.buf.numel() if ws else 0, _stream())
    _check(rc, "gcn_layer_fwd")
    return T, Z, Ho


def gcn_layer_fwd_form(ws: SpmmWorkspace, f_in: int, f_out: int, prec=GEMM_FP32) -> int:
    """Which form gcn_layer_fwd(want_t=False) takes: 2 sweep with the dense transform as epilogue,
    1 row-range kernel, 0 unsupported shape."""
    form = ctypes.c_int32(0)
    _check(lib().gcn_layer_fwd_form(_ptr(ws.buf) if ws else None, f_in, f_out, prec, ctypes.byref(form)),
           "gcn_layer_fwd_form")
    return form.value


def gcn_layer_bwd(rowptr, colidx, val, G, W, Zprev, Hprev, prec=GEMM_FP32, ws: SpmmWorkspace = None,
                  want_gprev=True, want_y=True):
    """S = A G, Gprev = (S W^T) .* [Zprev > 0], Y = Hprev^T S.  Returns (S, Gprev, Y)."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    val = _dev(val, torch.float32, "val")
    G = _dev(G, torch.float32, "G")
    W = _dev(W, torch.float32, "W")
    m, nnz = rowptr.numel() - 1, colidx.numel()
    f_in, f_out = W.shape
    dev = G.device
    S = torch.empty((m, f_out), dtype=torch.float32, device=dev)
    Gp = torch.empty((m, f_in), dtype=torch.float32, device=dev) if want_gprev else None
    Y = torch.empty((f_in, f_out), dtype=torch.float32, device=dev) if want_y else None
    yws = None
    if want_y:
        b = ctypes.c_size_t(0)
        _check(lib().gcn_bwd_workspace_bytes(m, f_in, f_out, ctypes.byref(b)), "gcn_bwd_workspace_bytes")
        yws = _ws(b.value, dev)
    rc = _calls().gcn_layer_bwd(_ptr(rowptr), _ptr(colidx), _ptr(val), m, nnz, _ptr(G), f_out, _ptr(W),
                             f_in, _ptr(Zprev), _ptr(Hprev), prec, _ptr(S), _ptr(Gp), _ptr(Y),
                             _ptr(ws.buf) if ws else None, ws.buf.numel() if ws else 0,
                             _ptr(yws), yws.numel() if yws is not None else 0, _stream())
    _check(rc, "gcn_layer_bwd")
    return S, Gp, Y


@dataclass
class ColBlocks:
    """Result of spmm_split_colblocks: nb CSR matrices sharing three buffers."""
    rowptr_blk: torch.Tensor      # int32 [nb, m+1]
    colidx_blk: torch.Tensor      # int32 [nnz]
    val_blk: torch.Tensor         # float32 [nnz]
    nnz_off: np.ndarray           # int64 [nb+1] (host)

    def block(self, q: int):
        a, b = int(self.nnz_off[q]), int(self.nnz_off[q + 1])
        return self.rowptr_blk[q], self.colidx_blk[a:b], self.val_blk[a:b]


def spmm_split_colblocks(rowptr, colidx, val, bounds) -> ColBlocks:
    """Split a CSR row block into one CSR per column range (Sec. 4.2; the A_iq of Alg. 2)."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    val = _dev(val, torch.float32, "val")
    m, nnz = rowptr.numel() - 1, colidx.numel()
    bounds = np.ascontiguousarray(bounds, dtype=np.int64)
    nb = bounds.size - 1
    dev = rowptr.device
    L = lib()
    wsb = ctypes.c_size_t(0)
    _check(L.spmm_split_workspace_bytes(m, nb, ctypes.byref(wsb)), "spmm_split_workspace_bytes")
    ws = _ws(wsb.value, dev)
    rp = torch.empty((nb, m + 1), dtype=torch.int32, device=dev)
    ci = torch.empty(max(nnz, 1), dtype=torch.int32, device=dev)
    va = torch.empty(max(nnz, 1), dtype=torch.float32, device=dev)
    off = np.zeros(nb + 1, dtype=np.int64)
    rc = L.spmm_split_colblocks(_ptr(rowptr), _ptr(colidx), _ptr(val), m, nnz,
                                _host(bounds), nb, _ptr(rp), _ptr(ci), _ptr(va),
                                _host(off), _ptr(ws), ws.numel(), _stream())
    _check(rc, "spmm_split_colblocks")
    return ColBlocks(rp, ci[:nnz], va[:nnz], off)


def spmm_stage_loop(stages, m: int, H, T0, T1, Z, accumulate_first=False, pack_stream=None):
    """Stage loop of Alg. 2 on one rank.  `stages` is a list of dicts with keys rowptr, colidx,
    val, rows and optionally ws (SpmmWorkspace).  Products run on the current stream, packs on
    `pack_stream` (a torch.cuda.Stream; None = the current stream)."""
    H = _dev(H, torch.float32, "H")
    Z = _dev(Z, torch.float32, "Z")
    T0 = _dev(T0, torch.float32, "T0")
    T1 = _dev(T1, torch.float32, "T1")
    n, f = H.shape
    arr = (_Stage * max(len(stages), 1))()
    for k, st in enumerate(stages):
        rp = _dev(st["rowptr"], torch.int32, "stage rowptr")
        ci = _dev(st["colidx"], torch.int32, "stage colidx")
        va = _dev(st["val"], torch.float32, "stage val")
        rows = _dev(st["rows"], torch.int32, "stage rows")
        if rp.numel() != m + 1:
            raise ValueError("stage rowptr must have m+1 entries")
        ws = st.get("ws")
        arr[k] = _Stage(rp.data_ptr(), ci.data_ptr() if ci.numel() else None,
                        va.data_ptr() if va.numel() else None, ci.numel(),
                        rows.data_ptr() if rows.numel() else None, rows.numel(),
                        ws.buf.data_ptr() if ws else None, ws.buf.numel() if ws else 0)
    cap = min(T0.shape[0], T1.shape[0])
    if T0.shape[1] != f or T1.shape[1] != f:
        raise ValueError("packed buffers must have H's width")
    ps = _stream() if pack_stream is None else pack_stream.cuda_stream
    rc = lib().spmm_stage_loop(ctypes.cast(arr, ctypes.c_void_p), len(stages), m, _ptr(H), n,
                               H.stride(0), f, _ptr(T0), _ptr(T1), cap, _ptr(Z), Z.stride(0),
                               int(accumulate_first), _stream(), ps)
    _check(rc, "spmm_stage_loop")
    return Z


def spmm_volume_stats(counts, f: int, elem_bytes: int = 4) -> dict:
    """Volume statistics of one SpMM from the P x P matrix of |NnzCols(i,q)| (host arithmetic)."""
    c = np.ascontiguousarray(counts, dtype=np.int64)
    if c.ndim != 2 or c.shape[0] != c.shape[1]:
        raise ValueError("counts must be P x P")
    out = np.zeros(8, dtype=np.float64)
    _check(lib().spmm_volume_stats(_host(c), c.shape[0], f, elem_bytes,
                                   _host(out)), "spmm_volume_stats")
    keys = ("total_bytes", "avg_bytes", "max_recv_bytes", "recv_imbalance_pct", "max_send_bytes",
            "send_imbalance_pct", "cut_rows", "cut_bytes")
    return dict(zip(keys, (float(x) for x in out)))


def spmm_csr_transpose(rowptr, colidx, val, n: int):
    """CSR of A^T for A = (rowptr, colidx, val) with n columns.  Returns (rowptr_t, colidx_t, val_t)."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    val = _dev(val, torch.float32, "val")
    m, nnz = rowptr.numel() - 1, colidx.numel()
    dev = rowptr.device
    L = lib()
    wsb = ctypes.c_size_t(0)
    _check(L.spmm_transpose_workspace_bytes(nnz, ctypes.byref(wsb)), "spmm_transpose_workspace_bytes")
    ws = _ws(wsb.value, dev)
    rpt = torch.empty(n + 1, dtype=torch.int32, device=dev)
    cit = torch.empty(max(nnz, 1), dtype=torch.int32, device=dev)
    vat = torch.empty(max(nnz, 1), dtype=torch.float32, device=dev)
    _check(L.spmm_csr_transpose(_ptr(rowptr), _ptr(colidx), _ptr(val), m, n, nnz, _ptr(rpt), _ptr(cit),
                                _ptr(vat), _ptr(ws), ws.numel(), _stream()), "spmm_csr_transpose")
    return rpt, cit[:nnz], vat[:nnz]


def _permute_ws(n: int, nnz: int, device):
    wsb = ctypes.c_size_t(0)
    _check(lib().spmm_permute_workspace_bytes(n, nnz, ctypes.byref(wsb)), "spmm_permute_workspace_bytes")
    return _ws(wsb.value, device)


def spmm_perm_from_labels(labels, n_parts: int):
    """Vertex order by part label (Sec. 5 / 6.1 renumbering).  Returns (perm, inv, part_off): perm[i] =
    old id of new vertex i, inv[v] = new id of old vertex v, part_off (host, n_parts+1)."""
    labels = _dev(labels, torch.int32, "labels")
    n = labels.numel()
    dev = labels.device
    ws = _permute_ws(n, n, dev)
    perm = torch.empty(max(n, 1), dtype=torch.int32, device=dev)
    inv = torch.empty(max(n, 1), dtype=torch.int32, device=dev)
    off = np.zeros(n_parts + 1, dtype=np.int64)
    _check(lib().spmm_perm_from_labels(_ptr(labels), n, n_parts, _ptr(perm), _ptr(inv),
                                       _host(off), _ptr(ws), ws.numel(), _stream()),
           "spmm_perm_from_labels")
    return perm[:n], inv[:n], off


def spmm_csr_permute_symmetric(rowptr, colidx, val, inv):
    """B = P A P^T with B[inv[r], inv[c]] = A[r, c].  Returns (rowptr_p, colidx_p, val_p)."""
    rowptr = _dev(rowptr, torch.int32, "rowptr")
    colidx = _dev(colidx, torch.int32, "colidx")
    val = _dev(val, torch.float32, "val")
    inv = _dev(inv, torch.int32, "inv")
    n, nnz = rowptr.numel() - 1, colidx.numel()
    if inv.numel() != n:
        raise ValueError("inv must have one entry per row")
    dev = rowptr.device
    ws = _permute_ws(n, nnz, dev)
    rpp = torch.empty(n + 1, dtype=torch.int32, device=dev)
    cip = torch.empty(max(nnz, 1), dtype=torch.int32, device=dev)
    vap = torch.empty(max(nnz, 1), dtype=torch.float32, device=dev)
    _check(lib().spmm_csr_permute_symmetric(_ptr(rowptr), _ptr(colidx), _ptr(val), n, nnz, _ptr(inv), _ptr(rpp),
                                            _ptr(cip), _ptr(vap), _ptr(ws), ws.numel(), _stream()),
           "spmm_csr_permute_symmetric")
    return rpp, cip[:nnz], vap[:nnz]


_DTYPE = {torch.float32: F32, torch.bfloat16: BF16}


def _typed(t: torch.Tensor, name: str, dtype=None):
    """A row-major matrix of fp32 or bfloat16 (of `dtype` where that is given), possibly a column slice of a wider one."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA/HIP tensor (there is no CPU path)")
    kind = t.dtype
    if t.dim() != 2 or (kind not in _DTYPE if dtype is None else kind is not dtype):
        raise ValueError(f"{name}: expected a 2-D tensor of " + (str(dtype) if dtype is not None else "float32 or bfloat16"))
    if not t.is_contiguous() and not _rows_apart(t):
        raise ValueError(f"{name}: rows must be contiguous (unit stride inside a row) and must not overlap")
    return t


def _shape(t: torch.Tensor, shape, name: str):
    if t.shape != shape:
        raise ValueError(f"{name}: expected {tuple(shape)}, got {tuple(t.shape)}")
    return t


def _weights(W: torch.Tensor, dtype):
    """Weight matrices one behind the other, each row-major: leading dimension and distance of two."""
    if not W.is_cuda:
        raise ValueError("W must be a CUDA/HIP tensor (there is no CPU path)")
    if W.dim() != 3 or W.dtype is not dtype:
        raise ValueError(f"W: expected a 3-D tensor of {dtype}")
    g, a, b = W.shape
    if W.is_contiguous():
        return b, a * b
    ld, stride = W.stride(1) if a > 1 else max(b, 1), W.stride(0) if g > 1 else 0
    if (b > 1 and W.stride(2) != 1) or ld < b or stride < 0:
        raise ValueError("W: rows must be contiguous (unit stride inside a row) and must not overlap")
    return ld, stride


def _offsets(off: torch.Tensor, name: str):
    off = _dev(off, torch.int32, name)
    if off.dim() != 1 or off.numel() < 2:
        raise ValueError(f"{name}: expected one offset more than there are parts")
    return off


def grouped_gemm_act(X, W, off, transW=False, prec=GEMM_FP32, act=ACT_IDENTITY, mask=None, out=None):
    """Y[r, :] = act(X[r, :] op(W[g])) .* [mask[r, :] > 0] for the rows off[g] <= r < off[g+1] of each type g; rows behind the
    last type are zeros.  X: m x kdim, W: types x kdim x nout (types x nout x kdim with transW), float32 or bfloat16;
    off: int32 on the device, one more than there are types."""
    X = _typed(X, "X")
    ldw, stride_w = _weights(W, X.dtype)
    off = _offsets(off, "off")
    m, kdim = X.shape
    types, nout = off.numel() - 1, W.shape[1 if transW else 2]
    _shape(W, (types, nout, kdim) if transW else (types, kdim, nout), "W")
    if mask is not None:
        _shape(_typed(mask, "mask", X.dtype), (m, nout), "mask")
    if out is None:
        out, ldy = X.new_empty((m, nout)), nout
    else:
        ldy = _ld(_shape(_typed(out, "out", X.dtype), (m, nout), "out"))
    _check(_calls().grouped_gemm_act(_DTYPE[X.dtype], X.data_ptr(), kdim if X.is_contiguous() else _ld(X), W.data_ptr(), ldw, stride_w,
                                     int(transW), off.data_ptr(), types, m, kdim, nout, prec, act, _ptr(mask),
                                     _ld(mask) if mask is not None else 0, out.data_ptr(), ldy, _stream()), "grouped_gemm_act")
    return out


def grouped_gemm_bwd(X, W, off, G, mask=None, prec=GEMM_FP32, want_dx=True, want_dw=True):
    """Gradients of grouped_gemm_act (transW = False, identity): dX[r, :] = (G[r, :] W[g]^T) .* [mask[r, :] > 0] in X's type and
    dW[g] = X_g^T G_g in float32.  Returns (dX, dW), None for what is not wanted (X or W may be None then: X only where
    want_dw is False, W never, its shape is needed)."""
    G = _typed(G, "G")
    ldw, stride_w = _weights(W, G.dtype)
    off = _offsets(off, "off")
    m, nout = G.shape
    types, kdim = off.numel() - 1, W.shape[1]
    _shape(W, (types, kdim, nout), "W")
    if X is not None:
        _shape(_typed(X, "X", G.dtype), (m, kdim), "X")
    elif want_dw:
        raise ValueError("the gradient of W needs X")
    if mask is not None:
        _shape(_typed(mask, "mask", G.dtype), (m, kdim), "mask")
    dX = G.new_empty((m, kdim)) if want_dx else None
    dW = ws = None
    if want_dw:
        dW = G.new_empty((types, kdim, nout), dtype=torch.float32)
        need = _bytes_of("grouped_gemm_bwd_workspace_bytes", m, types, kdim, nout)
        ws = G.new_empty(need, dtype=torch.uint8) if need else None
    _check(_calls().grouped_gemm_bwd(_DTYPE[G.dtype], _ptr(X), _ld(X) if X is not None else kdim, _ptr(W), ldw, stride_w, _ptr(off), types,
                                     m, kdim, nout, prec, _ptr(G), _ld(G), _ptr(mask), _ld(mask) if mask is not None else 0, _ptr(dX), kdim,
                                     _ptr(dW), _ptr(ws), ws.numel() if ws is not None else 0, _stream()), "grouped_gemm_bwd")
    return dX, dW


def _norm_args(X, groups, gamma, beta, seg, n_seg, out):
    """What both directions check; and out's place where it is not given."""
    X = _typed(X, "X")
    shape = X.shape
    if seg is not None:
        n_seg = _offsets(seg, "seg").numel() - 1
    if gamma is not None:
        _shape(_dev(gamma, torch.float32, "gamma"), shape[1:], "gamma")
    if beta is not None:
        _shape(_dev(beta, torch.float32, "beta"), shape[1:], "beta")
    whole = X.is_contiguous()
    if out is None:
        out, ldo = torch.empty_like(X) if whole else X.new_empty(shape), shape[1]
    else:
        ldo = _ld(_shape(_typed(out, "out", X.dtype), shape, "out"))
    return *shape, n_seg, out, shape[1] if whole else _ld(X), ldo


def group_norm_act(X, groups, gamma=None, beta=None, seg=None, n_seg=1, max_rows=0, eps=1e-5, act=ACT_IDENTITY, out=None):
    """Group norm with an activation, channels last: Y = act((X - mean) rstd gamma + beta), mean and variance over the rows of a
    segment and each of `groups` groups of channels.  seg: int32 on the device, one more than there are segments (rows behind
    the last are zeros in Y), or None for n_seg segments of equal length; max_rows: rows of the longest one where it is known.
    Returns (Y, mean, rstd), the last two float32, segments x groups."""
    m, c, n_seg, out, ldx, ldy = _norm_args(X, groups, gamma, beta, seg, n_seg, out)
    if seg is None and not max_rows and n_seg > 1:
        max_rows = m // n_seg
    kind = _DTYPE[X.dtype]
    need = _bytes_of("group_norm_workspace_bytes", kind, m, n_seg, max_rows, c, groups, max(ldx, ldy), 0)
    ws = X.new_empty(need, dtype=torch.uint8) if need else None
    mean = X.new_empty((n_seg, groups), dtype=torch.float32)
    rstd = torch.empty_like(mean)
    _check(_calls().group_norm_act_fwd(kind, X.data_ptr(), ldx, _ptr(seg), n_seg, max_rows, m, c, groups, _ptr(gamma), _ptr(beta),
                                       eps, act, out.data_ptr(), ldy, mean.data_ptr(), rstd.data_ptr(), _ptr(ws), need, _stream()),
           "group_norm_act_fwd")
    return out, mean, rstd


def group_norm_act_bwd(X, G, mean, rstd, groups, gamma=None, beta=None, seg=None, n_seg=1, max_rows=0, act=ACT_IDENTITY, out=None):
    """Gradients of group_norm_act for G = dLoss/dY, with the mean and rstd that it returned.  Returns (dX, dgamma, dbeta)."""
    m, c, n_seg, out, ldx, lddx = _norm_args(X, groups, gamma, beta, seg, n_seg, out)
    if seg is None and not max_rows and n_seg > 1:
        max_rows = m // n_seg
    _shape(_typed(G, "G", X.dtype), (m, c), "G")
    for name, t in (("mean", mean), ("rstd", rstd)):
        _shape(_dev(t, torch.float32, name), (n_seg, groups), name)
    kind, ldg = _DTYPE[X.dtype], _ld(G)
    need = _bytes_of("group_norm_workspace_bytes", kind, m, n_seg, max_rows, c, groups, max(ldx, ldg, lddx), 1)
    ws = X.new_empty(need, dtype=torch.uint8) if need else None
    dgamma = X.new_empty(c, dtype=torch.float32)
    dbeta = torch.empty_like(dgamma)
    _check(_calls().group_norm_act_bwd(kind, X.data_ptr(), ldx, G.data_ptr(), ldg, _ptr(seg), n_seg, max_rows, m, c, groups, _ptr(gamma),
                                       _ptr(beta), act, mean.data_ptr(), rstd.data_ptr(), out.data_ptr(), lddx, dgamma.data_ptr(),
                                       dbeta.data_ptr(), _ptr(ws), need, _stream()), "group_norm_act_bwd")
    return out, dgamma, dbeta


def _rows_in_python(grads, out):
    rows = []
    for g, o in zip(grads, grads if out is None else out, strict=True):
        kind = _DTYPE.get(g.dtype)
        if kind is None or not g.is_cuda or not g.is_contiguous():
            raise ValueError("gradients: expected contiguous float32 or bfloat16 CUDA/HIP tensors (there is no CPU path)")
        if o is not g and (o.dtype is not g.dtype or not o.is_cuda or not o.is_contiguous() or o.shape != g.shape):
            raise ValueError("out: expected contiguous tensors like the gradients")
        rows.append((g.data_ptr(), o.data_ptr(), g.numel(), kind))
    return np.array(rows, dtype=np.int64).tobytes()


_rows = None


def _listed(grads):
    return grads if isinstance(grads, (list, tuple)) else list(grads)


def _grad_list(grads, out=None):
    """struct sagnn_grad of the C header for each tensor, one behind the other."""
    global _rows
    if _rows is None:                      # csrc/gradlist.cpp, or the same in Python where it is not built for this torch
        ext = _extension("_gradlist", _build.GRADLIST) if _build.gradlist_fits() else None
        _rows = ext.rows if ext else _rows_in_python
    rows = _rows(grads, out)
    return rows, len(rows) // 32


@functools.lru_cache(maxsize=256)
def _bytes_of(query: str, *sizes) -> int:
    """What a workspace query of the library says, a function of the sizes alone."""
    b = ctypes.c_size_t(0)
    _check(getattr(lib(), query)(*sizes, ctypes.byref(b)), query)
    return b.value


def _grad_ws(grads, n):
    """Room for the sums, how much that is, and the norm's place."""
    like, need = grads[0] if n else torch.empty(0, device="cuda"), _bytes_of("grad_norm_workspace_bytes", n)
    return like.new_empty(need, dtype=torch.uint8), need, like.new_empty(1, dtype=torch.float32)


def grad_global_norm(grads):
    """The 2-norm over all tensors of the list, a float32 tensor of one element on the device."""
    grads = _listed(grads)
    rows, n = _grad_list(grads)
    ws, need, norm = _grad_ws(grads, n)
    _check(_calls().grad_global_norm(rows, n, norm.data_ptr(), ws.data_ptr(), need, _stream()), "grad_global_norm")
    return norm


def grad_clip_norm(grads, max_norm: float, norm=None, out=None):
    """Scales the tensors of the list by min(1, max_norm / norm), in place or into `out` (tensors like them).  norm: what
    grad_global_norm returned, perhaps joined across processes; None computes it.  Returns the norm (on the device)."""
    grads = _listed(grads)
    rows, n = _grad_list(grads, out)
    if norm is not None:
        _shape(_dev(norm, torch.float32, "norm"), (1,), "norm")
        _check(_calls().grad_scale_to_norm(rows, n, max_norm, _ptr(norm), _stream()), "grad_scale_to_norm")
        return norm
    ws, need, norm = _grad_ws(grads, n)
    _check(_calls().grad_clip_norm(rows, n, max_norm, norm.data_ptr(), ws.data_ptr(), need, _stream()), "grad_clip_norm")
    return norm


def _drop_args(p, seed, offset, row0):
    """Dropout as the library takes it: 65536ths, and the offset's two parts."""
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"p: expected a probability, got {p}")
    d_offset = None
    if isinstance(offset, torch.Tensor):
        if offset.numel() != 1:
            raise ValueError("offset: expected one element")
        d_offset, offset = _here(_dev(offset, torch.int64, "offset"), "offset").data_ptr(), 0
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset: expected 64 bits without a sign")
    return int(p * 65536 + 0.5), seed, offset, d_offset, row0


def _here(t, name="X"):
    """A tensor on the device whose current stream the call goes to: a launch elsewhere would neither wait for it nor be waited for."""
    if t.is_cuda and t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{name}: lies on {t.device}, which is not the current device")
    return t


def _lead(X, name="X", dtype=None):
    """A matrix on the current device: its address, leading dimension and rows and columns."""
    if X.is_cuda and X.is_contiguous() and X.dim() == 2 and (X.dtype in _DTYPE if dtype is None else X.dtype is dtype) and X.get_device() == torch._C._cuda_getDevice():
        m, c = X.shape
        return X.data_ptr(), c, m, c
    _here(_typed(X, name, dtype), name)
    return X.data_ptr(), _ld(X), *X.shape


def _like(t, X, name):
    """A matrix like X, or None: its address and leading dimension."""
    if t is None:
        return None, 0
    if t.dtype is X.dtype and t.shape == X.shape and t.is_contiguous() and t.get_device() == X.get_device():
        return t.data_ptr(), X.shape[1]
    _here(_shape(_typed(t, name, X.dtype), X.shape, name), name)
    return t.data_ptr(), _ld(t)


def _vector(t, n, name, dtype=torch.float32):
    """A vector of n values on the current device, or None: its address."""
    if t is None:
        return None
    _here(_shape(_dev(t, dtype, name), (n,), name), name)
    return t.data_ptr()


def dropout_add(X, p: float, seed: int, offset=0, residual=None, row0: int = 0, out=None):
    """Y = residual + dropout(X): each value is kept with probability 1 - p (to 2^-17) and divided by that, or 0.  The mask is a function of
    seed, offset, row0 + row and column; the gradient for X is the same call on dY without a residual, with the same seed, offset and row0.
    offset: an integer, or an int64 tensor of one element on the device that is read when the kernel runs (a captured graph counts it up).
    row0: the first row's number in the whole matrix where ranks share its rows.  X: m x C, float32 or bfloat16; residual like it."""
    x, ldx, m, c = _lead(X)
    y, ldy = _like(out, X, "out")
    if out is None:
        out = X.new_empty((m, c))
        y, ldy = out.data_ptr(), c
    r, ldr = _like(residual, X, "residual")
    _check(_calls().dropout_add(_DTYPE[X.dtype], x, ldx, r, ldr, m, c, *_drop_args(p, seed, offset, row0), y, ldy, _stream()), "dropout_add")
    return out


def _rms_norm(X, lead, gamma, residual, eps, p, seed, offset, row0, kind, y, ldy, scale, out_sum):
    x, ldx, m, c = lead
    S, s, lds = X, None, 0
    if residual is not None or p > 0.0:
        S = X.new_empty((m, c)) if out_sum is None else out_sum
        s, lds = _like(S, X, "out_sum")
    elif out_sum is not None:
        raise ValueError("out_sum: nothing is added or dropped, the sum is X")
    rstd = X.new_empty(m, dtype=torch.float32)
    r, ldr = _like(residual, X, "residual")
    _check(_calls().rms_norm_fwd(_DTYPE[X.dtype], x, ldx, r, ldr, m, c, _vector(gamma, c, "gamma"), eps, *_drop_args(p, seed, offset, row0),
                                 kind, y, ldy, scale, s, lds, rstd.data_ptr(), _stream()), "rms_norm_fwd")
    return S, rstd


def rms_norm(X, gamma=None, residual=None, eps: float = 1e-6, p: float = 0.0, seed: int = 0, offset=0, row0: int = 0, out=None, out_sum=None):
    """Root-mean-square norm of the rows of S = residual + dropout(X) (dropout_add's p, seed, offset, row0): Y = S rstd gamma,
    rstd = (mean(S^2) + eps)^-1/2.  X: m x C, float32 or bfloat16, residual like it; gamma: C, float32.  Returns (Y, S, rstd), S being X itself
    where nothing is added or dropped (None where out takes X's place then), rstd float32; out_sum may be the residual, which is updated in place then."""
    lead, over = _lead(X), False
    if out is None:
        out = X.new_empty(lead[2:])
        y, ldy = out.data_ptr(), lead[3]
    else:
        y, ldy = _like(out, X, "out")
        over = y == lead[0]
    S, rstd = _rms_norm(X, lead, gamma, residual, eps, p, seed, offset, row0, _DTYPE[X.dtype], y, ldy, None, out_sum)
    return out, None if over and S is X and out_sum is None else S, rstd


def rms_norm_e4m3(X, gamma=None, residual=None, eps: float = 1e-6, p: float = 0.0, seed: int = 0, offset=0, row0: int = 0, out_sum=None):
    """rms_norm with rows of 8 bits: Y[r, :] = scale[r] Q[r, :], Q torch.float8_e4m3fn, scale float32.  Returns (Q, scale, S, rstd).
    spmm_pack_rows_e4m3 reads them."""
    lead = _lead(X)
    Q, scale = X.new_empty(lead[2:], dtype=torch.float8_e4m3fn), X.new_empty(lead[2], dtype=torch.float32)
    S, rstd = _rms_norm(X, lead, gamma, residual, eps, p, seed, offset, row0, E4M3, Q.data_ptr(), lead[3], scale.data_ptr(), out_sum)
    return Q, scale, S, rstd


def rms_norm_bwd(S, G, rstd, gamma=None, grad_sum=None, p: float = 0.0, seed: int = 0, offset=0, row0: int = 0, want_dx=True, want_dgamma=True):
    """Gradients of rms_norm for G = dLoss/dY, with the S and rstd that it returned; grad_sum: the gradient that S has from elsewhere (the
    next residual).  Returns (dX, dR, dgamma): dX = dropout(dR), or dR itself where nothing was dropped; None for what is not wanted."""
    s, lds, m, c = _lead(S, "S")
    g, ldg = _like(G, S, "G")
    if g is None:
        raise ValueError("G is needed")
    d, ldd = _like(grad_sum, S, "grad_sum")
    drop = _drop_args(p, seed, offset, row0)
    dR = S.new_empty((m, c))
    dX = S.new_empty((m, c)) if want_dx and drop[0] else None
    dgamma = S.new_empty(c, dtype=torch.float32) if want_dgamma else None
    need = _bytes_of("rms_norm_bwd_workspace_bytes", m, c) if want_dgamma else 0
    ws = S.new_empty(need, dtype=torch.uint8) if need else None
    _check(_calls().rms_norm_bwd(_DTYPE[S.dtype], s, lds, g, ldg, d, ldd, m, c, _vector(gamma, c, "gamma"), _vector(rstd, m, "rstd"), *drop, _ptr(dX), c,
                                 dR.data_ptr(), c, _ptr(dgamma), _ptr(ws), need, _stream()), "rms_norm_bwd")
    return (dX if drop[0] else dR) if want_dx else None, dR, dgamma


def spmm_pack_rows_e4m3(Q, scale, rows=None, dtype=torch.float32, out=None):
    """out[i, :] = scale[rows[i]] Q[rows[i], :] for rows of 8 bits (rms_norm_e4m3's), widened to float32 or bfloat16; rows: int32, None: all of
    them.  A row number out of range gives zeros."""
    q, ldq, n, c = _lead(Q, "Q", torch.float8_e4m3fn)
    N = n if rows is None else rows.numel()
    at = _vector(rows, N, "rows", torch.int32)
    if out is None:
        out, o, ldo = Q.new_empty((N, c), dtype=dtype), None, c
        _typed(out, "dtype")
    else:
        o, ldo, *shape = _lead(out, "out")
        if shape != [N, c]:
            raise ValueError(f"out: expected {(N, c)}, got {tuple(out.shape)}")
    _check(_calls().spmm_pack_rows_e4m3(q, ldq, _vector(scale, n, "scale"), n, c, at, N, _DTYPE[out.dtype], o or out.data_ptr(), ldo, _stream()),
           "spmm_pack_rows_e4m3")
    return out


def _xent_args(H, W, labels, bias, transW):
    """What both directions check: H's rows and width, the classes, and the pointers that lead both calls."""
    h, ldh, m, k = _lead(H, "H")
    w, ldw, *shape = _lead(W, "W", H.dtype)
    n = shape[0 if transW else 1]
    if shape != ([n, k] if transW else [k, n]):
        raise ValueError(f"W: expected {k} {'columns' if transW else 'rows'}, got {tuple(W.shape)}")
    return m, k, n, (_DTYPE[H.dtype], h, ldh, w, ldw, int(transW), _vector(bias, n, "bias"), _vector(labels, m, "labels", torch.int32))


def softmax_xent(H, W, labels, bias=None, transW=False, prec=GEMM_FP32):
    """Softmax cross entropy over the classes of the logits H W + bias, which are not kept: loss[r] = lse[r] - logit[r, labels[r]], lse the
    logarithm of the row's sum of exponentials.  H: m x kdim, W: kdim x classes (classes x kdim with transW), float32 or bfloat16; labels: m, int32,
    one outside the classes (-1, say) for a row that has none: loss 0; bias: classes, float32.  Returns (loss, lse), float32."""
    m, k, n, args = _xent_args(H, W, labels, bias, transW)
    need = _bytes_of("softmax_xent_workspace_bytes", args[0], m, k, n, prec, 0)
    ws = H.new_empty(need, dtype=torch.uint8) if need else None
    loss = H.new_empty(m, dtype=torch.float32)
    lse = torch.empty_like(loss)
    _check(_calls().softmax_xent_fwd(*args, m, k, n, prec, loss.data_ptr(), lse.data_ptr(), _ptr(ws), need, _stream()), "softmax_xent_fwd")
    return loss, lse


def softmax_xent_bwd(H, W, labels, lse, grad=1.0, bias=None, transW=False, prec=GEMM_FP32, want_dh=True, want_dw=True):
    """Gradients of softmax_xent with the lse that it returned; grad: dLoss/d(loss), a number for all rows (one over how many labels there are, for
    their mean) or m, float32.  Returns (dH, dW, dbias), the first two in H's type, dbias float32; None for what is not wanted or not there."""
    m, k, n, args = _xent_args(H, W, labels, bias, transW)
    rows = isinstance(grad, torch.Tensor)
    need = _bytes_of("softmax_xent_bwd_workspace_bytes", args[0], m, k, n, prec, int(rows))
    ws = H.new_empty(need, dtype=torch.uint8)
    dH = H.new_empty((m, k)) if want_dh else None
    dW = H.new_empty(W.shape) if want_dw else None
    dbias = None if bias is None or not want_dw else torch.empty_like(bias)
    _check(_calls().softmax_xent_bwd(*args, _vector(lse, m, "lse"), _vector(grad, m, "grad") if rows else None, 1.0 if rows else grad, m, k, n, prec, _ptr(dH), k, _ptr(dW),
                                     _ptr(dbias), ws.data_ptr(), need, _stream()), "softmax_xent_bwd")
    return dH, dW, dbias
