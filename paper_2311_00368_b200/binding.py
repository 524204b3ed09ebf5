"""Thin Python binding over the C-ABI library ``libb2sp.so``: argument marshalling only.

Every step of the three ops runs inside the CUDA library; this module turns torch tensors
into raw device pointers + sizes, supplies a workspace and the current CUDA stream, and
raises on a non-zero status.  There is no CPU fallback: importing this module raises
``ImportError`` if the library has not been built, and calling an op without a CUDA device
fails in the library.

Function names and argument order follow ``include/b2sp.h`` (and ``include/b2sp_debug.h``).
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("B2SP_LIB") or os.path.join(_HERE, "libb2sp.so")  # B2SP_LIB: alternate build

ALGO_AUTO, ALGO_ROW, ALGO_ROW_NAT, ALGO_TILE, ALGO_TILE_PREPARED = 0, 1, 2, 3, 4
OP_SPMM, OP_SDDMM, OP_FUSEDMM = 0, 1, 2
ALGO_NAMES = {0: "auto", 1: "row", 2: "row_nat", 3: "tile", 4: "tile_prepared", -1: "none"}

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2311_00368_b200.build` "
        "(there is no fallback implementation)")

lib = ctypes.CDLL(LIB_PATH)

_i, _ll, _vp, _sz = ctypes.c_int, ctypes.c_longlong, ctypes.c_void_p, ctypes.c_size_t

lib.b2sp_version.restype = _i
lib.b2sp_status_string.restype = ctypes.c_char_p
lib.b2sp_status_string.argtypes = [_i]
lib.b2sp_workspace_bytes.restype = _sz
lib.b2sp_workspace_bytes.argtypes = [_i, _i, _i, _i, _i, _ll]
lib.b2sp_workspace_bytes_algo.restype = _sz
lib.b2sp_workspace_bytes_algo.argtypes = [_i, _i, _i, _i, _i, _i, _ll]
lib.b2sp_spmm.restype = _i
lib.b2sp_spmm.argtypes = [_i, _i, _i, _ll, _vp, _vp, _vp, _vp, _ll, _vp, _ll, _vp, _sz, _i, _vp]
lib.b2sp_sddmm.restype = _i
lib.b2sp_sddmm.argtypes = [_i, _i, _i, _ll, _vp, _vp, _vp, _vp, _ll, _vp, _ll, _vp, _vp, _sz, _i, _vp]
lib.b2sp_fusedmm.restype = _i
lib.b2sp_fusedmm.argtypes = [_i, _i, _i, _i, _ll, _vp, _vp, _vp, _vp, _ll, _vp, _ll, _vp, _ll, _vp, _ll,
                             _vp, _sz, _i, _vp]
lib.b2sp_spmm_bf16.restype = _i
lib.b2sp_spmm_bf16.argtypes = lib.b2sp_spmm.argtypes
lib.b2sp_sddmm_bf16.restype = _i
lib.b2sp_sddmm_bf16.argtypes = lib.b2sp_sddmm.argtypes
lib.b2sp_fusedmm_bf16.restype = _i
lib.b2sp_fusedmm_bf16.argtypes = lib.b2sp_fusedmm.argtypes
lib.b2sp_spmm_host.restype = _i
lib.b2sp_spmm_host.argtypes = [_i, _i, _i, _ll, _vp, _vp, _vp, _vp, _vp, _vp]
lib.b2sp_sddmm_host.restype = _i
lib.b2sp_sddmm_host.argtypes = [_i, _i, _i, _ll, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
lib.b2sp_fusedmm_host.restype = _i
lib.b2sp_fusedmm_host.argtypes = [_i, _i, _i, _i, _ll, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
lib.b2sp_spmm_static_scratch.restype = _i
lib.b2sp_spmm_static_scratch.argtypes = [_i, _i, _i, _ll, _vp, _vp, _vp, _vp, _ll, _vp, _ll, _vp]
lib.b2sp_workspace_bytes_batched.restype = _sz
lib.b2sp_workspace_bytes_batched.argtypes = [_i, _i, _i, _i, _i, _ll]
lib.b2sp_prepare_pattern_batched.restype = _i
lib.b2sp_prepare_pattern_batched.argtypes = [_i, _i, _i, _ll, _vp, _ll, _vp, _vp, _sz, _vp]
lib.b2sp_fusedmm_batched.restype = _i
lib.b2sp_fusedmm_batched.argtypes = [_i, _i, _i, _i, _i, _ll, _vp, _ll, _vp, _vp, _vp, _ll, _ll, _vp, _ll, _ll,
                                     _vp, _ll, _ll, _vp, _ll, _ll, _vp, _sz, _i, _vp]
lib.b2sp_fusedmm_batched_bf16.restype = _i
lib.b2sp_fusedmm_batched_bf16.argtypes = lib.b2sp_fusedmm_batched.argtypes
lib.b2sp_prepare_pattern.restype = _i
lib.b2sp_prepare_pattern.argtypes = [_i, _i, _ll, _vp, _vp, _vp, _sz, _vp]
lib.b2sp_validate_csr.restype = _i
lib.b2sp_validate_csr.argtypes = [_i, _i, _ll, _vp, _vp, _vp, _sz, _vp]
lib.b2sp_probe_fp32_peak.restype = _i
lib.b2sp_probe_fp32_peak.argtypes = [_i, _vp, ctypes.POINTER(ctypes.c_double), _vp]
lib.b2sp_probe_l2_pull.restype = _i
lib.b2sp_probe_l2_pull.argtypes = [_vp, ctypes.c_size_t, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), _vp]
lib.b2sp_device_status.restype = _i
lib.b2sp_device_status.argtypes = [_vp, _vp]
lib.b2sp_last_algo.restype = _i
lib.b2sp_last_algo.argtypes = [_i]
lib.b2sp_last_launches.restype = _i
lib.b2sp_last_launches.argtypes = [_i]
lib.b2sp_debug_force_k_splits.restype = None
lib.b2sp_debug_force_k_splits.argtypes = [_i]
lib.b2sp_debug_force_partition.restype = None
lib.b2sp_debug_force_partition.argtypes = [_i]
lib.b2sp_debug_window_table_offset.restype = _sz
lib.b2sp_debug_window_table_offset.argtypes = [_i]
lib.b2sp_debug_unsorted_flag_offset.restype = _sz
lib.b2sp_debug_unsorted_flag_offset.argtypes = []
lib.b2sp_debug_inject_wait_timeout.restype = _i
lib.b2sp_debug_inject_wait_timeout.argtypes = [_i, ctypes.c_ulonglong]


# Structures go to the library as packed bytes (a ctypes.Structure costs five times as long to fill as struct.pack).
_HEADS = struct.Struct("Pqqq").pack                        # b2sp_heads: data, ld, stride_head, stride_batch
_PROBLEM = struct.Struct("7ifPqPqPq").pack                 # b2sp_attention_problem, in the order of its members
_KV4 = struct.Struct("PqqPqqi4x").pack                     # b2sp_kv4
_ph = _pp = _pk = _vp
lib.b2sp_attention_count_tiles.restype = _i
lib.b2sp_attention_count_tiles.argtypes = [_i, _i, _i, _ll, _vp, _ll, _vp, _vp, _sz, ctypes.POINTER(_ll), _vp]
lib.b2sp_attention_plan_bytes.restype = _sz
lib.b2sp_attention_plan_bytes.argtypes = [_i, _i, _i, _ll, _ll]
lib.b2sp_attention_prepare.restype = _i
lib.b2sp_attention_prepare.argtypes = [_i, _i, _i, _ll, _vp, _ll, _vp, _ll, _vp, _sz, _vp]
lib.b2sp_attention_plan_status.restype = _i
lib.b2sp_attention_plan_status.argtypes = [_vp, _vp]
lib.b2sp_attention_workspace_bytes.restype = _sz
lib.b2sp_attention_workspace_bytes.argtypes = [_pp, _i]
lib.b2sp_attention_workspace_bytes_bf16.restype = _sz
lib.b2sp_attention_workspace_bytes_bf16.argtypes = [_pp, _i]
lib.b2sp_attention.restype = _i
lib.b2sp_attention.argtypes = [_pp, _ph, _ph, _ph, _ph, _vp, _vp, _sz, _i, _vp]
lib.b2sp_attention_bf16.restype = _i
lib.b2sp_attention_bf16.argtypes = lib.b2sp_attention.argtypes
lib.b2sp_attention_backward.restype = _i
lib.b2sp_attention_backward.argtypes = [_pp, _ph, _ph, _ph, _ph, _vp, _ph, _ph, _ph, _ph, _vp, _sz, _i, _vp]
lib.b2sp_attention_backward_bf16.restype = _i
lib.b2sp_attention_backward_bf16.argtypes = lib.b2sp_attention_backward.argtypes
lib.b2sp_attention_last_algo.restype = _i
lib.b2sp_attention_last_algo.argtypes = [_i]
lib.b2sp_attention_last_launches.restype = _i
lib.b2sp_attention_last_launches.argtypes = [_i]
for _name in ("b2sp_kv4_write", "b2sp_kv4_write_bf16"):
    getattr(lib, _name).restype = _i
    getattr(lib, _name).argtypes = [_i, _i, _i, _vp, _ll, _ll, _vp, _pk, _vp, _sz, _vp]
lib.b2sp_kv4_write_workspace_bytes.restype = _sz
lib.b2sp_kv4_write_workspace_bytes.argtypes = [_i, _i]
for _name in ("b2sp_kv4_read", "b2sp_kv4_read_bf16"):
    getattr(lib, _name).restype = _i
    getattr(lib, _name).argtypes = [_i, _i, _i, _vp, _pk, _vp, _ll, _ll, _vp]
lib.b2sp_attention_kv4_workspace_bytes.restype = _sz
lib.b2sp_attention_kv4_workspace_bytes.argtypes = [_i, _i, _i, _i, _ll]
lib.b2sp_attention_kv4.restype = _i
lib.b2sp_attention_kv4.argtypes = [_i, _i, _i, _i, _ll, _vp, _vp, _vp, _ll, _ll, _pk, _pk, ctypes.c_float, _vp, _ll, _ll, _vp, _vp, _sz, _vp]


class B2spError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib.b2sp_status_string(status).decode()} (status {status})")


def _check(status: int, where: str):
    if status != 0:
        raise B2spError(status, where)


# The argument marshalling is on the critical path of small calls (a few microseconds of GPU work): addresses and streams are
# passed as plain integers, which the declared argument types convert, and the stream is asked for without a Stream object.
def _ptr(t):
    return None if t is None else t.data_ptr()


try:
    _raw_stream = torch._C._cuda_getCurrentRawStream   # device index -> cudaStream_t of torch's current stream
except AttributeError:
    def _raw_stream(device_index):
        return torch.cuda.current_stream(device_index).cuda_stream


def _stream():
    return _raw_stream(torch.cuda.current_device())


def _ld(t):
    shape, strides = t.shape, t.stride()
    assert len(shape) == 2 and (shape[1] <= 1 or strides[1] == 1), "dense operands are row-major"
    return strides[0] if shape[0] > 1 else max(shape[1], strides[0])


def _want(t, dtype, name, cuda=True):
    if t is None:
        return
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}")
    if cuda and not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")


def version() -> int:
    return int(lib.b2sp_version())


def workspace_bytes(op: int, M: int, K: int, Kd: int, N: int, nnz: int, algo=None) -> int:
    """b2sp_workspace_bytes (upper bound over all algo values) or, with `algo`, b2sp_workspace_bytes_algo."""
    if algo is None:
        return int(lib.b2sp_workspace_bytes(op, M, K, Kd, N, nnz))
    return int(lib.b2sp_workspace_bytes_algo(op, algo, M, K, Kd, N, nnz))


class _Kept(threading.local):
    """Workspaces that this module keeps, per device and stream, for each thread of its own: a call's kernels pass partial results through
    its workspace, and the launches of two threads may take turns on one stream."""
    def __init__(self):
        self.workspaces = {}


_kept = _Kept()


_planner_setting = 0   # counts the calls of the debug hooks that change the planner's choice


# Sizes only, by the planner's setting: a size that another thread asked for while a hook took effect is not met again.
@functools.lru_cache(maxsize=4096)
def _workspace_need(op, M, K, Kd, N, nnz, algo, setting):
    return workspace_bytes(op, M, K, Kd, N, nnz, algo)


def _workspace(op, M, K, Kd, N, nnz, device, workspace, algo=0):
    if workspace is None:
        need = _workspace_need(op, M, K, Kd, N, nnz, algo, _planner_setting)
        if _capturing():   # (as in _scratch: it belongs to the graph)
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
            return workspace, need
        key, workspaces = (device.index, _raw_stream(device.index)), _kept.workspaces
        workspace = workspaces.get(key)
        if workspace is None or workspace.numel() < need:
            workspace = torch.empty(max(need, 1 << 20), dtype=torch.uint8, device=device)
            workspaces[key] = workspace
    return workspace, workspace.numel()


def probe_fp32_peak(iters: int = 4096, device=None) -> float:
    """b2sp_probe_fp32_peak: sustained FP32 FMA rate of the current device in GFLOP/s (synchronises)."""
    scratch = torch.zeros(1, dtype=torch.float32, device=device or "cuda")
    out = ctypes.c_double(0.0)
    _check(lib.b2sp_probe_fp32_peak(iters, _ptr(scratch), ctypes.byref(out), _stream()), "b2sp_probe_fp32_peak")
    return float(out.value)


def probe_l2_pull(device=None):
    """b2sp_probe_l2_pull: (GB/s per SM, GB/s of the whole GPU) of 32 KB bulk copies from L2 into shared memory (synchronises)."""
    scratch = torch.zeros((17 << 20) + 64, dtype=torch.uint8, device=device or "cuda")
    per_sm, total = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(lib.b2sp_probe_l2_pull(_ptr(scratch), scratch.numel(), ctypes.byref(per_sm), ctypes.byref(total), _stream()),
           "b2sp_probe_l2_pull")
    return float(per_sm.value), float(total.value)


def last_algo(op: int) -> int:
    return int(lib.b2sp_last_algo(op))


def last_launches(op: int) -> int:
    return int(lib.b2sp_last_launches(op))


def debug_force_k_splits(k_splits: int) -> None:
    """b2sp_debug_force_k_splits: override the dense-tile planner's K split (0 = planner's choice)."""
    global _planner_setting
    lib.b2sp_debug_force_k_splits(int(k_splits))
    _planner_setting += 1


def debug_force_partition(partition: int) -> None:
    """b2sp_debug_force_partition: 0 = planner's choice, 1 = tiles x K splits only, 2 = balanced wherever offered."""
    global _planner_setting
    lib.b2sp_debug_force_partition(int(partition))
    _planner_setting += 1


def debug_window_table_offset(M: int) -> int:
    """b2sp_debug_window_table_offset: where the window table of a pattern of M rows begins in a workspace, in bytes."""
    return int(lib.b2sp_debug_window_table_offset(M))


def debug_unsorted_flag_offset() -> int:
    """b2sp_debug_unsorted_flag_offset: the int of a workspace that says that its window table cannot be used."""
    return int(lib.b2sp_debug_unsorted_flag_offset())


def debug_inject_wait_timeout(chunk: int, limit_ns: int = 0) -> None:
    """b2sp_debug_inject_wait_timeout: make the dense-tile kernels' bounded waits run out (chunk >= 0) with a
    short limit, or switch the hook off again (chunk < 0)."""
    _check(lib.b2sp_debug_inject_wait_timeout(int(chunk), int(limit_ns)), "b2sp_debug_inject_wait_timeout")


def spmm(row_ptr, col_idx, values, D, K=None, out=None, workspace=None, algo=ALGO_AUTO, dtype=torch.float32):
    """b2sp_spmm: O = S @ D.  CSR tensors int32/fp32 on the GPU; D [K, N] fp32 row-major
    (dtype=torch.bfloat16: b2sp_spmm_bf16, D in bfloat16)."""
    _want(row_ptr, torch.int32, "row_ptr"); _want(col_idx, torch.int32, "col_idx")
    _want(values, torch.float32, "values"); _want(D, dtype, "D")
    M, nnz = row_ptr.numel() - 1, col_idx.numel()
    K = D.shape[0] if K is None else K
    N = D.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=D.device)
    ws, wsb = _workspace(OP_SPMM, M, K, 0, N, nnz, D.device, workspace, algo)
    fn, name = (lib.b2sp_spmm, "b2sp_spmm") if dtype == torch.float32 else (lib.b2sp_spmm_bf16, "b2sp_spmm_bf16")
    _check(fn(M, K, N, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(values), _ptr(D), _ld(D),
                         _ptr(out), _ld(out), _ptr(ws), wsb, algo, _stream()), name)
    return out


STATIC_SCRATCH_MAX_ROWS = 65536


def spmm_static_scratch(row_ptr, col_idx, values, D, K=None, out=None):
    """b2sp_spmm_static_scratch: SPMM for callers that may not allocate device memory.  The
    library's built-in scratch array replaces the workspace; M is limited to
    STATIC_SCRATCH_MAX_ROWS, and calls that could overlap on the GPU must not share a device.
    (`out` should be passed by such callers; it is only created here for convenience.)"""
    _want(row_ptr, torch.int32, "row_ptr"); _want(col_idx, torch.int32, "col_idx")
    _want(values, torch.float32, "values"); _want(D, torch.float32, "D")
    M, nnz = row_ptr.numel() - 1, col_idx.numel()
    K = D.shape[0] if K is None else K
    N = D.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=D.device)
    _check(lib.b2sp_spmm_static_scratch(M, K, N, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(values),
                                        _ptr(D), _ld(D), _ptr(out), _ld(out), _stream()),
           "b2sp_spmm_static_scratch")
    return out


def sddmm(row_ptr, col_idx, s_values, A, B, out=None, workspace=None, algo=ALGO_AUTO, dtype=torch.float32):
    """b2sp_sddmm: out[p] = s_p * <A[i], B[j]> on S's pattern; s_values=None means all ones
    (dtype=torch.bfloat16: b2sp_sddmm_bf16, A and B in bfloat16)."""
    _want(row_ptr, torch.int32, "row_ptr"); _want(col_idx, torch.int32, "col_idx")
    _want(s_values, torch.float32, "s_values"); _want(A, dtype, "A"); _want(B, dtype, "B")
    M, nnz = row_ptr.numel() - 1, col_idx.numel()
    K, Kd = B.shape
    if A.shape != (M, Kd):
        raise ValueError("A must be [M, Kd]")
    if out is None:
        out = torch.empty(nnz, dtype=torch.float32, device=A.device)
    ws, wsb = _workspace(OP_SDDMM, M, K, Kd, 0, nnz, A.device, workspace, algo)
    fn, name = (lib.b2sp_sddmm, "b2sp_sddmm") if dtype == torch.float32 else (lib.b2sp_sddmm_bf16, "b2sp_sddmm_bf16")
    _check(fn(M, K, Kd, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(s_values), _ptr(A), _ld(A),
                          _ptr(B), _ld(B), _ptr(out), _ptr(ws), wsb, algo, _stream()), name)
    return out


def fusedmm(row_ptr, col_idx, s_values, A, B, D, out=None, workspace=None, algo=ALGO_AUTO, dtype=torch.float32):
    """b2sp_fusedmm: O = (S .* (A @ B.T)) @ D in one pass; the sampled values never reach HBM
    (dtype=torch.bfloat16: b2sp_fusedmm_bf16, A, B and D in bfloat16)."""
    _want(row_ptr, torch.int32, "row_ptr"); _want(col_idx, torch.int32, "col_idx")
    _want(s_values, torch.float32, "s_values"); _want(A, dtype, "A"); _want(B, dtype, "B")
    _want(D, dtype, "D")
    M, nnz = row_ptr.numel() - 1, col_idx.numel()
    K, Kd = B.shape
    N = D.shape[1]
    if A.shape != (M, Kd) or D.shape[0] != K:
        raise ValueError("A must be [M, Kd] and D [K, N]")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=D.device)
    ws, wsb = _workspace(OP_FUSEDMM, M, K, Kd, N, nnz, D.device, workspace, algo)
    fn, name = (lib.b2sp_fusedmm, "b2sp_fusedmm") if dtype == torch.float32 else (lib.b2sp_fusedmm_bf16, "b2sp_fusedmm_bf16")
    _check(fn(M, K, Kd, N, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(s_values), _ptr(A),
                            _ld(A), _ptr(B), _ld(B), _ptr(D), _ld(D), _ptr(out), _ld(out), _ptr(ws), wsb,
                            algo, _stream()), name)
    return out


def _batch_dims(row_ptr, col_idx):
    """[batch, M + 1] row pointers and [batch, nnz_stride] column indices (a 1-D row_ptr: one shared pattern)."""
    if row_ptr.dim() == 1:
        return None, row_ptr.numel() - 1, 0, col_idx.shape[-1]
    assert row_ptr.stride(1) == 1 and col_idx.dim() == 2 and col_idx.stride(1) == 1
    return row_ptr.shape[0], row_ptr.shape[1] - 1, row_ptr.stride(0), col_idx.stride(0)


def _batch_stride(t, batch):
    """Element stride between the problems of a [batch, rows, cols] operand (0 for a shared [rows, cols] one)."""
    if t.dim() == 2:
        return 0
    assert t.dim() == 3 and t.shape[0] == batch and (t.shape[2] <= 1 or t.stride(2) == 1)
    return t.stride(0)


def workspace_bytes_batched(batch: int, M: int, K: int, Kd: int, N: int, nnz_stride: int) -> int:
    return int(lib.b2sp_workspace_bytes_batched(batch, M, K, Kd, N, nnz_stride))


def prepare_pattern_batched(row_ptr, col_idx, K, workspace, batch=None):
    """b2sp_prepare_pattern_batched: the window tables of a batch of patterns (row_ptr [batch, M + 1],
    col_idx [batch, nnz_stride]; 1-D tensors with `batch`: one pattern shared by all problems)."""
    nb, M, rps, nzs = _batch_dims(row_ptr, col_idx)
    nb = batch if nb is None else nb
    _check(lib.b2sp_prepare_pattern_batched(nb, M, K, nzs, _ptr(row_ptr), rps, _ptr(col_idx), _ptr(workspace),
                                            workspace.numel(), _stream()), "b2sp_prepare_pattern_batched")


def fusedmm_batched(row_ptr, col_idx, s_values, A, B, D, out=None, workspace=None, algo=ALGO_AUTO, dtype=torch.float32):
    """b2sp_fusedmm_batched: O[b] = (S[b] .* (A[b] @ B[b].T)) @ D[b] for all problems of a batch in one
    call.  row_ptr [batch, M + 1] (each problem's positions start at 0), col_idx / s_values
    [batch, nnz_stride] (rows padded to a common length), A [batch, M, Kd], B [batch, K, Kd],
    D [batch, K, N]; a 1-D row_ptr / col_idx / s_values or a 2-D dense operand is shared by all problems.
    dtype=torch.bfloat16: b2sp_fusedmm_batched_bf16 (A, B, D in bfloat16)."""
    _want(row_ptr, torch.int32, "row_ptr"); _want(col_idx, torch.int32, "col_idx")
    _want(s_values, torch.float32, "s_values"); _want(A, dtype, "A"); _want(B, dtype, "B")
    _want(D, dtype, "D")
    nb, M, rps, nzs = _batch_dims(row_ptr, col_idx)
    if nb is None:
        nb = max(t.shape[0] if t.dim() == 3 else 1 for t in (A, B, D))
    K, Kd, N = B.shape[-2], B.shape[-1], D.shape[-1]
    if out is None:
        out = torch.empty((nb, M, N), dtype=torch.float32, device=D.device)
    assert out.dim() == 3 and out.shape[0] == nb and out.stride(2) == 1
    if workspace is None:
        workspace = torch.empty(max(workspace_bytes_batched(nb, M, K, Kd, N, nzs), 1 << 20), dtype=torch.uint8,
                                device=D.device)
    ld = lambda t: t.stride(-2) if t.shape[-2] > 1 else max(t.shape[-1], t.stride(-2))
    fn, name = ((lib.b2sp_fusedmm_batched, "b2sp_fusedmm_batched") if dtype == torch.float32
                else (lib.b2sp_fusedmm_batched_bf16, "b2sp_fusedmm_batched_bf16"))
    _check(fn(nb, M, K, Kd, N, nzs, _ptr(row_ptr), rps, _ptr(col_idx), _ptr(s_values),
                                    _ptr(A), ld(A), _batch_stride(A, nb), _ptr(B), ld(B), _batch_stride(B, nb),
                                    _ptr(D), ld(D), _batch_stride(D, nb), _ptr(out), ld(out), out.stride(0),
                                    _ptr(workspace), workspace.numel(), algo, _stream()), name)
    return out


def _host(t, dtype, name):
    if t is None:
        return None
    if t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CPU tensor of {dtype}")
    return t


def spmm_host(row_ptr, col_idx, values, D, out):
    """b2sp_spmm_host: host tensors in, host tensor out (copies happen inside the library)."""
    for t, dt, n in ((row_ptr, torch.int32, "row_ptr"), (col_idx, torch.int32, "col_idx"),
                     (values, torch.float32, "values"), (D, torch.float32, "D"), (out, torch.float32, "out")):
        _host(t, dt, n)
    M, nnz = row_ptr.numel() - 1, col_idx.numel()
    K, N = D.shape
    _check(lib.b2sp_spmm_host(M, K, N, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(values), _ptr(D),
                              _ptr(out), _stream()), "b2sp_spmm_host")
    return out


def sddmm_host(row_ptr, col_idx, s_values, A, B, out):
    for t, dt, n in ((row_ptr, torch.int32, "row_ptr"), (col_idx, torch.int32, "col_idx"),
                     (s_values, torch.float32, "s_values"), (A, torch.float32, "A"),
                     (B, torch.float32, "B"), (out, torch.float32, "out")):
        _host(t, dt, n)
    M, nnz = row_ptr.numel() - 1, col_idx.numel()
    K, Kd = B.shape
    _check(lib.b2sp_sddmm_host(M, K, Kd, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(s_values), _ptr(A),
                               _ptr(B), _ptr(out), _stream()), "b2sp_sddmm_host")
    return out


def fusedmm_host(row_ptr, col_idx, s_values, A, B, D, out):
    for t, dt, n in ((row_ptr, torch.int32, "row_ptr"), (col_idx, torch.int32, "col_idx"),
                     (s_values, torch.float32, "s_values"), (A, torch.float32, "A"),
                     (B, torch.float32, "B"), (D, torch.float32, "D"), (out, torch.float32, "out")):
        _host(t, dt, n)
    M, nnz = row_ptr.numel() - 1, col_idx.numel()
    K, Kd = B.shape
    N = D.shape[1]
    _check(lib.b2sp_fusedmm_host(M, K, Kd, N, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(s_values),
                                 _ptr(A), _ptr(B), _ptr(D), _ptr(out), _stream()), "b2sp_fusedmm_host")
    return out


def prepare_pattern(row_ptr, col_idx, K, workspace):
    """b2sp_prepare_pattern: build S's window table in `workspace` once; later calls that pass the same
    workspace and algo=ALGO_TILE_PREPARED reuse it."""
    M, nnz = row_ptr.numel() - 1, col_idx.numel()
    _check(lib.b2sp_prepare_pattern(M, K, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(workspace),
                                    workspace.numel(), _stream()), "b2sp_prepare_pattern")


def validate_csr(row_ptr, col_idx, K) -> bool:
    """b2sp_validate_csr: True if the CSR arrays are well formed (synchronises)."""
    M, nnz = row_ptr.numel() - 1, col_idx.numel()
    ws = torch.empty(256, dtype=torch.uint8, device=row_ptr.device)
    st = lib.b2sp_validate_csr(M, K, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(ws), 256, _stream())
    if st == 3:
        return False
    _check(st, "b2sp_validate_csr")
    return True


def device_status(workspace) -> int:
    return int(lib.b2sp_device_status(_ptr(workspace), _stream()))


# ---- attention over a CSR pattern ------------------------------------------------------------------------------------------------
# The checks of these calls stand on the critical path of small ones: they are written out instead of shared, and run on shapes and strides
# that are fetched once.
def _ready(device, *others):
    """Raises where tensors are not on `device`, or that is not the current one."""
    if device.type != "cuda":
        raise ValueError("tensors must be on a CUDA device")
    for t in others:
        if t.device != device:
            raise ValueError(f"tensors on {device} and {t.device}")
    if device.index != _current_device():
        raise ValueError(f"tensors are on {device}, the current device is cuda:{_current_device()}: "
                         "call under torch.cuda.device(...)")


try:
    _current_device = torch._C._cuda_getDevice
except AttributeError:
    _current_device = torch.cuda.current_device
try:
    _capturing = torch._C._cuda_isCurrentStreamCapturing
except AttributeError:
    _capturing = torch.cuda.is_current_stream_capturing


def _scratch(need, device, workspace, stream):
    """`workspace`, or one that this module keeps per thread, device and stream; a call that is being captured gets one of its own, which
    belongs to the graph, so that graphs can be replayed side by side."""
    if workspace is not None:
        if workspace.dtype is not torch.uint8 or workspace.device != device:
            raise ValueError(f"workspace must be uint8 on {device}")
        return workspace
    if _capturing():
        return torch.empty(need, dtype=torch.uint8, device=device)
    key, workspaces = (device.index, stream, "attention"), _kept.workspaces
    workspace = workspaces.get(key)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1 << 20), dtype=torch.uint8, device=device)
        workspaces[key] = workspace
    return workspace


def _mask_dims(row_ptr, col_idx):
    """(patterns, M, row_ptr stride, nnz stride) of 1-D tensors (one pattern), [batch, .] or [batch, heads, .] ones."""
    if row_ptr.dtype is not torch.int32 or col_idx.dtype is not torch.int32:
        raise TypeError("row_ptr and col_idx must be torch.int32")
    a, b = row_ptr.shape, col_idx.shape
    n = len(a)
    if n != len(b) or not 1 <= n <= 3 or (n > 1 and a[:-1] != b[:-1]):
        raise ValueError("row_ptr and col_idx: [.], [batch, .] or [batch, heads, .], alike but for the last size")
    if a[-1] < 1:
        raise ValueError("row_ptr has M + 1 elements")
    if not (row_ptr.is_contiguous() and col_idx.is_contiguous()):
        raise ValueError("row_ptr and col_idx must be contiguous")
    return 1 if n == 1 else a[0] if n == 2 else a[0] * a[1], a[-1] - 1, a[-1], b[-1]


class AttentionPlan:
    """What b2sp_attention_prepare found out about a pattern, in device memory of its own; see attention_plan.  The plan holds on to the
    pattern's tensors: they must not change while it is used."""
    __slots__ = ("row_ptr", "col_idx", "K", "patterns", "M", "nnz_stride", "tiles", "memory", "pattern")


def attention_plan(row_ptr, col_idx, K):
    """b2sp_attention_count_tiles, _prepare and _plan_status: analyses a mask once for any number of attention calls on it
    (synchronises).  row_ptr [M + 1] and col_idx [nnz] for one mask that all problems share, [batch, .] for one per sequence,
    [batch, heads, .] for one per problem (col_idx padded to a common length).  The columns of a row must be distinct, in any order."""
    patterns, M, rps, nzs = _mask_dims(row_ptr, col_idx)
    device = row_ptr.device
    _ready(device, col_idx)
    if patterns < 1:
        raise ValueError("no pattern")
    tiles = _ll(0)
    ws = torch.empty(256, dtype=torch.uint8, device=device)
    args = (patterns, M, K, nzs, _ptr(row_ptr), rps, _ptr(col_idx))
    _check(lib.b2sp_attention_count_tiles(*args, _ptr(ws), 256, ctypes.byref(tiles), _stream()), "b2sp_attention_count_tiles")
    need = lib.b2sp_attention_plan_bytes(patterns, M, K, nzs, tiles.value)
    plan = AttentionPlan()
    plan.row_ptr, plan.col_idx, plan.K, plan.patterns, plan.M, plan.nnz_stride, plan.tiles = row_ptr, col_idx, K, patterns, M, nzs, tiles.value
    plan.pattern = (_ptr(row_ptr), _ptr(col_idx), K, patterns, M, nzs)
    plan.memory = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    _check(lib.b2sp_attention_prepare(*args, tiles.value, _ptr(plan.memory), plan.memory.numel(), _stream()), "b2sp_attention_prepare")
    _check(lib.b2sp_attention_plan_status(_ptr(plan.memory), _stream()), "b2sp_attention_plan_status")
    return plan


def _rows(t, shape, dtype, name):
    """A [batch, heads, rows, d] tensor as b2sp_heads."""
    s = t.stride()
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.shape != shape or (s[3] != 1 and shape[3] > 1):
        raise ValueError(f"{name} must be {list(shape)} with neighbouring elements along d")
    return _HEADS(t.data_ptr(), s[2], s[1], s[0])


@functools.lru_cache(maxsize=4096)
def _attention_need(sizes, nnz_stride, tiles, backward, dtype):
    """b2sp_attention_workspace_bytes, which goes by sizes only (tiles: -1 without a plan)."""
    fn = lib.b2sp_attention_workspace_bytes if dtype == torch.float32 else lib.b2sp_attention_workspace_bytes_bf16
    return fn(_PROBLEM(*sizes, 1.0, 256, sizes[3] + 1, 256, nnz_stride, 256 if tiles >= 0 else 0,
                                                               max(tiles, 0)), backward)


def _attention_problem(row_ptr, col_idx, q, k, scale, plan):
    """(sizes, nnz stride, b2sp_attention_problem, K's shape)"""
    patterns, M, rps, nzs = _mask_dims(row_ptr, col_idx)
    qs, ks = q.shape, k.shape
    if len(qs) != 4 or len(ks) != 4:
        raise ValueError("q, k and v must be [batch, heads, rows, d]")
    B, H, _, d = qs
    Hkv, K = ks[1], ks[2]
    if qs[2] != M or ks[0] != B or ks[3] != d or Hkv < 1 or H % Hkv:
        raise ValueError("q must be [batch, heads, M, d], k and v [batch, kv_heads, K, d], heads a multiple of kv_heads")
    n = len(row_ptr.shape)
    if n > 1 and (row_ptr.shape[0] != B or (n == 3 and row_ptr.shape[1] != H)):
        raise ValueError("row_ptr: [M + 1], [batch, M + 1] or [batch, heads, M + 1]")
    rp, ci = row_ptr.data_ptr(), col_idx.data_ptr()
    memory, tiles = 0, 0
    if plan is not None:
        if type(plan) is not AttentionPlan:
            raise TypeError("plan must come from attention_plan")
        if plan.pattern != (rp, ci, K, patterns, M, nzs):
            raise ValueError("the plan is of another pattern")
        memory, tiles = plan.memory.data_ptr(), plan.tiles
    sizes = (B, H, Hkv, M, K, d, patterns)
    return sizes, nzs, _PROBLEM(*sizes, d ** -0.5 if scale is None else scale, rp, rps, ci, nzs, memory, tiles)


def _lse(lse, shape):
    if lse.dtype is not torch.float32:
        raise TypeError("lse must be torch.float32")
    if lse.shape != shape or not lse.is_contiguous():
        raise ValueError(f"lse must be {list(shape)}, contiguous")


def attention(row_ptr, col_idx, q, k, v, scale=None, plan=None, out=None, lse=None, workspace=None, algo=ALGO_AUTO, dtype=torch.float32):
    """b2sp_attention: (O, lse), O = softmax(scale q k^T over the stored positions of each row) v.  q [batch, heads, M, d], k and v
    [batch, kv_heads, K, d] (any strides but the last; heads / kv_heads neighbouring query heads share a k and v), scale d ** -0.5
    unless given; the mask as in attention_plan, whose result goes into `plan`.  O is like q, in `dtype`; lse fp32 [batch, heads, M]
    (-inf, and a zero row of O, where a row stores nothing).  The results carry no autograd graph: attention_backward gives the gradients.
    dtype=torch.bfloat16: b2sp_attention_bf16."""
    sizes, nzs, p = _attention_problem(row_ptr, col_idx, q, k, scale, plan)
    qs, ks, device = q.shape, k.shape, q.device
    hq, hk, hv = _rows(q, qs, dtype, "q"), _rows(k, ks, dtype, "k"), _rows(v, ks, dtype, "v")
    _ready(device, k, v, row_ptr, col_idx)
    if out is None:
        out = torch.empty_like(q) if 0 not in q.stride() else torch.empty(qs, dtype=dtype, device=device)
    else:
        _ready(device, out)
    if lse is None:
        n, m = qs[1], qs[2]
        lse = torch.empty_strided(qs[:3], (n * m, m, 1), dtype=torch.float32, device=device)   # (half the price of torch.empty)
    else:
        _lse(lse, qs[:3])
        _ready(device, lse)
    stream = _raw_stream(device.index)
    ws = _scratch(_attention_need(sizes, nzs, -1 if plan is None else plan.tiles, 0, dtype), device, workspace, stream)
    fn, name = ((lib.b2sp_attention, "b2sp_attention") if dtype == torch.float32 else (lib.b2sp_attention_bf16, "b2sp_attention_bf16"))
    _check(fn(p, hq, hk, hv, _rows(out, qs, dtype, "out"), lse.data_ptr(), ws.data_ptr(), ws.numel(), algo, stream), name)
    return out, lse


def attention_backward(row_ptr, col_idx, q, k, v, out, lse, dout, plan, scale=None, dq=None, dk=None, dv=None, workspace=None,
                       algo=ALGO_AUTO, dtype=torch.float32):
    """b2sp_attention_backward: (dq, dk, dv) of sum(O * dout), from O and lse as attention left them; the probabilities are computed
    again.  dout is like q; dk and dv of shared heads are summed over the query heads that share them."""
    if plan is None:
        raise ValueError("the backward pass needs a plan")
    sizes, nzs, p = _attention_problem(row_ptr, col_idx, q, k, scale, plan)
    qs, ks, device = q.shape, k.shape, q.device
    _lse(lse, qs[:3])
    h = [_rows(t, s, dtype, n) for t, s, n in ((q, qs, "q"), (k, ks, "k"), (v, ks, "v"), (out, qs, "out"), (dout, qs, "dout"))]
    _ready(device, k, v, row_ptr, col_idx, out, lse, dout)
    # (gradients of operands that the caller expanded get elements of their own)
    fresh = lambda t: torch.empty_like(t) if 0 not in t.stride() or t.numel() == 0 else torch.empty(t.shape, dtype=t.dtype, device=t.device)  # noqa: E731
    given = [t for t in (dq, dk, dv) if t is not None]
    if given:
        _ready(device, *given)
    dq, dk, dv = fresh(q) if dq is None else dq, fresh(k) if dk is None else dk, fresh(v) if dv is None else dv
    stream = _raw_stream(device.index)
    ws = _scratch(_attention_need(sizes, nzs, plan.tiles, 1, dtype), device, workspace, stream)
    fn, name = ((lib.b2sp_attention_backward, "b2sp_attention_backward") if dtype == torch.float32
                else (lib.b2sp_attention_backward_bf16, "b2sp_attention_backward_bf16"))
    _check(fn(p, h[0], h[1], h[2], h[3], lse.data_ptr(), h[4], _rows(dq, qs, dtype, "dq"), _rows(dk, ks, dtype, "dk"), _rows(dv, ks, dtype, "dv"),
              ws.data_ptr(), ws.numel(), algo, stream), name)
    return dq, dk, dv


def attention_last_algo(backward=False) -> int:
    return int(lib.b2sp_attention_last_algo(int(backward)))


def attention_last_launches(backward=False) -> int:
    return int(lib.b2sp_attention_last_launches(int(backward)))


# ---- a cache of keys or values in 4 bits -----------------------------------------------------------------------------------------
def kv4_cache(heads: int, slots: int, d: int, device=None):
    """(codes, scales) of an empty cache for b2sp_kv4_write: uint8 [heads, slots, 16 * ceil(d / 32)] and bfloat16
    [heads, slots, ceil(d / 32)]; all rows read as zeros."""
    G = (d + 31) // 32
    return (torch.full((heads, slots, 16 * G), 0x88, dtype=torch.uint8, device=device or "cuda"),
            torch.zeros((heads, slots, G), dtype=torch.bfloat16, device=device or "cuda"))


def _kv4(codes, scales, heads, d, name):
    """A cache as b2sp_kv4."""
    if codes.dtype is not torch.uint8 or scales.dtype is not torch.bfloat16:
        raise TypeError(f"{name}codes must be torch.uint8, {name}scales torch.bfloat16")
    G, a, s, t = (d + 31) // 32, codes.shape, codes.stride(), scales.stride()
    if len(a) != 3 or a[0] != heads or a[2] != 16 * G or s[2] != 1:
        raise ValueError(f"{name}codes must be [heads, slots, 16 * ceil(d / 32)] with neighbouring bytes in the last dimension")
    if scales.shape != (heads, a[1], G) or (G > 1 and t[2] != 1):
        raise ValueError(f"{name}scales must be [heads, slots, ceil(d / 32)] with neighbouring elements in the last dimension")
    return _KV4(codes.data_ptr(), s[1], s[0], scales.data_ptr(), t[1], t[0], a[1])


_KV4_SCAN_TOKENS = 1024   # up to here b2sp_kv4_write needs no workspace


def _slot_list(slots):
    if slots.dtype is not torch.int32:
        raise TypeError("slots must be torch.int32")
    if slots.dim() != 1 or not slots.is_contiguous():
        raise ValueError("slots must be contiguous, one per token")
    return slots.shape[0]


def kv4_write(x, slots, codes, scales, workspace=None, dtype=torch.float32):
    """b2sp_kv4_write: the rows x [tokens, heads, d] are quantised into the rows `slots` (int32 [tokens]) of a cache (see kv4_cache); slots outside
    the cache are skipped, and of several tokens with one slot the last one's row stays.  dtype: x's, fp32 or bfloat16."""
    if x.dtype is not dtype:
        raise TypeError(f"x must be {dtype}")
    shape, s, device = x.shape, x.stride(), x.device
    if len(shape) != 3 or (shape[2] > 1 and s[2] != 1):
        raise ValueError("x must be [tokens, heads, d] with neighbouring elements along d")
    T, H, d = shape
    c = _kv4(codes, scales, H, d, "")
    if _slot_list(slots) != T:
        raise ValueError("slots must be contiguous, one per token")
    _ready(device, slots, codes, scales)
    stream, ws, size = _raw_stream(device.index), None, 0
    if T > _KV4_SCAN_TOKENS:
        ws = _scratch(lib.b2sp_kv4_write_workspace_bytes(T, codes.shape[1]), device, workspace, stream)
        ws, size = ws.data_ptr(), ws.numel()
    fn, name = (lib.b2sp_kv4_write, "b2sp_kv4_write") if dtype == torch.float32 else (lib.b2sp_kv4_write_bf16, "b2sp_kv4_write_bf16")
    _check(fn(T, H, d, x.data_ptr(), s[0], s[1], slots.data_ptr(), c, ws, size, stream), name)


def kv4_read(slots, codes, scales, d, out=None, dtype=torch.float32):
    """b2sp_kv4_read: [tokens, heads, d] in `dtype`, the values that the rows `slots` of a cache stand for (zeros outside the cache)."""
    H, device = codes.shape[0], codes.device
    c = _kv4(codes, scales, H, d, "")
    T = _slot_list(slots)
    if out is None:
        out = torch.empty_strided((T, H, d), (H * d, d, 1), dtype=dtype, device=device)
    s = out.stride()
    if out.dtype is not dtype:
        raise TypeError(f"out must be {dtype}")
    if out.shape != (T, H, d) or (d > 1 and s[2] != 1):
        raise ValueError("out must be [tokens, heads, d] with neighbouring elements along d")
    _ready(device, slots, scales, out)
    fn, name = (lib.b2sp_kv4_read, "b2sp_kv4_read") if dtype == torch.float32 else (lib.b2sp_kv4_read_bf16, "b2sp_kv4_read_bf16")
    _check(fn(T, H, d, slots.data_ptr(), c, out.data_ptr(), s[0], s[1], _raw_stream(device.index)), name)
    return out


@functools.lru_cache(maxsize=4096)
def _attention_kv4_need(M, heads, kv_heads, d, nnz):
    return lib.b2sp_attention_kv4_workspace_bytes(M, heads, kv_heads, d, nnz)


def attention_kv4(row_ptr, col_idx, q, k_codes, k_scales, v_codes, v_scales, scale=None, out=None, lse=None, workspace=None):
    """b2sp_attention_kv4: (O, lse) of query tokens q [M, heads, d] (bfloat16) over caches held in 4 bits; row i of the CSR arrays
    names the slots that token i sees, for all heads.  O is like q, lse fp32 [M, heads]; scale d ** -0.5 unless given."""
    if row_ptr.dtype is not torch.int32 or col_idx.dtype is not torch.int32 or q.dtype is not torch.bfloat16:
        raise TypeError("row_ptr and col_idx must be torch.int32, q torch.bfloat16")
    shape, s, device = q.shape, q.stride(), q.device
    if len(shape) != 3 or (shape[2] > 1 and s[2] != 1):
        raise ValueError("q must be [M, heads, d] with neighbouring elements along d")
    M, H, d = shape
    if row_ptr.shape != (M + 1,) or col_idx.dim() != 1 or not (row_ptr.is_contiguous() and col_idx.is_contiguous()):
        raise ValueError("row_ptr must be [M + 1] and col_idx [nnz], contiguous")
    Hkv, nnz = k_codes.shape[0], col_idx.shape[0]
    if Hkv < 1 or H % Hkv:
        raise ValueError("heads must be a multiple of the cache's")
    k, v = _kv4(k_codes, k_scales, Hkv, d, "k_"), _kv4(v_codes, v_scales, Hkv, d, "v_")
    if out is None:
        out = torch.empty_like(q) if 0 not in s else torch.empty(shape, dtype=q.dtype, device=device)
    t = out.stride()
    if out.dtype is not torch.bfloat16 or out.shape != shape or (d > 1 and t[2] != 1):
        raise ValueError("out must be like q, with neighbouring elements along d")
    if lse is None:
        lse = torch.empty_strided((M, H), (H, 1), dtype=torch.float32, device=device)
    else:
        _lse(lse, (M, H))
    _ready(device, row_ptr, col_idx, k_codes, k_scales, v_codes, v_scales, out, lse)
    stream = _raw_stream(device.index)
    ws = _scratch(_attention_kv4_need(M, H, Hkv, d, nnz), device, workspace, stream)
    _check(lib.b2sp_attention_kv4(M, H, Hkv, d, nnz, row_ptr.data_ptr(), col_idx.data_ptr(), q.data_ptr(), s[0], s[1], k, v,
                                  d ** -0.5 if scale is None else scale, out.data_ptr(), t[0], t[1], lse.data_ptr(), ws.data_ptr(),
                                  ws.numel(), stream), "b2sp_attention_kv4")
    return out, lse
