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


class _Heads(ctypes.Structure):
    """b2sp_heads"""
    _fields_ = [("data", _vp), ("ld", _ll), ("stride_head", _ll), ("stride_batch", _ll)]


class _AttentionProblem(ctypes.Structure):
    """b2sp_attention_problem"""
    _fields_ = [("batch", _i), ("heads", _i), ("kv_heads", _i), ("M", _i), ("K", _i), ("d", _i), ("patterns", _i),
                ("scale", ctypes.c_float), ("row_ptr", _vp), ("row_ptr_stride", _ll), ("col_idx", _vp), ("nnz_stride", _ll),
                ("plan", _vp), ("plan_tiles", _ll)]


class _Kv4(ctypes.Structure):
    """b2sp_kv4"""
    _fields_ = [("codes", _vp), ("code_ld", _ll), ("code_stride_head", _ll), ("scales", _vp), ("scale_ld", _ll),
                ("scale_stride_head", _ll), ("slots", _i)]


_ph, _pp, _pk = (ctypes.POINTER(t) for t in (_Heads, _AttentionProblem, _Kv4))
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


_ws_cache = {}


_planner_setting = 0   # counts the calls of the debug hooks that change the planner's choice


# Sizes only, by the planner's setting: a size that another thread asked for while a hook took effect is not met again.
@functools.lru_cache(maxsize=4096)
def _workspace_need(op, M, K, Kd, N, nnz, algo, setting):
    return workspace_bytes(op, M, K, Kd, N, nnz, algo)


def _workspace(op, M, K, Kd, N, nnz, device, workspace, algo=0):
    if workspace is None:
        need = _workspace_need(op, M, K, Kd, N, nnz, algo, _planner_setting)
        key = (device.index, _raw_stream(device.index))
        workspace = _ws_cache.get(key)
        if workspace is None or workspace.numel() < need:
            workspace = torch.empty(max(need, 1 << 20), dtype=torch.uint8, device=device)
            _ws_cache[key] = workspace
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
def _same_device(first, *others):
    """The device that all tensors are on, made the current one's index; raises where they differ."""
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError(f"tensors on {first.device} and {t.device}")
    return first.device


def _on_current_device(device):
    if device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is cuda:{torch.cuda.current_device()}: "
                         "call under torch.cuda.device(...)")


def _scratch(need, device, workspace):
    """`workspace`, or one that this module keeps per device and stream; a call that is being captured gets one of its own, which
    belongs to the graph, so that graphs can be replayed side by side."""
    if workspace is not None:
        return workspace
    if torch.cuda.is_current_stream_capturing():
        return torch.empty(need, dtype=torch.uint8, device=device)
    key = (device.index, _raw_stream(device.index), "attention")
    workspace = _ws_cache.get(key)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1 << 20), dtype=torch.uint8, device=device)
        _ws_cache[key] = workspace
    return workspace


def _mask_dims(row_ptr, col_idx):
    """(patterns, M, row_ptr stride, nnz stride) of 1-D tensors (one pattern), [batch, .] or [batch, heads, .] ones."""
    _want(row_ptr, torch.int32, "row_ptr"); _want(col_idx, torch.int32, "col_idx")
    if row_ptr.dim() != col_idx.dim() or not 1 <= row_ptr.dim() <= 3 or row_ptr.shape[:-1] != col_idx.shape[:-1]:
        raise ValueError("row_ptr and col_idx: [.], [batch, .] or [batch, heads, .], alike but for the last size")
    if row_ptr.shape[-1] < 1:
        raise ValueError("row_ptr has M + 1 elements")
    if not (row_ptr.is_contiguous() and col_idx.is_contiguous()):
        raise ValueError("row_ptr and col_idx must be contiguous")
    patterns = 1
    for n in row_ptr.shape[:-1]:
        patterns *= n
    return patterns, row_ptr.shape[-1] - 1, row_ptr.shape[-1], col_idx.shape[-1]


class AttentionPlan:
    """What b2sp_attention_prepare found out about a pattern, in device memory of its own; see attention_plan.  The plan holds on to the
    pattern's tensors: they must not change while it is used."""
    __slots__ = ("row_ptr", "col_idx", "K", "patterns", "M", "nnz_stride", "tiles", "memory")


def attention_plan(row_ptr, col_idx, K):
    """b2sp_attention_count_tiles, _prepare and _plan_status: analyses a mask once for any number of attention calls on it
    (synchronises).  row_ptr [M + 1] and col_idx [nnz] for one mask that all problems share, [batch, .] for one per sequence,
    [batch, heads, .] for one per problem (col_idx padded to a common length).  The columns of a row must be distinct, in any order."""
    patterns, M, rps, nzs = _mask_dims(row_ptr, col_idx)
    device = _same_device(row_ptr, col_idx)
    _on_current_device(device)
    if patterns < 1:
        raise ValueError("no pattern")
    tiles = _ll(0)
    ws = torch.empty(256, dtype=torch.uint8, device=device)
    args = (patterns, M, K, nzs, _ptr(row_ptr), rps, _ptr(col_idx))
    _check(lib.b2sp_attention_count_tiles(*args, _ptr(ws), 256, ctypes.byref(tiles), _stream()), "b2sp_attention_count_tiles")
    need = lib.b2sp_attention_plan_bytes(patterns, M, K, nzs, tiles.value)
    plan = AttentionPlan()
    plan.row_ptr, plan.col_idx, plan.K, plan.patterns, plan.M, plan.nnz_stride, plan.tiles = row_ptr, col_idx, K, patterns, M, nzs, tiles.value
    plan.memory = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    _check(lib.b2sp_attention_prepare(*args, tiles.value, _ptr(plan.memory), plan.memory.numel(), _stream()), "b2sp_attention_prepare")
    _check(lib.b2sp_attention_plan_status(_ptr(plan.memory), _stream()), "b2sp_attention_plan_status")
    return plan


def _heads(t):
    s = t.stride()
    return _Heads(t.data_ptr(), s[2], s[1], s[0])


def _attention_problem(row_ptr, col_idx, q, k, v, scale, plan, dtype):
    patterns, M, rps, nzs = _mask_dims(row_ptr, col_idx)
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _want(t, dtype, n)
        if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
            raise ValueError(f"{n} must be [batch, heads, rows, d] with neighbouring elements along d")
    B, H, _, d = q.shape
    Hkv, K = k.shape[1], k.shape[2]
    if q.shape[2] != M or k.shape != (B, Hkv, K, d) or v.shape != k.shape or Hkv < 1 or H % Hkv:
        raise ValueError("q must be [batch, heads, M, d], k and v [batch, kv_heads, K, d], heads a multiple of kv_heads")
    if row_ptr.dim() > 1 and (row_ptr.shape[0] != B or (row_ptr.dim() == 3 and row_ptr.shape[1] != H)):
        raise ValueError("row_ptr: [M + 1], [batch, M + 1] or [batch, heads, M + 1]")
    if plan is not None:
        if not isinstance(plan, AttentionPlan):
            raise TypeError("plan must come from attention_plan")
        if (plan.row_ptr.data_ptr(), plan.col_idx.data_ptr(), plan.K, plan.patterns, plan.M, plan.nnz_stride) != (
                row_ptr.data_ptr(), col_idx.data_ptr(), K, patterns, M, nzs):
            raise ValueError("the plan is of another pattern")
    _on_current_device(_same_device(q, k, v, row_ptr, col_idx, plan.memory if plan is not None else None))
    return _AttentionProblem(B, H, Hkv, M, K, d, patterns, d ** -0.5 if scale is None else scale, row_ptr.data_ptr(), rps,
                             col_idx.data_ptr(), nzs, plan.memory.data_ptr() if plan is not None else None, plan.tiles if plan is not None else 0)


def _given(t, shape, dtype, name, like):
    """An operand or output that the caller passes: of this shape and type, elements of its last dimension neighbours."""
    _want(t, dtype, name)
    if tuple(t.shape) != tuple(shape) or (shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name} must be {list(shape)} with neighbouring elements in the last dimension")
    _same_device(like, t)
    return t


def attention(row_ptr, col_idx, q, k, v, scale=None, plan=None, out=None, lse=None, workspace=None, algo=ALGO_AUTO, dtype=torch.float32):
    """b2sp_attention: (O, lse), O = softmax(scale q k^T over the stored positions of each row) v.  q [batch, heads, M, d], k and v
    [batch, kv_heads, K, d] (any strides but the last; heads / kv_heads neighbouring query heads share a k and v), scale d ** -0.5
    unless given; the mask as in attention_plan, whose result goes into `plan`.  O is like q, in `dtype`; lse fp32 [batch, heads, M]
    (-inf, and a zero row of O, where a row stores nothing).  dtype=torch.bfloat16: b2sp_attention_bf16."""
    p = _attention_problem(row_ptr, col_idx, q, k, v, scale, plan, dtype)
    out = torch.empty_like(q) if out is None else _given(out, q.shape, dtype, "out", q)
    if lse is None:
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    elif not _given(lse, q.shape[:3], torch.float32, "lse", q).is_contiguous():
        raise ValueError("lse must be contiguous")
    ws = _scratch(lib.b2sp_attention_workspace_bytes(ctypes.byref(p), 0), q.device, workspace)
    fn, name = ((lib.b2sp_attention, "b2sp_attention") if dtype == torch.float32 else (lib.b2sp_attention_bf16, "b2sp_attention_bf16"))
    _check(fn(ctypes.byref(p), _heads(q), _heads(k), _heads(v), _heads(out), _ptr(lse), _ptr(ws), ws.numel(), algo, _stream()), name)
    return out, lse


def attention_backward(row_ptr, col_idx, q, k, v, out, lse, dout, plan, scale=None, dq=None, dk=None, dv=None, workspace=None,
                       algo=ALGO_AUTO, dtype=torch.float32):
    """b2sp_attention_backward: (dq, dk, dv) of sum(O * dout), from O and lse as attention left them; the probabilities are computed
    again.  dout is like q; dk and dv of shared heads are summed over the query heads that share them."""
    if plan is None:
        raise ValueError("the backward pass needs a plan")
    p = _attention_problem(row_ptr, col_idx, q, k, v, scale, plan, dtype)
    _given(out, q.shape, dtype, "out", q); _given(dout, q.shape, dtype, "dout", q)
    if not _given(lse, q.shape[:3], torch.float32, "lse", q).is_contiguous():
        raise ValueError("lse must be contiguous")
    # (gradients of operands that the caller expanded get elements of their own)
    fresh = lambda t: torch.empty_like(t) if 0 not in t.stride() or t.numel() == 0 else torch.empty(t.shape, dtype=t.dtype, device=t.device)  # noqa: E731
    dq = fresh(q) if dq is None else _given(dq, q.shape, dtype, "dq", q)
    dk = fresh(k) if dk is None else _given(dk, k.shape, dtype, "dk", q)
    dv = fresh(v) if dv is None else _given(dv, v.shape, dtype, "dv", q)
    ws = _scratch(lib.b2sp_attention_workspace_bytes(ctypes.byref(p), 1), q.device, workspace)
    fn, name = ((lib.b2sp_attention_backward, "b2sp_attention_backward") if dtype == torch.float32
                else (lib.b2sp_attention_backward_bf16, "b2sp_attention_backward_bf16"))
    _check(fn(ctypes.byref(p), _heads(q), _heads(k), _heads(v), _heads(out), _ptr(lse), _heads(dout), _heads(dq), _heads(dk), _heads(dv),
              _ptr(ws), ws.numel(), algo, _stream()), name)
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
    _want(codes, torch.uint8, name + "codes"); _want(scales, torch.bfloat16, name + "scales")
    G = (d + 31) // 32
    if codes.dim() != 3 or codes.shape[0] != heads or codes.shape[2] != 16 * G or codes.stride(2) != 1:
        raise ValueError(f"{name}codes must be [heads, slots, 16 * ceil(d / 32)] with neighbouring bytes in the last dimension")
    if tuple(scales.shape) != (heads, codes.shape[1], G) or (G > 1 and scales.stride(2) != 1):
        raise ValueError(f"{name}scales must be [heads, slots, ceil(d / 32)] with neighbouring elements in the last dimension")
    return _Kv4(codes.data_ptr(), codes.stride(1), codes.stride(0), scales.data_ptr(), scales.stride(1), scales.stride(0), codes.shape[1])


_KV4_SCAN_TOKENS = 1024   # up to here b2sp_kv4_write needs no workspace


def _slot_list(slots, n=None):
    _want(slots, torch.int32, "slots")
    if slots.dim() != 1 or not slots.is_contiguous() or (n is not None and slots.numel() != n):
        raise ValueError("slots must be contiguous, one per token")
    return slots


def kv4_write(x, slots, codes, scales, workspace=None, dtype=torch.float32):
    """b2sp_kv4_write: the rows x [tokens, heads, d] are quantised into the rows `slots` (int32 [tokens]) of a cache (see kv4_cache); slots outside
    the cache are skipped, and of several tokens with one slot the last one's row stays.  dtype: x's, fp32 or bfloat16."""
    _want(x, dtype, "x")
    if x.dim() != 3 or (x.shape[2] > 1 and x.stride(2) != 1):
        raise ValueError("x must be [tokens, heads, d] with neighbouring elements along d")
    T, H, d = x.shape
    c = _kv4(codes, scales, H, d, "")
    _slot_list(slots, T)
    _on_current_device(_same_device(x, slots, codes, scales))
    fn, name = (lib.b2sp_kv4_write, "b2sp_kv4_write") if dtype == torch.float32 else (lib.b2sp_kv4_write_bf16, "b2sp_kv4_write_bf16")
    ws = workspace
    if T > _KV4_SCAN_TOKENS:
        ws = _scratch(lib.b2sp_kv4_write_workspace_bytes(T, c.slots), x.device, workspace)
    _check(fn(T, H, d, _ptr(x), x.stride(0), x.stride(1), _ptr(slots), c, _ptr(ws), 0 if ws is None else ws.numel(), _stream()), name)


def kv4_read(slots, codes, scales, d, out=None, dtype=torch.float32):
    """b2sp_kv4_read: [tokens, heads, d] in `dtype`, the values that the rows `slots` of a cache stand for (zeros outside the cache)."""
    H = codes.shape[0]
    c = _kv4(codes, scales, H, d, "")
    T = _slot_list(slots).numel()
    if out is None:
        out = torch.empty((T, H, d), dtype=dtype, device=codes.device)
    _given(out, (T, H, d), dtype, "out", codes)
    _on_current_device(_same_device(codes, slots, scales))
    fn, name = (lib.b2sp_kv4_read, "b2sp_kv4_read") if dtype == torch.float32 else (lib.b2sp_kv4_read_bf16, "b2sp_kv4_read_bf16")
    _check(fn(T, H, d, _ptr(slots), c, _ptr(out), out.stride(0), out.stride(1), _stream()), name)
    return out


def attention_kv4(row_ptr, col_idx, q, k_codes, k_scales, v_codes, v_scales, scale=None, out=None, lse=None, workspace=None):
    """b2sp_attention_kv4: (O, lse) of query tokens q [M, heads, d] (bfloat16) over caches held in 4 bits; row i of the CSR arrays
    names the slots that token i sees, for all heads.  O is like q, lse fp32 [M, heads]; scale d ** -0.5 unless given."""
    _want(row_ptr, torch.int32, "row_ptr"); _want(col_idx, torch.int32, "col_idx"); _want(q, torch.bfloat16, "q")
    if q.dim() != 3 or (q.shape[2] > 1 and q.stride(2) != 1) or row_ptr.dim() != 1 or col_idx.dim() != 1:
        raise ValueError("q must be [M, heads, d] with neighbouring elements along d, row_ptr [M + 1], col_idx [nnz]")
    if not (row_ptr.is_contiguous() and col_idx.is_contiguous()) or row_ptr.numel() != q.shape[0] + 1:
        raise ValueError("row_ptr must be [M + 1], contiguous as col_idx")
    M, H, d = q.shape
    Hkv, nnz = k_codes.shape[0], col_idx.numel()
    if Hkv < 1 or H % Hkv:
        raise ValueError("heads must be a multiple of the cache's")
    k, v = _kv4(k_codes, k_scales, Hkv, d, "k_"), _kv4(v_codes, v_scales, Hkv, d, "v_")
    out = torch.empty_like(q) if out is None else _given(out, q.shape, torch.bfloat16, "out", q)
    if lse is None:
        lse = torch.empty((M, H), dtype=torch.float32, device=q.device)
    elif not _given(lse, (M, H), torch.float32, "lse", q).is_contiguous():
        raise ValueError("lse must be contiguous")
    _on_current_device(_same_device(q, row_ptr, col_idx, k_codes, k_scales, v_codes, v_scales))
    ws = _scratch(lib.b2sp_attention_kv4_workspace_bytes(M, H, Hkv, d, nnz), q.device, workspace)
    _check(lib.b2sp_attention_kv4(M, H, Hkv, d, nnz, _ptr(row_ptr), _ptr(col_idx), _ptr(q), q.stride(0), q.stride(1), k, v,
                                  d ** -0.5 if scale is None else scale, _ptr(out), out.stride(0), out.stride(1), _ptr(lse), _ptr(ws),
                                  ws.numel(), _stream()), "b2sp_attention_kv4")
    return out, lse
