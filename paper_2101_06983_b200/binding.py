"""Thin ctypes binding over libgradcache.so (include/gradcache.h).

Argument marshalling only: torch tensors supply device memory and the current CUDA stream;
every numerical step runs inside the library's kernels.  There is no CPU fallback: if the
shared library is missing the import fails, and the calls need a CUDA device.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import _build

GC_F32, GC_BF16 = 0, 1
GC_MASK_NONE, GC_MASK_SELF = 0, 1
GC_OP_FWD, GC_OP_BWD, GC_OP_BUILD, GC_OP_BUILD_STORED = 0, 1, 2, 3
GC_DEV_POS_RANGE, GC_DEV_POS_MASKED, GC_DEV_WAIT_LIMIT, GC_DEV_GRAD_NONFINITE = 1, 2, 4, 8

EXPORTS = ("gc_workspace_bytes", "gc_plan_name", "gc_kernel_launches", "gc_loss_fwd",
           "gc_loss_bwd", "gc_build_cache", "gc_build_cache_stored", "gc_status_string",
           "gc_profile_enable",
           "gc_profile_read", "gc_profile_read_call", "gc_static_scratch_need", "gc_loss_fwd_static",
           "gc_cache_apply_workspace_bytes", "gc_cache_apply", "gc_shard_workspace_bytes",
           "gc_shard_fwd_dq", "gc_shard_dp", "gc_selftest_wait_limit", "gc_row_normalize",
           "gc_cosine_bwd", "gc_dtau_workspace_bytes", "gc_dtau", "gc_dist_begin",
           "gc_dist_accumulate", "gc_dist_finish", "gc_dist_w_block", "gc_dist_dot_block",
           "gc_multi_pos_workspace_bytes", "gc_build_cache_multi_pos",
           "gc_two_direction_workspace_bytes", "gc_build_cache_two_direction",
           "gc_grad_workspace_bytes", "gc_grad_norm", "gc_grad_scale", "gc_grad_clip",
           "gc_quantize_rows", "gc_matmul_i8", "gc_matmul_i8_plan_name")
GC_STATIC_SCRATCH_BYTES = 2 << 20


class _Tensor(ctypes.Structure):
    """gc_tensor of the C ABI."""
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld", ctypes.c_int64), ("ld_out", ctypes.c_int64),
                ("dtype", ctypes.c_int)]


class GradCacheError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (gc_status {status})")


def _load() -> ctypes.CDLL:
    path = _build.LIB
    if not os.path.exists(path):
        raise ImportError(
            f"{path} is missing: build it with `python -m paper_2101_06983_b200._build` "
            "(there is no fallback implementation)")
    lib = ctypes.CDLL(path)
    vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    common = [vp, i64, vp, i64, vp, i64, i64, i32, f32, i32, i32]
    lib.gc_workspace_bytes.restype = ctypes.c_size_t
    lib.gc_workspace_bytes.argtypes = [i32, i64, i64, i32, i32]
    lib.gc_plan_name.restype = ctypes.c_char_p
    lib.gc_plan_name.argtypes = [i32, i64, i64, i32, i32]
    lib.gc_kernel_launches.restype = i32
    lib.gc_kernel_launches.argtypes = [i32, i64, i64, i32, i32]
    lib.gc_status_string.restype = ctypes.c_char_p
    lib.gc_status_string.argtypes = [i32]
    lib.gc_loss_fwd.restype = i32
    lib.gc_loss_fwd.argtypes = common + [vp, vp, vp, vp, ctypes.c_size_t, vp, vp]
    lib.gc_loss_bwd.restype = i32
    lib.gc_loss_bwd.argtypes = common + [vp, vp, i64, vp, i64, vp, ctypes.c_size_t, vp, vp]
    lib.gc_build_cache.restype = i32
    lib.gc_build_cache.argtypes = common + [vp, vp, vp, vp, i64, vp, i64, vp, ctypes.c_size_t,
                                            vp, vp]
    lib.gc_build_cache_stored.restype = i32
    lib.gc_build_cache_stored.argtypes = lib.gc_build_cache.argtypes
    lib.gc_static_scratch_need.restype = ctypes.c_size_t
    lib.gc_static_scratch_need.argtypes = [i64, i64, i32, i32]
    lib.gc_loss_fwd_static.restype = i32
    lib.gc_loss_fwd_static.argtypes = common + [vp, vp, vp, vp, vp]
    lib.gc_cache_apply_workspace_bytes.restype = ctypes.c_size_t
    lib.gc_cache_apply_workspace_bytes.argtypes = [i64, i32, i32]
    lib.gc_cache_apply.restype = i32
    lib.gc_cache_apply.argtypes = [vp, i64, vp, i64, i64, i32, i32, i32, vp, i64, i32, vp,
                                   ctypes.c_size_t, vp, vp]
    lib.gc_shard_workspace_bytes.restype = ctypes.c_size_t
    lib.gc_shard_workspace_bytes.argtypes = [i64, i64, i32, i32, i64, i64]
    lib.gc_shard_fwd_dq.restype = i32
    lib.gc_shard_fwd_dq.argtypes = common + [i64, i64, vp, vp, vp, vp, i64, vp, ctypes.c_size_t,
                                             vp, vp]
    lib.gc_shard_dp.restype = i32
    lib.gc_shard_dp.argtypes = common + [vp, i64, i64, vp, i64, vp, ctypes.c_size_t, vp, vp]
    lib.gc_row_normalize.restype = i32
    lib.gc_row_normalize.argtypes = [vp, i64, i64, i32, i32, vp, i64, vp, vp]
    lib.gc_cosine_bwd.restype = i32
    lib.gc_cosine_bwd.argtypes = [vp, i64, i64, i32, i32, vp, vp, i64, vp, i64, vp]
    lib.gc_dtau_workspace_bytes.restype = ctypes.c_size_t
    lib.gc_dtau_workspace_bytes.argtypes = [i64]
    lib.gc_dtau.restype = i32
    lib.gc_dtau.argtypes = [vp, i64, vp, i64, i64, i32, f32, i32, vp, vp, ctypes.c_size_t, vp]
    lib.gc_multi_pos_workspace_bytes.restype = ctypes.c_size_t
    lib.gc_multi_pos_workspace_bytes.argtypes = [i64, i64, i32, i32, i64]
    lib.gc_build_cache_multi_pos.restype = i32
    lib.gc_build_cache_multi_pos.argtypes = [vp, i64, vp, i64, vp, vp, i64, i64, i64, i32, f32, i32,
                                             i32, vp, vp, vp, i64, vp, i64, vp, ctypes.c_size_t,
                                             vp, vp]
    lib.gc_two_direction_workspace_bytes.restype = ctypes.c_size_t
    lib.gc_two_direction_workspace_bytes.argtypes = [i64, i64, i32, i32]
    lib.gc_build_cache_two_direction.restype = i32
    lib.gc_build_cache_two_direction.argtypes = [vp, i64, vp, i64, vp, i64, i64, i32, f32, i32, vp,
                                                 vp, vp, i64, vp, i64, vp, ctypes.c_size_t, vp, vp]
    lib.gc_dist_begin.restype = i32
    lib.gc_dist_begin.argtypes = [vp, vp, vp, i64, vp]
    lib.gc_dist_accumulate.restype = i32
    lib.gc_dist_accumulate.argtypes = [vp, i64, i64, i64, i64, i64, vp, i64, i64, f32, i32, vp, vp, vp, vp]
    lib.gc_dist_finish.restype = i32
    lib.gc_dist_finish.argtypes = [vp, vp, vp, vp, i64, i64, i32, vp, vp, vp, vp]
    lib.gc_dist_w_block.restype = i32
    lib.gc_dist_w_block.argtypes = [vp, i64, i64, i64, i64, i64, vp, vp, i64, i64, f32, i32, vp, i64, vp]
    lib.gc_dist_dot_block.restype = i32
    lib.gc_dist_dot_block.argtypes = [vp, i64, vp, i64, i64, i64, i32, i32, i64, i64, i64, i64, vp, i64, vp]
    lib.gc_grad_workspace_bytes.restype = ctypes.c_size_t
    lib.gc_grad_workspace_bytes.argtypes = [i64]
    lib.gc_grad_norm.restype = i32
    lib.gc_grad_norm.argtypes = [vp, i64, vp, vp, vp, ctypes.c_size_t, vp, vp]
    lib.gc_grad_scale.restype = i32
    lib.gc_grad_scale.argtypes = [vp, i64, vp, f32, vp, vp]
    lib.gc_grad_clip.restype = i32
    lib.gc_grad_clip.argtypes = [vp, i64, f32, vp, vp, vp, ctypes.c_size_t, vp, vp]
    lib.gc_quantize_rows.restype = i32
    lib.gc_quantize_rows.argtypes = [vp, i64, i64, i64, i32, vp, i64, vp, vp]
    lib.gc_matmul_i8.restype = i32
    lib.gc_matmul_i8.argtypes = [vp, i64, vp, vp, i64, vp, i64, i64, i64, i32, vp, i64, vp, vp]
    lib.gc_matmul_i8_plan_name.restype = ctypes.c_char_p
    lib.gc_matmul_i8_plan_name.argtypes = [i64, i64, i64, i32]
    lib.gc_selftest_wait_limit.restype = i32
    lib.gc_selftest_wait_limit.argtypes = [ctypes.c_uint64, vp, vp, vp]
    lib.gc_profile_enable.restype = i32
    lib.gc_profile_enable.argtypes = [i32]
    lib.gc_profile_read.restype = i32
    lib.gc_profile_read.argtypes = [ctypes.POINTER(f32)] * 3
    lib.gc_profile_read_call.restype = i32
    lib.gc_profile_read_call.argtypes = [i64] + [ctypes.POINTER(f32)] * 3
    return lib


_lib = _load()
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch.cuda.current_device


def status_string(status: int) -> str:
    return _lib.gc_status_string(int(status)).decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return GC_F32
    if t.dtype == torch.bfloat16:
        return GC_BF16
    raise TypeError(f"Q/P must be float32 or bfloat16, got {t.dtype}")


_CODES = {torch.float32: GC_F32, torch.bfloat16: GC_BF16}


def gc_workspace_bytes(op: int, B: int, N: int, d: int, dtype: int) -> int:
    return int(_lib.gc_workspace_bytes(op, B, N, d, dtype))


def gc_plan_name(op: int, B: int, N: int, d: int, dtype: int) -> str:
    return _lib.gc_plan_name(op, B, N, d, dtype).decode()


def gc_kernel_launches(op: int, B: int, N: int, d: int, dtype: int) -> int:
    return int(_lib.gc_kernel_launches(op, B, N, d, dtype))


def _ptr(t):
    # the integer itself: a ctypes object per argument costs more than the conversion of an int
    return None if t is None else t.data_ptr()


def _common(Q, P, pos_idx, tau, mask_mode):
    qs, ps = Q.shape, P.shape
    if len(qs) != 2 or len(ps) != 2 or Q.stride(1) != 1 or P.stride(1) != 1:
        raise ValueError("Q and P must be 2-D with unit stride along d")
    if pos_idx.dtype is not torch.int32 or not pos_idx.is_contiguous():
        raise TypeError("pos_idx must be a contiguous int32 tensor")
    B, d = qs
    N = ps[0]
    if P.dtype is not Q.dtype or ps[1] != d:
        raise ValueError("Q and P must share dtype and width")
    code = _dtype_code(Q)
    return (Q.data_ptr(), Q.stride(0), P.data_ptr(), P.stride(0), pos_idx.data_ptr(), B, N, d,
            float(tau), int(mask_mode), code), B, N, d, code


def _stream():
    """The current stream of the current device as an integer.  Asked for on every call, so taken from
    torch's own query (0.3 us against 3 us for building a Stream object: a sixth of a small call)."""
    return _raw_stream(_current_device())


def alloc_workspace(op: int, B: int, N: int, d: int, dtype: int, device) -> torch.Tensor:
    """A workspace tensor of the size gc_workspace_bytes reports (torch memory is 512-byte
    aligned, which covers the 256-byte requirement)."""
    n = max(gc_workspace_bytes(op, B, N, d, dtype), 256)
    return torch.empty(n, dtype=torch.uint8, device=device)


def gc_loss_fwd(Q, P, pos_idx, tau, mask_mode, loss, row_lse, pos_logit=None, ws=None,
                dev_status=None):
    """Eq. 1: writes loss[1], row_lse[B] and optionally pos_logit[B] (all float32 on device)."""
    args, B, N, d, code = _common(Q, P, pos_idx, tau, mask_mode)
    if ws is None:
        ws = alloc_workspace(GC_OP_FWD, B, N, d, code, Q.device)
    rc = _lib.gc_loss_fwd(*args, _ptr(loss), _ptr(row_lse), _ptr(pos_logit), _ptr(ws),
                          ws.numel(), _ptr(dev_status), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_loss_fwd")


def gc_static_scratch_need(B: int, N: int, d: int, dtype: int) -> int:
    return int(_lib.gc_static_scratch_need(B, N, d, dtype))


def gc_loss_fwd_static(Q, P, pos_idx, tau, mask_mode, loss, row_lse, pos_logit=None,
                       dev_status=None):
    """gc_loss_fwd without a caller workspace: the scratch is a fixed array inside the library
    (GC_STATIC_SCRATCH_BYTES).  Nothing is allocated by the call; all outputs are the caller's.
    Raises GradCacheError with GC_ERR_LIMIT (9) when the problem needs more scratch than that.
    Calls on one device share the array, so they must not overlap on the GPU."""
    args, B, N, d, code = _common(Q, P, pos_idx, tau, mask_mode)
    rc = _lib.gc_loss_fwd_static(*args, _ptr(loss), _ptr(row_lse), _ptr(pos_logit),
                                 _ptr(dev_status), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_loss_fwd_static")


def gc_loss_bwd(Q, P, pos_idx, tau, mask_mode, row_lse, dQ, dP, ws=None, dev_status=None):
    """Eq. 5-7 given row_lse: overwrites dQ[B x d] and dP[N x d] (either may be None)."""
    args, B, N, d, code = _common(Q, P, pos_idx, tau, mask_mode)
    if ws is None:
        ws = alloc_workspace(GC_OP_BWD, B, N, d, code, Q.device)
    rc = _lib.gc_loss_bwd(*args, _ptr(row_lse), _ptr(dQ), 0 if dQ is None else dQ.stride(0),
                          _ptr(dP), 0 if dP is None else dP.stride(0), _ptr(ws), ws.numel(),
                          _ptr(dev_status), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_loss_bwd")


def gc_build_cache(Q, P, pos_idx, tau, mask_mode, loss, row_lse, dQ, dP, pos_logit=None,
                   ws=None, dev_status=None):
    """Step 2 of Section 3.3: loss, row_lse and the representation gradient cache dQ, dP."""
    args, B, N, d, code = _common(Q, P, pos_idx, tau, mask_mode)
    if ws is None:
        ws = alloc_workspace(GC_OP_BUILD, B, N, d, code, Q.device)
    rc = _lib.gc_build_cache(*args, _ptr(loss), _ptr(row_lse), _ptr(pos_logit), _ptr(dQ),
                             dQ.stride(0), _ptr(dP), dP.stride(0), _ptr(ws), ws.numel(),
                             _ptr(dev_status), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_build_cache")


def gc_build_cache_stored(Q, P, pos_idx, tau, mask_mode, loss, row_lse, dQ, dP, pos_logit=None,
                          ws=None, dev_status=None):
    """gc_build_cache by way of a stored B x N bf16 weight matrix and two GEMMs (comparison plan)."""
    args, B, N, d, code = _common(Q, P, pos_idx, tau, mask_mode)
    if ws is None:
        ws = alloc_workspace(GC_OP_BUILD_STORED, B, N, d, code, Q.device)
    rc = _lib.gc_build_cache_stored(*args, _ptr(loss), _ptr(row_lse), _ptr(pos_logit), _ptr(dQ),
                                    dQ.stride(0), _ptr(dP), dP.stride(0), _ptr(ws), ws.numel(),
                                    _ptr(dev_status), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_build_cache_stored")


def gc_cache_apply_workspace_bytes(rows: int, d: int, d_in: int) -> int:
    return int(_lib.gc_cache_apply_workspace_bytes(rows, d, d_in))


def gc_cache_apply(U, X, dW, accumulate: bool, ws=None, dev_status=None):
    """Step 3 for a linear encoder (Eq. 8-9): dW[d x d_in] (+)= U^T X with U [rows x d] float32
    (rows of the cache) and X [rows x d_in] bfloat16 (the same rows' encoder inputs)."""
    if U.dim() != 2 or X.dim() != 2 or dW.dim() != 2 or U.stride(1) != 1 or X.stride(1) != 1 \
            or dW.stride(1) != 1:
        raise ValueError("U, X and dW must be 2-D with unit stride along their rows")
    if U.dtype != torch.float32 or dW.dtype != torch.float32:
        raise TypeError("U and dW must be float32")
    rows, d = U.shape
    d_in = X.shape[1]
    if X.shape[0] != rows or tuple(dW.shape) != (d, d_in):
        raise ValueError("shape mismatch")
    if ws is None:
        ws = torch.empty(max(gc_cache_apply_workspace_bytes(rows, d, d_in), 256),
                         dtype=torch.uint8, device=U.device)
    rc = _lib.gc_cache_apply(_ptr(U), U.stride(0), _ptr(X), X.stride(0), rows, d, d_in,
                             _dtype_code(X), _ptr(dW), dW.stride(0), 1 if accumulate else 0,
                             _ptr(ws), ws.numel(), _ptr(dev_status), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_cache_apply")


def gc_shard_workspace_bytes(B: int, N: int, d: int, dtype: int, q_count: int, p_count: int) -> int:
    return int(_lib.gc_shard_workspace_bytes(B, N, d, dtype, q_count, p_count))


def gc_shard_fwd_dq(Q, P, pos_idx, tau, q0, q_count, loss_part, row_lse, dQ, pos_logit=None,
                    ws=None, dev_status=None, mask_mode=GC_MASK_NONE):
    """Section 3.4, local queries [q0, q0 + q_count) of the gathered batch: writes their entries
    of row_lse[B], dQ[q_count x d] and loss_part[1] (this rank's share of the loss of Eq. 1)."""
    args, B, N, d, code = _common(Q, P, pos_idx, tau, mask_mode)
    if ws is None:
        ws = torch.empty(max(gc_shard_workspace_bytes(B, N, d, code, q_count, N), 256),
                         dtype=torch.uint8, device=Q.device)
    rc = _lib.gc_shard_fwd_dq(*args, q0, q_count, _ptr(loss_part), _ptr(row_lse), _ptr(pos_logit),
                              _ptr(dQ), dQ.stride(0), _ptr(ws), ws.numel(), _ptr(dev_status),
                              _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_shard_fwd_dq")


def gc_shard_dp(Q, P, pos_idx, tau, row_lse, p0, p_count, dP, ws=None, dev_status=None,
                mask_mode=GC_MASK_NONE):
    """Section 3.4, local passages [p0, p0 + p_count) of the gathered batch, given row_lse of all
    B queries: writes dP[p_count x d]."""
    args, B, N, d, code = _common(Q, P, pos_idx, tau, mask_mode)
    if ws is None:
        ws = torch.empty(max(gc_shard_workspace_bytes(B, N, d, code, B, p_count), 256),
                         dtype=torch.uint8, device=Q.device)
    rc = _lib.gc_shard_dp(*args, _ptr(row_lse), p0, p_count, _ptr(dP), dP.stride(0), _ptr(ws),
                          ws.numel(), _ptr(dev_status), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_shard_dp")


def gc_row_normalize(X, Xn, inv_norm) -> None:
    """Xn[i] = X[i]/|X[i]| (dtype of X) and inv_norm[i] = 1/|X[i]| (float32): the unit rows of the
    cosine-similarity loss."""
    rows, d = X.shape
    rc = _lib.gc_row_normalize(_ptr(X), X.stride(0), rows, d, _dtype_code(X), _ptr(Xn),
                               Xn.stride(0), _ptr(inv_norm), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_row_normalize")


def gc_cosine_bwd(X, inv_norm, dXn, dX) -> None:
    """dX[i] = inv_norm[i] (dXn[i] - n_i <n_i, dXn[i]>): cache rows of the unit rows taken back
    through the normalisation (dX may be dXn)."""
    rows, d = X.shape
    rc = _lib.gc_cosine_bwd(_ptr(X), X.stride(0), rows, d, _dtype_code(X), _ptr(inv_norm),
                            _ptr(dXn), dXn.stride(0), _ptr(dX), dX.stride(0), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_cosine_bwd")


def gc_dtau(Q, dQ, tau, dtau, ws=None) -> None:
    """dtau[0] = dL/dtau = -(1/tau) sum_i <Q_i, dQ_i> (Q: the rows the sweeps saw)."""
    B, d = Q.shape
    if ws is None:
        ws = torch.empty(max(int(_lib.gc_dtau_workspace_bytes(B)), 256), dtype=torch.uint8,
                         device=Q.device)
    rc = _lib.gc_dtau(_ptr(Q), Q.stride(0), _ptr(dQ), dQ.stride(0), B, d, float(tau),
                      _dtype_code(Q), _ptr(dtau), _ptr(ws), ws.numel(), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_dtau")


def gc_build_cache_multi_pos(Q, P, pos_ptr, pos_list, tau, mask_mode, loss, row_lse, dQ, dP,
                             ws=None, dev_status=None) -> None:
    """Several positives per query (CSR lists pos_ptr [B + 1], pos_list, int32): loss and cache
    rows of the mean-over-positives loss (Section 3.3, Step 2)."""
    B, d = Q.shape
    N = P.shape[0]
    n_pos = pos_list.numel()
    code = _dtype_code(Q)
    if ws is None:
        ws = torch.empty(max(int(_lib.gc_multi_pos_workspace_bytes(B, N, d, code, n_pos)), 256),
                         dtype=torch.uint8, device=Q.device)
    rc = _lib.gc_build_cache_multi_pos(_ptr(Q), Q.stride(0), _ptr(P), P.stride(0), _ptr(pos_ptr),
                                       _ptr(pos_list), n_pos, B, N, d, float(tau), int(mask_mode),
                                       code, _ptr(loss), _ptr(row_lse), _ptr(dQ), dQ.stride(0),
                                       _ptr(dP), dP.stride(0), _ptr(ws), ws.numel(),
                                       _ptr(dev_status), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_build_cache_multi_pos")


def gc_build_cache_two_direction(Q, P, pos_idx, tau, loss, row_lse, dQ, dP, ws=None,
                                 dev_status=None) -> None:
    """L = (L_row + L_col) / 2 over the B positive pairs (Section 3.3, Step 2), no mask."""
    B, d = Q.shape
    N = P.shape[0]
    code = _dtype_code(Q)
    if ws is None:
        ws = torch.empty(max(int(_lib.gc_two_direction_workspace_bytes(B, N, d, code)), 256),
                         dtype=torch.uint8, device=Q.device)
    rc = _lib.gc_build_cache_two_direction(_ptr(Q), Q.stride(0), _ptr(P), P.stride(0),
                                           _ptr(pos_idx), B, N, d, float(tau), code, _ptr(loss),
                                           _ptr(row_lse), _ptr(dQ), dQ.stride(0), _ptr(dP),
                                           dP.stride(0), _ptr(ws), ws.numel(), _ptr(dev_status),
                                           _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_build_cache_two_direction")


class DistanceCache:
    """Section 5 in tiled form: per-row state of the first pass over the distance blocks, then
    row_lse / loss, then blocks of the Distance Gradient Cache w = dL/dd.  Marshalling only."""

    def __init__(self, pos_idx, B, N, tau, mask_mode=GC_MASK_NONE):
        dev = pos_idx.device
        self.pos, self.B, self.N, self.tau, self.mask = pos_idx, B, N, float(tau), int(mask_mode)
        self.run_m = torch.empty(B, device=dev)
        self.run_l = torch.empty(B, device=dev)
        self.pos_d = torch.empty(B, device=dev)
        self.row_lse = torch.empty(B, device=dev)
        self.loss = torch.zeros(1, device=dev)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=dev)
        rc = _lib.gc_dist_begin(_ptr(self.run_m), _ptr(self.run_l), _ptr(self.pos_d), B, _stream())
        if rc != 0:
            raise GradCacheError(rc, "gc_dist_begin")

    def accumulate(self, D_block, i0, j0):
        bq, bn = D_block.shape
        rc = _lib.gc_dist_accumulate(_ptr(D_block), D_block.stride(0), i0, bq, j0, bn, _ptr(self.pos),
                                     self.B, self.N, self.tau, self.mask, _ptr(self.run_m),
                                     _ptr(self.run_l), _ptr(self.pos_d), _stream())
        if rc != 0:
            raise GradCacheError(rc, "gc_dist_accumulate")

    def finish(self):
        rc = _lib.gc_dist_finish(_ptr(self.run_m), _ptr(self.run_l), _ptr(self.pos_d), _ptr(self.pos),
                                 self.B, self.N, self.mask, _ptr(self.row_lse), _ptr(self.loss),
                                 _ptr(self.dev_status), _stream())
        if rc != 0:
            raise GradCacheError(rc, "gc_dist_finish")

    def w_block(self, D_block, i0, j0, W_block):
        bq, bn = D_block.shape
        rc = _lib.gc_dist_w_block(_ptr(D_block), D_block.stride(0), i0, bq, j0, bn, _ptr(self.pos),
                                  _ptr(self.row_lse), self.B, self.N, self.tau, self.mask,
                                  _ptr(W_block), W_block.stride(0), _stream())
        if rc != 0:
            raise GradCacheError(rc, "gc_dist_w_block")


def gc_dist_dot_block(Q, P, i0, bq, j0, bn, D_block) -> None:
    """D_block[r][c] = <Q[i0 + r], P[j0 + c]>: a block of dot-product distances (float32)."""
    B, d = Q.shape
    N = P.shape[0]
    rc = _lib.gc_dist_dot_block(_ptr(Q), Q.stride(0), _ptr(P), P.stride(0), B, N, d, _dtype_code(Q),
                                i0, bq, j0, bn, _ptr(D_block), D_block.stride(0), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_dist_dot_block")


def _on_device(dev, *others):
    """The library launches on the current device's current stream: refuses tensors that live elsewhere (dev: a
    tensor's device, -1 for the host; others: those of the other tensors)."""
    for d in others:
        if d != dev:
            raise ValueError(f"tensors must be on one CUDA device, got devices {dev} and {d}")
    if dev < 0 or dev != _current_device():
        raise ValueError("tensors must be on the current CUDA device")


def _scalar(t, dtype, name):
    if t is not None and (t.dtype is not dtype or t.numel() < 1):
        raise TypeError(f"{name} must be a {dtype} tensor of one value")


def _dense(t) -> bool:
    """Whether the values of t fill one stretch of memory, in whatever order of dimensions."""
    run = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz > 1):
        if stride != run:
            return False
        run *= size
    return True


def _as_matrix(t, like=None):
    """(rows, cols, pitch) of a tensor: one row where its values fill one stretch of memory (and those of
    `like`, a tensor of the same shape, lie in the same order), else a matrix with unit stride along its rows."""
    if t.numel() == 0:
        return 1, 0, 0
    # (the stride of a dimension of size 1 says nothing)
    if _dense(t) and (like is None or (_dense(like) and all(
            a == b for a, b, size in zip(t.stride(), like.stride(), t.shape) if size > 1))):
        return 1, t.numel(), t.numel()
    if t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1):
        return t.shape[0], t.shape[1], t.stride(0)
    if t.dim() == 1:
        return t.shape[0], 1, t.stride(0)
    raise ValueError("a gradient must be dense, or a matrix with unit stride along its rows")


class GradList:
    """A list of gradients as gc_grad_norm, gc_grad_scale and gc_grad_clip take it, described once: float32 or
    bfloat16 CUDA tensors on one device, any shapes, each dense or a matrix with unit stride along its rows.
    `out`: tensors of the same shapes and types that the clipped gradients go to (default: in place).  It
    holds the tensors; make a new one when they are replaced (writing to them needs none)."""

    def __init__(self, grads, out=None):
        self.grads = list(grads)
        self.out = None if out is None else list(out)
        if self.out is not None and len(self.out) != len(self.grads):
            raise ValueError("out must hold one tensor for each gradient")
        self.n = len(self.grads)
        self.tensors = (_Tensor * max(self.n, 1))()
        self.address = ctypes.addressof(self.tensors)
        self.device = self.grads[0].get_device() if self.grads else None
        for i, g in enumerate(self.grads):
            o = None if self.out is None else self.out[i]
            for t in (g, o):
                if t is not None and (not t.is_cuda or t.get_device() != self.device):
                    raise ValueError("gradients must be CUDA tensors of one device")
            code = _dtype_code(g)
            if o is not None and (o.dtype != g.dtype or o.shape != g.shape):
                raise ValueError("out must have the shapes and types of the gradients")
            x = self.tensors[i]
            x.data, x.dtype = g.data_ptr(), code
            x.rows, x.cols, x.ld = _as_matrix(g, o)
            if o is not None:
                x.out = o.data_ptr()
                rows, cols, x.ld_out = _as_matrix(o, g)
                if (rows, cols) != (x.rows, x.cols):
                    raise ValueError("a gradient that is not dense needs an out of two dimensions, and the "
                                     "other way round")


def gc_grad_workspace_bytes(n: int) -> int:
    return int(_lib.gc_grad_workspace_bytes(n))


def _grad_args(grads, *others):
    """(GradList, current device): everything lives there."""
    if not isinstance(grads, GradList):
        grads = GradList(grads)
    dev = grads.device
    if dev is None:
        dev = _current_device()
    _on_device(dev, *[t.get_device() for t in others if t is not None])
    return grads, dev


def _grad_ws(grads, dev):
    return torch.empty(gc_grad_workspace_bytes(grads.n), dtype=torch.uint8, device=torch.device("cuda", dev))


def gc_grad_norm(grads, norm=None, sq_sum=None, ws=None, dev_status=None) -> None:
    """norm[0] (float32) = 2-norm over all tensors of `grads` (a GradList, or a sequence of tensors), sq_sum[0]
    (float64) its square; either may be left out.  A NaN or an infinity sets GC_DEV_GRAD_NONFINITE."""
    _scalar(norm, torch.float32, "norm")
    _scalar(sq_sum, torch.float64, "sq_sum")
    _scalar(dev_status, torch.int32, "dev_status")
    grads, dev = _grad_args(grads, ws, norm, sq_sum, dev_status)
    if ws is None:
        ws = _grad_ws(grads, dev)
    rc = _lib.gc_grad_norm(grads.address, grads.n, _ptr(sq_sum), _ptr(norm), ws.data_ptr(), ws.numel(),
                           _ptr(dev_status), _raw_stream(dev))
    if rc != 0:
        raise GradCacheError(rc, "gc_grad_norm")


def gc_grad_scale(grads, sq_sum, max_norm, dev_status=None) -> None:
    """Scales the gradients (in place, or into the list's `out`) by min(1, max_norm / (n + 1e-6)), with n^2 =
    sq_sum[0] (float64): of gc_grad_norm, or summed over ranks that hold different gradients."""
    _scalar(sq_sum, torch.float64, "sq_sum")
    _scalar(dev_status, torch.int32, "dev_status")
    grads, dev = _grad_args(grads, None, sq_sum, dev_status)
    rc = _lib.gc_grad_scale(grads.address, grads.n, _ptr(sq_sum), max_norm, _ptr(dev_status),
                            _raw_stream(dev))
    if rc != 0:
        raise GradCacheError(rc, "gc_grad_scale")


def gc_grad_clip(grads, max_norm, norm, sq_sum=None, ws=None, dev_status=None) -> None:
    """norm[0] = 2-norm over all tensors, which are scaled (in place, or into the list's `out`) by
    min(1, max_norm / (norm + 1e-6)); left as they are, with GC_DEV_GRAD_NONFINITE set, where a value is not
    finite."""
    _scalar(norm, torch.float32, "norm")
    _scalar(sq_sum, torch.float64, "sq_sum")
    _scalar(dev_status, torch.int32, "dev_status")
    grads, dev = _grad_args(grads, ws, norm, sq_sum, dev_status)
    if ws is None:
        ws = _grad_ws(grads, dev)
    rc = _lib.gc_grad_clip(grads.address, grads.n, max_norm, _ptr(sq_sum), _ptr(norm), ws.data_ptr(),
                           ws.numel(), _ptr(dev_status), _raw_stream(dev))
    if rc != 0:
        raise GradCacheError(rc, "gc_grad_clip")


def gc_quantize_rows(X, q, scale) -> None:
    """scale[i] (float32) = max |X[i]| times 1/127 and q[i] (int8) = X[i] / scale[i] to the nearest integer."""
    shape, xs, qs = X.shape, X.stride(), q.stride()
    if len(xs) != 2 or q.shape != shape or xs[1] != 1 or qs[1] != 1:
        raise ValueError("X and q must be 2-D of one shape with unit stride along their rows")
    rows, d = shape
    code = _CODES.get(X.dtype)
    if code is None or q.dtype is not torch.int8 or scale.dtype is not torch.float32 or not scale.is_contiguous():
        raise TypeError("X must be float32 or bfloat16, q int8, scale contiguous float32")
    if scale.numel() != rows:
        raise ValueError("scale must hold one value for each row")
    dev = X.get_device()
    _on_device(dev, q.get_device(), scale.get_device())
    rc = _lib.gc_quantize_rows(X.data_ptr(), xs[0], rows, d, code, q.data_ptr(), qs[0], scale.data_ptr(),
                               _raw_stream(dev))
    if rc != 0:
        raise GradCacheError(rc, "gc_quantize_rows")


def gc_matmul_i8_plan_name(rows: int, cols: int, k: int, out_dtype: int) -> str:
    return _lib.gc_matmul_i8_plan_name(rows, cols, k, out_dtype).decode()


def gc_matmul_i8(A, a_scale, B, b_scale, out, dev_status=None) -> None:
    """out[i][j] = a_scale[i] b_scale[j] sum_k A[i][k] B[j][k] with A, B int8 (gc_quantize_rows), out float32 or
    bfloat16: the linear encoder's output (A inputs, B = W), or scores of queries against passages."""
    sa, sb, so = A.stride(), B.stride(), out.stride()
    if len(sa) != 2 or len(sb) != 2 or len(so) != 2 or sa[1] != 1 or sb[1] != 1 or so[1] != 1:
        raise ValueError("A, B and out must be 2-D with unit stride along their rows")
    rows, k = A.shape
    cols, kb = B.shape
    if kb != k or out.shape != (rows, cols) or a_scale.numel() != rows or b_scale.numel() != cols:
        raise ValueError("shape mismatch")
    code, i8, f32 = _CODES.get(out.dtype), torch.int8, torch.float32
    if code is None or A.dtype is not i8 or B.dtype is not i8:
        raise TypeError("A and B must be int8, out float32 or bfloat16")
    if a_scale.dtype is not f32 or b_scale.dtype is not f32 or not a_scale.is_contiguous() \
            or not b_scale.is_contiguous():
        raise TypeError("scales must be contiguous float32")
    _scalar(dev_status, torch.int32, "dev_status")
    dev = A.get_device()
    _on_device(dev, a_scale.get_device(), B.get_device(), b_scale.get_device(), out.get_device(),
               dev if dev_status is None else dev_status.get_device())
    rc = _lib.gc_matmul_i8(A.data_ptr(), sa[0], a_scale.data_ptr(), B.data_ptr(), sb[0], b_scale.data_ptr(), rows,
                           cols, k, code, out.data_ptr(), so[0], _ptr(dev_status), _raw_stream(dev))
    if rc != 0:
        raise GradCacheError(rc, "gc_matmul_i8")


def gc_selftest_wait_limit(limit_ns: int, dev_status, waited_ns=None) -> None:
    """Runs the library's bounded on-chip wait with a limit of `limit_ns` on a barrier nothing
    arrives on: ORs GC_DEV_WAIT_LIMIT into dev_status[0] (int32) and writes the time waited to
    waited_ns[0] (int64 tensor, optional)."""
    rc = _lib.gc_selftest_wait_limit(int(limit_ns), _ptr(dev_status), _ptr(waited_ns), _stream())
    if rc != 0:
        raise GradCacheError(rc, "gc_selftest_wait_limit")


def gc_profile_enable(sets) -> None:
    """Per-kernel timing on (sets >= 1 event sets, True = 1) or off (0 / False)."""
    rc = _lib.gc_profile_enable(int(sets))
    if rc != 0:
        raise GradCacheError(rc, "gc_profile_enable")


def gc_profile_read(call: int | None = None) -> tuple[float, float, float]:
    """Milliseconds of the forward sweep, dQ sweep and dP sweep kernels of call number `call`
    since the enable (default: the most recent call)."""
    a, b, c = ctypes.c_float(), ctypes.c_float(), ctypes.c_float()
    if call is None:
        rc = _lib.gc_profile_read(ctypes.byref(a), ctypes.byref(b), ctypes.byref(c))
    else:
        rc = _lib.gc_profile_read_call(int(call), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c))
    if rc != 0:
        raise GradCacheError(rc, "gc_profile_read")
    return a.value, b.value, c.value


def problem_tensors(prob, device="cuda"):
    """(Q, P, pos_idx) device tensors for an inputs.Problem, in its dtype.  Shared rows stay one
    buffer (Q is P)."""
    import numpy as np
    if prob.dtype == "bf16":
        Q = torch.from_numpy(prob.Q_bits.view(np.int16)).view(torch.bfloat16).to(device)
        P = Q if prob.shared else torch.from_numpy(prob.P_bits.view(np.int16)).view(
            torch.bfloat16).to(device)
    else:
        Q = torch.from_numpy(prob.Q).to(device)
        P = Q if prob.shared else torch.from_numpy(prob.P).to(device)
    return Q, P, torch.from_numpy(prob.pos_idx).to(device)


class Outputs:
    """Device buffers for one problem size, allocated once and reused across calls."""

    def __init__(self, B: int, N: int, d: int, dtype: int, device="cuda", op: int = GC_OP_BUILD):
        f = dict(dtype=torch.float32, device=device)
        self.loss = torch.zeros(1, **f)
        self.row_lse = torch.empty(B, **f)
        self.pos_logit = torch.empty(B, **f)
        self.dQ = torch.empty(B, d, **f)
        self.dP = torch.empty(N, d, **f)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=device)
        self.ws = alloc_workspace(op, B, N, d, dtype, device)


def build_cache(Q, P, pos_idx, tau=1.0, mask_mode=GC_MASK_NONE, out: Outputs | None = None):
    """Convenience wrapper: allocates outputs (or reuses `out`) and calls gc_build_cache."""
    B, d = Q.shape
    N = P.shape[0]
    if out is None:
        out = Outputs(B, N, d, _dtype_code(Q), Q.device)
    out.dev_status.zero_()
    gc_build_cache(Q, P, pos_idx, tau, mask_mode, out.loss, out.row_lse, out.dQ, out.dP,
                   out.pos_logit, out.ws, out.dev_status)
    return out
