"""ctypes binding of libzr.so (argument marshalling only).

Functions carry the names of the C ABI in include/zr.h.  Tensors are torch
tensors living on the GPU; only their data pointers, shapes and strides cross
the boundary.  There is no CPU fallback: if the library is not built the
import raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Tuple, Union

import torch

DROP_N, DROP_K = 0, 1
W_KN, W_NK = 0, 1
WS_FRESH, WS_HOLDS_FORWARD = 0, 1
ZERO, AVERAGE, SAME = 0, 1, 2
F32, BF16 = 0, 1
MX_E4M3, MX_E2M1, MX_INT8 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4
NORM_RMS, NORM_LAYER = 0, 1

_LIB_PATH = os.environ.get("ZR_LIBZR_PATH") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libzr.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(
        f"{_LIB_PATH} is missing: build it first (python -m paper_2401_11469_amd.build); "
        "there is no fallback path")
_lib = ctypes.CDLL(_LIB_PATH)

_vp, _i32, _i64, _f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double

_lib.zr_status_string.argtypes = [ctypes.c_int]
_lib.zr_status_string.restype = ctypes.c_char_p
_lib.zr_keep_count.argtypes = [_i64, _f64]
_lib.zr_keep_count.restype = _i64
_lib.zr_resize_select.argtypes = [_vp, _i32, _i32, _f64, _vp, _vp, _i64, _vp]
_lib.zr_resize_select.restype = ctypes.c_int
_lib.zr_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32, ctypes.c_int, ctypes.c_int]
_lib.zr_workspace_bytes.restype = ctypes.c_size_t
_lib.zr_resized_linear_fwd.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _i32,
                                       _vp, _i32, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, _vp,
                                       _vp, ctypes.c_size_t, _vp]
_lib.zr_resized_linear_fwd.restype = ctypes.c_int
_lib.zr_resized_linear_bwd.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64,
                                       _i32, _i32, _i32, _vp, _i32,
                                       ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, _vp, _vp,
                                       _vp, ctypes.c_size_t, ctypes.c_int, _vp]
_lib.zr_resized_linear_bwd.restype = ctypes.c_int
_lib.zr_impute.argtypes = [_vp, _i64, _i32, _i32, _i32, _vp, _i32, ctypes.c_int, _vp, ctypes.c_int, _vp]
_lib.zr_impute.restype = ctypes.c_int
_lib.zr_extract_kept_columns.argtypes = [_vp, _i64, _i32, _i32, _vp, _i32, _vp, _i64, ctypes.c_int, _vp]
_lib.zr_extract_kept_columns.restype = ctypes.c_int
_lib.zr_debug_record_kernel_names.argtypes = [ctypes.c_int]
_lib.zr_debug_record_kernel_names.restype = None
_lib.zr_debug_last_kernel.argtypes = []
_lib.zr_debug_last_kernel.restype = ctypes.c_char_p
_lib.zr_priority_scores.argtypes = [_vp, _vp, _i64, _i32, _i32, ctypes.c_int, _vp, _vp, _i32, _vp, ctypes.c_int,
                                    _vp, ctypes.c_size_t, _vp]
_lib.zr_priority_workspace_bytes.argtypes = [_i32, _i32, ctypes.c_int]
_lib.zr_priority_workspace_bytes.restype = ctypes.c_size_t
_lib.zr_priority_scores.restype = ctypes.c_int
_lib.zr_priority_scores_static.argtypes = [_vp, _vp, _i64, _i32, _i32, ctypes.c_int, _vp, _vp, _i32, _vp, ctypes.c_int, _vp]
_lib.zr_priority_scores_static.restype = ctypes.c_int
_lib.zr_priority_static_scratch_bytes.argtypes = []
_lib.zr_priority_static_scratch_bytes.restype = ctypes.c_size_t
_lib.zr_pruning_ratio.argtypes = [_f64, _f64, _f64, _f64]
_lib.zr_pruning_ratio.restype = _f64
_lib.zr_count_above.argtypes = [_vp, _i32, ctypes.c_float, _vp, _vp]
_lib.zr_count_above.restype = ctypes.c_int
_lib.zr_layer_ratio.argtypes = [_i64, _i64, _f64, _f64]
_lib.zr_layer_ratio.restype = _f64
_lib.zr_migration_range.argtypes = [_i32, _i32, _i32, _i64, ctypes.POINTER(_i64), ctypes.POINTER(_i64)]
_lib.zr_migration_range.restype = ctypes.c_int
_lib.zr_migrated_accumulate.argtypes = [_vp, _i64, _vp, _i64, ctypes.c_int, _vp, _i64, _i32, _i32, _i32, ctypes.c_int, _vp]
_lib.zr_migrated_accumulate.restype = ctypes.c_int
_lib.zr_select_workspace_bytes.argtypes = [_i32]
_lib.zr_select_workspace_bytes.restype = ctypes.c_size_t
_lib.zr_resize_select_ws.argtypes = [_vp, _i32, _f64, _vp, _vp, _vp, ctypes.c_size_t, _vp]
_lib.zr_resize_select_ws.restype = ctypes.c_int
_lib.zr_resize_select_multi.argtypes = [_i32, ctypes.POINTER(_vp), ctypes.POINTER(_i32), ctypes.POINTER(_f64),
                                        ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp]
_lib.zr_resize_select_multi.restype = ctypes.c_int
_lib.zr_debug_time_next_product.argtypes = [_vp, _vp]
_lib.zr_debug_time_next_product.restype = ctypes.c_int
_lib.zr_debug_mfma_rate.argtypes = [_i32, _i32, _vp, ctypes.POINTER(_f64), _vp]
_lib.zr_debug_mfma_rate.restype = ctypes.c_int
_lib.zr_validate_keep_idx.argtypes = [_vp, _i32, _i32, _vp, _vp]
_lib.zr_validate_keep_idx.restype = ctypes.c_int
_lib.zr_mx_row_bytes.argtypes = [_i32, ctypes.c_int]
_lib.zr_mx_row_bytes.restype = ctypes.c_size_t
_lib.zr_mx_scale_bytes.argtypes = [_i32]
_lib.zr_mx_scale_bytes.restype = ctypes.c_size_t
_lib.zr_mx_quantize.argtypes = [_vp, _i64, _i32, _i32, ctypes.c_int, _vp, _i32, ctypes.c_int, ctypes.c_int, _vp, _i64, _vp, _i64, _vp]
_lib.zr_mx_quantize.restype = ctypes.c_int
_lib.zr_mx_dequantize.argtypes = [_vp, _i64, _vp, _i64, _i32, _i32, ctypes.c_int, _vp, _i64, ctypes.c_int, _vp]
_lib.zr_mx_dequantize.restype = ctypes.c_int
_lib.zr_mx_linear_fwd.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_int, _vp, _i64, _vp, _i64, ctypes.c_int, _vp, _i64,
                                  _i32, _i32, _i32, _vp, _i32, ctypes.c_int, ctypes.c_int, ctypes.c_int, _vp, _vp]
_lib.zr_mx_linear_fwd.restype = ctypes.c_int
_lib.zr_mx_bwd_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32, ctypes.c_int, ctypes.c_int]
_lib.zr_mx_bwd_workspace_bytes.restype = ctypes.c_size_t
_lib.zr_resized_linear_bwd_mx.argtypes = [_vp, _i64, _vp, _i64, ctypes.c_int, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64,
                                          _i32, _i32, _i32, _vp, _i32, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                          _vp, _vp, _vp, ctypes.c_size_t, _vp]
_lib.zr_resized_linear_bwd_mx.restype = ctypes.c_int
_int, _size = ctypes.c_int, ctypes.c_size_t
_lib.zr_dropout.argtypes = [_vp, _i64, _vp, _i64, _i32, _i32, _f64, _vp, _int, _vp]
_lib.zr_dropout.restype = _int
for _f in (_lib.zr_act_fwd_workspace_bytes, _lib.zr_act_bwd_workspace_bytes):
    _f.argtypes = [_i32, _i32, _i32, _i32, _int, _int]
    _f.restype = _size
_lib.zr_resized_linear_act_fwd.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _i32, _vp, _i32, _int, _int, _int,
                                           _vp, _int, _vp, _i64, _f64, _vp, _vp, _i64, _vp, _i64, _vp, _size, _vp]
_lib.zr_resized_linear_act_fwd.restype = _int
_lib.zr_resized_linear_act_bwd.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _i64,
                                           _i32, _i32, _i32, _vp, _i32, _int, _int, _int, _int, _f64, _vp, _vp, _size, _vp]
_lib.zr_resized_linear_act_bwd.restype = _int
_lib.zr_block_join_workspace_bytes.argtypes = [_i32, _i32]
_lib.zr_block_join_workspace_bytes.restype = _size
_lib.zr_block_join_fwd.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _int, _int, _f64, _f64, _vp, _f64,
                                   _vp, _vp, _vp, _vp, _vp, _vp, _int, _vp]
_lib.zr_block_join_fwd.restype = _int
_lib.zr_block_join_bwd.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _int, _int, _f64, _f64, _vp, _f64,
                                   _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _size, _int, _vp]
_lib.zr_block_join_bwd.restype = _int


class ZrError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"libzr status {status}: {_lib.zr_status_string(status).decode()}")


def _check(status: int) -> None:
    if status != 0:
        raise ZrError(status)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _mat(t: Optional[torch.Tensor], name: str):
    """(pointer, leading dimension) of a 2-D row-major CUDA tensor."""
    if t is None:
        return None, 0
    if not t.is_cuda or t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name}: need a 2-D GPU tensor with unit column stride")
    return t.data_ptr(), t.stride(0)


def _stream(stream) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def workspace_bytes(M: int, K: int, N: int, n_keep: int, mode: int, dtype) -> int:
    code = dtype if isinstance(dtype, int) else (BF16 if dtype == torch.bfloat16 else F32)
    return int(_lib.zr_workspace_bytes(M, K, N, n_keep, mode, code))


def _ws(workspace: Optional[torch.Tensor]):
    if workspace is None:
        return None, 0
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace: need a contiguous GPU tensor")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def keep_count(n: int, ratio: float) -> int:
    return int(_lib.zr_keep_count(n, ratio))


def status_string(status: int) -> str:
    return _lib.zr_status_string(status).decode()


def resize_select(scores: torch.Tensor, ratio: float, keep_idx: Optional[torch.Tensor] = None,
                  drop_idx: Optional[torch.Tensor] = None, want_drop: bool = True,
                  stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """scores: fp32 [n] or [batch, n] on the GPU.  Returns (keep_idx, drop_idx) as int32
    tensors of row length n' and n - n' (views of buffers with a common pitch)."""
    if scores.dtype != torch.float32 or not scores.is_cuda or not scores.is_contiguous():
        raise ValueError("scores: need a contiguous fp32 GPU tensor")
    batched = scores.dim() == 2
    n = scores.shape[-1]
    batch = scores.shape[0] if batched else 1
    n_keep = keep_count(n, ratio)
    if n_keep < 1:
        raise ZrError(3)
    ld = max(n_keep, n - n_keep, 1)
    if keep_idx is None:
        keep_idx = torch.empty((batch, ld), dtype=torch.int32, device=scores.device)
    if drop_idx is None and want_drop:
        drop_idx = torch.empty((batch, ld), dtype=torch.int32, device=scores.device)
    for t in (keep_idx, drop_idx):
        if t is not None and (t.dtype != torch.int32 or t.dim() != 2 or t.stride(1) != 1
                              or t.stride(0) != keep_idx.stride(0) or t.shape[0] < batch):
            raise ValueError("index buffers: int32 [batch, ld] with a common pitch")
    _check(_lib.zr_resize_select(scores.data_ptr(), n, batch, float(ratio), keep_idx.data_ptr(),
                                 None if drop_idx is None else drop_idx.data_ptr(),
                                 keep_idx.stride(0), _stream(stream)))
    k = keep_idx[:batch, :n_keep]
    d = None if drop_idx is None else drop_idx[:batch, :n - n_keep]
    if not batched:
        k = k[0]
        d = None if d is None else d[0]
    return k, d


def select_workspace_bytes(n: int) -> int:
    return int(_lib.zr_select_workspace_bytes(n))


def resize_select_ws(scores: torch.Tensor, ratio: float, workspace: Optional[torch.Tensor],
                     keep_idx: Optional[torch.Tensor] = None, drop_idx: Optional[torch.Tensor] = None,
                     want_drop: bool = True, stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """One fp32 vector [n] on the GPU, with a scratch buffer (select_workspace_bytes(n) bytes) that lets a
    long vector be selected by many workgroups.  Returns (keep_idx[n'], drop_idx[n - n'])."""
    if scores.dtype != torch.float32 or not scores.is_cuda or not scores.is_contiguous() or scores.dim() != 1:
        raise ValueError("scores: need a contiguous 1-D fp32 GPU tensor")
    n = scores.shape[0]
    n_keep = keep_count(n, ratio)
    if n_keep < 1:
        raise ZrError(3)
    if keep_idx is None:
        keep_idx = torch.empty(n_keep, dtype=torch.int32, device=scores.device)
    if drop_idx is None and want_drop:
        drop_idx = torch.empty(max(n - n_keep, 1), dtype=torch.int32, device=scores.device)
    for t, need in ((keep_idx, n_keep), (drop_idx, n - n_keep)):
        if t is not None and (t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous() or t.numel() < need):
            raise ValueError("index buffers: contiguous int32 vectors of at least n' and n - n' entries")
    _check(_lib.zr_resize_select_ws(scores.data_ptr(), n, float(ratio), keep_idx.data_ptr(),
                                    None if drop_idx is None else drop_idx.data_ptr(), *_ws(workspace), _stream(stream)))
    return keep_idx[:n_keep], None if drop_idx is None else drop_idx[:n - n_keep]


def resize_select_multi(scores, ratios, keep_idx=None, drop_idx=None, stream=None):
    """One launch for several score vectors (lists of 1-D fp32 GPU tensors and ratios).
    Returns lists of kept / dropped index tensors (views of the given buffers, or new ones)."""
    cnt = len(scores)
    ns = [int(s.numel()) for s in scores]
    nk = [keep_count(n, r) for n, r in zip(ns, ratios)]
    if keep_idx is None:
        keep_idx = [torch.empty(n, dtype=torch.int32, device=s.device) for n, s in zip(ns, scores)]
    if drop_idx is None:
        drop_idx = [torch.empty(n, dtype=torch.int32, device=s.device) for n, s in zip(ns, scores)]
    for s in scores:
        if s.dtype != torch.float32 or not s.is_cuda or not s.is_contiguous():
            raise ValueError("scores: contiguous fp32 GPU tensors")
    PV, PI, PD = _vp * cnt, _i32 * cnt, _f64 * cnt
    _check(_lib.zr_resize_select_multi(cnt, PV(*[s.data_ptr() for s in scores]), PI(*ns), PD(*[float(r) for r in ratios]),
                                       PV(*[k.data_ptr() for k in keep_idx]), PV(*[d.data_ptr() for d in drop_idx]),
                                       _stream(stream)))
    return ([k.view(-1)[:c] for k, c in zip(keep_idx, nk)],
            [d.view(-1)[:n - c] for d, n, c in zip(drop_idx, ns, nk)])


def resized_linear_fwd(X: torch.Tensor, W: torch.Tensor, keep_idx: torch.Tensor, mode: int,
                       policy: int = ZERO, prev_Y: Optional[torch.Tensor] = None,
                       Y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                       stream=None, w_layout: int = W_KN) -> torch.Tensor:
    """W is [K, N] (w_layout=W_KN) or [N, K] (W_NK)."""
    M, K = X.shape
    N = W.shape[1] if w_layout == W_KN else W.shape[0]
    if tuple(W.shape) != ((K, N) if w_layout == W_KN else (N, K)) or W.dtype != X.dtype:
        raise ValueError("W must be [K, N] (W_KN) or [N, K] (W_NK) with X's dtype")
    if Y is None:
        Y = torch.empty((M, N), dtype=X.dtype, device=X.device)
    (xp, ldx), (wp, ldw), (yp, ldy) = _mat(X, "X"), _mat(W, "W"), _mat(Y, "Y")
    pp, ldp = _mat(prev_Y, "prev_Y")
    if prev_Y is not None and ldp != ldy:
        raise ValueError("prev_Y must share Y's leading dimension")
    _check(_lib.zr_resized_linear_fwd(xp, ldx, wp, ldw, yp, ldy, M, K, N,
                                      keep_idx.data_ptr(), keep_idx.numel(), mode, w_layout, _dtype_code(X),
                                      policy, pp, *_ws(workspace), _stream(stream)))
    return Y


def resized_linear_bwd(X: torch.Tensor, W: torch.Tensor, dY: torch.Tensor, keep_idx: torch.Tensor,
                       mode: int, policy: int = ZERO, prev_dX: Optional[torch.Tensor] = None,
                       prev_dW: Optional[torch.Tensor] = None, dX: Optional[torch.Tensor] = None,
                       dW: Optional[torch.Tensor] = None, need_dX: bool = True, need_dW: bool = True,
                       workspace: Optional[torch.Tensor] = None, stream=None,
                       w_layout: int = W_KN,
                       workspace_holds_forward: bool = False) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """W and dW are [K, N] (w_layout=W_KN) or [N, K] (W_NK).  workspace_holds_forward: the
    workspace is the one the forward call of this layer step used and is untouched since."""
    M, K = X.shape
    N = dY.shape[1]
    wshape = (K, N) if w_layout == W_KN else (N, K)
    if dY.shape[0] != M or tuple(W.shape) != wshape:
        raise ValueError("dY must be [M, N] and W [K, N] (W_KN) or [N, K] (W_NK)")
    if need_dX and dX is None:
        dX = torch.empty((M, K), dtype=X.dtype, device=X.device)
    if need_dW and dW is None:
        dW = torch.empty(wshape, dtype=X.dtype, device=X.device)
    (xp, ldx), (wp, ldw), (gp, ldg) = _mat(X, "X"), _mat(W, "W"), _mat(dY, "dY")
    (dxp, lddx), (dwp, lddw) = _mat(dX if need_dX else None, "dX"), _mat(dW if need_dW else None, "dW")
    (pxp, ldpx), (pwp, ldpw) = _mat(prev_dX, "prev_dX"), _mat(prev_dW, "prev_dW")
    if (prev_dX is not None and need_dX and ldpx != lddx) or (prev_dW is not None and need_dW and ldpw != lddw):
        raise ValueError("previous tensors must share the outputs' leading dimensions")
    _check(_lib.zr_resized_linear_bwd(xp, ldx, wp, ldw, gp, ldg, dxp, lddx, dwp, lddw, M, K, N,
                                      keep_idx.data_ptr(), keep_idx.numel(), mode, w_layout, _dtype_code(X),
                                      policy, pxp, pwp, *_ws(workspace), 1 if workspace_holds_forward else 0,
                                      _stream(stream)))
    return (dX if need_dX else None), (dW if need_dW else None)


def impute(out: torch.Tensor, axis: int, keep_idx: torch.Tensor, policy: int = ZERO,
           prev: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """In place: fills the slices of ``out`` not listed in keep_idx along ``axis``."""
    op, ld = _mat(out, "out")
    pp, ldp = _mat(prev, "prev")
    if prev is not None and ldp != ld:
        raise ValueError("prev must share out's leading dimension")
    _check(_lib.zr_impute(op, ld, out.shape[0], out.shape[1], axis, keep_idx.data_ptr(),
                          keep_idx.numel(), policy, pp, _dtype_code(out), _stream(stream)))
    return out


def extract_kept_columns(inp: torch.Tensor, keep_idx: torch.Tensor, out: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """out[r, q] = inp[r, keep_idx[q]], zero padded to a multiple of 64 columns (bf16)."""
    rows, n = inp.shape
    width = (keep_idx.numel() + 63) // 64 * 64
    if out is None:
        out = torch.empty((rows, width), dtype=inp.dtype, device=inp.device)
    (ip, ld), (op, ldo) = _mat(inp, "inp"), _mat(out, "out")
    _check(_lib.zr_extract_kept_columns(ip, ld, rows, n, keep_idx.data_ptr(), keep_idx.numel(), op, ldo,
                                        _dtype_code(inp), _stream(stream)))
    return out


class MX(NamedTuple):
    """A matrix [rows, n] in blocks of 32 values with a power of two each: elements uint8 [rows, >= mx_row_bytes(n, fmt)],
    scales uint8 [rows, >= mx_scale_bytes(n)] (zr.h has the layout)."""
    q: torch.Tensor
    scales: torch.Tensor
    n: int
    fmt: int


def mx_row_bytes(n: int, fmt: int) -> int:
    return int(_lib.zr_mx_row_bytes(n, fmt))


def mx_scale_bytes(n: int) -> int:
    return int(_lib.zr_mx_scale_bytes(n))


def mx_empty(rows: int, n: int, fmt: int, device="cuda") -> MX:
    return MX(torch.empty((rows, mx_row_bytes(n, fmt)), dtype=torch.uint8, device=device),
              torch.empty((rows, mx_scale_bytes(n)), dtype=torch.uint8, device=device), n, fmt)


# The calls below are made once a layer and token while decoding, where the host's part of a call is longer than the GPU's:
# attributes are looked up once, the current stream without an object for it (by torch's public calls where it has no shorter way).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_get_device = getattr(torch._C, "_cuda_getDevice", None) or (lambda: torch.cuda.current_device())
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _here() -> int:
    """The current GPU, on which the kernels run."""
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return _get_device()


def _on(stream, here: int) -> int:
    if stream is None:
        return _raw_stream(here)
    if stream.device.index != here:
        raise ValueError("stream: of another GPU")
    return stream.cuda_stream


def _empty(shape, dtype, device, stream, returned: bool = True) -> torch.Tensor:
    """Memory for a call on `stream`, of that stream's own: another's may still be read by work that was queued there before it was freed.
    What the caller gets back is also kept from reuse until the current stream has done what it has queued when it is freed."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if returned:
        t.record_stream(torch.cuda.current_stream())
    return t


def _mx_empty(rows: int, n: int, fmt: int, device, stream, returned: bool = True) -> MX:
    return MX(_empty((rows, mx_row_bytes(n, fmt)), torch.uint8, device, stream, returned),
              _empty((rows, mx_scale_bytes(n)), torch.uint8, device, stream, returned), n, fmt)


def _grid(t: Optional[torch.Tensor], here: int, name: str):
    """(pointer, leading dimension) of a 2-D tensor on the current GPU."""
    if t.get_device() != here:
        raise ValueError(f"{name}: must be on the current GPU")
    st = t.stride()
    if len(st) != 2 or st[1] != 1:
        raise ValueError(f"{name}: need a 2-D tensor with unit column stride")
    return t.data_ptr(), st[0]


def _list(keep_idx: Optional[torch.Tensor], here: int):
    """(pointer, length) of a kept list, None: (None, 0)."""
    if keep_idx is None:
        return None, 0
    if (keep_idx.dtype is not torch.int32 or keep_idx.dim() != 1 or not keep_idx.is_contiguous()
            or keep_idx.get_device() != here):
        raise ValueError("keep_idx: need a contiguous int32 vector on the current GPU")
    if keep_idx.numel() == 0:       # (an empty tensor's pointer is null, which would mean that nothing is pruned)
        raise ZrError(3)
    return keep_idx.data_ptr(), keep_idx.numel()


def _mx(m: Optional[MX], rows: int, n: int, here: int, name: str):
    """(elements, pitch, scales, pitch, format) of a matrix in blocks of the given size."""
    if m is None:
        return None, 0, None, 0, 0
    q, s, held, fmt = m
    if held != n or q.shape[0] != rows or s.shape[0] != rows:
        raise ValueError(f"{name}: need {rows} rows of {n} values in blocks")
    if q.dtype is not torch.uint8 or s.dtype is not torch.uint8:
        raise ValueError(f"{name}: elements and scales are uint8")
    if q.shape[1] << (fmt == MX_E2M1) < (n + 127) // 128 * 128 or s.shape[1] < (n + 511) // 512 * 16:
        raise ValueError(f"{name}: its rows do not hold {n} values")
    return (*_grid(q, here, name), *_grid(s, here, name), fmt)


def _code(dtype) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}")
    return code


def mx_quantize(src: torch.Tensor, fmt: int, axis: int = 1, keep_idx: Optional[torch.Tensor] = None,
                out: Optional[MX] = None, stream=None) -> MX:
    """src [rows, cols] in blocks along `axis` (0: the transpose in blocks), of the kept indices of that axis alone."""
    here = _here()
    on = _on(stream, here)
    sp, ld = _grid(src, here, "src")
    rows, cols = src.shape
    held, n = (rows, cols) if axis == 1 else (cols, rows)
    kp, nk = _list(keep_idx, here)
    if kp is not None:
        n = nk
    if out is None:
        out = _mx_empty(held, n, fmt, src.device, stream)
    if out.fmt != fmt:
        raise ValueError("out is of another format")
    qp, ldq, scp, lds, _ = _mx(out, held, n, here, "out")
    st = _lib.zr_mx_quantize(sp, ld, rows, cols, axis, kp, n, _code(src.dtype), fmt, qp, ldq, scp, lds, on)
    if st:
        raise ZrError(st)
    return out


def mx_dequantize(m: MX, dtype=torch.bfloat16, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The values [rows, n] that m stands for, in `dtype` (or in out's)."""
    here = _here()
    on = _on(stream, here)
    rows = m.q.shape[0]
    if out is None:
        out = _empty((rows, m.n), dtype, m.q.device, stream)
    if out.shape != (rows, m.n):
        raise ValueError("out must be [rows, n]")
    op, ldo = _grid(out, here, "out")
    qp, ldq, scp, lds, fmt = _mx(m, rows, m.n, here, "m")
    st = _lib.zr_mx_dequantize(qp, ldq, scp, lds, rows, m.n, fmt, op, ldo, _code(out.dtype), on)
    if st:
        raise ZrError(st)
    return out


def mx_linear_fwd(X: Union[torch.Tensor, MX], W: MX, keep_idx: Optional[torch.Tensor] = None, mode: int = DROP_K,
                  policy: int = ZERO, prev_Y: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
                  x_fmt: int = MX_E4M3, x_mx: Optional[MX] = None, K: Optional[int] = None, dtype=torch.bfloat16,
                  stream=None) -> torch.Tensor:
    """X [M, K] (put into blocks of x_fmt by the call, into x_mx where given: the checkpoint for resized_linear_bwd_mx;
    without x_mx at most 16 rows keep none, for more one is allocated), or X in blocks already (K: the layer's, for DROP_K; dtype: of Y).
    W in blocks: [N, n_keep] (DROP_K) or the whole shard [N, K] (DROP_N).  keep_idx None: nothing is pruned."""
    here = _here()
    on = _on(stream, here)
    N = W.q.shape[0]
    kp, nk = _list(keep_idx, here)
    if type(X) is MX:
        if x_mx is not None:
            raise ValueError("x_mx: X is in blocks already")
        x_mx, x_fmt, M = X, X.fmt, X.q.shape[0]
        K = X.n if K is None else K
        xp, ldx, dt = None, 0, dtype if Y is None else Y.dtype
        c = nk if kp is not None and mode == DROP_K else K
    else:
        xp, ldx = _grid(X, here, "X")
        M, K = X.shape
        dt = X.dtype
        c = nk if kp is not None and mode == DROP_K else K
        if x_mx is None:
            if M > 16:
                x_mx = _mx_empty(M, c, x_fmt, X.device, stream, returned=False)
        elif x_mx.fmt != x_fmt:
            raise ValueError("x_mx is of another format")
    if Y is None:
        Y = _empty((M, N), dt, W.q.device, stream)
    elif Y.dtype is not dt or Y.shape != (M, N):
        raise ValueError("Y must be [M, N] of X's dtype")
    yp, ldy = _grid(Y, here, "Y")
    pp = None
    if prev_Y is not None:
        pp, ldp = _grid(prev_Y, here, "prev_Y")
        if ldp != ldy or prev_Y.dtype is not dt or prev_Y.shape != (M, N):
            raise ValueError("prev_Y must be like Y, its leading dimension too")
    xq, ldxq, xs, ldxs, _ = _mx(x_mx, M, c, here, "X")
    wq, ldwq, ws, ldws, w_fmt = _mx(W, N, c, here, "W")
    st = _lib.zr_mx_linear_fwd(xp, ldx, xq, ldxq, xs, ldxs, x_fmt, wq, ldwq, ws, ldws, w_fmt, yp, ldy, M, K, N, kp, nk,
                               mode, _code(dt), policy, pp, on)
    if st:
        raise ZrError(st)
    return Y


def mx_bwd_workspace_bytes(M: int, K: int, N: int, n_keep: int, mode: int, dtype) -> int:
    return int(_lib.zr_mx_bwd_workspace_bytes(M, K, N, n_keep, mode, dtype if isinstance(dtype, int) else _code(dtype)))


def _bwd_scratch(M: int, K: int, N: int, n_keep: int, mode: int, dt) -> int:
    """Bytes for a call that is given no buffer: without the place of the columns that a call on uncompressed X extracts, which
    are side by side in a DROP_K checkpoint.  (With them 20 of 211 large calls split their contraction into more slices, 17 of those
    to no gain.)"""
    size = mx_bwd_workspace_bytes(M, K, N, n_keep, mode, dt)
    return size - 2 * M * ((n_keep + 63) // 64 * 64) if mode == DROP_K and dt is torch.bfloat16 else size


def resized_linear_bwd_mx(X: Optional[MX], W: torch.Tensor, dY: torch.Tensor, keep_idx: torch.Tensor, mode: int, policy: int = ZERO,
                          prev_dX: Optional[torch.Tensor] = None, prev_dW: Optional[torch.Tensor] = None,
                          dX: Optional[torch.Tensor] = None, dW: Optional[torch.Tensor] = None, need_dX: bool = True,
                          need_dW: bool = True, workspace: Optional[torch.Tensor] = None, stream=None,
                          w_layout: int = W_KN) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """resized_linear_bwd from the checkpoint of X: [M, n_keep] in blocks (DROP_K) or [M, K] (DROP_N).  workspace: of
    mx_bwd_workspace_bytes bytes (zr.h says how far less will do), needed for dW (None: allocated)."""
    here = _here()
    on = _on(stream, here)
    M, N = dY.shape
    wshape = W.shape
    K = wshape[0] if w_layout == W_KN else wshape[1]
    dt = dY.dtype
    if wshape != ((K, N) if w_layout == W_KN else (N, K)) or W.dtype is not dt:
        raise ValueError("dY must be [M, N] and W [K, N] (W_KN) or [N, K] (W_NK) of its dtype")
    kp, n_keep = _list(keep_idx, here)
    wp, ldw = _grid(W, here, "W")
    gp, ldg = _grid(dY, here, "dY")

    def result(need, t, prev, shape, name):
        """(tensor, pointer, leading dimension, previous one's pointer) of an output."""
        if not need:
            return None, None, 0, None
        if t is None:
            t = _empty(shape, dt, dY.device, stream)
        elif t.shape != shape or t.dtype is not dt:
            raise ValueError(f"{name}: wrong shape or dtype")
        p, ld = _grid(t, here, name)
        pp = None
        if prev is not None:
            pp, ldp = _grid(prev, here, "prev_" + name)
            if ldp != ld or prev.shape != shape or prev.dtype is not dt:
                raise ValueError(f"prev_{name} must be like {name}, its leading dimension too")
        return t, p, ld, pp

    dX, dxp, lddx, pxp = result(need_dX, dX, prev_dX, (M, K), "dX")
    dW, dwp, lddw, pwp = result(need_dW, dW, prev_dW, wshape, "dW")
    xq, ldxq, xs, ldxs, fmt = _mx(X if need_dW else None, M, n_keep if mode == DROP_K else K, here, "X")
    if workspace is None and need_dW:
        workspace = _empty(_bwd_scratch(M, K, N, n_keep, mode, dt), torch.uint8, dY.device, stream, returned=False)
    if workspace is not None and workspace.get_device() != here:
        raise ValueError("workspace: must be on the current GPU")
    st = _lib.zr_resized_linear_bwd_mx(xq, ldxq, xs, ldxs, fmt, wp, ldw, gp, ldg, dxp, lddx, dwp, lddw, M, K, N,
                                       kp, n_keep, mode, w_layout, _code(dt), policy, pxp, pwp,
                                       *_ws(workspace), on)
    if st:
        raise ZrError(st)
    return dX, dW


# ---- around the products of a block: bias, activation, gate, dropout, residual, norms ----
def _vec(t: Optional[torch.Tensor], n: int, dt, here: int, name: str):
    """Pointer of a vector of n values of dtype dt, None: None."""
    if t is None:
        return None
    if t.dtype is not dt or t.shape != (n,) or not t.is_contiguous() or t.get_device() != here:
        raise ValueError(f"{name}: need a contiguous vector of {n} {dt} on the current GPU")
    return t.data_ptr()


def _like(t: Optional[torch.Tensor], shape, dt, here: int, name: str):
    """(pointer, leading dimension) of a matrix of this shape and dtype, None: (None, 0)."""
    if t is None:
        return None, 0
    ld, one = t.stride() if t.dtype is dt and t.shape == shape else (0, 0)
    if one != 1 or t.get_device() != here:
        raise ValueError(f"{name}: need {tuple(shape)} of {dt} with unit column stride, on the current GPU")
    return t.data_ptr(), ld


def _generator(rng: Optional[torch.Tensor], here: int):
    """Pointer to seed and offset: two 64-bit integers in GPU memory."""
    if rng is None:
        return None
    if rng.dtype not in (torch.int64, torch.uint64) or rng.numel() != 2 or not rng.is_contiguous() or rng.get_device() != here:
        raise ValueError("rng: need two contiguous 64-bit integers, seed and offset, on the current GPU")
    return rng.data_ptr()


def _scratch(workspace: Optional[torch.Tensor], here: int):
    if workspace is None:
        return None, 0
    if workspace.get_device() != here:
        raise ValueError("workspace: must be on the current GPU")
    return _ws(workspace)


def dropout(x: torch.Tensor, p: float, rng: Optional[torch.Tensor], out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x with elements dropped with probability p and the others scaled up; the same call on a gradient is the backward pass.
    rng: seed and offset in GPU memory (zr.h says which draw an element looks at)."""
    here = _here()
    on = _on(stream, here)
    xp, ldx = _grid(x, here, "x")
    if out is None:
        out = _empty(x.shape, x.dtype, x.device, stream)
    op, ldo = _like(out, x.shape, x.dtype, here, "out")
    st = _lib.zr_dropout(xp, ldx, op, ldo, x.shape[0], x.shape[1], p, _generator(rng, here) if p else None, _code(x.dtype), on)
    if st:
        raise ZrError(st)
    return out


def act_workspace_bytes(M: int, K: int, N: int, n_keep: int, mode: int, dtype, backward: bool = False) -> int:
    f = _lib.zr_act_bwd_workspace_bytes if backward else _lib.zr_act_fwd_workspace_bytes
    return int(f(M, K, N, n_keep, mode, dtype if isinstance(dtype, int) else _code(dtype)))


def _layer(X_shape, W: torch.Tensor, N: int, dt, w_layout: int):
    K = W.shape[0] if w_layout == W_KN else W.shape[1]
    if W.shape != ((K, N) if w_layout == W_KN else (N, K)) or W.dtype is not dt or (X_shape is not None and X_shape[1] != K):
        raise ValueError("need X [M, K], W [K, N] (W_KN) or [N, K] (W_NK), all of one dtype")
    return K


def resized_linear_act_fwd(X: torch.Tensor, W: torch.Tensor, keep_idx: Optional[torch.Tensor] = None, mode: int = DROP_K,
                           bias: Optional[torch.Tensor] = None, act: int = ACT_NONE, gate: Optional[torch.Tensor] = None, p: float = 0.0,
                           rng: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
                           Z: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None,
                           w_layout: int = W_KN) -> torch.Tensor:
    """Y = residual + dropout(act(X W + bias) * gate), with the kept list of resized_linear_fwd (None: nothing is pruned).
    Z, where given, receives X W + bias for the backward pass.  workspace: optional, of act_workspace_bytes bytes."""
    here = _here()
    on = _on(stream, here)
    xp, ldx = _grid(X, here, "X")
    wp, ldw = _grid(W, here, "W")
    M, dt = X.shape[0], X.dtype
    N = W.shape[1] if w_layout == W_KN else W.shape[0]
    K = _layer(X.shape, W, N, dt, w_layout)
    kp, nk = _list(keep_idx, here)
    if Y is None:
        Y = _empty((M, N), dt, X.device, stream)
    yp, ldy = _like(Y, (M, N), dt, here, "Y")
    zp, ldz = _like(Z, (M, N), dt, here, "Z")
    gp, ldg = _like(gate, (M, N), dt, here, "gate")
    rp, ldr = _like(residual, (M, N), dt, here, "residual")
    st = _lib.zr_resized_linear_act_fwd(xp, ldx, wp, ldw, yp, ldy, M, K, N, kp, nk, mode, w_layout, _code(dt),
                                        _vec(bias, N, dt, here, "bias"), act, gp, ldg, p, _generator(rng, here) if p else None, rp, ldr, zp, ldz,
                                        *_scratch(workspace, here), on)
    if st:
        raise ZrError(st)
    return Y


def resized_linear_act_bwd(X: Optional[torch.Tensor], W: torch.Tensor, dY: torch.Tensor, keep_idx: Optional[torch.Tensor] = None,
                           mode: int = DROP_K, act: int = ACT_NONE, Z: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                           p: float = 0.0, rng: Optional[torch.Tensor] = None, dX: Optional[torch.Tensor] = None,
                           dW: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None,
                           need_dX: bool = True, need_dW: bool = True, workspace: Optional[torch.Tensor] = None, stream=None,
                           w_layout: int = W_KN) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """The gradients of resized_linear_act_fwd: (dX, dW); dbias and dgate are computed where tensors for them are given.  The
    residual's gradient is dY.  workspace: of act_workspace_bytes(backward=True) bytes (None: allocated)."""
    here = _here()
    on = _on(stream, here)
    M, N = dY.shape
    dt = dY.dtype
    K = _layer(None, W, N, dt, w_layout)
    kp, nk = _list(keep_idx, here)
    xp, ldx = _like(X, (M, K), dt, here, "X")
    wp, ldw = _grid(W, here, "W")
    gyp, ldgy = _grid(dY, here, "dY")
    zp, ldz = _like(Z, (M, N), dt, here, "Z")
    gp, ldg = _like(gate, (M, N), dt, here, "gate")
    dgp, lddg = _like(dgate, (M, N), dt, here, "dgate")
    if not need_dX:
        dX = None
    elif dX is None:
        dX = _empty((M, K), dt, dY.device, stream)
    if not need_dW:
        dW = None
    elif dW is None:
        dW = _empty(tuple(W.shape), dt, dY.device, stream)
    dxp, lddx = _like(dX, (M, K), dt, here, "dX")
    dwp, lddw = _like(dW, W.shape, dt, here, "dW")
    if workspace is None:
        n_keep = nk if kp is not None else N if mode == DROP_N else K
        workspace = _empty(act_workspace_bytes(M, K, N, n_keep, mode, dt, True), torch.uint8, dY.device, stream, returned=False)
    st = _lib.zr_resized_linear_act_bwd(xp, ldx, wp, ldw, gyp, ldgy, zp, ldz, gp, ldg, dxp, lddx, dwp, lddw,
                                        _vec(dbias, N, dt, here, "dbias"), dgp, lddg, M, K, N, kp, nk, mode, w_layout, _code(dt), act, p,
                                        _generator(rng, here) if p else None, *_scratch(workspace, here), on)
    if st:
        raise ZrError(st)
    return dX, dW


def block_join_workspace_bytes(rows: int, cols: int) -> int:
    return int(_lib.zr_block_join_workspace_bytes(rows, cols))


def block_join_fwd(y: torch.Tensor, x: torch.Tensor, norm: int = NORM_RMS, post: bool = False, pre: bool = True, eps: float = 1e-5,
                   p: float = 0.0, rng: Optional[torch.Tensor] = None, scale: float = 1.0, bias: Optional[torch.Tensor] = None,
                   gate: Optional[torch.Tensor] = None, post_w: Optional[torch.Tensor] = None, post_b: Optional[torch.Tensor] = None,
                   pre_w: Optional[torch.Tensor] = None, pre_b: Optional[torch.Tensor] = None, x_out: Optional[torch.Tensor] = None,
                   h: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """x_out = x + scale * gate * post(dropout(y + bias)), h = pre(x_out) with the norms that are asked for: (x_out, h or None)."""
    here = _here()
    on = _on(stream, here)
    yp, ldy = _grid(y, here, "y")
    shape, dt = y.shape, y.dtype
    rows, cols = shape
    xp, ldx = _like(x, shape, dt, here, "x")
    if x_out is None:
        x_out = _empty(tuple(shape), dt, y.device, stream)
    if not pre:
        h = None
    elif h is None:
        h = _empty(tuple(shape), dt, y.device, stream)
    op, ldo = _like(x_out, shape, dt, here, "x_out")
    hp, ldh = _like(h, shape, dt, here, "h")
    st = _lib.zr_block_join_fwd(yp, ldy, xp, ldx, op, ldo, hp, ldh, rows, cols, (1 if post else 0) | (2 if pre else 0), norm, eps, p,
                                _generator(rng, here) if p else None, scale, _vec(bias, cols, dt, here, "bias"), _vec(gate, cols, dt, here, "gate"),
                                _vec(post_w, cols, dt, here, "post_w"), _vec(post_b, cols, dt, here, "post_b"),
                                _vec(pre_w, cols, dt, here, "pre_w"), _vec(pre_b, cols, dt, here, "pre_b"), _code(dt), on)
    if st:
        raise ZrError(st)
    return x_out, h


def block_join_bwd(dx_out: Optional[torch.Tensor], dh: Optional[torch.Tensor], x_out: Optional[torch.Tensor], y: Optional[torch.Tensor],
                   norm: int = NORM_RMS, post: bool = False, pre: bool = True, eps: float = 1e-5, p: float = 0.0,
                   rng: Optional[torch.Tensor] = None, scale: float = 1.0, bias: Optional[torch.Tensor] = None,
                   gate: Optional[torch.Tensor] = None, post_w: Optional[torch.Tensor] = None, post_b: Optional[torch.Tensor] = None,
                   pre_w: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None, dy: Optional[torch.Tensor] = None,
                   dbias: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None, dpost_w: Optional[torch.Tensor] = None,
                   dpost_b: Optional[torch.Tensor] = None, dpre_w: Optional[torch.Tensor] = None, dpre_b: Optional[torch.Tensor] = None,
                   need_dx: bool = True, need_dy: bool = True, workspace: Optional[torch.Tensor] = None,
                   stream=None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """The gradients of block_join_fwd from those at x_out (None: zeros) and h, x_out and y: (dx, dy); a vector's gradient is
    computed where a tensor for it is given.  workspace: of block_join_workspace_bytes bytes (None: allocated where needed)."""
    here = _here()
    on = _on(stream, here)
    first = next((t for t in (dx_out, dh) if t is not None), None)
    if first is None:
        raise ZrError(1)
    shape, dt = first.shape, first.dtype
    rows, cols = shape
    gp, ldg = _like(dx_out, shape, dt, here, "dx_out")
    hp, ldh = _like(dh, shape, dt, here, "dh")
    xp, ldx = _like(x_out, shape, dt, here, "x_out")
    yp, ldy = _like(y, shape, dt, here, "y")
    if not need_dx:
        dx = None
    elif dx is None:
        dx = _empty(tuple(shape), dt, first.device, stream)
    if not need_dy:
        dy = None
    elif dy is None:
        dy = _empty(tuple(shape), dt, first.device, stream)
    dxp, lddx = _like(dx, shape, dt, here, "dx")
    dyp, lddy = _like(dy, shape, dt, here, "dy")
    sums = [_vec(t, cols, dt, here, n) for t, n in ((dbias, "dbias"), (dgate, "dgate"), (dpost_w, "dpost_w"), (dpost_b, "dpost_b"),
                                                    (dpre_w, "dpre_w"), (dpre_b, "dpre_b"))]
    if workspace is None and any(s is not None for s in sums):
        workspace = _empty(block_join_workspace_bytes(rows, cols), torch.uint8, first.device, stream, returned=False)
    st = _lib.zr_block_join_bwd(gp, ldg, hp, ldh, xp, ldx, yp, ldy, dxp, lddx, dyp, lddy, rows, cols,
                                (1 if post else 0) | (2 if pre else 0), norm, eps, p, _generator(rng, here) if p else None, scale,
                                _vec(bias, cols, dt, here, "bias"), _vec(gate, cols, dt, here, "gate"),
                                _vec(post_w, cols, dt, here, "post_w"), _vec(post_b, cols, dt, here, "post_b"),
                                _vec(pre_w, cols, dt, here, "pre_w"), *sums, *_scratch(workspace, here), _code(dt), on)
    if st:
        raise ZrError(st)
    return dx, dy


def priority_scores(W_t: torch.Tensor, W_prev: torch.Tensor, mode: int,
                    prev_scores: Optional[torch.Tensor] = None, prev_keep_idx: Optional[torch.Tensor] = None,
                    scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    K, N = W_t.shape
    (tp, ld), (pp, ldp) = _mat(W_t, "W_t"), _mat(W_prev, "W_prev")
    if W_prev.shape != W_t.shape or ldp != ld or W_prev.dtype != W_t.dtype:
        raise ValueError("W_prev must match W_t in shape, leading dimension and dtype")
    n = N if mode == DROP_N else K
    if scores is None:
        scores = torch.empty(n, dtype=torch.float32, device=W_t.device)
    _check(_lib.zr_priority_scores(tp, pp, ld, K, N, mode,
                                   None if prev_scores is None else prev_scores.data_ptr(),
                                   None if prev_keep_idx is None else prev_keep_idx.data_ptr(),
                                   0 if prev_keep_idx is None else prev_keep_idx.numel(),
                                   scores.data_ptr(), _dtype_code(W_t), *_ws(workspace), _stream(stream)))
    return scores


def priority_scores_static(W_t: torch.Tensor, W_prev: torch.Tensor, mode: int, scores: torch.Tensor,
                           prev_scores: Optional[torch.Tensor] = None, prev_keep_idx: Optional[torch.Tensor] = None,
                           stream=None) -> torch.Tensor:
    """zr_priority_scores_static: the library's own scratch, nothing allocated (the caller brings `scores`)."""
    K, N = W_t.shape
    (tp, ld), (pp, ldp) = _mat(W_t, "W_t"), _mat(W_prev, "W_prev")
    if W_prev.shape != W_t.shape or ldp != ld or W_prev.dtype != W_t.dtype:
        raise ValueError("W_prev must match W_t in shape, leading dimension and dtype")
    _check(_lib.zr_priority_scores_static(tp, pp, ld, K, N, mode,
                                          None if prev_scores is None else prev_scores.data_ptr(),
                                          None if prev_keep_idx is None else prev_keep_idx.data_ptr(),
                                          0 if prev_keep_idx is None else prev_keep_idx.numel(),
                                          scores.data_ptr(), _dtype_code(W_t), _stream(stream)))
    return scores


def priority_static_scratch_bytes() -> int:
    return int(_lib.zr_priority_static_scratch_bytes())


def priority_workspace_bytes(K: int, N: int, mode: int) -> int:
    return int(_lib.zr_priority_workspace_bytes(K, N, mode))


def pruning_ratio(T_i: float, T_avg: float, M_i: float, gamma_max: float = 0.9) -> float:
    return float(_lib.zr_pruning_ratio(T_i, T_avg, M_i, gamma_max))


def count_above(scores: torch.Tensor, theta: float, count: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    if count is None:
        count = torch.empty(1, dtype=torch.int32, device=scores.device)
    _check(_lib.zr_count_above(scores.data_ptr(), scores.numel(), float(theta), count.data_ptr(), _stream(stream)))
    return count


def layer_ratio(count_above_: int, L: int, alpha: float, gamma: float) -> float:
    return float(_lib.zr_layer_ratio(int(count_above_), int(L), alpha, gamma))


def migration_range(r_i: int, r_k: int, e: int, L_mig: int):
    b, en = _i64(0), _i64(0)
    _check(_lib.zr_migration_range(r_i, r_k, e, L_mig, ctypes.byref(b), ctypes.byref(en)))
    return int(b.value), int(en.value)


def migrated_accumulate(out: torch.Tensor, A: torch.Tensor, B: torch.Tensor, b_transposed: bool, stream=None) -> torch.Tensor:
    """out += A @ B (or A @ B.T); A, B, out may be column/row slices of larger matrices."""
    M, C = A.shape
    N = out.shape[1]
    if out.shape[0] != M or tuple(B.shape) != ((N, C) if b_transposed else (C, N)):
        raise ValueError("shape mismatch")
    if not (A.dtype == B.dtype == out.dtype):
        raise ValueError("dtype mismatch")
    (ap, lda), (bp, ldb), (op, ldo) = _mat(A, "A"), _mat(B, "B"), _mat(out, "out")
    _check(_lib.zr_migrated_accumulate(ap, lda, bp, ldb, 1 if b_transposed else 0, op, ldo, M, N, C,
                                       _dtype_code(out), _stream(stream)))
    return out


def debug_time_next_product(start: "torch.cuda.Event", stop: "torch.cuda.Event") -> None:
    """The next product records the two events right around its GEMM launch(es).
    The events must have been created with enable_timing=True and recorded once
    before (torch creates the HIP event lazily)."""
    _check(_lib.zr_debug_time_next_product(start.cuda_event, stop.cuda_event))


def debug_mfma_rate(blocks: int, iters: int, stream=None) -> float:
    """Launches the register-only MFMA loop (time it with events); returns the FLOPs it performs."""
    sink = torch.empty(blocks, dtype=torch.float32, device="cuda")
    flops = ctypes.c_double(0.0)
    _check(_lib.zr_debug_mfma_rate(blocks, iters, sink.data_ptr(), ctypes.byref(flops), _stream(stream)))
    return float(flops.value)


def debug_record_kernel_names(on: bool = True) -> None:
    """Switches the recording of GEMM kernel names on or off for this thread (off by default)."""
    _lib.zr_debug_record_kernel_names(1 if on else 0)


def debug_last_kernel() -> str:
    return _lib.zr_debug_last_kernel().decode()


def validate_keep_idx(keep_idx: torch.Tensor, n: int, stream=None) -> bool:
    flag = torch.zeros(1, dtype=torch.int32, device=keep_idx.device)
    st = _lib.zr_validate_keep_idx(keep_idx.data_ptr(), keep_idx.numel(), n, flag.data_ptr(), _stream(stream))
    if st == 0:
        return True
    if st == 4:
        return False
    raise ZrError(st)
