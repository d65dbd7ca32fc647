"""ctypes binding of the attention entry points (include/attn.h): argument marshalling only."""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass

from . import binding as _b
from .binding import KNN_ERR_HIP, KNN_ERR_INVALID_ARG, KNN_OK, KnnError, knn_status_string

ATTN_MAX_D = 128
ATTN_BF16, ATTN_F16 = 0, 1

ATTN_SYMBOLS = ("attn_plan", "attn_grad_plan", "attn_apply", "attn_grad")


class RowsStruct(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64), ("hs", ctypes.c_int64)]


class OptionsStruct(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("scale", ctypes.c_double),
                ("cap", ctypes.c_double), ("slopes", ctypes.c_void_p), ("docs", ctypes.c_int64),
                ("starts", ctypes.c_void_p), ("k_starts", ctypes.c_void_p), ("prefix", ctypes.c_void_p)]


class AttnPlanStruct(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("m", ctypes.c_int64), ("hq", ctypes.c_int32), ("hkv", ctypes.c_int32),
                ("d", ctypes.c_int32), ("tile_rows", ctypes.c_int32), ("n_splits", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("workspace_bytes", ctypes.c_uint64),
                ("min_limit_bytes", ctypes.c_uint64)]


@dataclass(frozen=True)
class AttnPlan:
    n: int
    m: int
    hq: int
    hkv: int
    d: int
    tile_rows: int
    n_splits: int
    workspace_bytes: int
    min_limit_bytes: int


_ready = False


def _load():
    global _ready
    lib = _b.load()
    if not _ready:
        i64, i32, u64, vp, ptr = ctypes.c_int64, ctypes.c_int32, ctypes.c_uint64, ctypes.c_void_p, ctypes.POINTER
        shape, rows = [i64, i64, i32, i32, i32], ptr(RowsStruct)
        lib.attn_plan.argtypes = lib.attn_grad_plan.argtypes = shape + [u64, ptr(AttnPlanStruct)]
        lib.attn_apply.argtypes = [rows, rows, rows] + shape + [ptr(OptionsStruct), u64, vp, u64, rows, vp, vp]
        lib.attn_grad.argtypes = [rows, rows, rows, rows, vp, rows] + shape + [ptr(OptionsStruct), u64, vp, u64, rows,
                                                                              rows, rows, vp]
        for name in ATTN_SYMBOLS:
            getattr(lib, name).restype = ctypes.c_int
        _ready = True
    return lib


def _raise(st: int, plan=None):
    detail = knn_status_string(st)
    if st == KNN_ERR_HIP:
        detail += " (" + _load().knn_last_hip_error().decode() + ")"
    raise KnnError(st, detail, int(plan.min_limit_bytes) if plan is not None else 0)


def _plan(fn, n, m, hq, hkv, d, mem_limit_bytes) -> AttnPlan:
    ps = AttnPlanStruct()
    st = int(fn(n, m, hq, hkv, d, mem_limit_bytes, ctypes.byref(ps)))
    if st != KNN_OK:
        _raise(st, ps)
    return AttnPlan(*(getattr(ps, f[0]) for f in AttnPlanStruct._fields_ if f[0] != "reserved"))


def attn_plan(n: int, m: int, hq: int, hkv: int, d: int, mem_limit_bytes: int) -> AttnPlan:
    return _plan(_load().attn_plan, n, m, hq, hkv, d, mem_limit_bytes)


def attn_grad_plan(n: int, m: int, hq: int, hkv: int, d: int, mem_limit_bytes: int) -> AttnPlan:
    return _plan(_load().attn_grad_plan, n, m, hq, hkv, d, mem_limit_bytes)


def _refuse(text):
    raise KnnError(KNN_ERR_INVALID_ARG, text)


def _rows(t):
    """[rows, heads, d] with unit stride along d."""
    return RowsStruct(t.data_ptr() if t.numel() else None, t.stride(0), t.stride(1))


def _check_rows(name, t, like, shape):
    if not t.is_cuda or t.device != like.device or t.dtype != like.dtype or tuple(t.shape) != tuple(shape):
        _refuse(f"{name} must be {tuple(shape)} in {like.dtype} on {like.device}")
    if t.shape[2] > 1 and t.stride(2) != 1:
        _refuse(f"{name} must have unit stride along its last dimension")


def _words(name, t, device, count, dtype):
    if t is None:
        return None
    if not t.is_cuda or t.device != device or t.dtype != dtype or t.dim() != 1 or not t.is_contiguous() or \
            (count is not None and t.numel() != count):
        _refuse(f"{name} must be contiguous {dtype}" + ("" if count is None else f" with {count} entries") + f" on {device}")
    return t.data_ptr()


def _dtype(Q):
    import torch

    if not Q.is_cuda:
        _refuse("Q must be a device tensor (no CPU path exists)")
    if Q.dtype not in (torch.bfloat16, torch.float16):
        _refuse("Q, K and V must be bfloat16 or float16")
    return ATTN_BF16 if Q.dtype == torch.bfloat16 else ATTN_F16


def _shape(Q, K, V):
    if Q.dim() != 3 or K.dim() != 3 or V.dim() != 3:
        _refuse("Q, K and V must be [rows, heads, d]")
    (n, hq, d), (m, hkv, _) = Q.shape, K.shape
    _check_rows("Q", Q, Q, Q.shape)
    _check_rows("K", K, Q, (m, hkv, d))
    _check_rows("V", V, Q, (m, hkv, d))
    return n, m, hq, hkv, d


def _options(Q, scale, causal, cap, slopes, starts, k_starts, prefix):
    import torch

    dtype = _dtype(Q)
    if k_starts is None:
        k_starts = starts
    if starts is None and k_starts is not None:
        _refuse("k_starts needs starts")
    docs = 1 if starts is None else starts.numel() - 1
    if docs < 1:
        _refuse("starts must hold at least two entries")
    o = OptionsStruct(dtype, int(bool(causal)), 1.0 / math.sqrt(Q.shape[2]) if scale is None else float(scale),
                      float(cap), _words("slopes", slopes, Q.device, Q.shape[1], torch.float32), docs,
                      _words("starts", starts, Q.device, docs + 1, torch.int32),
                      _words("k_starts", k_starts, Q.device, docs + 1, torch.int32),
                      _words("prefix", prefix, Q.device, docs, torch.int32))
    return o


def _workspace(workspace, nbytes, device):
    import torch

    if workspace is None:
        return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    if not workspace.is_cuda or workspace.device != device or workspace.dtype != torch.uint8 or \
            not workspace.is_contiguous():
        _refuse(f"workspace must be contiguous uint8 on {device}")
    return workspace


def attn_apply(Q, K, V, mem_limit_bytes: int, scale=None, causal: bool = False, cap: float = 0.0, slopes=None,
               starts=None, k_starts=None, prefix=None, workspace=None, out=None):
    """attn_apply(Q[n,hq,d], K[m,hkv,d], V[m,hkv,d], mem_limit_bytes, ...) -> (O [n,hq,d], lse fp32 [hq,n]).

    O = softmax(scores) V without the n x m matrix; Q, K, V all bfloat16 or all float16, any strides
    with a unit one along d, hkv a divisor of hq.  scale (default 1 / sqrt(d)); causal; cap: scores
    become cap * tanh(score / cap); slopes fp32 [hq]: minus slope * distance; starts, k_starts int32
    [docs + 1] (k_starts = starts unless given): rows see keys of their own document; prefix int32
    [docs]: keys at a document's start that all its rows see although causal.  Rows outside the
    documents keep what `out` (O, lse) holds there.  The workspace (uint8, attn_plan's bytes) is
    allocated here unless given.  Work is enqueued on torch's current stream; no synchronisation is done.
    """
    import torch

    options = _options(Q, scale, causal, cap, slopes, starts, k_starts, prefix)
    n, m, hq, hkv, d = _shape(Q, K, V)
    plan = attn_plan(n, m, hq, hkv, d, mem_limit_bytes)
    with torch.cuda.device(Q.device):
        workspace = _workspace(workspace, plan.workspace_bytes, Q.device)
        if out is None:
            O = torch.empty((n, hq, d), dtype=Q.dtype, device=Q.device)
            lse = torch.empty((hq, n), dtype=torch.float32, device=Q.device)
        else:
            O, lse = out
            _check_rows("O", O, Q, (n, hq, d))
            _check_lse(lse, hq, n, Q.device)
        st = int(_load().attn_apply(_rows(Q), _rows(K), _rows(V), n, m, hq, hkv, d, options, mem_limit_bytes,
                                    workspace.data_ptr(), workspace.numel(), _rows(O), lse.data_ptr(),
                                    torch.cuda.current_stream(Q.device).cuda_stream))
    if st != KNN_OK:
        _raise(st)
    return O, lse


def _check_lse(lse, hq, n, device):
    import torch

    if not lse.is_cuda or lse.device != device or lse.dtype != torch.float32 or tuple(lse.shape) != (hq, n) or \
            not lse.is_contiguous():
        _refuse(f"lse must be contiguous float32 [{hq}, {n}] on {device}")


def attn_grad(Q, K, V, O, lse, dO, mem_limit_bytes: int, scale=None, causal: bool = False, cap: float = 0.0,
              slopes=None, starts=None, k_starts=None, prefix=None, workspace=None, out=None):
    """attn_grad(Q, K, V, O, lse, dO, mem_limit_bytes, ...) -> (dQ [n,hq,d], dK [m,hkv,d], dV [m,hkv,d]).

    The gradients of sum(dO * O) by Q, K and V; O and lse as attn_apply gave them for the same Q, K, V and
    options.  Heads that share a K and V add up.  The workspace (uint8, attn_grad_plan's bytes) is allocated here
    unless given; `out` takes the three gradients.  The same inputs give the same bits.
    """
    import torch

    options = _options(Q, scale, causal, cap, slopes, starts, k_starts, prefix)
    n, m, hq, hkv, d = _shape(Q, K, V)
    _check_rows("O", O, Q, (n, hq, d))
    _check_rows("dO", dO, Q, (n, hq, d))
    _check_lse(lse, hq, n, Q.device)
    plan = attn_grad_plan(n, m, hq, hkv, d, mem_limit_bytes)
    with torch.cuda.device(Q.device):
        workspace = _workspace(workspace, plan.workspace_bytes, Q.device)
        if out is None:
            dQ = torch.empty((n, hq, d), dtype=Q.dtype, device=Q.device)
            dK, dV = (torch.empty((m, hkv, d), dtype=Q.dtype, device=Q.device) for _ in range(2))
        else:
            dQ, dK, dV = out
            _check_rows("dQ", dQ, Q, (n, hq, d))
            _check_rows("dK", dK, Q, (m, hkv, d))
            _check_rows("dV", dV, Q, (m, hkv, d))
        st = int(_load().attn_grad(_rows(Q), _rows(K), _rows(V), _rows(O), lse.data_ptr(), _rows(dO), n, m, hq, hkv, d,
                                   options, mem_limit_bytes, workspace.data_ptr(), workspace.numel(), _rows(dQ),
                                   _rows(dK), _rows(dV), torch.cuda.current_stream(Q.device).cuda_stream))
    if st != KNN_OK:
        _raise(st)
    return dQ, dK, dV
