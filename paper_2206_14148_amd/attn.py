"""ctypes binding of the attention entry points (include/attn.h): argument marshalling only."""
from __future__ import annotations

import contextlib
import ctypes
import math
from dataclasses import dataclass

try:  # plans need no tensors
    import torch
except ImportError:
    torch = None

from . import binding as _b
from .binding import KNN_ERR_HIP, KNN_ERR_INVALID_ARG, KNN_OK, KnnError, knn_status_string

ATTN_MAX_D = 128
ATTN_BF16, ATTN_F16 = 0, 1

ATTN_INT8, ATTN_E4M3 = 0, 1

ATTN_SYMBOLS = ("attn_plan", "attn_grad_plan", "attn_apply", "attn_grad", "attn_cache_row", "attn_cache_map",
                "attn_cache_append", "attn_cache_plan", "attn_cache_apply")


class RowsStruct(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64), ("hs", ctypes.c_int64)]


class OptionsStruct(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("scale", ctypes.c_double),
                ("cap", ctypes.c_double), ("slopes", ctypes.c_void_p), ("docs", ctypes.c_int64),
                ("starts", ctypes.c_void_p), ("k_starts", ctypes.c_void_p), ("prefix", ctypes.c_void_p)]


class AttnPlanStruct(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("m", ctypes.c_int64), ("hq", ctypes.c_int32), ("hkv", ctypes.c_int32),
                ("d", ctypes.c_int32), ("tile_rows", ctypes.c_int32), ("n_splits", ctypes.c_int32),
                ("row_splits", ctypes.c_int32), ("workspace_bytes", ctypes.c_uint64),
                ("min_limit_bytes", ctypes.c_uint64)]


class CacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("blocks", ctypes.c_int64), ("hkv", ctypes.c_int32),
                ("d", ctypes.c_int32), ("block", ctypes.c_int32), ("code", ctypes.c_int32)]


class AttnCachePlanStruct(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("longest", ctypes.c_int64), ("nq", ctypes.c_int32), ("hq", ctypes.c_int32),
                ("hkv", ctypes.c_int32), ("d", ctypes.c_int32), ("range_tokens", ctypes.c_int32),
                ("n_ranges", ctypes.c_int32), ("workspace_bytes", ctypes.c_uint64),
                ("min_limit_bytes", ctypes.c_uint64)]


@dataclass(frozen=True)
class AttnCachePlan:
    batch: int
    longest: int
    nq: int
    hq: int
    hkv: int
    d: int
    range_tokens: int
    n_ranges: int
    workspace_bytes: int
    min_limit_bytes: int


@dataclass(frozen=True)
class AttnPlan:
    n: int
    m: int
    hq: int
    hkv: int
    d: int
    tile_rows: int
    n_splits: int
    row_splits: int
    workspace_bytes: int
    min_limit_bytes: int


_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = _b.load()
        i64, i32, u64, vp, ptr = ctypes.c_int64, ctypes.c_int32, ctypes.c_uint64, ctypes.c_void_p, ctypes.POINTER
        shape, rows = [i64, i64, i32, i32, i32], ptr(RowsStruct)
        lib.attn_plan.argtypes = lib.attn_grad_plan.argtypes = shape + [u64, ptr(AttnPlanStruct)]
        lib.attn_apply.argtypes = [rows, rows, rows] + shape + [ptr(OptionsStruct), u64, vp, u64, rows, vp, vp]
        lib.attn_grad.argtypes = [rows, rows, rows, rows, vp, rows] + shape + [ptr(OptionsStruct), u64, vp, u64, rows,
                                                                              rows, rows, vp]
        cache = ptr(CacheStruct)
        lib.attn_cache_row.argtypes = [i32]
        lib.attn_cache_map.argtypes = [vp, vp, i64, vp, i64, i32, vp, i64, vp, vp, i64, vp, vp]
        lib.attn_cache_append.argtypes = [cache, i32, rows, rows, i64, vp, vp]
        lib.attn_cache_plan.argtypes = [i64, i32, i32, i32, i32, i64, u64, ptr(AttnCachePlanStruct)]
        lib.attn_cache_apply.argtypes = [cache, i32, rows, i64, i32, i32, vp, i64, vp, ctypes.c_double, ctypes.c_double,
                                         vp, u64, vp, u64, rows, vp]
        for name in ATTN_SYMBOLS:
            getattr(lib, name).restype = ctypes.c_int
        _lib = lib
    return _lib


_same_device = contextlib.nullcontext()


def _on(device):
    """The device as the current one; nothing to do where it is."""
    return _same_device if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _stream(device) -> int:
    # (the object that torch makes around it would cost more than all checks of a call)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw else torch.cuda.current_stream(device).cuda_stream


def _raise(st: int, plan=None):
    detail = knn_status_string(st)
    if st == KNN_ERR_HIP:
        detail += " (" + _load().knn_last_hip_error().decode() + ")"
    raise KnnError(st, detail, int(plan.min_limit_bytes) if plan is not None else 0)


def _planned(fn, ps, *shape):
    st = int(fn(*shape, ctypes.byref(ps)))
    if st != KNN_OK:
        _raise(st, ps)
    return ps


def _as(cls, ps):
    return cls(*(getattr(ps, name) for name in cls.__dataclass_fields__))


def attn_plan(n: int, m: int, hq: int, hkv: int, d: int, mem_limit_bytes: int) -> AttnPlan:
    return _as(AttnPlan, _planned(_load().attn_plan, AttnPlanStruct(), n, m, hq, hkv, d, mem_limit_bytes))


def attn_grad_plan(n: int, m: int, hq: int, hkv: int, d: int, mem_limit_bytes: int) -> AttnPlan:
    return _as(AttnPlan, _planned(_load().attn_grad_plan, AttnPlanStruct(), n, m, hq, hkv, d, mem_limit_bytes))


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
    if not Q.is_cuda:
        _refuse("Q must be a device tensor (no CPU path exists)")
    if Q.dtype not in (torch.bfloat16, torch.float16):
        _refuse("Q, K and V must be bfloat16 or float16")
    return ATTN_BF16 if Q.dtype == torch.bfloat16 else ATTN_F16


def _shape(Q, K, V):
    _dtype(Q)
    if Q.dim() != 3 or K.dim() != 3 or V.dim() != 3:
        _refuse("Q, K and V must be [rows, heads, d]")
    (n, hq, d), (m, hkv, _) = Q.shape, K.shape
    _check_rows("Q", Q, Q, Q.shape)
    _check_rows("K", K, Q, (m, hkv, d))
    _check_rows("V", V, Q, (m, hkv, d))
    return n, m, hq, hkv, d


def _options(Q, scale, causal, cap, slopes, starts, k_starts, prefix):
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
    """(the tensor, which the call keeps alive, its address and size)"""
    if workspace is None:
        if not nbytes:
            return None, None, 0
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return workspace, workspace.data_ptr(), nbytes
    if not workspace.is_cuda or workspace.device != device or workspace.dtype != torch.uint8 or \
            not workspace.is_contiguous():
        _refuse(f"workspace must be contiguous uint8 on {device}")
    return workspace, workspace.data_ptr(), workspace.numel()


def attn_apply(Q, K, V, mem_limit_bytes: int, scale=None, causal: bool = False, cap: float = 0.0, slopes=None,
               starts=None, k_starts=None, prefix=None, workspace=None, out=None):
    """attn_apply(Q[n,hq,d], K[m,hkv,d], V[m,hkv,d], mem_limit_bytes, ...) -> (O [n,hq,d], lse fp32 [hq,n]).

    O = softmax(scores) V without the n x m matrix; Q, K, V all bfloat16 or all float16, any strides
    with a unit one along d, hkv a divisor of hq.  scale (default 1 / sqrt(d)); causal; cap: scores
    become cap * tanh(score / cap); slopes fp32 [hq]: minus slope * distance; starts, k_starts int32
    [docs + 1] (k_starts = starts unless given): rows see keys of their own document; prefix int32
    [docs]: keys at a document's start that all its rows see although causal.  Rows outside the
    documents keep what `out` (O, lse) holds there.  d is 128 at most.  The call is not recorded for autograd, whatever
    its inputs ask for: attn_grad gives the gradients.  The workspace (uint8, attn_plan's bytes) is allocated here unless given.  Work is enqueued on torch's current stream; no synchronisation is done.
    """
    n, m, hq, hkv, d = _shape(Q, K, V)
    plan = _planned(_load().attn_plan, AttnPlanStruct(), n, m, hq, hkv, d, mem_limit_bytes)
    options = _options(Q, scale, causal, cap, slopes, starts, k_starts, prefix)
    with _on(Q.device):
        workspace, ws, ws_bytes = _workspace(workspace, plan.workspace_bytes, Q.device)
        if out is None:
            O = torch.empty((n, hq, d), dtype=Q.dtype, device=Q.device)
            lse = torch.empty((hq, n), dtype=torch.float32, device=Q.device)
        else:
            O, lse = out
            _check_rows("O", O, Q, (n, hq, d))
            _check_lse(lse, hq, n, Q.device)
        st = int(_load().attn_apply(_rows(Q), _rows(K), _rows(V), n, m, hq, hkv, d, options, mem_limit_bytes,
                                    ws, ws_bytes, _rows(O), lse.data_ptr(),
                                    _stream(Q.device)))
    if st != KNN_OK:
        _raise(st)
    return O, lse


def _check_lse(lse, hq, n, device):
    if not lse.is_cuda or lse.device != device or lse.dtype != torch.float32 or tuple(lse.shape) != (hq, n) or \
            not lse.is_contiguous():
        _refuse(f"lse must be contiguous float32 [{hq}, {n}] on {device}")


def attn_grad(Q, K, V, O, lse, dO, mem_limit_bytes: int, scale=None, causal: bool = False, cap: float = 0.0,
              slopes=None, starts=None, k_starts=None, prefix=None, workspace=None, out=None):
    """attn_grad(Q, K, V, O, lse, dO, mem_limit_bytes, ...) -> (dQ [n,hq,d], dK [m,hkv,d], dV [m,hkv,d]).

    The gradients of sum(dO * O) by Q, K and V; O and lse as attn_apply gave them for the same Q, K, V and
    options.  Heads that share a K and V add up.  The workspace (uint8, attn_grad_plan's bytes) is allocated here
    unless given; `out` takes the three gradients.  The same inputs give the same bits.  In float16 P and the scores'
    gradients are scaled by powers of two, so dO may be of any magnitude that its gradients have in float16.
    """
    n, m, hq, hkv, d = _shape(Q, K, V)
    _check_rows("O", O, Q, (n, hq, d))
    _check_rows("dO", dO, Q, (n, hq, d))
    _check_lse(lse, hq, n, Q.device)
    plan = _planned(_load().attn_grad_plan, AttnPlanStruct(), n, m, hq, hkv, d, mem_limit_bytes)
    options = _options(Q, scale, causal, cap, slopes, starts, k_starts, prefix)
    with _on(Q.device):
        workspace, ws, ws_bytes = _workspace(workspace, plan.workspace_bytes, Q.device)
        if out is None:
            dQ = torch.empty((n, hq, d), dtype=Q.dtype, device=Q.device)
            dK, dV = (torch.empty((m, hkv, d), dtype=Q.dtype, device=Q.device) for _ in range(2))
        else:
            dQ, dK, dV = out
            _check_rows("dQ", dQ, Q, (n, hq, d))
            _check_rows("dK", dK, Q, (m, hkv, d))
            _check_rows("dV", dV, Q, (m, hkv, d))
        st = int(_load().attn_grad(_rows(Q), _rows(K), _rows(V), _rows(O), lse.data_ptr(), _rows(dO), n, m, hq, hkv, d,
                                   options, mem_limit_bytes, ws, ws_bytes, _rows(dQ),
                                   _rows(dK), _rows(dV), _stream(Q.device)))
    if st != KNN_OK:
        _raise(st)
    return dQ, dK, dV


def attn_cache_row(d: int) -> int:
    """Entries of a row in a cache of rows of d: 64 or 128."""
    row = int(_load().attn_cache_row(d))
    if row == 0:
        _refuse(f"d must be in 1 .. {ATTN_MAX_D}")
    return row


@dataclass(frozen=True)
class AttnCache:
    """Keys and values of earlier rows as 8-bit codes in blocks: k [blocks, hkv, block, row], v [blocks, hkv, row,
    block] (int8 or float8_e4m3fn, contiguous), k_scale, v_scale fp32 [blocks, hkv]; row = attn_cache_row(d)."""
    k: "object"
    v: "object"
    k_scale: "object"
    v_scale: "object"
    d: int

    @staticmethod
    def empty(blocks: int, hkv: int, d: int, block: int, code: str = "int8", device="cuda") -> "AttnCache":
        """A cache of nothing yet; code "int8" or "e4m3"."""
        dtype = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}.get(code)
        if dtype is None:
            _refuse('code must be "int8" or "e4m3"')
        row = attn_cache_row(d)
        k = torch.zeros((blocks, hkv, block, row), dtype=torch.uint8, device=device).view(dtype)
        v = torch.zeros((blocks, hkv, row, block), dtype=torch.uint8, device=device).view(dtype)
        scales = [torch.zeros((blocks, hkv), dtype=torch.float32, device=device) for _ in range(2)]
        return AttnCache(k, v, scales[0], scales[1], d)

    @staticmethod
    def blocks_within(limit_bytes: int, hkv: int, d: int, block: int) -> int:
        """How many blocks limit_bytes hold, scales included."""
        return _b.knn_chunk_rows(limit_bytes, hkv * (2 * block * attn_cache_row(d) + 8))

    def _struct(self):
        k, v, ks, vs = self.k, self.v, self.k_scale, self.v_scale
        if k.dim() != 4 or not k.is_cuda:
            _refuse("k and v must be 4-D device tensors")
        blocks, hkv, block, row = shape = k.shape
        if row != (64 if self.d <= 64 else 128) or not 1 <= self.d <= ATTN_MAX_D or v.shape != (blocks, hkv, row, block):
            _refuse("k must be [blocks, hkv, block, attn_cache_row(d)] and v the same with the last two exchanged")
        code = _codes().get(k.dtype)
        device = k.device
        if code is None or v.dtype != k.dtype or v.device != device or not k.is_contiguous() or not v.is_contiguous():
            _refuse("k and v must be contiguous, both int8 or both float8_e4m3fn, on one device")
        for t in (ks, vs):
            if t.dtype != torch.float32 or t.device != device or t.shape != shape[:2] or not t.is_contiguous():
                _refuse("k_scale and v_scale must be contiguous float32 [blocks, hkv] on the device of k")
        return CacheStruct(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), blocks, hkv, self.d, block, code)


def _codes():
    return {torch.int8: ATTN_INT8, torch.float8_e4m3fn: ATTN_E4M3}


def attn_cache_plan(batch: int, nq: int, hq: int, hkv: int, d: int, longest: int, mem_limit_bytes: int) -> AttnCachePlan:
    return _as(AttnCachePlan, _planned(_load().attn_cache_plan, AttnCachePlanStruct(), batch, nq, hq, hkv, d, longest,
                                       mem_limit_bytes))


def _check_table(table, batch, device):
    if not table.is_cuda or table.device != device or table.dtype != torch.int32 or table.dim() != 2 or \
            table.shape[0] != batch or not table.is_contiguous():
        _refuse(f"table must be contiguous int32 [{batch}, width] on {device}")


def attn_cache_map(lengths, news, table, free, block: int, n_slots: int, out=None):
    """attn_cache_map(lengths[batch], news[batch], table[batch,width], free[n], block, n_slots)
    -> (table, starts int32 [batch+1], slots int64 [n_slots], used int32 [1]).

    A step's block tables and slots from the requests' lengths after it and their numbers of new tokens (all int32):
    `table` is completed in place with blocks from `free`, in order; the new tokens of request i are rows starts[i] ..
    starts[i + 1] - 1 and go to slots; -1 behind the last and where there is no block.  `used` entries of `free` are
    needed; more than it has: too few.  `out` takes (starts, slots, used).
    """
    if not lengths.is_cuda:
        _refuse("lengths must be a device tensor (no CPU path exists)")
    if n_slots < 0:
        _refuse("n_slots must not be negative")
    device, batch = lengths.device, lengths.numel()
    _check_table(table, batch, device)
    pointers = (_words("lengths", lengths, device, batch, torch.int32), _words("news", news, device, batch, torch.int32))
    free_ptr = _words("free", free, device, None, torch.int32)
    with _on(device):
        if out is None:
            starts = torch.empty((batch + 1,), dtype=torch.int32, device=device)
            slots = torch.empty((n_slots,), dtype=torch.int64, device=device)
            used = torch.empty((1,), dtype=torch.int32, device=device)
        else:
            starts, slots, used = out
            _words("starts", starts, device, batch + 1, torch.int32)
            _words("slots", slots, device, n_slots, torch.int64)
            _words("used", used, device, 1, torch.int32)
        st = int(_load().attn_cache_map(*pointers, batch, table.data_ptr(), table.shape[1], block, free_ptr, free.numel(),
                                        starts.data_ptr(), slots.data_ptr(), n_slots, used.data_ptr(),
                                        _stream(device)))
    if st != KNN_OK:
        _raise(st)
    return table, starts, slots, used


def attn_cache_append(cache: AttnCache, K, V, slots) -> None:
    """attn_cache_append(cache, K[count,hkv,d], V[count,hkv,d], slots int64 [count]): new rows into the cache.

    The slots of one block must stand together; -1 is passed over, within a block as well.  A block's scale grows with its largest magnitude,
    codes that it holds already follow; a block that gets its token 0 is begun anew.
    """
    c = cache._struct()
    if not K.is_cuda or K.device != cache.k.device:
        _refuse("K and V must be on the cache's device")
    dtype = _dtype(K)
    if K.dim() != 3 or V.dim() != 3:
        _refuse("K and V must be [rows, heads, d]")
    count = K.shape[0]
    _check_rows("K", K, K, (count, c.hkv, c.d))
    _check_rows("V", V, K, (count, c.hkv, c.d))
    at = _words("slots", slots, K.device, count, torch.int64)
    with _on(K.device):
        st = int(_load().attn_cache_append(c, dtype, _rows(K), _rows(V), count, at,
                                           _stream(K.device)))
    if st != KNN_OK:
        _raise(st)


def attn_cache_apply(Q, cache: AttnCache, table, lengths, mem_limit_bytes: int, scale=None, cap: float = 0.0, slopes=None,
                     workspace=None, out=None):
    """attn_cache_apply(Q[batch,nq,hq,d], cache, table int32 [batch,width], lengths int32 [batch], ...) -> O like Q.

    Attention of the last nq rows of each request over the `lengths` tokens that the cache holds of it, the rows'
    own among them: row t sees tokens up to lengths - nq + t.  scale, cap and slopes as in attn_apply.  The workspace
    (uint8, attn_cache_plan's bytes for longest = width * block) is allocated here unless given.
    """
    c = cache._struct()
    if not Q.is_cuda or Q.device != cache.k.device or Q.dim() != 4:
        _refuse("Q must be [batch, nq, hq, d] on the cache's device")
    dtype = _dtype(Q)
    batch, nq, hq, d = Q.shape
    if d != c.d or (d > 1 and Q.stride(3) != 1):
        _refuse("Q must have the cache's d and unit stride along it")
    _check_table(table, batch, Q.device)
    at = _words("lengths", lengths, Q.device, batch, torch.int32)
    tilt = _words("slopes", slopes, Q.device, hq, torch.float32)
    plan = _planned(_load().attn_cache_plan, AttnCachePlanStruct(), batch, nq, hq, c.hkv, d, table.shape[1] * c.block,
                    mem_limit_bytes)
    with _on(Q.device):
        workspace, ws, ws_bytes = _workspace(workspace, plan.workspace_bytes, Q.device)
        O = torch.empty((batch, nq, hq, d), dtype=Q.dtype, device=Q.device) if out is None else out
        if not O.is_cuda or O.device != Q.device or O.dtype != Q.dtype or O.shape != Q.shape or (d > 1 and O.stride(3) != 1):
            _refuse(f"out must be {tuple(Q.shape)} in {Q.dtype} on {Q.device} with unit stride along its last dimension")
        flat = []
        for t in (Q, O):
            if batch > 1 and nq > 1 and t.stride(0) != nq * t.stride(1):
                _refuse("the rows of all requests must lie evenly apart (stride(0) == nq * stride(1))")
            flat.append(RowsStruct(t.data_ptr() if t.numel() else None, t.stride(1) if nq > 1 else t.stride(0), t.stride(2)))
        st = int(_load().attn_cache_apply(c, dtype, flat[0], batch, nq, hq, table.data_ptr(), table.shape[1], at,
                                          1.0 / math.sqrt(d) if scale is None else float(scale), float(cap), tilt,
                                          mem_limit_bytes, ws, ws_bytes, flat[1],
                                          _stream(Q.device)))
    if st != KNN_OK:
        _raise(st)
    return O
