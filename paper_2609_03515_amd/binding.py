"""ctypes binding of libinertiakv.so: argument marshalling only.

Every function carries the name of the C entry point it calls and takes torch tensors for device buffers;
it passes their device pointers and the current HIP stream, and raises KVError on a non-zero status.  All
computation happens in the HIP kernels behind the C ABI; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libinertiakv.so")

KV_OK, KV_ERR_INVALID_ARG, KV_ERR_UNSUPPORTED, KV_ERR_WORKSPACE, KV_ERR_HIP = 0, -1, -2, -3, -4
KV_F32, KV_BF16 = 0, 1
KV_INIT_MEAN, KV_INIT_MIN, KV_INIT_ZERO = 0, 1, 2
KV_RULE_EMA, KV_RULE_SINGLE_STEP, KV_RULE_CUMULATIVE = 0, 1, 2
KV_SCORE_ATTENTION, KV_SCORE_VNORM, KV_SCORE_ENTROPY, KV_SCORE_NORMS_EMITTED = 0, 1, 2, 4
KV_EMIT_SCORES, KV_EMIT_VNORMS = 1, 2
KV_FAULT_EXCHANGE_TIMEOUT, KV_FAULT_CACHE, KV_FAULT_NO_PAGES, KV_FAULT_SHARED_PAGE = 1, 2, 4, 8
KV_PATH_LDS, KV_PATH_EXCHANGE, KV_PATH_LOGITS = 0, 1, 2
KV_PHASES = 5
PHASES = ("append", "score", "fold", "select", "compact")

EXPORTED = ("kv_workspace_bytes", "kv_score_ema", "kv_topk_select", "kv_compact", "kv_evict_step",
            "kv_append", "kv_attend_score", "kv_evict_finish", "kv_rank_trace_state_bytes", "kv_score_merge",
            "kv_score_plan", "kv_fault_status", "kv_set_exchange_wait_limit", "kv_evict_step_static",
            "kv_value_norms", "kv_q4_pool_bytes", "kv_q4_workspace_bytes", "kv_q4_reserve", "kv_q4_store", "kv_q4_load",
            "kv_q4_store_rotary", "kv_q4_window_workspace_bytes", "kv_q4_attend_window", "kv_q4_shared_workspace_bytes",
            "kv_q4_attend_shared", "kv_q4_attend", "kv_q4_fork", "kv_q4_free", "kv_q4_compact", "kv_q4_evict", "kv_status_string")
KV_STATIC_SCRATCH_BYTES = 64 << 20
KV_TRACE_COUNTS = 10


class KVError(RuntimeError):
    def __init__(self, fn, status):
        super().__init__(f"{fn} failed: {status_string(status)} ({status})")
        self.status = status


class KvShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("capacity", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class KvParams(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("budget", ctypes.c_int32), ("refresh_period", ctypes.c_int32),
                ("score_free", ctypes.c_int32), ("nonrefresh_init", ctypes.c_int32),
                ("recency_bias", ctypes.c_float), ("recency_window", ctypes.c_int32), ("rule", ctypes.c_int32),
                ("score_variant", ctypes.c_int32), ("score_merge", ctypes.c_int32)]


class KvTrace(ctypes.Structure):
    _fields_ = [("begin", ctypes.c_void_p * KV_PHASES), ("end", ctypes.c_void_p * KV_PHASES)]


class KvScoreInfo(ctypes.Structure):
    _fields_ = [("merge", ctypes.c_int32), ("path", ctypes.c_int32), ("chunks", ctypes.c_int32)]


class KvRankTrace(ctypes.Structure):
    _fields_ = [("k", ctypes.c_int32), ("max_pos", ctypes.c_int32), ("state", ctypes.c_void_p),
                ("counts", ctypes.c_void_p), ("raw_keep", ctypes.c_void_p), ("ema_keep", ctypes.c_void_p)]


class KvQ4Shape(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("batch", "layers", "n_q_heads", "n_kv_heads", "head_dim", "dtype",
                                                    "page_rows", "n_pages", "max_pages")]


class KvQ4Buffers(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("pool", "table", "len", "refs", "u", "pos")]


class KvRotary(ctypes.Structure):
    _fields_ = [("dim", ctypes.c_int32), ("adjacent", ctypes.c_int32), ("axes", ctypes.c_int32), ("scale", ctypes.c_float),
                ("inv_freq", ctypes.c_float * 64), ("axis", ctypes.c_uint8 * 64)]


class KvQ4Strides(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int64) for name in ("layer", "batch", "head", "row")]


_lib = None


def load_library(path: str = LIB_PATH):
    """Loads the built library; raises if it is missing (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2609_03515_amd.build.build()")
    lib = ctypes.CDLL(path)
    vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    shp, prm, trc = ctypes.POINTER(KvShape), ctypes.POINTER(KvParams), ctypes.POINTER(KvTrace)
    rtr = ctypes.POINTER(KvRankTrace)
    lib.kv_workspace_bytes.argtypes = [shp, i32, ctypes.POINTER(sz)]
    lib.kv_score_ema.argtypes = [shp, i32, vp, vp, vp, i32, f32, f32, i32, vp, vp, vp, sz, vp]
    lib.kv_topk_select.argtypes = [shp, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.kv_compact.argtypes = [shp, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.kv_evict_step.argtypes = [shp, prm, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp,
                                  ctypes.POINTER(i32), vp, vp, trc, rtr, vp, sz, vp]
    lib.kv_append.argtypes = [shp, prm, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.kv_attend_score.argtypes = [shp, i32, i32, i32, vp, vp, vp, vp, i32, f32, i32, i32, vp, vp, sz, vp]
    lib.kv_evict_finish.argtypes = [shp, prm, i32, i32, vp, vp, vp, vp, vp, ctypes.POINTER(i32), vp, vp, rtr, vp,
                                    sz, vp]
    lib.kv_value_norms.argtypes = [shp, i32, vp, vp, vp]
    lib.kv_rank_trace_state_bytes.argtypes = [i32, i32, ctypes.POINTER(sz)]
    lib.kv_score_merge.argtypes = [shp, i32, prm, ctypes.POINTER(i32)]
    lib.kv_score_plan.argtypes = [shp, i32, prm, ctypes.POINTER(KvScoreInfo)]
    lib.kv_fault_status.argtypes = [vp, sz, vp, i32, vp]
    lib.kv_set_exchange_wait_limit.argtypes = [i32]
    lib.kv_evict_step_static.argtypes = [shp, prm, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp,
                                         ctypes.POINTER(i32), vp, vp, trc, rtr, vp]
    qsh, buf, std = ctypes.POINTER(KvQ4Shape), ctypes.POINTER(KvQ4Buffers), ctypes.POINTER(KvQ4Strides)
    lib.kv_q4_pool_bytes.argtypes = [qsh, ctypes.POINTER(sz)]
    lib.kv_q4_workspace_bytes.argtypes = [qsh, i32, i32, ctypes.POINTER(sz)]
    lib.kv_q4_reserve.argtypes = [qsh, buf, vp, vp, i32, vp, vp, sz, vp]
    lib.kv_q4_store.argtypes = [qsh, buf, i32, i32, i32, vp, vp, vp, std, vp, std, vp, sz, vp]
    lib.kv_q4_load.argtypes = lib.kv_q4_store.argtypes
    lib.kv_q4_store_rotary.argtypes = [qsh, buf, i32, i32, i32, vp, vp, ctypes.POINTER(KvRotary), vp, vp, std, vp, std, vp, std,
                                       vp, std, vp, sz, vp]
    lib.kv_q4_attend.argtypes = [qsh, buf, i32, i32, i32, vp, vp, f32, i32, vp, vp, f32, vp, vp, vp, sz, vp]
    lib.kv_q4_window_workspace_bytes.argtypes = [qsh, i32, i32, i32, ctypes.POINTER(sz)]
    lib.kv_q4_attend_window.argtypes = [qsh, buf, i32, i32, i32, i32, vp, vp, std, i32, i32, vp, std, vp, sz, vp]
    lib.kv_q4_shared_workspace_bytes.argtypes = [qsh, i32, i32, ctypes.POINTER(sz)]
    lib.kv_q4_attend_shared.argtypes = [qsh, buf, i32, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.kv_q4_fork.argtypes = [qsh, buf, i32, vp, vp, vp, sz, vp]
    lib.kv_q4_free.argtypes = [qsh, buf, i32, vp, vp, sz, vp]
    lib.kv_q4_compact.argtypes = [qsh, buf, i32, vp, vp, sz, vp]
    lib.kv_q4_evict.argtypes = [qsh, buf, i32, vp, vp, vp, sz, vp]
    for fn in EXPORTED[:-1]:
        getattr(lib, fn).restype = i32
    lib.kv_status_string.argtypes = [i32]
    lib.kv_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().kv_status_string(int(status)).decode()


def _check(fn, status):
    if status != KV_OK:
        raise KVError(fn, status)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


# torch's raw handle of a device's current stream, and the current device: internal names, None in a torch without them
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        # the current device's current stream.  Building torch's Stream object for it took 2.9 us of a call's 13
        # (one eviction step) or 10 (one layer's attention); the raw handle takes 0.2
        if _raw_stream is not None and _device is not None and torch.cuda.is_initialized():
            return _raw_stream(_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_shape(batch, layers, n_q_heads, n_kv_heads, head_dim, capacity, dtype) -> KvShape:
    if isinstance(dtype, str):
        dtype = {"f32": KV_F32, "bf16": KV_BF16}[dtype]
    elif dtype in (torch.float32, torch.bfloat16):
        dtype = KV_F32 if dtype == torch.float32 else KV_BF16
    return KvShape(batch, layers, n_q_heads, n_kv_heads, head_dim, capacity, dtype)


def make_params(alpha, budget, refresh_period=1, score_free=False, nonrefresh_init="mean", recency_bias=0.0,
                recency_window=0, rule="ema", vnorm=False, entropy=False, norms_emitted=False,
                score_merge=0) -> KvParams:
    init = {"mean": KV_INIT_MEAN, "min": KV_INIT_MIN}[nonrefresh_init] if isinstance(nonrefresh_init, str) \
        else int(nonrefresh_init)
    rl = {"ema": KV_RULE_EMA, "single": KV_RULE_SINGLE_STEP, "cumulative": KV_RULE_CUMULATIVE}[rule] \
        if isinstance(rule, str) else int(rule)
    variant = (KV_SCORE_VNORM if vnorm else 0) | (KV_SCORE_ENTROPY if entropy else 0) | \
        (KV_SCORE_NORMS_EMITTED if norms_emitted else 0)
    return KvParams(float(alpha), int(budget), int(refresh_period), int(bool(score_free)), init,
                    float(recency_bias), int(recency_window), rl, variant, int(score_merge))


def kv_workspace_bytes(shape: KvShape, n_max: int) -> int:
    out = ctypes.c_size_t(0)
    _check("kv_workspace_bytes", load_library().kv_workspace_bytes(ctypes.byref(shape), int(n_max),
                                                                    ctypes.byref(out)))
    return out.value


def kv_score_merge(shape: KvShape, n: int, params: KvParams) -> int:
    out = ctypes.c_int32(0)
    _check("kv_score_merge", load_library().kv_score_merge(ctypes.byref(shape), int(n), ctypes.byref(params),
                                                            ctypes.byref(out)))
    return out.value


def kv_score_plan(shape: KvShape, n: int, params: KvParams) -> KvScoreInfo:
    out = KvScoreInfo()
    _check("kv_score_plan", load_library().kv_score_plan(ctypes.byref(shape), int(n), ctypes.byref(params),
                                                          ctypes.byref(out)))
    return out


def kv_fault_status(ws, out=None, clear=False, stream=None):
    """Queues the copy of the workspace's fault word into `out` (a device int32/uint32 tensor of one element,
    or None) and/or its clearing."""
    _check("kv_fault_status", load_library().kv_fault_status(_ptr(ws), _ws_bytes(ws), _ptr(out), int(bool(clear)),
                                                              _stream(stream)))


def kv_set_exchange_wait_limit(polls: int) -> int:
    return int(load_library().kv_set_exchange_wait_limit(int(polls)))


def kv_score_ema(shape, n, q, k, pos, cur_pos, alpha, recency_bias, recency_window, u, s_out, ws, stream=None):
    _check("kv_score_ema", load_library().kv_score_ema(
        ctypes.byref(shape), int(n), _ptr(q), _ptr(k), _ptr(pos), int(cur_pos), float(alpha),
        float(recency_bias), int(recency_window), _ptr(u), _ptr(s_out), _ptr(ws),
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def kv_topk_select(shape, n, budget, u, pos, keep, ws, stream=None):
    _check("kv_topk_select", load_library().kv_topk_select(
        ctypes.byref(shape), int(n), int(budget), _ptr(u), _ptr(pos), _ptr(keep), _ptr(ws),
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def kv_compact(shape, n, budget, keep, k, v, u, pos, ws, stream=None, v_norms=None):
    _check("kv_compact", load_library().kv_compact(
        ctypes.byref(shape), int(n), int(budget), _ptr(keep), _ptr(k), _ptr(v), _ptr(u), _ptr(pos), _ptr(v_norms),
        _ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def kv_value_norms(shape, n, v, v_norms, stream=None):
    """Fills the value-norm cache v_norms [layers][batch][n_kv][cap] float for rows [0, n) from V."""
    _check("kv_value_norms", load_library().kv_value_norms(ctypes.byref(shape), int(n), _ptr(v), _ptr(v_norms),
                                                            _stream(stream)))


def kv_evict_step(shape, params, t, n_in, new_pos, q, k_new, v_new, k, v, u, pos, ws, keep_out=None,
                  s_out=None, trace: KvTrace | None = None, rank_trace: KvRankTrace | None = None,
                  stream=None, v_norms=None) -> int:
    """Returns n_out = min(B, n_in + 1)."""
    n_out = ctypes.c_int32(-1)
    _check("kv_evict_step", load_library().kv_evict_step(
        ctypes.byref(shape), ctypes.byref(params), int(t), int(n_in), int(new_pos), _ptr(q), _ptr(k_new),
        _ptr(v_new), _ptr(k), _ptr(v), _ptr(u), _ptr(pos), _ptr(v_norms), ctypes.byref(n_out), _ptr(keep_out),
        _ptr(s_out),
        ctypes.byref(trace) if trace is not None else None,
        ctypes.byref(rank_trace) if rank_trace is not None else None, _ptr(ws),
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))
    return n_out.value


def kv_evict_step_static(shape, params, t, n_in, new_pos, q, k_new, v_new, k, v, u, pos, keep_out=None,
                         s_out=None, trace: KvTrace | None = None, rank_trace: KvRankTrace | None = None,
                         stream=None, v_norms=None) -> int:
    """kv_evict_step with the library's static scratch instead of a workspace.  Returns n_out."""
    n_out = ctypes.c_int32(-1)
    _check("kv_evict_step_static", load_library().kv_evict_step_static(
        ctypes.byref(shape), ctypes.byref(params), int(t), int(n_in), int(new_pos), _ptr(q), _ptr(k_new),
        _ptr(v_new), _ptr(k), _ptr(v), _ptr(u), _ptr(pos), _ptr(v_norms), ctypes.byref(n_out), _ptr(keep_out),
        _ptr(s_out),
        ctypes.byref(trace) if trace is not None else None,
        ctypes.byref(rank_trace) if rank_trace is not None else None, _stream(stream)))
    return n_out.value


def kv_rank_trace_state_bytes(batch: int, max_pos: int) -> int:
    out = ctypes.c_size_t(0)
    _check("kv_rank_trace_state_bytes", load_library().kv_rank_trace_state_bytes(int(batch), int(max_pos),
                                                                                  ctypes.byref(out)))
    return out.value


def make_rank_trace(k, max_pos, state, counts, raw_keep=None, ema_keep=None) -> KvRankTrace:
    """state: a zero-filled device tensor of kv_rank_trace_state_bytes() bytes; counts: int32 device tensor
    [batch][KV_TRACE_COUNTS].  Keep the tensors alive while the struct is in use."""
    return KvRankTrace(int(k), int(max_pos), _ptr(state), _ptr(counts), _ptr(raw_keep), _ptr(ema_keep))


def _ws_bytes(ws):
    return ws.numel() * ws.element_size() if ws is not None else 0


def kv_append(shape, params, t, n_in, new_pos, k_new, v_new, k, v, u, pos, stream=None, v_norms=None):
    _check("kv_append", load_library().kv_append(
        ctypes.byref(shape), ctypes.byref(params), int(t), int(n_in), int(new_pos), _ptr(k_new), _ptr(v_new),
        _ptr(k), _ptr(v), _ptr(u), _ptr(pos), _ptr(v_norms), _stream(stream)))


def kv_attend_score(shape, layer0, layer_count, n, q, k, v, pos, cur_pos, recency_bias, recency_window,
                    emit_scores, o, ws, stream=None):
    _check("kv_attend_score", load_library().kv_attend_score(
        ctypes.byref(shape), int(layer0), int(layer_count), int(n), _ptr(q), _ptr(k), _ptr(v), _ptr(pos),
        int(cur_pos), float(recency_bias), int(recency_window), int(emit_scores), _ptr(o), _ptr(ws),
        _ws_bytes(ws), _stream(stream)))


def kv_evict_finish(shape, params, t, n, k, v, u, pos, ws, keep_out=None, s_out=None,
                    rank_trace: KvRankTrace | None = None, stream=None, v_norms=None) -> int:
    """Returns n_out = min(B, n)."""
    n_out = ctypes.c_int32(-1)
    _check("kv_evict_finish", load_library().kv_evict_finish(
        ctypes.byref(shape), ctypes.byref(params), int(t), int(n), _ptr(k), _ptr(v), _ptr(u), _ptr(pos),
        _ptr(v_norms), ctypes.byref(n_out), _ptr(keep_out), _ptr(s_out),
        ctypes.byref(rank_trace) if rank_trace is not None else None, _ptr(ws), _ws_bytes(ws), _stream(stream)))
    return n_out.value


def workspace(shape: KvShape, n_max: int, device="cuda") -> torch.Tensor:
    """A caller-owned workspace tensor of kv_workspace_bytes() bytes (256-byte aligned by the allocator), its
    fault word cleared on the current stream."""
    nbytes = kv_workspace_bytes(shape, n_max)
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    kv_fault_status(ws, None, clear=True)
    return ws


class KvCache:
    """One cache's device buffers (caller-owned torch tensors) and its cached row count n, for `evict_step`.

    k, v: [layers][batch][n_kv_heads][capacity][head_dim] of the shape's dtype; u: [batch][capacity] f32;
    pos: [batch][capacity] int32; ws: a workspace of kv_workspace_bytes(shape, capacity) bytes; v_norms: the
    optional per-row value-norm cache [layers][batch][n_kv_heads][capacity] f32 (VNorm scoring)."""

    def __init__(self, shape: KvShape, k, v, u, pos, n: int, ws, v_norms=None):
        self.shape, self.k, self.v, self.u, self.pos, self.n, self.ws = shape, k, v, u, pos, int(n), ws
        self.v_norms = v_norms

    @classmethod
    def allocate(cls, shape: KvShape, device="cuda", v_norms=False) -> "KvCache":
        """Zero-filled buffers for `shape` with n = 0; the caller fills the prefill rows and sets n."""
        dt = torch.float32 if shape.dtype == KV_F32 else torch.bfloat16
        rows = (shape.layers, shape.batch, shape.n_kv_heads, shape.capacity)
        return cls(shape, torch.zeros(rows + (shape.head_dim,), dtype=dt, device=device),
                   torch.zeros(rows + (shape.head_dim,), dtype=dt, device=device),
                   torch.zeros(shape.batch, shape.capacity, dtype=torch.float32, device=device),
                   torch.zeros(shape.batch, shape.capacity, dtype=torch.int32, device=device), 0,
                   workspace(shape, shape.capacity, device),
                   torch.zeros(rows, dtype=torch.float32, device=device) if v_norms else None)


def evict_step(cache: KvCache, q, k_new, v_new, t: int, params: KvParams, new_pos: int, keep_out=None,
               s_out=None, stream=None) -> int:
    """One decode step t (1-based) through kv_evict_step on `cache`'s buffers: the newcomer (q, k_new, v_new at
    position new_pos) is appended, and on refresh steps the cache is scored, folded, selected and compacted to
    the budget.  Sets cache.n to the new row count and returns it; raises KVError on a non-zero status."""
    cache.n = kv_evict_step(cache.shape, params, t, cache.n, new_pos, q, k_new, v_new, cache.k, cache.v,
                            cache.u, cache.pos, cache.ws, keep_out=keep_out, s_out=s_out, stream=stream,
                            v_norms=cache.v_norms)
    return cache.n


def faults(ws, clear=False) -> int:
    """The workspace's fault word (kv_fault bits), read after synchronising the current stream."""
    out = torch.zeros(1, dtype=torch.int32, device=ws.device)
    kv_fault_status(ws, out, clear=clear)
    return int(out.item()) & 0xffffffff


# --- Paged 4-bit cache ----------------------------------------------------------------------------------------
def make_q4_shape(batch, layers, n_q_heads, n_kv_heads, head_dim, page_rows, n_pages, max_pages, dtype) -> KvQ4Shape:
    if isinstance(dtype, str):
        dtype = {"f32": KV_F32, "bf16": KV_BF16}[dtype]
    elif dtype in (torch.float32, torch.bfloat16):
        dtype = KV_F32 if dtype == torch.float32 else KV_BF16
    return KvQ4Shape(batch, layers, n_q_heads, n_kv_heads, head_dim, dtype, page_rows, n_pages, max_pages)


def kv_q4_pool_bytes(shape: KvQ4Shape) -> int:
    out = ctypes.c_size_t(0)
    _check("kv_q4_pool_bytes", load_library().kv_q4_pool_bytes(ctypes.byref(shape), ctypes.byref(out)))
    return out.value


def kv_q4_workspace_bytes(shape: KvQ4Shape, n_max: int, layer_count: int) -> int:
    out = ctypes.c_size_t(0)
    _check("kv_q4_workspace_bytes", load_library().kv_q4_workspace_bytes(ctypes.byref(shape), int(n_max),
                                                                          int(layer_count), ctypes.byref(out)))
    return out.value


def q4_workspace(shape: KvQ4Shape, n_max: int, layer_count: int, device="cuda") -> torch.Tensor:
    """A caller-owned workspace tensor of kv_q4_workspace_bytes() bytes, its fault word cleared on the current stream."""
    ws = torch.empty(kv_q4_workspace_bytes(shape, n_max, layer_count), dtype=torch.uint8, device=device)
    kv_fault_status(ws, None, clear=True)
    return ws


def _q4_buffer(name, needed):
    """A buffer of a KvQ4Cache: what is assigned is checked and is what the calls see from then on."""

    def get(cache):
        return cache._tensors[name]

    def put(cache, t):
        dtype, numel = cache._sizes[name]
        if (needed if t is None else t.device != cache._place or not _q4_ok(t, dtype, numel, cache._device)):
            raise KVError("KvQ4Cache." + name, KV_ERR_INVALID_ARG)
        cache._tensors[name] = t
        setattr(cache._addresses, name, _ptr(t))

    return property(get, put)


class KvQ4Cache:
    """One paged 4-bit cache's device buffers (caller-owned, contiguous torch tensors) for the kv_q4 calls.

    pool: uint8, kv_q4_pool_bytes(shape); table: [batch][max_pages] int32; len: [batch] int32; refs: [n_pages] int32;
    u: [batch][capacity] f32 and pos: [batch][capacity] int32 (nullable: not kept), capacity = max_pages * page_rows.
    A buffer may be replaced by assigning another (cache.u = u_out, say); one whose storage is changed under the same tensor
    (resize_, set_) has to be assigned again.  The shape is a copy of the caller's, and shape and buffers (the addresses) give copies."""

    def __init__(self, shape: KvQ4Shape, pool, table, len, refs, u=None, pos=None):
        cap = shape.max_pages * shape.page_rows
        self._place, self._device = pool.device, pool.get_device()
        self._own, self._addresses, self._tensors = KvQ4Shape.from_buffer_copy(shape), KvQ4Buffers(), {}
        i32 = torch.int32
        self._sizes = {"pool": (torch.uint8, kv_q4_pool_bytes(shape)), "table": (i32, shape.batch * shape.max_pages),
                       "len": (i32, shape.batch), "refs": (i32, shape.n_pages), "u": (torch.float32, shape.batch * cap),
                       "pos": (i32, shape.batch * cap)}
        self.pool, self.table, self.len, self.refs, self.u, self.pos = pool, table, len, refs, u, pos
        self.element = torch.float32 if shape.dtype == KV_F32 else torch.bfloat16
        # what every call passes or compares with, taken once (building it took 4 us of a call's 13)
        self._shape, self._buffers = ctypes.byref(self._own), ctypes.byref(self._addresses)
        self._batch, self._rows = shape.batch, shape.batch * cap
        self._heads, self._dim, self._query = shape.n_kv_heads, shape.head_dim, (shape.batch, shape.n_q_heads, shape.head_dim)

    pool, table, len, refs = (_q4_buffer(name, True) for name in ("pool", "table", "len", "refs"))
    u, pos = _q4_buffer("u", False), _q4_buffer("pos", False)

    @property
    def shape(self) -> KvQ4Shape:
        return KvQ4Shape.from_buffer_copy(self._own)

    @property
    def buffers(self) -> KvQ4Buffers:
        return KvQ4Buffers.from_buffer_copy(self._addresses)

    @classmethod
    def allocate(cls, shape: KvQ4Shape, device="cuda") -> "KvQ4Cache":
        """Buffers of an empty cache."""
        cap = shape.max_pages * shape.page_rows
        return cls(shape, torch.empty(kv_q4_pool_bytes(shape), dtype=torch.uint8, device=device),
                   torch.full((shape.batch, shape.max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(shape.batch, dtype=torch.int32, device=device),
                   torch.zeros(shape.n_pages, dtype=torch.int32, device=device),
                   torch.zeros(shape.batch, cap, dtype=torch.float32, device=device),
                   torch.zeros(shape.batch, cap, dtype=torch.int32, device=device))


def _q4_ok(t, dtype, numel, device):
    """Whether a buffer that a kernel indexes without knowing its size is none, or has the type, place, layout and size."""
    return t is None or (t.dtype is dtype and t.numel() >= numel and t.get_device() == device and t.is_contiguous())


def _q4_heads(cache, t, layers):
    """Whether queries or outputs have the cache's type and place, and the heads of `layers` layers at least, in order."""
    if t is None:
        return False
    s = tuple(t.shape)
    return (t.dtype is cache.element and t.get_device() == cache._device and t.is_contiguous()
            and (s == cache._query and layers == 1 or s[1:] == cache._query and s[0] >= layers))


def _q4_tail(fn, cache, ws, stream):
    """The last arguments of a call, workspace and stream: the workspace has to lie with the cache, and the cache on the current
    device, a GPU."""
    dev = cache._device
    if dev < 0 or dev != (torch.cuda.current_device() if _device is None else _device()) or (
            ws is not None and (ws.dtype is not torch.uint8 or ws.get_device() != dev or not ws.is_contiguous())):
        raise KVError(fn, KV_ERR_INVALID_ARG)
    handle = _raw_stream(dev) if stream is None and _raw_stream is not None else _stream(stream)
    return (None, 0, handle) if ws is None else (ws.data_ptr(), ws.numel(), handle)


def kv_q4_reserve(cache: KvQ4Cache, add, new_pos, ws, granted=None, init="mean", stream=None):
    """add, new_pos, granted: [batch] int32 (new_pos and granted nullable); init: "mean", "min" or "zero"."""
    n, dev = cache._batch, cache._device
    if not (_q4_ok(add, torch.int32, n, dev) and _q4_ok(new_pos, torch.int32, n, dev) and _q4_ok(granted, torch.int32, n, dev)):
        raise KVError("kv_q4_reserve", KV_ERR_INVALID_ARG)
    mode = {"mean": KV_INIT_MEAN, "min": KV_INIT_MIN, "zero": KV_INIT_ZERO}.get(init, -1) if isinstance(init, str) else int(init)
    tail = _q4_tail("kv_q4_reserve", cache, ws, stream)
    _check("kv_q4_reserve", load_library().kv_q4_reserve(cache._shape, cache._buffers, _ptr(add), _ptr(new_pos), mode,
                                                         _ptr(granted), *tail))


def _q4_rows(fn, cache, layer0, layer_count, rows, k, v, ws, first, count, stream):
    # (a decode step's rows are bound by the host: 7.3 us a call with a helper per tensor, 6.7 so, of which the kernel is 3.5)
    n, heads, dev, element = cache._batch, cache._heads, cache._device, cache.element
    shape = (layer_count, n, heads, rows, cache._dim)
    ks, vs = k.stride(), v.stride()
    if not (k.shape == shape and v.shape == shape and k.dtype is element and v.dtype is element and ks[4] == 1 and vs[4] == 1
            and k.get_device() == dev and v.get_device() == dev
            and (first is None or _q4_ok(first, torch.int32, n, dev)) and (count is None or _q4_ok(count, torch.int32, n, dev))):
        raise KVError(fn, KV_ERR_INVALID_ARG)
    tail = _q4_tail(fn, cache, ws, stream)
    # (the stride of an extent of 1 is not used, and may be anything)
    ln, bn, hn, rn = layer_count > 1, n > 1, heads > 1, rows > 1
    k_strides = KvQ4Strides(ks[0] * ln, ks[1] * bn, ks[2] * hn, ks[3] * rn)
    v_strides = k_strides if ks == vs else KvQ4Strides(vs[0] * ln, vs[1] * bn, vs[2] * hn, vs[3] * rn)
    _check(fn, getattr(load_library(), fn)(cache._shape, cache._buffers, layer0, layer_count, rows, _ptr(first), _ptr(count),
                                           k.data_ptr(), k_strides, v.data_ptr(), v_strides, *tail))


def kv_q4_store(cache: KvQ4Cache, layer0, layer_count, rows, k, v, ws, first=None, count=None, stream=None):
    """k, v: [layer_count][batch][n_kv_heads][rows][head_dim] in any strides with contiguous rows; first, count: [batch]."""
    _q4_rows("kv_q4_store", cache, layer0, layer_count, rows, k, v, ws, first, count, stream)


def kv_q4_load(cache: KvQ4Cache, layer0, layer_count, rows, k, v, ws, first=None, count=None, stream=None):
    """As kv_q4_store, into k and v."""
    _q4_rows("kv_q4_load", cache, layer0, layer_count, rows, k, v, ws, first, count, stream)


def make_rotary(inv_freq, axis=None, pairs="halves", scale=1.0, axes=None) -> KvRotary:
    """inv_freq: the pairs' angles per position, dim / 2 numbers (held as float32); axis: each pair's axis (all 0 without);
    pairs: "halves" (elements i and i + dim / 2) or "adjacent" (2 i and 2 i + 1); axes: how many there are (the largest + 1)."""
    inv_freq = [float(x) for x in inv_freq]
    axis = [0] * len(inv_freq) if axis is None else [int(x) for x in axis]
    if not 0 < len(inv_freq) <= 64 or len(axis) != len(inv_freq) or not all(0 <= x < 256 for x in axis) or pairs not in ("halves", "adjacent"):
        raise KVError("make_rotary", KV_ERR_INVALID_ARG)
    r = KvRotary(2 * len(inv_freq), int(pairs == "adjacent"), max(axis) + 1 if axes is None else int(axes), float(scale))
    r.inv_freq[: len(inv_freq)] = inv_freq
    r.axis[: len(axis)] = axis
    return r


def _q4_spread(cache, layer_count, heads, rows, a, b):
    """Strides of two tensors [layer_count][batch][heads][rows][head_dim] of the cache's type and place, whose rows are contiguous; None
    where one is not so.  (The stride of an extent of 1 is not used, and may be anything.)"""
    shape, dev, element = (layer_count, cache._batch, heads, rows, cache._dim), cache._device, cache.element
    s, t = a.stride(), b.stride()
    if not (a.shape == shape and b.shape == shape and a.dtype is element and b.dtype is element and s[4] == 1 and t[4] == 1
            and a.get_device() == dev and b.get_device() == dev):
        return None
    ln, bn, hn, rn = layer_count > 1, cache._batch > 1, heads > 1, rows > 1
    first = KvQ4Strides(s[0] * ln, s[1] * bn, s[2] * hn, s[3] * rn)
    return first, first if s == t else KvQ4Strides(t[0] * ln, t[1] * bn, t[2] * hn, t[3] * rn)


def kv_q4_store_rotary(cache: KvQ4Cache, layer0, layer_count, rows, k, v, rotary: KvRotary, positions, ws, first=None, count=None,
                       q=None, q_out=None, stream=None):
    """k, v, first, count as kv_q4_store; positions: [axes][batch][rows] int32, contiguous; q, q_out: [layer_count][batch]
    [n_q_heads][rows][head_dim] in any strides with contiguous rows (q_out may be q)."""
    n, dev = cache._batch, cache._device
    kv = _q4_spread(cache, layer_count, cache._heads, rows, k, v)
    qs = (None, None) if q is None or q_out is None else _q4_spread(cache, layer_count, cache._query[1], rows, q, q_out)
    if (kv is None or qs is None or (q is None) != (q_out is None) or not _q4_ok(positions, torch.int32, rotary.axes * n * rows, dev)
            or (first is not None and not _q4_ok(first, torch.int32, n, dev)) or (count is not None and not _q4_ok(count, torch.int32, n, dev))):
        raise KVError("kv_q4_store_rotary", KV_ERR_INVALID_ARG)
    tail = _q4_tail("kv_q4_store_rotary", cache, ws, stream)
    _check("kv_q4_store_rotary", load_library().kv_q4_store_rotary(
        cache._shape, cache._buffers, layer0, layer_count, rows, _ptr(first), _ptr(count), rotary, _ptr(positions), k.data_ptr(), kv[0],
        v.data_ptr(), kv[1], _ptr(q), qs[0], _ptr(q_out), qs[1], *tail))


def kv_q4_attend(cache: KvQ4Cache, layer0, layer_count, n_max, q, o, ws, cur_pos=None, recency_bias=0.0, recency_window=0,
                 s_out=None, alpha=0.0, u_prior=None, u_out=None, stream=None):
    """q, o: [layer_count][batch][n_q_heads][head_dim] (of more layers: the first ones; of one layer, its dimension may be left
    out); cur_pos: [batch] int32; s_out: [layer_count][batch][n_max] f32; u_prior, u_out: [batch][capacity] f32."""
    n, dev, f32 = cache._batch, cache._device, torch.float32
    if not (_q4_heads(cache, q, layer_count) and _q4_heads(cache, o, layer_count) and _q4_ok(cur_pos, torch.int32, n, dev)
            and _q4_ok(s_out, f32, layer_count * n * n_max, dev) and _q4_ok(u_prior, f32, cache._rows, dev)
            and _q4_ok(u_out, f32, cache._rows, dev)):
        raise KVError("kv_q4_attend", KV_ERR_INVALID_ARG)
    tail = _q4_tail("kv_q4_attend", cache, ws, stream)
    _check("kv_q4_attend", load_library().kv_q4_attend(
        cache._shape, cache._buffers, layer0, layer_count, n_max, _ptr(q), _ptr(cur_pos), recency_bias, recency_window, _ptr(o),
        _ptr(s_out), alpha, _ptr(u_prior), _ptr(u_out), *tail))


def kv_q4_window_workspace_bytes(shape: KvQ4Shape, n_max: int, rows: int, layer_count: int) -> int:
    out = ctypes.c_size_t(0)
    _check("kv_q4_window_workspace_bytes", load_library().kv_q4_window_workspace_bytes(
        ctypes.byref(shape), int(n_max), int(rows), int(layer_count), ctypes.byref(out)))
    return out.value


def kv_q4_shared_workspace_bytes(shape: KvQ4Shape, n_max: int, layer_count: int) -> int:
    out = ctypes.c_size_t(0)
    _check("kv_q4_shared_workspace_bytes", load_library().kv_q4_shared_workspace_bytes(
        ctypes.byref(shape), int(n_max), int(layer_count), ctypes.byref(out)))
    return out.value


def q4_window_workspace(shape: KvQ4Shape, n_max: int, rows: int, layer_count: int, device="cuda") -> torch.Tensor:
    """A caller-owned workspace tensor of kv_q4_window_workspace_bytes() bytes, its fault word cleared on the current stream."""
    ws = torch.empty(kv_q4_window_workspace_bytes(shape, n_max, rows, layer_count), dtype=torch.uint8, device=device)
    kv_fault_status(ws, None, clear=True)
    return ws


def q4_shared_workspace(shape: KvQ4Shape, n_max: int, layer_count: int, device="cuda") -> torch.Tensor:
    """As q4_window_workspace, for kv_q4_attend_shared."""
    ws = torch.empty(kv_q4_shared_workspace_bytes(shape, n_max, layer_count), dtype=torch.uint8, device=device)
    kv_fault_status(ws, None, clear=True)
    return ws


def kv_q4_attend_window(cache: KvQ4Cache, layer0, layer_count, n_max, rows, q, o, ws, window=0, sinks=0, count=None, stream=None):
    """q, o: [layer_count][batch][n_q_heads][rows][head_dim] in any strides with contiguous rows; count: [batch] int32."""
    strides = _q4_spread(cache, layer_count, cache._query[1], rows, q, o)
    if strides is None or not _q4_ok(count, torch.int32, cache._batch, cache._device):
        raise KVError("kv_q4_attend_window", KV_ERR_INVALID_ARG)
    tail = _q4_tail("kv_q4_attend_window", cache, ws, stream)
    _check("kv_q4_attend_window", load_library().kv_q4_attend_window(
        cache._shape, cache._buffers, layer0, layer_count, n_max, rows, _ptr(count), q.data_ptr(), strides[0], window, sinks,
        o.data_ptr(), strides[1], *tail))


def kv_q4_attend_shared(cache: KvQ4Cache, layer0, layer_count, n_max, group, q, o, ws, stream=None):
    """q, o as kv_q4_attend; group: [batch] int32, equal for slots that share pages."""
    if not (_q4_heads(cache, q, layer_count) and _q4_heads(cache, o, layer_count) and _q4_ok(group, torch.int32, cache._batch, cache._device)):
        raise KVError("kv_q4_attend_shared", KV_ERR_INVALID_ARG)
    tail = _q4_tail("kv_q4_attend_shared", cache, ws, stream)
    _check("kv_q4_attend_shared", load_library().kv_q4_attend_shared(cache._shape, cache._buffers, layer0, layer_count, n_max, _ptr(group),
                                                                     _ptr(q), _ptr(o), *tail))


def kv_q4_fork(cache: KvQ4Cache, src, dst, ws, stream=None):
    """src, dst: int32 tensors of the same size (at most batch)."""
    n = src.numel()
    if dst.numel() != n or not (_q4_ok(src, torch.int32, n, cache._device) and _q4_ok(dst, torch.int32, n, cache._device)):
        raise KVError("kv_q4_fork", KV_ERR_INVALID_ARG)
    tail = _q4_tail("kv_q4_fork", cache, ws, stream)
    _check("kv_q4_fork", load_library().kv_q4_fork(cache._shape, cache._buffers, n, _ptr(src), _ptr(dst), *tail))


def kv_q4_free(cache: KvQ4Cache, slots, ws, stream=None):
    """slots: int32 tensor of at most batch entries."""
    if not _q4_ok(slots, torch.int32, 0, cache._device):
        raise KVError("kv_q4_free", KV_ERR_INVALID_ARG)
    tail = _q4_tail("kv_q4_free", cache, ws, stream)
    _check("kv_q4_free", load_library().kv_q4_free(cache._shape, cache._buffers, slots.numel(), _ptr(slots), *tail))


def kv_q4_compact(cache: KvQ4Cache, n_max, keep, ws, stream=None):
    """keep: [batch][capacity] uint8."""
    if not _q4_ok(keep, torch.uint8, cache._rows, cache._device):
        raise KVError("kv_q4_compact", KV_ERR_INVALID_ARG)
    tail = _q4_tail("kv_q4_compact", cache, ws, stream)
    _check("kv_q4_compact", load_library().kv_q4_compact(cache._shape, cache._buffers, n_max, _ptr(keep), *tail))


def kv_q4_evict(cache: KvQ4Cache, n_max, budget, ws, keep_out=None, stream=None):
    """budget: [batch] int32; keep_out: [batch][capacity] uint8."""
    dev = cache._device
    if not (_q4_ok(budget, torch.int32, cache._batch, dev) and _q4_ok(keep_out, torch.uint8, cache._rows, dev)):
        raise KVError("kv_q4_evict", KV_ERR_INVALID_ARG)
    tail = _q4_tail("kv_q4_evict", cache, ws, stream)
    _check("kv_q4_evict", load_library().kv_q4_evict(cache._shape, cache._buffers, n_max, _ptr(budget), _ptr(keep_out),
                                                     *tail))


# --- HIP events for the timing hooks (runtime plumbing, no computation) -------------------------------------
_hip = None


def _hip_runtime():
    global _hip
    if _hip is None:
        _hip = ctypes.CDLL("libamdhip64.so")
        _hip.hipEventCreate.argtypes = [ctypes.POINTER(ctypes.c_void_p)]
        _hip.hipEventCreateWithFlags.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_uint]
        _hip.hipEventDestroy.argtypes = [ctypes.c_void_p]
        _hip.hipEventSynchronize.argtypes = [ctypes.c_void_p]
        _hip.hipEventElapsedTime.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.c_void_p, ctypes.c_void_p]
        _hip.hipEventRecord.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    return _hip


HIP_EVENT_DISABLE_SYSTEM_FENCE = 0x20000000  # hipEventDisableSystemFence


class HipEvent:
    """A HIP event.  timing_only: created with hipEventDisableSystemFence, so recording it does not write back
    and invalidate the caches (a timestamp between kernels that leaves them undisturbed); read it only after
    the stream has been synchronized."""

    def __init__(self, timing_only: bool = False):
        self.handle = ctypes.c_void_p()
        if timing_only:
            rc = _hip_runtime().hipEventCreateWithFlags(ctypes.byref(self.handle), HIP_EVENT_DISABLE_SYSTEM_FENCE)
        else:
            rc = _hip_runtime().hipEventCreate(ctypes.byref(self.handle))
        if rc != 0:
            raise RuntimeError(f"hipEventCreate failed ({rc})")

    def record(self, stream=None):
        rc = _hip_runtime().hipEventRecord(self.handle, _stream(stream))
        if rc != 0:
            raise RuntimeError(f"hipEventRecord failed ({rc})")

    def elapsed_ms(self, later: "HipEvent") -> float:
        _hip_runtime().hipEventSynchronize(later.handle)
        out = ctypes.c_float(0)
        rc = _hip_runtime().hipEventElapsedTime(ctypes.byref(out), self.handle, later.handle)
        if rc != 0:
            raise RuntimeError(f"hipEventElapsedTime failed ({rc})")
        return out.value

    def __del__(self):
        if _hip is not None and self.handle:
            _hip.hipEventDestroy(self.handle)
            self.handle = ctypes.c_void_p()


def make_trace(pairs: dict) -> KvTrace:
    """pairs: phase name -> (begin HipEvent, end HipEvent)."""
    tr = KvTrace()
    for i, name in enumerate(PHASES):
        if name in pairs:
            tr.begin[i] = pairs[name][0].handle.value
            tr.end[i] = pairs[name][1].handle.value
    return tr
