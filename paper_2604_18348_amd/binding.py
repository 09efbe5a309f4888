"""ctypes binding of libadacluster.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/adacluster.h),
takes torch CUDA tensors, allocates the outputs with torch and passes raw device
pointers plus the current torch stream.  No step of the method runs in Python,
and there is no fallback: a missing library or a failing call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import operator
import struct
import threading
import warnings
from dataclasses import dataclass, replace

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("ADACLUSTER_LIB") or os.path.join(_HERE, "_lib", "libadacluster.so")
MAX_STAGES = 16

F32, BF16 = 0, 1
SCORE_TQ, SCORE_BOX, SCORE_DOT = 0, 1, 2
SELECT_TOPK, SELECT_TOPP = 0, 1


class CParams(ctypes.Structure):
    _fields_ = [("H", ctypes.c_int32), ("N", ctypes.c_int32), ("d", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("q_clusters", ctypes.c_int32),
                ("q_iters", ctypes.c_int32), ("k_iters", ctypes.c_int32),
                ("q_init_mode", ctypes.c_int32), ("k_init_mode", ctypes.c_int32), ("k_m0", ctypes.c_int32),
                ("k_m_min", ctypes.c_int32), ("k_max_clusters", ctypes.c_int32),
                ("k_max_stages", ctypes.c_int32), ("tau_abs", ctypes.c_float),
                ("tau_factor", ctypes.c_float), ("min_unassigned_frac", ctypes.c_float),
                ("score_mode", ctypes.c_int32), ("select_mode", ctypes.c_int32),
                ("topk", ctypes.c_int32), ("top_p", ctypes.c_float),
                ("softmax_scale", ctypes.c_float), ("q_no_norm", ctypes.c_int32)]


class COutputs(ctypes.Structure):
    _names = ["q_labels", "q_centroids", "q_assign_centroids", "q_sizes", "q_mean_norm",
              "k_labels", "k_centroids", "k_assign_centroids", "k_box_min", "k_box_max",
              "k_sizes", "k_count", "full_flag", "k_stage_offs", "k_stage_of", "tau_used",
              "sel_idx", "sel_cnt"]
    _fields_ = [(n, ctypes.c_void_p) for n in _names]


class CHeadStats(ctypes.Structure):
    _fields_ = [("k_count", ctypes.c_int32), ("full_flag", ctypes.c_int32), ("stages", ctypes.c_int32),
                ("q_tiles", ctypes.c_int32), ("unassigned", ctypes.c_int32 * (MAX_STAGES + 1)),
                ("reserved", ctypes.c_int32), ("executed_pairs", ctypes.c_int64), ("issued_pairs", ctypes.c_int64)]


class CBlockParams(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "d", "dtype", "bits", "page", "num_pages", "max_pages", "max_q", "qblock",
                                               "causal", "topk", "keep_first", "q_rows", "k_rows")]
                + [("softmax_scale", ctypes.c_float)]
                + [(n, ctypes.c_int64 * k) for n, k in (("q_stride", 2), ("o_stride", 2), ("k_stride", 3), ("v_stride", 3),
                                                        ("new_k_stride", 2), ("new_v_stride", 2), ("do_stride", 2), ("dq_stride", 2),
                                                        ("dk_stride", 2), ("dv_stride", 2))])


@dataclass
class Params:
    H: int
    N: int
    d: int
    dtype: int = BF16
    q_clusters: int = 65
    q_iters: int = 3
    k_iters: int = 3
    q_init_mode: int = 0
    k_init_mode: int = 0
    k_m0: int = 100
    k_m_min: int = 16
    k_max_clusters: int = 1024
    k_max_stages: int = 10
    tau_abs: float = 0.0
    tau_factor: float = 1.5
    min_unassigned_frac: float = 0.0
    score_mode: int = SCORE_TQ
    select_mode: int = SELECT_TOPK
    topk: int = 64
    top_p: float = 0.9
    softmax_scale: float = 0.0
    q_no_norm: int = 0

    def c(self) -> CParams:
        return CParams(*_param_values(self))      # (dataclasses.asdict copies every value on its way: 10 us)

    @property
    def cap(self) -> int:
        return self.k_max_clusters + self.k_m0


@dataclass
class BlockParams:
    """adacluster_block_params without what follows from the tensors of a call (pages of the pool, rows, strides)."""
    B: int
    Hq: int
    Hkv: int
    d: int
    dtype: int = BF16
    bits: int = 0
    page: int = 64
    max_pages: int = 1
    max_q: int = 1
    qblock: int = 1
    causal: int = 1
    topk: int = 0
    keep_first: int = 1
    softmax_scale: float = 0.0

    @property
    def blocks(self) -> int:
        return -(-self.max_q // max(1, self.qblock))


@dataclass
class BlockCache:
    """Tensors of a paged cache: k, v [num_pages,Hkv,page,d] of the params dtype in any strides, or with bits=4 the codes,
    uint8 [num_pages,Hkv,page,d/2], and k_meta, v_meta, bfloat16 [num_pages,Hkv,page,d/64,2], contiguous; boxes
    [num_pages,Hkv,2,d]."""
    k: torch.Tensor
    v: torch.Tensor
    k_meta: torch.Tensor = None
    v_meta: torch.Tensor = None
    boxes: torch.Tensor = None


_param_values = operator.attrgetter(*(name for name, _ in CParams._fields_))
_lib = None


def load_library():
    """Loads the shared library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2604_18348_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER(CParams)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.adacluster_centroid_capacity.argtypes = [P]
    lib.adacluster_workspace_bytes.argtypes = [P, ctypes.POINTER(sz)]
    lib.adacluster_last_error.argtypes = [ctypes.c_char_p, sz]
    lib.adacluster_qcluster.argtypes = [P] + [vp] * 6 + [vp, sz, vp]
    lib.adacluster_kcluster.argtypes = [P] + [vp] * 12 + [vp, sz, vp]
    lib.adacluster_select.argtypes = [P] + [vp] * 10 + [vp, sz, vp]
    lib.adacluster_sparse_attn.argtypes = [P] + [vp] * 9 + [vp, sz, vp]
    lib.adacluster_attn.argtypes = [P] + [vp] * 4 + [ctypes.POINTER(COutputs), vp, sz, vp]
    lib.adacluster_dense_attn.argtypes = [P] + [vp] * 4 + [vp, sz, vp]
    lib.adacluster_compactness.argtypes = [P] + [vp] * 4 + [vp, sz, vp]
    lib.adacluster_compactness_noalloc.argtypes = [P] + [vp] * 4 + [vp]
    lib.adacluster_mfma_probe.argtypes = [ctypes.c_int32, vp, sz, ctypes.POINTER(ctypes.c_double), vp]
    lib.adacluster_stats_fetch.argtypes = [P, vp, sz, ctypes.POINTER(CHeadStats), vp]
    lib.adacluster_quest_scores.argtypes = [ctypes.c_int32] * 7 + [vp] * 5
    BP = vp                                            # (the bytes of a CBlockParams, or a pointer to one)
    lib.adacluster_block_workspace_bytes.argtypes = [BP, ctypes.c_int32, ctypes.POINTER(sz)]
    lib.adacluster_cache_append.argtypes = [BP] + [vp] * 11
    lib.adacluster_cache_read.argtypes = [BP] + [vp] * 10
    lib.adacluster_block_boxes.argtypes = [BP] + [vp] * 4
    lib.adacluster_block_select.argtypes = [BP] + [vp] * 9 + [sz, vp]
    lib.adacluster_block_attn.argtypes = [BP] + [vp] * 13 + [sz, vp]
    lib.adacluster_block_attn_backward.argtypes = [BP] + [vp] * 13 + [sz, vp]
    lib.adacluster_prefix_workspace_bytes.argtypes = [BP, ctypes.c_int32, ctypes.POINTER(sz)]
    lib.adacluster_prefix_attn.argtypes = [BP, ctypes.c_int32] + [vp] * 13 + [sz, vp]
    lib.adacluster_weights_workspace_bytes.argtypes = [BP, ctypes.POINTER(sz)]
    lib.adacluster_cache_weights.argtypes = [BP] + [vp] * 8 + [ctypes.c_float, vp, vp, sz, vp]
    lib.adacluster_cache_evict.argtypes = [BP] + [vp] * 3 + [ctypes.c_int32] * 2 + [vp] * 10
    lib.adacluster_profile_enable.argtypes = [ctypes.c_int]
    lib.adacluster_profile_read.argtypes = [ctypes.POINTER(ctypes.c_float)]
    for n in ("profile_enable", "profile_read", "centroid_capacity", "workspace_bytes", "last_error", "qcluster", "kcluster", "select",
              "sparse_attn", "attn", "dense_attn", "compactness", "compactness_noalloc", "quest_scores", "stats_fetch", "mfma_probe",
              "block_workspace_bytes", "cache_append", "cache_read", "block_boxes", "block_select", "block_attn", "block_attn_backward",
              "prefix_workspace_bytes", "prefix_attn", "weights_workspace_bytes", "cache_weights", "cache_evict"):
        getattr(lib, "adacluster_" + n).restype = ctypes.c_int
    _lib = lib
    return lib


EXPORTED = ["adacluster_centroid_capacity", "adacluster_workspace_bytes", "adacluster_last_error",
            "adacluster_qcluster", "adacluster_kcluster", "adacluster_select",
            "adacluster_sparse_attn", "adacluster_attn", "adacluster_dense_attn", "adacluster_compactness",
            "adacluster_compactness_noalloc", "adacluster_quest_scores", "adacluster_stats_fetch", "adacluster_mfma_probe",
            "adacluster_block_workspace_bytes", "adacluster_cache_append", "adacluster_cache_read", "adacluster_block_boxes",
            "adacluster_block_select", "adacluster_block_attn", "adacluster_block_attn_backward",
            "adacluster_prefix_workspace_bytes", "adacluster_prefix_attn", "adacluster_weights_workspace_bytes",
            "adacluster_cache_weights", "adacluster_cache_evict",
            "adacluster_profile_enable", "adacluster_profile_read"]

STAGES = ["qcluster", "kcluster", "select", "permute", "plan", "attention", "kreduce"]


def adacluster_profile_enable(on: bool):
    _check(load_library().adacluster_profile_enable(1 if on else 0), "profile_enable")


def adacluster_profile_read():
    """Stage times (ms) of the last profiled call as a dict; stages that did not run are absent."""
    arr = (ctypes.c_float * len(STAGES))()
    _check(load_library().adacluster_profile_read(arr), "profile_read")
    return {n: float(arr[i]) for i, n in enumerate(STAGES) if arr[i] >= 0}


class AdaClusterError(RuntimeError):
    pass


def _check(rc, what):
    if rc != 0:
        buf = ctypes.create_string_buffer(256)
        load_library().adacluster_last_error(buf, 256)
        raise AdaClusterError(f"{what} failed with code {rc}: {buf.value.decode()}")


def _ptr(t):
    return None if t is None else t.data_ptr()      # (the argument types make it a pointer)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _tdtype(p: Params):
    return torch.bfloat16 if p.dtype == BF16 else torch.float32


def _check_qkv(p: Params, *ts):
    for t in ts:
        if not (t.is_cuda and t.is_contiguous() and t.dtype == _tdtype(p) and t.shape == (p.H, p.N, p.d)):
            raise ValueError("tensor must be a contiguous CUDA tensor [H,N,d] of the params dtype")


def adacluster_workspace_bytes(p: Params) -> int:
    out = ctypes.c_size_t(0)
    cp = p.c()
    _check(load_library().adacluster_workspace_bytes(ctypes.byref(cp), ctypes.byref(out)), "workspace_bytes")
    return out.value


_ws_cache = threading.local()      # .of: {(device, stream): (size, tensor)}


def workspace(p: Params, device="cuda"):
    """A torch uint8 workspace of the required size for calls on the current stream: kept from call to call, for every host thread, device
    and stream by itself (calls of two threads or streams at once must not share scratch), until one of another size is asked for there.
    While the stream is being captured it is a tensor of its own instead, which torch takes from the graph's pool and which therefore lives as
    long as the graph.  Whoever captures without torch, or goes on with it on another stream, holds a workspace and passes it as `ws`."""
    n = adacluster_workspace_bytes(p)
    device, at = torch.device(device), "host"
    if device.type == "cuda":
        i = torch.cuda.current_device() if device.index is None else device.index
        device, at = torch.device("cuda", i), (i, _raw_stream(i))
    if at != "host" and torch.cuda.is_current_stream_capturing():
        t = torch.empty(n + 256, dtype=torch.uint8, device=device)
    else:
        kept = _ws_cache.__dict__.setdefault("of", {})
        if at not in kept or kept[at][0] != n:
            kept.pop(at, None)                           # (the old one goes before the new one comes)
            kept[at] = n, torch.empty(n + 256, dtype=torch.uint8, device=device)
        t = kept[at][1]
    off = (-t.data_ptr()) % 256
    return t[off:off + n]


def adacluster_qcluster(p: Params, Q, q_centroids_init=None, ws=None):
    _check_qkv(p, Q)
    dev = Q.device
    ws = workspace(p, dev) if ws is None else ws
    i32, f32 = torch.int32, torch.float32
    out = dict(
        q_labels=torch.empty((p.H, p.N), dtype=i32, device=dev),
        q_centroids=(q_centroids_init.clone() if q_centroids_init is not None
                     else torch.empty((p.H, p.q_clusters, p.d), dtype=f32, device=dev)),
        q_assign_centroids=torch.empty((p.H, p.q_clusters, p.d), dtype=f32, device=dev),
        q_sizes=torch.empty((p.H, p.q_clusters), dtype=i32, device=dev),
        q_mean_norm=torch.empty((p.H, p.q_clusters), dtype=f32, device=dev))
    cp = p.c()
    _check(load_library().adacluster_qcluster(
        ctypes.byref(cp), _ptr(Q), _ptr(out["q_labels"]), _ptr(out["q_centroids"]),
        _ptr(out["q_assign_centroids"]), _ptr(out["q_sizes"]), _ptr(out["q_mean_norm"]),
        _ptr(ws), ws.numel(), _stream()), "adacluster_qcluster")
    return out


def adacluster_kcluster(p: Params, K, want_box=True, ws=None, prev=None):
    """`prev` (warm start, k_init_mode 1): dict with k_centroids, k_count, full_flag of an earlier call."""
    _check_qkv(p, K)
    dev = K.device
    ws = workspace(p, dev) if ws is None else ws
    i32, f32 = torch.int32, torch.float32
    cap = p.cap
    out = dict(
        k_labels=torch.empty((p.H, p.N), dtype=i32, device=dev),
        k_centroids=torch.zeros((p.H, cap, p.d), dtype=f32, device=dev),
        k_assign_centroids=torch.zeros((p.H, cap, p.d), dtype=f32, device=dev),
        k_box_min=torch.zeros((p.H, cap, p.d), dtype=f32, device=dev) if want_box else None,
        k_box_max=torch.zeros((p.H, cap, p.d), dtype=f32, device=dev) if want_box else None,
        k_sizes=torch.empty((p.H, cap), dtype=i32, device=dev),
        k_count=torch.empty((p.H,), dtype=i32, device=dev),
        full_flag=torch.empty((p.H,), dtype=i32, device=dev),
        k_stage_offs=torch.empty((p.H, MAX_STAGES + 1), dtype=i32, device=dev),
        k_stage_of=torch.empty((p.H, p.N), dtype=i32, device=dev),
        tau_used=torch.zeros((1,), dtype=f32, device=dev))
    if prev is not None:
        out["k_centroids"] = prev["k_centroids"].clone()
        out["k_count"] = prev["k_count"].clone()
        out["full_flag"] = prev["full_flag"].clone()
    cp = p.c()
    _check(load_library().adacluster_kcluster(
        ctypes.byref(cp), _ptr(K), _ptr(out["k_labels"]), _ptr(out["k_centroids"]),
        _ptr(out["k_assign_centroids"]), _ptr(out["k_box_min"]), _ptr(out["k_box_max"]),
        _ptr(out["k_sizes"]), _ptr(out["k_count"]), _ptr(out["full_flag"]), _ptr(out["k_stage_offs"]),
        _ptr(out["k_stage_of"]), _ptr(out["tau_used"]), _ptr(ws), ws.numel(), _stream()),
        "adacluster_kcluster")
    return out


def adacluster_select(p: Params, q_centroids, q_mean_norm, k_centroids, k_box_min, k_box_max, k_sizes,
                      k_count, full_flag, ws=None):
    dev = q_centroids.device
    ws = workspace(p, dev) if ws is None else ws
    sel_idx = torch.empty((p.H, p.q_clusters, p.cap), dtype=torch.int32, device=dev)
    sel_cnt = torch.empty((p.H, p.q_clusters), dtype=torch.int32, device=dev)
    cp = p.c()
    _check(load_library().adacluster_select(
        ctypes.byref(cp), _ptr(q_centroids), _ptr(q_mean_norm), _ptr(k_centroids), _ptr(k_box_min),
        _ptr(k_box_max), _ptr(k_sizes), _ptr(k_count), _ptr(full_flag), _ptr(sel_idx), _ptr(sel_cnt),
        _ptr(ws), ws.numel(), _stream()), "adacluster_select")
    return sel_idx, sel_cnt


def adacluster_sparse_attn(p: Params, Q, K, V, q_labels, k_labels, k_count, sel_idx, sel_cnt, out=None, ws=None):
    _check_qkv(p, Q, K, V)
    ws = workspace(p, Q.device) if ws is None else ws
    O = torch.empty_like(Q) if out is None else out
    cp = p.c()
    _check(load_library().adacluster_sparse_attn(
        ctypes.byref(cp), _ptr(Q), _ptr(K), _ptr(V), _ptr(q_labels), _ptr(k_labels), _ptr(k_count),
        _ptr(sel_idx), _ptr(sel_cnt), _ptr(O), _ptr(ws), ws.numel(), _stream()), "adacluster_sparse_attn")
    return O


def adacluster_compactness(p: Params, K, k_labels, k_centroids, ws=None):
    """Per-head mean squared reconstruction error of a key clustering (Sec. 3.2.1) -> float32 [H]."""
    ws = workspace(p, K.device) if ws is None else ws
    mse = torch.empty((p.H,), dtype=torch.float32, device=K.device)
    cp = p.c()
    _check(load_library().adacluster_compactness(
        ctypes.byref(cp), _ptr(K), _ptr(k_labels), _ptr(k_centroids), _ptr(mse), _ptr(ws), ws.numel(), _stream()),
        "adacluster_compactness")
    return mse


def adacluster_compactness_noalloc(p: Params, K, k_labels, k_centroids, out=None):
    """adacluster_compactness without a workspace: partial sums in the library's own device array.  `out`
    lets the caller pass the [H] float32 result tensor, so that the call itself allocates nothing."""
    mse = torch.empty((p.H,), dtype=torch.float32, device=K.device) if out is None else out
    cp = p.c()
    _check(load_library().adacluster_compactness_noalloc(
        ctypes.byref(cp), _ptr(K), _ptr(k_labels), _ptr(k_centroids), _ptr(mse), _stream()),
        "adacluster_compactness_noalloc")
    return mse


def adacluster_stats_fetch(p: Params, ws):
    """Per-head figures of the last adacluster_attn call on `ws` -> list of dicts (waits for the stream)."""
    arr = (CHeadStats * p.H)()
    cp = p.c()
    _check(load_library().adacluster_stats_fetch(ctypes.byref(cp), _ptr(ws), ws.numel(), arr, _stream()),
           "adacluster_stats_fetch")
    return [dict(k_count=r.k_count, full_flag=r.full_flag, stages=r.stages, q_tiles=r.q_tiles,
                 unassigned=list(r.unassigned), executed_pairs=r.executed_pairs, issued_pairs=r.issued_pairs)
            for r in arr]


def adacluster_mfma_probe(iters: int, sink):
    """Enqueues the register-only MFMA loop on the current stream; returns the flops of the launch."""
    fl = ctypes.c_double(0.0)
    _check(load_library().adacluster_mfma_probe(int(iters), _ptr(sink), sink.numel(), ctypes.byref(fl), _stream()),
           "adacluster_mfma_probe")
    return fl.value


QUEST_ALU, QUEST_MFMA = 0, 1


def adacluster_quest_scores(Q, R_pos, R_neg, form, clamp=False, out=None):
    """Quest scores (Eq. 1 / Eq. 2) of query rows Q [H,Lq,d] against pages with maxima R_pos and minima
    R_neg [H,Lk,d] -> float32 [H,Lq,Lk]."""
    H, Lq, d = Q.shape
    Lk = R_pos.shape[1]
    assert R_pos.shape == (H, Lk, d) and R_neg.shape == (H, Lk, d)
    assert Q.dtype == R_pos.dtype == R_neg.dtype and Q.dtype in (torch.float32, torch.bfloat16)
    assert Q.is_contiguous() and R_pos.is_contiguous() and R_neg.is_contiguous()
    S = torch.empty((H, Lq, Lk), dtype=torch.float32, device=Q.device) if out is None else out
    _check(load_library().adacluster_quest_scores(
        H, Lq, Lk, d, BF16 if Q.dtype == torch.bfloat16 else F32, int(form), 1 if clamp else 0,
        _ptr(Q), _ptr(R_pos), _ptr(R_neg), _ptr(S), _stream()), "adacluster_quest_scores")
    return S


def alloc_outputs(p: Params, dev, want_box=False, want_stage=True):
    """Device tensors for every intermediate of the fused call."""
    i32, f32 = torch.int32, torch.float32
    cap = p.cap
    o = dict(
        q_labels=torch.empty((p.H, p.N), dtype=i32, device=dev),
        q_centroids=torch.empty((p.H, p.q_clusters, p.d), dtype=f32, device=dev),
        q_assign_centroids=torch.empty((p.H, p.q_clusters, p.d), dtype=f32, device=dev),
        q_sizes=torch.empty((p.H, p.q_clusters), dtype=i32, device=dev),
        q_mean_norm=torch.empty((p.H, p.q_clusters), dtype=f32, device=dev),
        k_labels=torch.empty((p.H, p.N), dtype=i32, device=dev),
        k_centroids=torch.zeros((p.H, cap, p.d), dtype=f32, device=dev),
        k_assign_centroids=torch.zeros((p.H, cap, p.d), dtype=f32, device=dev),
        k_box_min=torch.zeros((p.H, cap, p.d), dtype=f32, device=dev) if want_box else None,
        k_box_max=torch.zeros((p.H, cap, p.d), dtype=f32, device=dev) if want_box else None,
        k_sizes=torch.empty((p.H, cap), dtype=i32, device=dev),
        k_count=torch.empty((p.H,), dtype=i32, device=dev),
        full_flag=torch.empty((p.H,), dtype=i32, device=dev),
        k_stage_offs=torch.empty((p.H, MAX_STAGES + 1), dtype=i32, device=dev) if want_stage else None,
        k_stage_of=torch.empty((p.H, p.N), dtype=i32, device=dev) if want_stage else None,
        tau_used=torch.empty((1,), dtype=f32, device=dev),
        sel_idx=torch.empty((p.H, p.q_clusters, cap), dtype=i32, device=dev),
        sel_cnt=torch.empty((p.H, p.q_clusters), dtype=i32, device=dev))
    return o


def adacluster_attn(p: Params, Q, K, V, outs=None, out=None, ws=None):
    """Fused call.  `outs`: dict from alloc_outputs (or None to keep intermediates in the workspace)."""
    _check_qkv(p, Q, K, V)
    ws = workspace(p, Q.device) if ws is None else ws
    O = torch.empty_like(Q) if out is None else out
    co = None
    if outs is not None:
        co = COutputs(*[_ptr(outs.get(n)) for n in COutputs._names])
    cp = p.c()
    _check(load_library().adacluster_attn(
        ctypes.byref(cp), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), ctypes.byref(co) if co is not None else None,
        _ptr(ws), ws.numel(), _stream()), "adacluster_attn")
    return O


def adacluster_dense_attn(p: Params, Q, K, V, out=None, ws=None):
    _check_qkv(p, Q, K, V)
    ws = workspace(p, Q.device) if ws is None else ws
    O = torch.empty_like(Q) if out is None else out
    cp = p.c()
    _check(load_library().adacluster_dense_attn(
        ctypes.byref(cp), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(ws), ws.numel(), _stream()),
        "adacluster_dense_attn")
    return O


# ---- attention over pages of keys ---------------------------------------------------------------------------------------

BLOCK_SELECT, BLOCK_ATTN, BLOCK_BACKWARD = 0, 1, 2
_block_values = operator.attrgetter("B", "Hq", "Hkv", "d", "dtype", "bits", "page")
_block_more = operator.attrgetter("max_pages", "max_q", "qblock", "causal", "topk", "keep_first")
_block_pack = struct.Struct("@16if22q").pack      # CBlockParams; a token's step of generation is a few calls of 20 us, of which ctypes.Structure would be 5
_NO2, _NO3 = (0, 0), (0, 0, 0)


def _block_c(p: BlockParams, q_rows, k_rows=0, num_pages=0, q=_NO2, o=_NO2, k=_NO3, v=_NO3, new_k=_NO2, new_v=_NO2, d_o=_NO2, dq=_NO2, dk=_NO2,
             dv=_NO2) -> bytes:
    """adacluster_block_params as bytes; the rest are the strides."""
    return _block_pack(*_block_values(p), num_pages, *_block_more(p), q_rows, k_rows, p.softmax_scale, *q, *o, *k, *v, *new_k, *new_v, *d_o, *dq,
                       *dk, *dv)


def _rows(name, t, dtype, heads, d, device):
    """A [rows, heads, d] tensor with d contiguous; its strides of rows and heads."""
    s = t.shape
    if len(s) != 3 or s[1] != heads or s[2] != d or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be a [rows, {heads}, {d}] tensor of {dtype} on {device}")
    a, b, c = t.stride()
    if c != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return a, b


def _gpu(t):
    if not t.is_cuda:
        raise ValueError("tensors must be on a GPU: %s must be a CUDA tensor" % type(t).__name__)
    return t.device


def _ints(name, t, shape, device):
    if t.shape != shape or t.dtype != torch.int32 or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {tuple(shape)} on {device}")


def _pool(p: BlockParams, cache: BlockCache, device, boxes):
    """Checks a cache; its number of pages and the strides of k and v (page, token, head)."""
    ck, cv, Hkv, page, d = cache.k, cache.v, p.Hkv, p.page, p.d
    n = ck.shape[0]
    if boxes:
        _boxes(cache.boxes, (n, Hkv, 2, d), p, device)
    if p.bits == 4:
        for name, t, shape, dt in (("k", ck, (n, Hkv, page, d // 2), torch.uint8), ("v", cv, (n, Hkv, page, d // 2), torch.uint8),
                                   ("k_meta", cache.k_meta, (n, Hkv, page, d // 64, 2), torch.bfloat16),
                                   ("v_meta", cache.v_meta, (n, Hkv, page, d // 64, 2), torch.bfloat16)):
            if t is None or t.shape != shape or t.dtype != dt or not t.is_contiguous() or t.device != device:
                raise ValueError(f"cache.{name} must be a contiguous {dt} tensor {shape} on {device}")
        return n, _NO3, _NO3
    shape, dt = (n, Hkv, page, d), _tdtype(p)
    out = [n]
    for name, t in (("k", ck), ("v", cv)):
        a, b, c, e = t.stride() if t.dim() == 4 else (0, 0, 0, 0)
        if t.shape != shape or t.dtype != dt or e != 1 or t.device != device:
            raise ValueError(f"cache.{name} must be a {dt} tensor {shape} on {device}, its last dimension contiguous")
        out.append((a, c, b))
    return out


def _boxes(t, shape, p, device):
    if t is None or t.shape != shape or t.dtype != _tdtype(p) or not t.is_contiguous() or t.device != device:
        raise ValueError(f"boxes must be a contiguous {_tdtype(p)} tensor {tuple(shape)} on {device}")


@functools.lru_cache(maxsize=1024)
def _block_bytes(cp: bytes, call):
    """Workspace of a call: it follows from the parameters alone."""
    n = ctypes.c_size_t(0)
    _check(load_library().adacluster_block_workspace_bytes(cp, call, ctypes.byref(n)), "block_workspace_bytes")
    return n.value


def _block_ws(cp, call, device, ws):
    if ws is None:
        # a tensor of its own for every call: torch hands memory out by stream, and to a captured graph from that graph's pool
        n = _block_bytes(cp, call)
        return (torch.empty(n, dtype=torch.uint8, device=device), n) if n else (None, 0)
    if ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.device != device:
        raise ValueError(f"ws must be a contiguous uint8 tensor on {device}")
    return ws, ws.numel()


def _on(device, name, *args):
    """Calls an entry point on the current stream of the device that owns the tensors, which has to be the current one for a launch."""
    i = device.index
    fn = getattr(load_library(), name)
    if i == torch.cuda.current_device():
        rc = fn(*args, _raw_stream(i))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _raw_stream(i))
    if rc:
        _check(rc, name)


def _raw_stream(i):
    return torch._C._cuda_getCurrentRawStream(i)      # (torch.cuda.current_stream(i).cuda_stream makes an object on the way: 2 us)


def alloc_cache(p: BlockParams, num_pages, device="cuda"):
    """A BlockCache of num_pages empty pages."""
    z = lambda *s, dt: torch.zeros(s, dtype=dt, device=device)  # noqa: E731
    n, dt = num_pages, _tdtype(p)
    boxes = z(n, p.Hkv, 2, p.d, dt=dt)
    if p.bits == 4:
        codes = lambda: z(n, p.Hkv, p.page, p.d // 2, dt=torch.uint8)  # noqa: E731
        meta = lambda: z(n, p.Hkv, p.page, p.d // 64, 2, dt=torch.bfloat16)  # noqa: E731
        return BlockCache(codes(), codes(), meta(), meta(), boxes)
    return BlockCache(z(n, p.Hkv, p.page, p.d, dt=dt), z(n, p.Hkv, p.page, p.d, dt=dt), None, None, boxes)


def adacluster_block_workspace_bytes(p: BlockParams, call, q_rows, k_rows=0, num_pages=0) -> int:
    if not q_rows:                                      # a step without queries
        return 0
    return _block_bytes(_block_c(p, q_rows, k_rows, num_pages), call)


def adacluster_cache_append(p: BlockParams, k, v, cu_new, seq_lens, page_table, cache: BlockCache):
    """Writes new tokens k, v [rows,Hkv,d] into the cache behind the seq_lens[b] tokens that sequence b holds."""
    dev, dt = _gpu(k), _tdtype(p)
    rows = k.shape[0]
    if v.shape[0] != rows:
        raise ValueError("k and v must have the same rows")
    _ints("cu_new", cu_new, (p.B + 1,), dev)
    _ints("seq_lens", seq_lens, (p.B,), dev)
    _ints("page_table", page_table, (p.B, p.max_pages), dev)
    n, ks, vs = _pool(p, cache, dev, True)
    cp = _block_c(p, rows, 0, n, k=ks, v=vs, new_k=_rows("k", k, dt, p.Hkv, p.d, dev), new_v=_rows("v", v, dt, p.Hkv, p.d, dev))
    if rows:
        _on(dev, "adacluster_cache_append", cp, k.data_ptr(), v.data_ptr(), cu_new.data_ptr(), seq_lens.data_ptr(), page_table.data_ptr(),
            cache.k.data_ptr(), cache.v.data_ptr(), _ptr(cache.k_meta), _ptr(cache.v_meta), cache.boxes.data_ptr())


def adacluster_cache_read(p: BlockParams, cache: BlockCache, cu_new, first, page_table, rows, out=None):
    """Tokens of the cache as values -> k, v [rows,Hkv,d]: of sequence b those from position first[b] on, to its rows by cu_new.
    Rows that belong to no sequence, or to positions past max_pages * page, are not written: without `out` they hold anything."""
    dev, dt = _gpu(cache.k), _tdtype(p)
    _ints("cu_new", cu_new, (p.B + 1,), dev)
    _ints("first", first, (p.B,), dev)
    _ints("page_table", page_table, (p.B, p.max_pages), dev)
    n, ks, vs = _pool(p, cache, dev, False)
    shape = (rows, p.Hkv, p.d)
    if out is None:
        out = torch.empty(shape, dtype=dt, device=dev), torch.empty(shape, dtype=dt, device=dev)
    else:
        for t in out:
            if t.shape != shape or t.dtype != dt or not t.is_contiguous() or t.device != dev:
                raise ValueError(f"out must be two contiguous {dt} tensors {shape} on {dev}")
    if rows:
        _on(dev, "adacluster_cache_read", _block_c(p, rows, 0, n, k=ks, v=vs), cu_new.data_ptr(), first.data_ptr(), page_table.data_ptr(),
            cache.k.data_ptr(), cache.v.data_ptr(), _ptr(cache.k_meta), _ptr(cache.v_meta), out[0].data_ptr(), out[1].data_ptr())
    return out


def adacluster_block_boxes(p: BlockParams, k, cu_k, out=None):
    """Boxes of packed keys [rows,Hkv,d] -> [B,max_pages,Hkv,2,d]."""
    dev, dt = _gpu(k), _tdtype(p)
    _ints("cu_k", cu_k, (p.B + 1,), dev)
    shape = (p.B, p.max_pages, p.Hkv, 2, p.d)
    boxes = torch.empty(shape, dtype=dt, device=dev) if out is None else out
    _boxes(boxes, shape, p, dev)
    strides = _rows("k", k, dt, p.Hkv, p.d, dev)
    if not k.shape[0]:                                  # no keys: every page is past its sequence's last
        return boxes.zero_()
    _on(dev, "adacluster_block_boxes", _block_c(p, 1, k.shape[0], k=(0, *strides)), k.data_ptr(), cu_k.data_ptr(), boxes.data_ptr())
    return boxes


def _keys_of(p, cu_k, seq_lens, page_table, dev, paged):
    if paged:
        if seq_lens is None or page_table is None:
            raise ValueError("a paged cache needs seq_lens and page_table")
        _ints("seq_lens", seq_lens, (p.B,), dev)
        _ints("page_table", page_table, (p.B, p.max_pages), dev)
    else:
        if cu_k is None:
            raise ValueError("packed keys need cu_k")
        _ints("cu_k", cu_k, (p.B + 1,), dev)


def adacluster_block_select(p: BlockParams, q, cu_q, boxes, cu_k=None, seq_lens=None, page_table=None, k_rows=None, ws=None):
    """Pages of every block of queries -> sel_idx [B,blocks,Hkv,topk], sel_cnt [B,blocks,Hkv].  cu_k: packed keys (k_rows: rows of
    the key tensor, where it has fewer than cu_k says); seq_lens and page_table: a paged cache."""
    dev = _gpu(q)
    paged = cu_k is None
    n = boxes.shape[0]
    cp = _block_c(p, q.shape[0], 0 if paged else (2 ** 31 - 1 if k_rows is None else k_rows), n if paged else 0,
                  q=_rows("q", q, _tdtype(p), p.Hq, p.d, dev))
    _ints("cu_q", cu_q, (p.B + 1,), dev)
    _keys_of(p, cu_k, seq_lens, page_table, dev, paged)
    _boxes(boxes, (n, p.Hkv, 2, p.d) if paged else (p.B, p.max_pages, p.Hkv, 2, p.d), p, dev)
    idx = torch.empty((p.B, p.blocks, p.Hkv, p.topk), dtype=torch.int32, device=dev)
    cnt = torch.empty((p.B, p.blocks, p.Hkv), dtype=torch.int32, device=dev)
    if not q.shape[0] or k_rows == 0:                   # a step without queries, or without keys
        return idx.fill_(-1), cnt.zero_()
    ws, size = _block_ws(cp, BLOCK_SELECT, dev, ws)
    _on(dev, "adacluster_block_select", cp, q.data_ptr(), cu_q.data_ptr(), _ptr(cu_k), _ptr(seq_lens), _ptr(page_table), boxes.data_ptr(),
        idx.data_ptr(), cnt.data_ptr(), _ptr(ws), size)
    return idx, cnt


def adacluster_block_attn(p: BlockParams, q, cu_q, k=None, v=None, cu_k=None, cache: BlockCache = None, seq_lens=None, page_table=None,
                          sel_idx=None, out=None, lse=None, ws=None):
    """Attention of q [rows,Hq,d] over packed k, v [rows,Hkv,d] with cu_k, or over a cache with seq_lens and page_table; over the
    pages of sel_idx, or all -> o like q, lse float32 [rows,Hq].  Rows that belong to no sequence are not written: without `out` and
    `lse` they hold anything.  Nothing is recorded for autograd: the gradients are adacluster_block_attn_backward's, called from the
    backward method of a torch.autograd.Function, say (a call on tensors that require gradients, with gradients enabled, warns)."""
    dev, dt = _gpu(q), _tdtype(p)
    if torch.is_grad_enabled() and (q.requires_grad or cache is None and any(t is not None and t.requires_grad for t in (k, v))):
        warnings.warn("adacluster_block_attn records nothing for autograd: no gradient reaches q, k or v through its output "
                      "(adacluster_block_attn_backward has the gradients)", stacklevel=2)
    rows = q.shape[0]
    _ints("cu_q", cu_q, (p.B + 1,), dev)
    _keys_of(p, cu_k, seq_lens, page_table, dev, cache is not None)
    km = vm = None
    n = k_rows = 0
    if cache is not None:
        n, ks, vs = _pool(p, cache, dev, False)
        k, v, km, vm, cu_k = cache.k, cache.v, cache.k_meta, cache.v_meta, None
    else:
        k_rows, ks, vs = _kv(p, k, v, dev)
    if sel_idx is not None:
        _ints("sel_idx", sel_idx, (p.B, p.blocks, p.Hkv, p.topk), dev)
    o = torch.empty_like(q) if out is None else out
    if lse is None:
        lse = torch.empty((rows, p.Hq), dtype=torch.float32, device=dev)
    else:
        _lse(lse, rows, p, dev)
    if o.shape[0] != rows:
        raise ValueError("out must have the rows of q")
    if cache is None and not k_rows and rows:           # every sequence is without keys
        k = v = _row_of_none(p.Hkv, p.d, dt, dev)
        k_rows, ks, vs, cu_k, sel_idx = 1, _NO3, _NO3, torch.zeros_like(cu_k), None
    cp = _block_c(p, rows, k_rows, n, q=_rows("q", q, dt, p.Hq, p.d, dev), o=_rows("out", o, dt, p.Hq, p.d, dev), k=ks, v=vs)
    if not rows:
        return o, lse
    ws, size = _block_ws(cp, BLOCK_ATTN, dev, ws)
    _on(dev, "adacluster_block_attn", cp, q.data_ptr(), cu_q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(km), _ptr(vm), _ptr(cu_k), _ptr(seq_lens),
        _ptr(page_table), _ptr(sel_idx), o.data_ptr(), lse.data_ptr(), _ptr(ws), size)
    return o, lse


def _kv(p, k, v, dev):
    if k is None or v is None or k.shape[0] != v.shape[0]:
        raise ValueError("k and v must be given, with the same rows")
    dt = _tdtype(p)
    return k.shape[0], (0, *_rows("k", k, dt, p.Hkv, p.d, dev)), (0, *_rows("v", v, dt, p.Hkv, p.d, dev))


def _row_of_none(heads, d, dt, dev):
    """What a call is given in the place of a tensor without rows: a row that belongs to no sequence."""
    return torch.zeros((1, heads, d), dtype=dt, device=dev)


def _lse(lse, rows, p, dev):
    if lse.shape != (rows, p.Hq) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.device != dev:
        raise ValueError(f"lse must be a contiguous float32 tensor {(rows, p.Hq)} on {dev}")


def adacluster_block_attn_backward(p: BlockParams, q, k, v, o, lse, d_o, cu_q, cu_k, sel_idx=None, outs=None, ws=None):
    """Gradients of adacluster_block_attn over packed keys -> dq, dk, dv (like q, k, v).  Without `outs`, rows that belong to no
    sequence are zero."""
    dev, dt = _gpu(q), _tdtype(p)
    rows = q.shape[0]
    k_rows, ks, vs = _kv(p, k, v, dev)
    _lse(lse, rows, p, dev)
    _ints("cu_q", cu_q, (p.B + 1,), dev)
    _ints("cu_k", cu_k, (p.B + 1,), dev)
    if sel_idx is not None:
        _ints("sel_idx", sel_idx, (p.B, p.blocks, p.Hkv, p.topk), dev)
    dq, dk, dv = (torch.zeros_like(t) for t in (q, k, v)) if outs is None else outs
    if not (o.shape[0] == d_o.shape[0] == dq.shape[0] == rows and dk.shape[0] == dv.shape[0] == k_rows):
        raise ValueError("o, d_o and dq must have the rows of q, dk and dv those of k")
    at = lambda name, t, heads: _rows(name, t, dt, heads, p.d, dev)  # noqa: E731
    strides = dict(q=at("q", q, p.Hq), o=at("o", o, p.Hq), k=ks, v=vs, d_o=at("d_o", d_o, p.Hq), dq=at("dq", dq, p.Hq), dk=at("dk", dk, p.Hkv),
                   dv=at("dv", dv, p.Hkv))
    grads = dq, dk, dv
    if not rows and not k_rows:
        return grads
    if not rows:                                        # every sequence is without queries: dk and dv are zero
        p, rows, ws, sel_idx = replace(p, max_q=1), 1, None, None
        q = o = d_o = dq = _row_of_none(p.Hq, p.d, dt, dev)
        lse, cu_q = torch.zeros((1, p.Hq), device=dev), torch.zeros_like(cu_q)
        strides.update(q=_NO2, o=_NO2, d_o=_NO2, dq=_NO2)
    elif not k_rows:                                    # ... without keys: dq is zero
        k = v = dk = dv = _row_of_none(p.Hkv, p.d, dt, dev)
        k_rows, cu_k, sel_idx = 1, torch.zeros_like(cu_k), None
        strides.update(k=_NO3, v=_NO3, dk=_NO2, dv=_NO2)
    cp = _block_c(p, rows, k_rows, 0, **strides)
    ws, size = _block_ws(cp, BLOCK_BACKWARD, dev, ws)
    _on(dev, "adacluster_block_attn_backward", cp, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(),
        cu_q.data_ptr(), cu_k.data_ptr(), _ptr(sel_idx), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(ws), size)
    return grads


# ---- a cache whose sequences share prefixes and drop tokens ---------------------------------------------------------------


@functools.lru_cache(maxsize=1024)
def _prefix_bytes(cp: bytes, groups):
    n = ctypes.c_size_t(0)
    _check(load_library().adacluster_prefix_workspace_bytes(cp, groups, ctypes.byref(n)), "prefix_workspace_bytes")
    return n.value


def adacluster_prefix_workspace_bytes(p: BlockParams, groups, q_rows, num_pages) -> int:
    if not q_rows:                                      # a step without queries
        return 0
    return _prefix_bytes(_block_c(p, q_rows, 0, num_pages), groups)


def adacluster_prefix_attn(p: BlockParams, q, cu_q, cache: BlockCache, seq_lens, page_table, cu_group, prefix_lens, out=None, lse=None, ws=None):
    """adacluster_block_attn of q [rows,Hq,d] over all pages of a cache, for groups of sequences that share their first prefix_lens[g]
    positions: sequences cu_group[g] .. cu_group[g+1]-1, whose shared pages (the first one's) are read once -> o like q, lse float32
    [rows,Hq].  Rows that belong to no sequence are not written: without `out` and `lse` they hold anything.  Nothing is
    recorded for autograd (queries that require gradients, with gradients enabled, warn)."""
    dev, dt = _gpu(q), _tdtype(p)
    if torch.is_grad_enabled() and q.requires_grad:
        warnings.warn("adacluster_prefix_attn records nothing for autograd: no gradient reaches q through its output", stacklevel=2)
    rows, groups = q.shape[0], prefix_lens.shape[0]
    _ints("cu_q", cu_q, (p.B + 1,), dev)
    _ints("cu_group", cu_group, (groups + 1,), dev)
    _ints("prefix_lens", prefix_lens, (groups,), dev)
    _keys_of(p, None, seq_lens, page_table, dev, True)
    n, ks, vs = _pool(p, cache, dev, False)
    o = torch.empty_like(q) if out is None else out
    if lse is None:
        lse = torch.empty((rows, p.Hq), dtype=torch.float32, device=dev)
    else:
        _lse(lse, rows, p, dev)
    if o.shape[0] != rows:
        raise ValueError("out must have the rows of q")
    cp = _block_c(p, rows, 0, n, q=_rows("q", q, dt, p.Hq, p.d, dev), o=_rows("out", o, dt, p.Hq, p.d, dev), k=ks, v=vs)
    if not rows:
        return o, lse
    if ws is None:
        size = _prefix_bytes(cp, groups)
        ws = torch.empty(size, dtype=torch.uint8, device=dev)
    else:
        ws, size = _block_ws(cp, None, dev, ws)
    _on(dev, "adacluster_prefix_attn", cp, groups, q.data_ptr(), cu_q.data_ptr(), cache.k.data_ptr(), cache.v.data_ptr(), _ptr(cache.k_meta),
        _ptr(cache.v_meta), seq_lens.data_ptr(), page_table.data_ptr(), cu_group.data_ptr(), prefix_lens.data_ptr(), o.data_ptr(), lse.data_ptr(),
        _ptr(ws), size)
    return o, lse


@functools.lru_cache(maxsize=1024)
def _weights_bytes(cp: bytes):
    n = ctypes.c_size_t(0)
    _check(load_library().adacluster_weights_workspace_bytes(cp, ctypes.byref(n)), "weights_workspace_bytes")
    return n.value


def adacluster_weights_workspace_bytes(p: BlockParams, q_rows, num_pages) -> int:
    return _weights_bytes(_block_c(p, max(1, q_rows), 0, num_pages))


def _weights(name, t, p, dev):
    shape = (p.B, p.Hkv, p.max_pages * p.page)
    if t.shape != shape or t.dtype != torch.float32 or not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{name} must be a contiguous float32 tensor {shape} on {dev}")


def adacluster_cache_weights(p: BlockParams, q, cu_q, lse, cache: BlockCache, seq_lens, page_table, weights=None, decay=1.0, out=None, ws=None):
    """decay * weights + what every cached key gets from the queries q [rows,Hq,d] whose attention over all keys left lse [rows,Hq], summed
    over queries and the heads that share the key -> float32 [B,Hkv,max_pages*page], 0 from a sequence's last key on.  weights None: from
    nothing.  out: may be weights.  Nothing is recorded for autograd (as in adacluster_prefix_attn)."""
    dev, dt = _gpu(q), _tdtype(p)
    if torch.is_grad_enabled() and (q.requires_grad or lse.requires_grad or weights is not None and weights.requires_grad):
        warnings.warn("adacluster_cache_weights records nothing for autograd: no gradient reaches q, lse or weights through its output", stacklevel=2)
    rows = q.shape[0]
    _ints("cu_q", cu_q, (p.B + 1,), dev)
    _keys_of(p, None, seq_lens, page_table, dev, True)
    _lse(lse, rows, p, dev)
    n, ks, _ = _pool(p, cache, dev, False)
    if weights is not None:
        _weights("weights", weights, p, dev)
    if out is None:
        out = torch.empty((p.B, p.Hkv, p.max_pages * p.page), dtype=torch.float32, device=dev)
    else:
        _weights("out", out, p, dev)
    strides = _rows("q", q, dt, p.Hq, p.d, dev)
    if not rows:                                        # a step without queries: what was there, decayed
        q, lse, strides, rows, cu_q = _row_of_none(p.Hq, p.d, dt, dev), torch.zeros((1, p.Hq), device=dev), _NO2, 1, torch.zeros_like(cu_q)
    cp = _block_c(p, rows, 0, n, q=strides, k=ks)
    if ws is None:
        size = _weights_bytes(cp)
        ws = torch.empty(size, dtype=torch.uint8, device=dev) if size else None
    else:
        ws, size = _block_ws(cp, None, dev, ws)
    _on(dev, "adacluster_cache_weights", cp, q.data_ptr(), cu_q.data_ptr(), lse.data_ptr(), cache.k.data_ptr(), _ptr(cache.k_meta), seq_lens.data_ptr(),
        page_table.data_ptr(), _ptr(weights), decay, out.data_ptr(), _ptr(ws), size)
    return out


def adacluster_cache_evict(p: BlockParams, cache: BlockCache, seq_lens, page_table, weights, keep, recent, new_table, out=None):
    """Moves the `keep` tokens of every sequence and head that stay (its first keep_first pages, its last `recent` tokens, the others by
    weight) to the pages of new_table -> kept int32 [B,Hkv,keep] (-1 behind the end), new lengths int32 [B], new weights like weights (out:
    where to).  A page of new_table may be one of page_table only where all its tokens stay in their place."""
    dev = _gpu(cache.k)
    _keys_of(p, None, seq_lens, page_table, dev, True)
    _ints("new_table", new_table, (p.B, p.max_pages), dev)
    _weights("weights", weights, p, dev)
    n, ks, vs = _pool(p, cache, dev, True)
    if out is None:
        out = torch.empty_like(weights)
    else:
        _weights("out", out, p, dev)
    keep, recent = operator.index(keep), operator.index(recent)
    if keep < 1:
        raise ValueError("keep must be at least 1")
    kept = torch.empty((p.B, p.Hkv, keep), dtype=torch.int32, device=dev)
    lens = torch.empty((p.B,), dtype=torch.int32, device=dev)
    _on(dev, "adacluster_cache_evict", _block_c(p, 1, 0, n, k=ks, v=vs), seq_lens.data_ptr(), page_table.data_ptr(), weights.data_ptr(), keep, recent,
        new_table.data_ptr(), kept.data_ptr(), lens.data_ptr(), out.data_ptr(), cache.k.data_ptr(), cache.v.data_ptr(), _ptr(cache.k_meta),
        _ptr(cache.v_meta), cache.boxes.data_ptr())
    return kept, lens, out
