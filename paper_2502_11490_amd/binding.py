"""ctypes marshalling for include/gmpgr_ann.h.  PyTorch is used for device memory and the
current HIP stream only."""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

import numpy as np
import torch

ANN_OK, ANN_EINVAL, ANN_ENOMEM, ANN_EDEVICE, ANN_ENOTIMPL, ANN_EWORKSPACE = 0, -1, -2, -3, -4, -5
ANN_F32, ANN_BF16, ANN_F8, ANN_F16 = 0, 1, 2, 3
ANN_VALIDATE, ANN_MLP_GENERIC = 1, 2
ANN_SILU, ANN_GELU, ANN_SIGMOID, ANN_RELU = 0, 1, 2, 3

_HERE = os.path.dirname(os.path.abspath(__file__))
# GMPGR_ANN_LIB names another build of the same library (measurement builds with other tuning constants)
_LIB_PATH = os.environ.get("GMPGR_ANN_LIB") or os.path.join(_HERE, "libgmpgr_ann.so")
_lib = None

EXPORTS = [
    "ann_graph_load", "ann_graph_free", "ann_mlp_load", "ann_mlp_free", "ann_mlp_uses_mfma",
    "ann_search_workspace_bytes", "ann_search", "ann_search_ragged", "ann_search_layers_workspace_bytes",
    "ann_search_layers", "ann_search_walkers_workspace_bytes", "ann_search_walkers",
    "ann_search_stream_workspace_bytes", "ann_search_stream", "ann_stream_open", "ann_stream_submit", "ann_stream_step",
    "ann_stream_drain", "ann_stream_close", "ann_score_pairs", "ann_score_pairs_noalloc", "ann_graph_set_locality", "ann_search_visited_set_is_bitmap", "ann_brute_force", "ann_brute_force_workspace_bytes", "ann_rerank", "ann_rerank_workspace_bytes", "ann_users_add_noise", "ann_quantize_e4m3",
    "ann_layer_norm", "ann_layer_norm_backward_workspace_bytes", "ann_layer_norm_backward", "ann_dropout",
    "ann_gated_ffn_workspace_bytes", "ann_gated_ffn", "ann_gated_ffn_backward_workspace_bytes", "ann_gated_ffn_backward",
    "ann_search_stats", "ann_set_progress_timeout", "ann_profile_enable", "ann_profile_read", "ann_profile_copy", "ann_last_error",
]


class AnnError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ann error {code}: {msg}")
        self.code = code


class Stats(ctypes.Structure):
    _fields_ = [("pairs_scored", ctypes.c_int64), ("nodes_expanded", ctypes.c_int64),
                ("max_query_iters", ctypes.c_int64), ("visited_overflow", ctypes.c_int64),
                ("queries", ctypes.c_int64), ("adjacency_bytes", ctypes.c_int64),
                ("embedding_bytes", ctypes.c_int64), ("pair_list_bytes", ctypes.c_int64)]


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libgmpgr_ann.so (built by paper_2502_11490_amd/build.py).  Raises if it is missing:
    there is no other implementation to fall back to."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} not found: build it with `python -m paper_2502_11490_amd.build` "
            "(or __graft_entry__.build()); the library has no CPU fallback")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, u32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_size_t
    lib.ann_graph_load.argtypes = [vp, vp, i64, i32, i32, i32, u32, vp, ctypes.POINTER(vp)]
    lib.ann_graph_load.restype = ctypes.c_int
    lib.ann_graph_free.argtypes = [vp]
    lib.ann_graph_free.restype = None
    lib.ann_mlp_load.argtypes = [i32, ctypes.POINTER(i32), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                 ctypes.POINTER(ctypes.c_float), i32, i32, u32, vp, ctypes.POINTER(vp)]
    lib.ann_mlp_load.restype = ctypes.c_int
    lib.ann_mlp_free.argtypes = [vp]
    lib.ann_mlp_free.restype = None
    lib.ann_mlp_uses_mfma.argtypes = [vp]
    lib.ann_mlp_uses_mfma.restype = ctypes.c_int
    lib.ann_search_workspace_bytes.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32]
    lib.ann_search_workspace_bytes.restype = sz
    lib.ann_search.argtypes = [vp, vp, vp, i32, vp, i32, i32, i32, i32, i32, vp, sz, vp, vp, vp]
    lib.ann_search.restype = ctypes.c_int
    lib.ann_search_ragged.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp, vp, i32, i32, i32, i32, vp, sz, vp, vp, vp]
    lib.ann_search_ragged.restype = ctypes.c_int
    pi32 = ctypes.POINTER(i32)
    lib.ann_search_layers_workspace_bytes.argtypes = [ctypes.POINTER(vp), i32, vp, i32, i32, pi32, pi32, pi32, i32]
    lib.ann_search_layers_workspace_bytes.restype = sz
    lib.ann_search_layers.argtypes = [ctypes.POINTER(vp), i32, vp, vp, i32, vp, i32, pi32, pi32, pi32, i32, vp, sz,
                                      vp, vp, vp]
    lib.ann_search_layers.restype = ctypes.c_int
    lib.ann_search_walkers_workspace_bytes.argtypes = [vp, vp, i32, i32, i32, i32]
    lib.ann_search_walkers_workspace_bytes.restype = sz
    lib.ann_search_walkers.argtypes = [vp, vp, vp, i32, vp, i32, i32, i32, vp, sz, vp, vp, vp]
    lib.ann_search_walkers.restype = ctypes.c_int
    lib.ann_search_stream_workspace_bytes.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, i32]
    lib.ann_search_stream_workspace_bytes.restype = sz
    lib.ann_search_stream.argtypes = [vp, vp, vp, i32, vp, i32, i32, i32, i32, i32, i32, vp, sz, vp, vp, vp]
    lib.ann_search_stream.restype = ctypes.c_int
    lib.ann_stream_open.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp, ctypes.POINTER(vp)]
    lib.ann_stream_open.restype = ctypes.c_int
    lib.ann_stream_submit.argtypes = [vp, i32]
    lib.ann_stream_step.argtypes = [vp, i32]
    lib.ann_stream_drain.argtypes = [vp]
    lib.ann_stream_close.argtypes = [vp]
    for name in ("ann_stream_submit", "ann_stream_step", "ann_stream_drain", "ann_stream_close"):
        getattr(lib, name).restype = ctypes.c_int
    lib.ann_score_pairs.argtypes = [vp, vp, vp, i32, i64, vp, vp, vp, i32, vp]
    lib.ann_score_pairs.restype = ctypes.c_int
    lib.ann_score_pairs_noalloc.argtypes = [vp, vp, vp, i32, i64, vp, vp, vp, vp]
    lib.ann_score_pairs_noalloc.restype = ctypes.c_int
    lib.ann_search_visited_set_is_bitmap.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32]
    lib.ann_search_visited_set_is_bitmap.restype = ctypes.c_int
    lib.ann_graph_set_locality.argtypes = [vp, vp, vp]
    lib.ann_graph_set_locality.restype = ctypes.c_int
    lib.ann_brute_force.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, ctypes.c_size_t, vp]
    lib.ann_brute_force.restype = ctypes.c_int
    lib.ann_brute_force_workspace_bytes.argtypes = [vp, vp, i32, i32]
    lib.ann_brute_force_workspace_bytes.restype = ctypes.c_size_t
    lib.ann_rerank_workspace_bytes.argtypes = [vp, vp, i32, i32, i32]
    lib.ann_rerank_workspace_bytes.restype = ctypes.c_size_t
    lib.ann_rerank.argtypes = [vp, vp, vp, i32, vp, i32, i32, vp, vp, vp, ctypes.c_size_t, vp]
    lib.ann_rerank.restype = ctypes.c_int
    lib.ann_users_add_noise.argtypes = [vp, vp, i32, i32, i32, ctypes.c_double, ctypes.c_uint64, ctypes.c_uint64, vp]
    lib.ann_users_add_noise.restype = ctypes.c_int
    lib.ann_quantize_e4m3.argtypes = [vp, i32, i64, ctypes.c_float, vp, vp]
    lib.ann_quantize_e4m3.restype = ctypes.c_int
    f64, u64 = ctypes.c_double, ctypes.c_uint64
    lib.ann_layer_norm.argtypes = [vp, i64, vp, vp, i64, i32, i32, f64, vp, i64, vp, vp, vp]
    lib.ann_layer_norm.restype = ctypes.c_int
    lib.ann_layer_norm_backward_workspace_bytes.argtypes = [i64, i32, i32]
    lib.ann_layer_norm_backward_workspace_bytes.restype = sz
    lib.ann_layer_norm_backward.argtypes = [vp, i64, vp, i64, vp, vp, vp, i64, i32, i32, vp, i64, vp, vp, vp, sz, vp]
    lib.ann_layer_norm_backward.restype = ctypes.c_int
    lib.ann_dropout.argtypes = [vp, vp, vp, i64, i32, f64, u64, u64, vp, vp]
    lib.ann_dropout.restype = ctypes.c_int
    lib.ann_gated_ffn_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
    lib.ann_gated_ffn_workspace_bytes.restype = sz
    lib.ann_gated_ffn.argtypes = [vp, i64, vp, vp, vp, vp, i64, i32, i32, i32, i32, i32, vp, i64, vp, vp, sz, vp]
    lib.ann_gated_ffn.restype = ctypes.c_int
    lib.ann_gated_ffn_backward_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
    lib.ann_gated_ffn_backward_workspace_bytes.restype = sz
    lib.ann_gated_ffn_backward.argtypes = [vp, i64, vp, i64, vp, vp, vp, i64, i32, i32, i32, i32, i32, vp, i64, vp, vp, vp,
                                           vp, vp, sz, vp]
    lib.ann_gated_ffn_backward.restype = ctypes.c_int
    lib.ann_search_stats.argtypes = [vp, ctypes.POINTER(Stats), vp]
    lib.ann_search_stats.restype = ctypes.c_int
    lib.ann_set_progress_timeout.argtypes = [ctypes.c_double]
    lib.ann_set_progress_timeout.restype = ctypes.c_int
    lib.ann_profile_enable.argtypes = [ctypes.c_int]
    lib.ann_profile_enable.restype = ctypes.c_int
    lib.ann_profile_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.ann_profile_read.restype = ctypes.c_int
    lib.ann_profile_copy.argtypes = [vp, vp, sz, vp]
    lib.ann_profile_copy.restype = ctypes.c_int
    lib.ann_last_error.argtypes = []
    lib.ann_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def ann_last_error() -> str:
    return load_library().ann_last_error().decode()


def _check(rc: int):
    if rc != ANN_OK:
        raise AnnError(rc, ann_last_error())


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return ANN_F32
    if t.dtype == torch.bfloat16:
        return ANN_BF16
    if t.dtype == torch.float8_e4m3fn:
        return ANN_F8
    if t.dtype == torch.float16:
        return ANN_F16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dev_ptr(t: Optional[torch.Tensor], name: str, dtype=None) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _queries_ptr(queries: torch.Tensor, m, Q: Optional[int] = None) -> Optional[int]:
    """User vectors must be [Q][d_user] in the metric's element type (bf16 for the 8-bit metric, whose user half
    stays 16-bit): the library takes a bare pointer and could not tell.  With Q given, the row count is checked
    too (the kernels read Q rows)."""
    want = {ANN_F32: torch.float32, ANN_BF16: torch.bfloat16, ANN_F16: torch.float16, ANN_F8: torch.bfloat16}[m.dtype]
    if queries.dim() != 2 or queries.shape[1] != m.d_user:
        raise ValueError(f"queries must be [Q][{m.d_user}], got {tuple(queries.shape)}")
    if Q is not None and queries.shape[0] != Q:
        raise ValueError(f"queries has {queries.shape[0]} rows, entries has {Q}")
    return _dev_ptr(queries, "queries", want)


def _entries_shape(entries: torch.Tensor):
    if entries.dim() != 2:
        raise ValueError(f"entries must be [Q][E], got {tuple(entries.shape)}")
    return int(entries.shape[0]), int(entries.shape[1])


def _check_out(out_ids, out_scores, Q: int, k: int) -> None:
    """Caller-supplied result arrays must be exactly [Q][k]: the library writes Q * k elements into each."""
    for name, t in (("out_ids", out_ids), ("out_scores", out_scores)):
        if t is None or tuple(t.shape) != (Q, k):
            raise ValueError(f"{name} must be [{Q}][{k}], got {None if t is None else tuple(t.shape)}")


def _per_query_ptr(t: torch.Tensor, name: str, Q: int) -> Optional[int]:
    if t is None or t.numel() != Q:
        raise ValueError(f"{name} must hold one int32 per query ({Q}), got {None if t is None else t.numel()}")
    return _dev_ptr(t, name, torch.int32)


class Graph:
    """Owns the C handle and keeps the borrowed tensors alive."""

    def __init__(self, handle, adj, emb):
        self.handle, self.adj, self.emb = handle, adj, emb

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.ann_graph_free(self.handle)
            self.handle = None


class Mlp:
    def __init__(self, handle, dims, d_user, dtype):
        self.handle, self.dims, self.d_user, self.dtype = handle, list(dims), d_user, dtype

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.ann_mlp_free(self.handle)
            self.handle = None


def ann_graph_load(adj: torch.Tensor, emb: torch.Tensor, flags: int = 0, stream=None) -> Graph:
    lib = load_library()
    if adj.dim() != 2 or emb.dim() != 2 or adj.shape[0] != emb.shape[0]:
        raise ValueError("adj must be [N,R] and emb [N,d]")
    h = ctypes.c_void_p()
    rc = lib.ann_graph_load(_dev_ptr(adj, "adj", torch.int32), _dev_ptr(emb, "emb"), adj.shape[0], adj.shape[1],
                            emb.shape[1], _dtype_code(emb), flags, _stream_ptr(stream), ctypes.byref(h))
    _check(rc)
    return Graph(h, adj, emb)


def ann_graph_set_locality(g: Graph, rank: Optional[torch.Tensor], stream=None) -> None:
    """Addresses the visited bitmap of searches on `g` by rank [N] (int32 permutation of the ids, device; None
    removes it).  Results do not change; the tensor is kept alive with the graph."""
    if rank is not None and (rank.dim() != 1 or rank.shape[0] != g.adj.shape[0]):
        raise ValueError(f"rank must be [{g.adj.shape[0]}], got {tuple(rank.shape)}")
    _check(load_library().ann_graph_set_locality(g.handle, _dev_ptr(rank, "rank", torch.int32), _stream_ptr(stream)))
    g.rank = rank


def ann_search_visited_set_is_bitmap(g: Graph, m: Mlp, Q: int, E: int, W: int, L: int, k: int, max_iters: int = 0) -> bool:
    rc = load_library().ann_search_visited_set_is_bitmap(g.handle, m.handle, Q, E, W, L, k, max_iters)
    if rc < 0:
        _check(rc)
    return rc == 1


def _host_bytes(t) -> np.ndarray:
    """Host copy of a weight tensor as a contiguous numpy array (bf16 as raw uint16)."""
    if isinstance(t, torch.Tensor):
        t = t.detach().to("cpu").contiguous()
        if t.dtype == torch.bfloat16:
            return t.view(torch.int16).numpy().view(np.uint16).copy()
        return t.numpy().copy()
    return np.ascontiguousarray(t)


def ann_mlp_load(W: Sequence, b: Sequence, head_w, d_user: int, dtype: int, flags: int = 0, stream=None) -> Mlp:
    """W[l]: [out,in] torch tensors (fp32, bf16 or fp16, matching dtype) or numpy arrays (bf16 as uint16 bits);
    b[l]: [out] fp32; head_w: [J] fp32."""
    lib = load_library()
    n = len(W)
    Wh = [_host_bytes(w) for w in W]
    # the 8-bit metric takes bf16 weights and quantises them
    want = {ANN_F32: np.float32, ANN_F16: np.float16}.get(dtype, np.uint16)
    for w in Wh:
        if w.dtype != want:
            raise TypeError(f"weights must be {np.dtype(want).name if want != np.uint16 else 'bf16'}")
    bh = [np.ascontiguousarray(_host_bytes(x), dtype=np.float32) for x in b]
    hw = np.ascontiguousarray(_host_bytes(head_w), dtype=np.float32)
    dims = [Wh[0].shape[1]] + [w.shape[0] for w in Wh]
    for l in range(n):
        if Wh[l].shape != (dims[l + 1], dims[l]) or bh[l].shape != (dims[l + 1],):
            raise ValueError("layer shapes do not chain")
    if hw.shape != (dims[-1],):
        raise ValueError("head_w must have one weight per head")
    dims_c = (ctypes.c_int32 * (n + 1))(*dims)
    W_c = (ctypes.c_void_p * n)(*[w.ctypes.data for w in Wh])
    b_c = (ctypes.c_void_p * n)(*[x.ctypes.data for x in bh])
    h = ctypes.c_void_p()
    rc = lib.ann_mlp_load(n, dims_c, W_c, b_c, hw.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), d_user, dtype,
                          flags, _stream_ptr(stream), ctypes.byref(h))
    _check(rc)
    return Mlp(h, dims, d_user, dtype)


def ann_mlp_uses_mfma(m: Mlp) -> bool:
    return bool(load_library().ann_mlp_uses_mfma(m.handle))


def ann_search_workspace_bytes(g: Graph, m: Mlp, Q: int, E: int, W_max: int, L_max: int, k: int,
                               max_iters_max: int) -> int:
    n = load_library().ann_search_workspace_bytes(g.handle, m.handle, Q, E, W_max, L_max, k, max_iters_max)
    if n == 0:
        raise AnnError(ANN_EINVAL, ann_last_error())
    return int(n)


def _alloc_out(Q, k, device):
    return (torch.empty((Q, k), dtype=torch.int32, device=device),
            torch.empty((Q, k), dtype=torch.float32, device=device))


def ann_search(g: Graph, m: Mlp, queries: torch.Tensor, entries: torch.Tensor, W: int, L: int, k: int,
               max_iters: int = 0, workspace: Optional[torch.Tensor] = None, out_ids=None, out_scores=None,
               stream=None):
    """Returns (ids [Q,k] int32, scores [Q,k] fp32) on the device.  `workspace` is a uint8 device tensor of at
    least ann_search_workspace_bytes(...) bytes; one is allocated when omitted."""
    lib = load_library()
    Q, E = _entries_shape(entries)
    if workspace is None:
        workspace = torch.empty(ann_search_workspace_bytes(g, m, Q, E, W, L, k, max_iters), dtype=torch.uint8,
                                device=queries.device)
    if out_ids is None:
        out_ids, out_scores = _alloc_out(Q, k, queries.device)
    _check_out(out_ids, out_scores, Q, k)
    rc = lib.ann_search(g.handle, m.handle, _queries_ptr(queries, m, Q), Q, _dev_ptr(entries, "entries", torch.int32),
                        E, W, L, k, max_iters, _dev_ptr(workspace, "workspace", torch.uint8), workspace.numel(),
                        _dev_ptr(out_ids, "out_ids", torch.int32), _dev_ptr(out_scores, "out_scores", torch.float32),
                        _stream_ptr(stream))
    _check(rc)
    return out_ids, out_scores


def ann_search_ragged(g: Graph, m: Mlp, queries, entries, W_q, L_q, iters_q, W_max: int, L_max: int, k: int,
                      max_iters_max: int, workspace: Optional[torch.Tensor] = None, out_ids=None, out_scores=None,
                      stream=None):
    lib = load_library()
    Q, E = _entries_shape(entries)
    if workspace is None:
        workspace = torch.empty(ann_search_workspace_bytes(g, m, Q, E, W_max, L_max, k, max_iters_max),
                                dtype=torch.uint8, device=queries.device)
    if out_ids is None:
        out_ids, out_scores = _alloc_out(Q, k, queries.device)
    _check_out(out_ids, out_scores, Q, k)
    for name, t in (("W_q", W_q), ("L_q", L_q), ("iters_q", iters_q)):  # sizes first: they need no device
        if t is None or t.numel() != Q:
            raise ValueError(f"{name} must hold one int32 per query ({Q}), got {None if t is None else t.numel()}")
    rc = lib.ann_search_ragged(g.handle, m.handle, _queries_ptr(queries, m, Q), Q,
                               _dev_ptr(entries, "entries", torch.int32), E, _per_query_ptr(W_q, "W_q", Q),
                               _per_query_ptr(L_q, "L_q", Q), _per_query_ptr(iters_q, "iters_q", Q), W_max,
                               L_max, k, max_iters_max, _dev_ptr(workspace, "workspace", torch.uint8),
                               workspace.numel(), _dev_ptr(out_ids, "out_ids", torch.int32),
                               _dev_ptr(out_scores, "out_scores", torch.float32), _stream_ptr(stream))
    _check(rc)
    return out_ids, out_scores


def ann_search_walkers_workspace_bytes(g: Graph, m: Mlp, Q: int, E: int, T: int, k: int) -> int:
    nbytes = load_library().ann_search_walkers_workspace_bytes(g.handle, m.handle, Q, E, T, k)
    if nbytes == 0:
        raise AnnError(-1, ann_last_error())
    return nbytes


def ann_search_walkers(g: Graph, m: Mlp, queries: torch.Tensor, entries: torch.Tensor, T: int, k: int,
                       workspace: Optional[torch.Tensor] = None, out_ids=None, out_scores=None, stream=None):
    """One walker per seed, T greedy hops each, one shared result list.  Returns (ids [Q,k], scores [Q,k])."""
    lib = load_library()
    Q, E = _entries_shape(entries)
    if workspace is None:
        workspace = torch.empty(ann_search_walkers_workspace_bytes(g, m, Q, E, T, k), dtype=torch.uint8,
                                device=queries.device)
    if out_ids is None:
        out_ids, out_scores = _alloc_out(Q, k, queries.device)
    _check_out(out_ids, out_scores, Q, k)
    rc = lib.ann_search_walkers(g.handle, m.handle, _queries_ptr(queries, m, Q), Q,
                                _dev_ptr(entries, "entries", torch.int32), E, T, k,
                                _dev_ptr(workspace, "workspace", torch.uint8), workspace.numel(),
                                _dev_ptr(out_ids, "out_ids", torch.int32),
                                _dev_ptr(out_scores, "out_scores", torch.float32), _stream_ptr(stream))
    _check(rc)
    return out_ids, out_scores


def ann_search_stream_workspace_bytes(g: Graph, m: Mlp, Q_total: int, slots: int, E: int, W: int, L: int, k: int,
                                      max_iters: int = 0) -> int:
    nbytes = load_library().ann_search_stream_workspace_bytes(g.handle, m.handle, Q_total, slots, E, W, L, k, max_iters)
    if nbytes == 0:
        raise AnnError(-1, ann_last_error())
    return nbytes


def ann_search_stream(g: Graph, m: Mlp, queries: torch.Tensor, entries: torch.Tensor, slots: int, W: int, L: int,
                      k: int, max_iters: int = 0, workspace: Optional[torch.Tensor] = None, out_ids=None,
                      out_scores=None, stream=None):
    """All queries, `slots` of them in flight at a time; a finished query's slot goes to the next one.
    Returns (ids [Q_total,k], scores [Q_total,k])."""
    lib = load_library()
    Q, E = _entries_shape(entries)
    if workspace is None:
        workspace = torch.empty(ann_search_stream_workspace_bytes(g, m, Q, slots, E, W, L, k, max_iters),
                                dtype=torch.uint8, device=queries.device)
    if out_ids is None:
        out_ids, out_scores = _alloc_out(Q, k, queries.device)
    _check_out(out_ids, out_scores, Q, k)
    rc = lib.ann_search_stream(g.handle, m.handle, _queries_ptr(queries, m, Q), Q,
                               _dev_ptr(entries, "entries", torch.int32), E, slots, W, L, k, max_iters,
                               _dev_ptr(workspace, "workspace", torch.uint8), workspace.numel(),
                               _dev_ptr(out_ids, "out_ids", torch.int32),
                               _dev_ptr(out_scores, "out_scores", torch.float32), _stream_ptr(stream))
    _check(rc)
    return out_ids, out_scores


class Stream:
    """An open stream (ann_stream_open): queries are written into rows of `queries` / `entries` and submitted
    while earlier ones are being searched; results land in the same rows of `out_ids` / `out_scores`.  The
    object keeps the caller's arrays and the workspace alive."""

    def __init__(self, g: Graph, m: Mlp, queries: torch.Tensor, entries: torch.Tensor, slots: int, W: int, L: int,
                 k: int, max_iters: int = 0, workspace: Optional[torch.Tensor] = None, out_ids=None, out_scores=None,
                 stream=None):
        lib = load_library()
        cap, E = _entries_shape(entries)
        if workspace is None:
            workspace = torch.empty(ann_search_stream_workspace_bytes(g, m, cap, slots, E, W, L, k, max_iters),
                                    dtype=torch.uint8, device=queries.device)
        if out_ids is None:
            out_ids, out_scores = _alloc_out(cap, k, queries.device)
        _check_out(out_ids, out_scores, cap, k)
        self.g, self.m, self.queries, self.entries, self.workspace = g, m, queries, entries, workspace
        self.out_ids, self.out_scores, self.capacity = out_ids, out_scores, cap
        self.handle = ctypes.c_void_p()
        _check(lib.ann_stream_open(g.handle, m.handle, cap, slots, E, W, L, k, max_iters, _queries_ptr(queries, m, cap),
                                   _dev_ptr(entries, "entries", torch.int32), _dev_ptr(out_ids, "out_ids", torch.int32),
                                   _dev_ptr(out_scores, "out_scores", torch.float32),
                                   _dev_ptr(workspace, "workspace", torch.uint8), workspace.numel(), _stream_ptr(stream),
                                   ctypes.byref(self.handle)))

    def submit(self, n: int) -> None:
        _check(load_library().ann_stream_submit(self.handle, n))

    def step(self, rounds: int) -> None:
        _check(load_library().ann_stream_step(self.handle, rounds))

    def drain(self) -> None:
        _check(load_library().ann_stream_drain(self.handle))

    def close(self) -> None:
        if getattr(self, "handle", None):
            _check(load_library().ann_stream_close(self.handle))
            self.handle = None

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.ann_stream_close(self.handle)
            self.handle = None


def ann_stream_open(g: Graph, m: Mlp, queries, entries, slots: int, W: int, L: int, k: int, max_iters: int = 0,
                    **kw) -> Stream:
    return Stream(g, m, queries, entries, slots, W, L, k, max_iters, **kw)


def _layer_args(graphs: Sequence[Graph], W_l, L_l, K_l):
    n = len(graphs)
    if not (len(W_l) == len(L_l) == len(K_l) == n):
        raise ValueError("W_l, L_l, K_l need one entry per layer")
    handles = (ctypes.c_void_p * n)(*[g.handle for g in graphs])
    arr = lambda v: (ctypes.c_int32 * n)(*[int(x) for x in v])
    return n, handles, arr(W_l), arr(L_l), arr(K_l)


def ann_search_layers_workspace_bytes(graphs: Sequence[Graph], m: Mlp, Q: int, E: int, W_l, L_l, K_l,
                                      max_iters: int = 0) -> int:
    n, handles, W, L, K = _layer_args(graphs, W_l, L_l, K_l)
    nbytes = load_library().ann_search_layers_workspace_bytes(handles, n, m.handle, Q, E, W, L, K, max_iters)
    if nbytes == 0:
        raise AnnError(-1, ann_last_error())
    return nbytes


def ann_search_layers(graphs: Sequence[Graph], m: Mlp, queries: torch.Tensor, entries: torch.Tensor, W_l, L_l, K_l,
                      max_iters: int = 0, workspace: Optional[torch.Tensor] = None, out_ids=None, out_scores=None,
                      stream=None):
    """Layer-by-layer search, coarsest graph first; K_l[-1] results per query.  Returns (ids, scores)."""
    lib = load_library()
    Q, E = _entries_shape(entries)
    n, handles, W, L, K = _layer_args(graphs, W_l, L_l, K_l)
    if workspace is None:
        workspace = torch.empty(ann_search_layers_workspace_bytes(graphs, m, Q, E, W_l, L_l, K_l, max_iters),
                                dtype=torch.uint8, device=queries.device)
    if out_ids is None:
        out_ids, out_scores = _alloc_out(Q, int(K_l[-1]), queries.device)
    _check_out(out_ids, out_scores, Q, int(K_l[-1]))
    rc = lib.ann_search_layers(handles, n, m.handle, _queries_ptr(queries, m, Q), Q,
                               _dev_ptr(entries, "entries", torch.int32), E, W, L, K, max_iters,
                               _dev_ptr(workspace, "workspace", torch.uint8), workspace.numel(),
                               _dev_ptr(out_ids, "out_ids", torch.int32),
                               _dev_ptr(out_scores, "out_scores", torch.float32), _stream_ptr(stream))
    _check(rc)
    return out_ids, out_scores


def ann_score_pairs(g: Graph, m: Mlp, queries: torch.Tensor, q_idx: torch.Tensor, item: torch.Tensor,
                    out: Optional[torch.Tensor] = None, tile_rows: int = 0, stream=None) -> torch.Tensor:
    lib = load_library()
    M = q_idx.numel()
    if item.numel() != M:
        raise ValueError(f"q_idx names {M} pairs, item {item.numel()}")
    if out is None:
        out = torch.empty(M, dtype=torch.float32, device=queries.device)
    if out.numel() != M:
        raise ValueError(f"out must hold {M} scores, got {out.numel()}")
    rc = lib.ann_score_pairs(g.handle, m.handle, _queries_ptr(queries, m), queries.shape[0], M,
                             _dev_ptr(q_idx, "q_idx", torch.int32), _dev_ptr(item, "item", torch.int32),
                             _dev_ptr(out, "out", torch.float32), tile_rows, _stream_ptr(stream))
    _check(rc)
    return out


def ann_score_pairs_noalloc(g: Graph, m: Mlp, queries: torch.Tensor, q_idx: torch.Tensor, item: torch.Tensor,
                            out: torch.Tensor, stream=None) -> torch.Tensor:
    """ann_score_pairs without any allocation: `out` ([M] fp32) is the caller's, the library's scratch is a
    fixed array on the device.  Only enqueues; synchronise the stream before reading `out`."""
    lib = load_library()
    M = q_idx.numel()
    if item.numel() != M or out.numel() != M:
        raise ValueError(f"q_idx names {M} pairs, item {item.numel()}, out {out.numel()}")
    rc = lib.ann_score_pairs_noalloc(g.handle, m.handle, _queries_ptr(queries, m), queries.shape[0], M,
                                     _dev_ptr(q_idx, "q_idx", torch.int32), _dev_ptr(item, "item", torch.int32),
                                     _dev_ptr(out, "out", torch.float32), _stream_ptr(stream))
    _check(rc)
    return out


def _workspace_args(workspace: Optional[torch.Tensor]):
    if workspace is None:
        return None, 0
    return _dev_ptr(workspace, "workspace", torch.uint8), workspace.numel()


def ann_brute_force_workspace_bytes(g: Graph, m: Mlp, Q: int, k: int) -> int:
    n = load_library().ann_brute_force_workspace_bytes(g.handle, m.handle, Q, k)
    if n == 0:
        raise AnnError(ANN_EINVAL, ann_last_error())
    return int(n)


def ann_rerank_workspace_bytes(g: Graph, m: Mlp, Q: int, n: int, k: int) -> int:
    b = load_library().ann_rerank_workspace_bytes(g.handle, m.handle, Q, n, k)
    if b == 0:
        raise AnnError(ANN_EINVAL, ann_last_error())
    return int(b)


def ann_brute_force(g: Graph, m: Mlp, queries: torch.Tensor, k: int, out_ids: Optional[torch.Tensor] = None,
                    out_scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Exhaustive search: the k most relevant items of the whole table per query (ids [Q][k] int32, relevances
    [Q][k] fp32; relevance descending, ties by ascending id).  With a `workspace` (uint8 device tensor of
    ann_brute_force_workspace_bytes) the call only enqueues; without one it allocates and synchronises."""
    lib = load_library()
    Q = queries.shape[0]
    if out_ids is None:
        out_ids = torch.empty(Q, k, dtype=torch.int32, device=queries.device)
    if out_scores is None:
        out_scores = torch.empty(Q, k, dtype=torch.float32, device=queries.device)
    _check_out(out_ids, out_scores, Q, k)
    ws, ws_bytes = _workspace_args(workspace)
    rc = lib.ann_brute_force(g.handle, m.handle, _queries_ptr(queries, m), Q, k,
                             _dev_ptr(out_ids, "out_ids", torch.int32),
                             _dev_ptr(out_scores, "out_scores", torch.float32), ws, ws_bytes, _stream_ptr(stream))
    _check(rc)
    return out_ids, out_scores


def ann_rerank(g: Graph, m: Mlp, queries: torch.Tensor, cand: torch.Tensor, k: int,
               out_ids: Optional[torch.Tensor] = None, out_scores: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, stream=None):
    """The k most relevant of each query's candidates cand [Q][n] (int32; ids outside the table are skipped)
    under this metric: ids [Q][k] int32, relevances [Q][k] fp32.  `workspace` as for ann_brute_force
    (ann_rerank_workspace_bytes)."""
    lib = load_library()
    Q = queries.shape[0]
    if cand.dim() != 2 or cand.shape[0] != Q:
        raise ValueError(f"cand must be [{Q}][n], got {tuple(cand.shape)}")
    if out_ids is None:
        out_ids = torch.empty(Q, k, dtype=torch.int32, device=queries.device)
    if out_scores is None:
        out_scores = torch.empty(Q, k, dtype=torch.float32, device=queries.device)
    _check_out(out_ids, out_scores, Q, k)
    ws, ws_bytes = _workspace_args(workspace)
    rc = lib.ann_rerank(g.handle, m.handle, _queries_ptr(queries, m), Q, _dev_ptr(cand, "cand", torch.int32),
                        cand.shape[1], k, _dev_ptr(out_ids, "out_ids", torch.int32),
                        _dev_ptr(out_scores, "out_scores", torch.float32), ws, ws_bytes, _stream_ptr(stream))
    _check(rc)
    return out_ids, out_scores


def ann_users_add_noise(users: torch.Tensor, sigma: float, seed: int, draw: int = 0,
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """users + sigma * N(0, I) (Eq. 5), same dtype and shape; `out` may be `users`."""
    if users.dim() != 2:
        raise ValueError("users must be [Q][d]")
    if out is None:
        out = torch.empty_like(users)
    if out.shape != users.shape or out.dtype != users.dtype:
        raise ValueError("out must have the shape and dtype of users")
    Q, d = users.shape
    _check(load_library().ann_users_add_noise(_dev_ptr(users, "users") if Q else None, _dev_ptr(out, "out") if Q else None,
                                              Q, d, _dtype_code(users), float(sigma), int(seed), int(draw),
                                              _stream_ptr(stream)))
    return out


def ann_quantize_e4m3(src: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """e4m3(scale * src) as a torch.float8_e4m3fn tensor of the same shape (src: fp32 or bf16, on the device)."""
    if out is None:
        out = torch.empty(src.shape, dtype=torch.float8_e4m3fn, device=src.device)
    if out.shape != src.shape or out.dtype != torch.float8_e4m3fn:
        raise ValueError("out must be float8_e4m3fn with the shape of src")
    code = _dtype_code(src)
    if code == ANN_F8:
        raise TypeError("src must be fp32 or bf16")
    n = src.numel()
    _check(load_library().ann_quantize_e4m3(_dev_ptr(src, "src") if n else None, code, n, float(scale),
                                            _dev_ptr(out, "out") if n else None, _stream_ptr(stream)))
    return out


# ---- the block of a projector: y = x + dropout(ffn(layer_norm(x))) ----
#
# Tensors of one call lie on one device; the call goes to that device's current stream, or to `stream`, a stream of it.
# Results and workspaces that the call makes belong to the stream it goes to; that its inputs are there, and stay until it
# has read them, is the caller's to see to.  Gradients are calls of their own: these functions leave no trace in autograd, also
# where a tensor requires gradients.

_ROW_CODE = {torch.float32: ANN_F32, torch.bfloat16: ANN_BF16, torch.float16: ANN_F16}


def _row_code(t: torch.Tensor, name: str) -> int:
    code = _ROW_CODE.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be fp32, bf16 or fp16, got {t.dtype}")
    return code


def _row_shape(t: torch.Tensor, name: str):
    """(rows, width, row stride) of a [..., width] tensor: dense, or [rows][width] whose rows are."""
    if t.dim() < 1 or t.shape[-1] < 1:
        raise ValueError(f"{name} must be [..., width] with a width of at least 1, got {tuple(t.shape)}")
    d = t.shape[-1]
    if t.is_contiguous():
        return t.numel() // d, d, d
    if t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= d:
        return t.shape[0], d, t.stride(0)
    raise ValueError(f"{name} must be contiguous, or [rows][width] with contiguous rows; strides {t.stride()}")


def _like(t: torch.Tensor, name: str, x: torch.Tensor, shape, dtype=None) -> None:
    """t must have this shape, x's device and type (or `dtype`)."""
    if t.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != (dtype or x.dtype):
        raise TypeError(f"{name} must be {dtype or x.dtype}, got {t.dtype}")
    if t.device != x.device:
        raise ValueError(f"{name} is on {t.device}, the rows are on {x.device}")


def _dense(t: Optional[torch.Tensor], name: str, x: torch.Tensor, shape, dtype=None) -> Optional[int]:
    if t is None:
        return None
    _like(t, name, x, shape, dtype)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _place(x: torch.Tensor, stream):
    """What makes x's device, and `stream` where one is given, the current ones while a call allocates and launches;
    None where they are that already (the usual case, which entering a context would lengthen by microseconds)."""
    if stream is not None:
        if stream.device != x.device:
            raise ValueError(f"stream is on {stream.device}, the rows are on {x.device}")
        return torch.cuda.stream(stream)
    if not x.is_cuda or torch._C._cuda_getDevice() == x.get_device():
        return None
    return torch.cuda.device(x.device)


def _current(x: torch.Tensor) -> int:
    """The current stream of x's device as the library takes it."""
    if not x.is_cuda:
        raise ValueError("the rows must be a device tensor")
    return torch._C._cuda_getCurrentRawStream(x.get_device())


def _row_workspace(workspace: Optional[torch.Tensor], need: int, x: torch.Tensor) -> torch.Tensor:
    """The caller's workspace, or a fresh one."""
    if need == 0:
        raise AnnError(ANN_EINVAL, ann_last_error())
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    elif workspace.device != x.device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {x.device}")
    return workspace


def ann_layer_norm(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                   eps: float = 1e-5, save: bool = False, out: Optional[torch.Tensor] = None, stream=None):
    """Layer norm over the last dimension of x [..., d]; gamma, beta [d] of x's type (None = ones, zeros).  `out` may be
    x.  With save=True (out, mean, rstd), the last two fp32 [rows], for ann_layer_norm_backward; autograd does not see the call."""
    place = _place(x, stream)
    if place is not None:
        with place:
            return ann_layer_norm(x, gamma, beta, eps, save, out)
    code = _row_code(x, "x")
    M, d, ld = _row_shape(x, "x")
    gp, bp = _dense(gamma, "gamma", x, (d,)), _dense(beta, "beta", x, (d,))
    if out is None:
        out, ld_out = torch.empty(x.shape, dtype=x.dtype, device=x.device), d
    else:
        _like(out, "out", x, x.shape)
        ld_out = _row_shape(out, "out")[2]
    mean = rstd = mp = rp = None
    if save:
        mean, rstd = torch.empty((2, M), dtype=torch.float32, device=x.device)
        mp, rp = mean.data_ptr(), rstd.data_ptr()
    rc = load_library().ann_layer_norm(x.data_ptr(), ld, gp, bp, M, d, code, eps, out.data_ptr(), ld_out, mp, rp, _current(x))
    if rc:
        _check(rc)
    return (out, mean, rstd) if save else out


def ann_layer_norm_backward_workspace_bytes(M: int, d: int, dtype: int) -> int:
    n = load_library().ann_layer_norm_backward_workspace_bytes(M, d, dtype)
    if n == 0:
        raise AnnError(ANN_EINVAL, ann_last_error())
    return int(n)


def ann_layer_norm_backward(dout: torch.Tensor, x: torch.Tensor, gamma: Optional[torch.Tensor], mean: torch.Tensor,
                            rstd: torch.Tensor, need_dx: bool = True, need_dparams: bool = True,
                            workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, dgamma, dbeta) of ann_layer_norm(x, gamma, beta, save=True); None for what is not needed."""
    place = _place(x, stream)
    if place is not None:
        with place:
            return ann_layer_norm_backward(dout, x, gamma, mean, rstd, need_dx, need_dparams, workspace)
    code = _row_code(x, "x")
    M, d, ld = _row_shape(x, "x")
    _like(dout, "dout", x, x.shape)
    ld_dout = _row_shape(dout, "dout")[2]
    gp = _dense(gamma, "gamma", x, (d,))
    mp, rp = _dense(mean, "mean", x, (M,), torch.float32), _dense(rstd, "rstd", x, (M,), torch.float32)
    lib = load_library()
    dx = dgamma = dbeta = dgp = dbp = wp = None
    wb = 0
    if need_dx:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if need_dparams:
        dgamma, dbeta = torch.empty((2, d), dtype=x.dtype, device=x.device)
        workspace = _row_workspace(workspace, lib.ann_layer_norm_backward_workspace_bytes(M, d, code), x)
        dgp, dbp, wp, wb = dgamma.data_ptr(), dbeta.data_ptr(), workspace.data_ptr(), workspace.numel()
    rc = lib.ann_layer_norm_backward(dout.data_ptr(), ld_dout, x.data_ptr(), ld, gp, mp, rp, M, d, code,
                                     dx.data_ptr() if need_dx else None, d, dgp, dbp, wp, wb, _current(x))
    if rc:
        _check(rc)
    return dx, dgamma, dbeta


def ann_dropout(x: torch.Tensor, p: float, seed: int, draw: int = 0, residual: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, draw_dev: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """residual + dropout of x (None = no residual), the choice a pure function of (seed, draw, element): the gradient
    of x is ann_dropout(dout, p, seed, draw).  Contiguous tensors of one shape; `out` may be x or residual.  draw_dev
    (one int64 on the device) is added to `draw` when the kernel runs: the replays of a recorded call draw anew.  Autograd does
    not see the call."""
    place = _place(x, stream)
    if place is not None:
        with place:
            return ann_dropout(x, p, seed, draw, residual, out, draw_dev)
    code = _row_code(x, "x")
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    rp = _dense(residual, "residual", x, x.shape)
    dp = None
    if draw_dev is not None:
        if draw_dev.numel() != 1 or draw_dev.device != x.device or draw_dev.dtype not in (torch.int64, torch.uint64):
            raise ValueError(f"draw_dev must be one int64 on {x.device}")
        dp = draw_dev.data_ptr()
    if out is None:
        out = torch.empty_like(x)
        op = out.data_ptr()
    else:
        op = _dense(out, "out", x, x.shape)
    rc = load_library().ann_dropout(x.data_ptr(), rp, op, x.numel(), code, p, seed, draw, dp, _current(x))
    if rc:
        _check(rc)
    return out


def _ffn_shapes(x, w_in, w_out):
    code = _row_code(x, "x")
    M, D, ld = _row_shape(x, "x")
    if w_in.dim() != 2 or w_out.dim() != 2 or w_in.shape[0] != 2 * w_out.shape[1]:
        raise ValueError(f"w_in must be [2 * d_hidden][d_in] and w_out [d_out][d_hidden], got {tuple(w_in.shape)}, "
                         f"{tuple(w_out.shape)}")
    O, F = w_out.shape
    return code, M, D, F, O, ld, _dense(w_in, "w_in", x, (2 * F, D)), _dense(w_out, "w_out", x, (O, F))


def ann_gated_ffn_workspace_bytes(M: int, d_in: int, d_hidden: int, d_out: int, dtype: int) -> int:
    n = load_library().ann_gated_ffn_workspace_bytes(M, d_in, d_hidden, d_out, dtype)
    if n == 0:
        raise AnnError(ANN_EINVAL, ann_last_error())
    return int(n)


def ann_gated_ffn(x: torch.Tensor, w_in: torch.Tensor, w_out: torch.Tensor, b_in: Optional[torch.Tensor] = None,
                  b_out: Optional[torch.Tensor] = None, act: int = ANN_SILU, save: bool = False,
                  out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """(act(gate) * up) w_out^T + b_out with [gate | up] = x w_in^T + b_in: x [..., d_in], w_in [2 * d_hidden][d_in] (the gate's
    rows first), w_out [d_out][d_hidden], all of one type.  With save=True (out, pre), pre [rows][2 * d_hidden] fp32, for
    ann_gated_ffn_backward; autograd does not see the call."""
    place = _place(x, stream)
    if place is not None:
        with place:
            return ann_gated_ffn(x, w_in, w_out, b_in, b_out, act, save, out, workspace)
    code, M, D, F, O, ld, wip, wop = _ffn_shapes(x, w_in, w_out)
    bip, bop = _dense(b_in, "b_in", x, (2 * F,)), _dense(b_out, "b_out", x, (O,))
    shape, ld_out = x.shape[:-1] + (O,), O
    if out is None:
        out = torch.empty(shape, dtype=x.dtype, device=x.device)
    else:
        _like(out, "out", x, shape)
        ld_out = _row_shape(out, "out")[2]
    lib = load_library()
    pre = torch.empty((M, 2 * F), dtype=torch.float32, device=x.device) if save else None
    workspace = _row_workspace(workspace, lib.ann_gated_ffn_workspace_bytes(M, D, F, O, code), x)
    rc = lib.ann_gated_ffn(x.data_ptr(), ld, wip, bip, wop, bop, M, D, F, O, act, code, out.data_ptr(), ld_out,
                           pre.data_ptr() if save else None, workspace.data_ptr(), workspace.numel(), _current(x))
    if rc:
        _check(rc)
    return (out, pre) if save else out


def ann_gated_ffn_backward_workspace_bytes(M: int, d_in: int, d_hidden: int, d_out: int, dtype: int) -> int:
    n = load_library().ann_gated_ffn_backward_workspace_bytes(M, d_in, d_hidden, d_out, dtype)
    if n == 0:
        raise AnnError(ANN_EINVAL, ann_last_error())
    return int(n)


def ann_gated_ffn_backward(dout: torch.Tensor, x: torch.Tensor, pre: torch.Tensor, w_in: torch.Tensor,
                           w_out: torch.Tensor, act: int = ANN_SILU, bias: bool = False, need_dx: bool = True,
                           need_dw: bool = True, workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, dw_in, dw_out, db_in, db_out) of ann_gated_ffn(..., save=True); None for what is not needed (the last two
    are given with bias=True)."""
    place = _place(x, stream)
    if place is not None:
        with place:
            return ann_gated_ffn_backward(dout, x, pre, w_in, w_out, act, bias, need_dx, need_dw, workspace)
    code, M, D, F, O, ld, wip, wop = _ffn_shapes(x, w_in, w_out)
    _like(dout, "dout", x, x.shape[:-1] + (O,))
    ld_dout = _row_shape(dout, "dout")[2]
    pp = _dense(pre, "pre", x, (M, 2 * F), torch.float32)
    lib = load_library()
    new = lambda *shape: torch.empty(shape, dtype=x.dtype, device=x.device)  # noqa: E731
    dx = new(*x.shape) if need_dx else None
    dw_in, dw_out = (new(2 * F, D), new(O, F)) if need_dw else (None, None)
    db_in, db_out = (new(2 * F), new(O)) if bias else (None, None)
    workspace = _row_workspace(workspace, lib.ann_gated_ffn_backward_workspace_bytes(M, D, F, O, code), x)
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    rc = lib.ann_gated_ffn_backward(dout.data_ptr(), ld_dout, x.data_ptr(), ld, pp, wip, wop, M, D, F, O, act, code,
                                    ptr(dx), D, ptr(dw_in), ptr(db_in), ptr(dw_out), ptr(db_out),
                                    workspace.data_ptr(), workspace.numel(), _current(x))
    if rc:
        _check(rc)
    return dx, dw_in, dw_out, db_in, db_out


def ann_search_stats(workspace: torch.Tensor, stream=None) -> Stats:
    st = Stats()
    _check(load_library().ann_search_stats(_dev_ptr(workspace, "workspace", torch.uint8), ctypes.byref(st),
                                           _stream_ptr(stream)))
    return st


def ann_set_progress_timeout(seconds: float) -> None:
    _check(load_library().ann_set_progress_timeout(float(seconds)))


STAGES = ("score", "round", "pack")


def ann_profile_enable(on: bool) -> None:
    _check(load_library().ann_profile_enable(1 if on else 0))


def ann_profile_read() -> dict:
    """{stage: (milliseconds, launches)} since the last read."""
    ms = (ctypes.c_double * len(STAGES))()
    n = (ctypes.c_int64 * len(STAGES))()
    _check(load_library().ann_profile_read(ms, n))
    return {name: (float(ms[i]), int(n[i])) for i, name in enumerate(STAGES)}


def ann_profile_copy(dst: torch.Tensor, src: torch.Tensor, stream=None) -> None:
    """Reference copy of known size for hardware traffic counters (dst, src: same-size device tensors)."""
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("dst and src must have the same size")
    _check(load_library().ann_profile_copy(_dev_ptr(dst, "dst"), _dev_ptr(src, "src"), nbytes, _stream_ptr(stream)))
