"""Binding of include/nats_serve.h: a tree of drafted tokens read against the decode state and the cache, the commit of its
accepted path, the attention weights that the cache's rows get, and the eviction by them.

Argument marshalling only, as in binding.py; tensors must be on torch's current device, work goes on torch's current stream.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import binding as nb
from .binding import NATS_LINEAR_GDN, _check, _dtype_code, _ptr, _require, _require_workspace, _stream_ptr

MAX_NODES = 64   # NATS_TREE_MAX_NODES


class TreeParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("T", ctypes.c_int32), ("d", ctypes.c_int32),
                ("cap", ctypes.c_int32), ("dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("la_scale", ctypes.c_float), ("combine_mode", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("linear_op", ctypes.c_int32), ("freeze_on_softmax", ctypes.c_int32), ("group", ctypes.c_int32),
                ("q_nla", ctypes.c_void_p), ("k_nla", ctypes.c_void_p)]


class CacheWeightsParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("T", ctypes.c_int32), ("d", ctypes.c_int32),
                ("cap", ctypes.c_int32), ("dtype", ctypes.c_int32), ("q_group", ctypes.c_int32),
                ("vis_group", ctypes.c_int32), ("softmax_scale", ctypes.c_float), ("decay", ctypes.c_float)]


class CacheEvictParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32), ("cap", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("keep", ctypes.c_int32), ("recent", ctypes.c_int32)]


def declare(lib) -> None:
    """Argument types of the entry points; called where the library is loaded."""
    vp, size = ctypes.c_void_p, ctypes.c_size_t
    lib.nats_hybrid_attn_decode_tree_workspace_bytes.restype = size
    lib.nats_hybrid_attn_decode_tree_workspace_bytes.argtypes = [ctypes.POINTER(TreeParams)]
    lib.nats_hybrid_attn_decode_tree.restype = ctypes.c_int
    lib.nats_hybrid_attn_decode_tree.argtypes = [ctypes.POINTER(TreeParams)] + [vp] * 17 + [size, vp]
    lib.nats_hybrid_attn_tree_commit.restype = ctypes.c_int
    lib.nats_hybrid_attn_tree_commit.argtypes = [ctypes.POINTER(TreeParams)] + [vp] * 14
    lib.nats_hybrid_attn_tree_commit_ex.restype = ctypes.c_int
    lib.nats_hybrid_attn_tree_commit_ex.argtypes = [ctypes.POINTER(TreeParams)] + [vp] * 15
    lib.nats_cache_weights_workspace_bytes.restype = size
    lib.nats_cache_weights_workspace_bytes.argtypes = [ctypes.POINTER(CacheWeightsParams), ctypes.c_int32]
    lib.nats_cache_weights.restype = ctypes.c_int
    lib.nats_cache_weights.argtypes = [ctypes.POINTER(CacheWeightsParams)] + [vp] * 7 + [size, vp]
    for evict in (lib.nats_cache_evict, lib.nats_cache_evict_clear):
        evict.restype = ctypes.c_int
        evict.argtypes = [ctypes.POINTER(CacheEvictParams)] + [vp] * 6


def _require_here(*tensors: Optional[torch.Tensor]) -> None:
    for t in tensors:
        if t is not None and t.is_cuda and t.device.index != torch.cuda.current_device():
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{torch.cuda.current_device()}")


def _cache_shape(k_cache):
    if k_cache.dim() != 4:
        raise ValueError(f"k_cache must have 4 dimensions, got {tuple(k_cache.shape)}")
    return k_cache.shape


def _tree_shape(k, k_cache, group):
    """(B, H, T, d, cap, H * group)"""
    B, HG, cap, d = _cache_shape(k_cache)
    if k.dim() != 4:
        raise ValueError(f"k must have 4 dimensions, got {tuple(k.shape)}")
    H, T = k.shape[1], k.shape[2]
    if group < 1 or H * group != HG:
        raise ValueError(f"{HG} heads of the cache are not group {group} times the {H} of k")
    return B, H, T, d, cap, HG


def decode_tree_workspace_bytes(B, H, T, d, cap, dtype_code, group: int = 1) -> int:
    """nats_hybrid_attn_decode_tree_workspace_bytes."""
    p = TreeParams(B, H, T, d, cap, dtype_code, 0.0, 0.0, 0, 0.0, 0, 0, group, None, None)
    return int(nb.load_library().nats_hybrid_attn_decode_tree_workspace_bytes(ctypes.byref(p)))


def hybrid_attn_decode_tree(state, k_cache, v_cache, cache_len, q, k, v, alpha, beta, mask, parent, *, n_nodes=None,
                            softmax_scale: float = 0.0, la_scale: float = 0.0, combine_mode: int = 0, rms_eps: float = 0.0,
                            linear_op: int = NATS_LINEAR_GDN, freeze_on_softmax: bool = False, q_nla=None, k_nla=None,
                            w_nla=None, w_la=None, group: int = 1, out=None, lse=None, workspace=None):
    """nats_hybrid_attn_decode_tree: a tree of T <= 64 drafted tokens per sequence (parent [B,T] i32; -1: follows the last
    committed token) read against state and cache, which stay as they are -> (o [B,H*G,T,d], lse [B,H*G,T] f32).  q, k
    [B,H,T,d], alpha, beta, mask [B,H,T]; everything else has H * group heads.  n_nodes [B] i32: nodes from there on give rows
    of 0 and lse -inf.  workspace: uint8 tensor of decode_tree_workspace_bytes(...) bytes, allocated for the call if None."""
    lib = nb.load_library()
    r = nb._host.decode_tree(state, k_cache, v_cache, cache_len, q, k, v, alpha, beta, mask, parent, n_nodes, q_nla, k_nla, w_nla,
                             w_la, out, lse, workspace, softmax_scale, la_scale, combine_mode, rms_eps, linear_op, freeze_on_softmax,
                             group)
    if r is not None:
        if type(r) is int:
            _check(r)
        return r
    # an argument that the host path does not take: the checks below say which
    B, H, T, d, cap, HG = _tree_shape(k, k_cache, group)
    dt = k_cache.dtype
    _require(state, "state", (B, HG, d, d), torch.float32)
    _require(k_cache, "k_cache", (B, HG, cap, d), dt)
    _require(v_cache, "v_cache", (B, HG, cap, d), dt)
    _require(cache_len, "cache_len", (B, HG), torch.int32)
    _require(q, "q", (B, H, T, d), dt)
    _require(k, "k", (B, H, T, d), dt)
    _require(v, "v", (B, HG, T, d), dt)
    _require(alpha, "alpha", (B, H, T), torch.float32)
    _require(beta, "beta", (B, H, T), torch.float32)
    _require(mask, "mask", (B, H, T), torch.uint8)
    _require(parent, "parent", (B, T), torch.int32)
    _require(n_nodes, "n_nodes", (B,), torch.int32)
    _require(q_nla, "q_nla", (B, HG, T, d), dt)
    _require(k_nla, "k_nla", (B, HG, T, d), dt)
    _require(w_nla, "w_nla", (B, HG, T), torch.float32)
    _require(w_la, "w_la", (B, HG, T), torch.float32)
    _require_here(state, k_cache, v_cache, cache_len, q, k, v, alpha, beta, mask, parent, n_nodes, q_nla, k_nla, w_nla, w_la, out,
                  lse, workspace)
    p = TreeParams(B, H, T, d, cap, _dtype_code(k_cache), softmax_scale, la_scale, combine_mode, rms_eps, linear_op,
                   int(freeze_on_softmax), group, q_nla.data_ptr() if q_nla is not None else None,
                   k_nla.data_ptr() if k_nla is not None else None)
    o = torch.empty_like(v) if out is None else out
    _require(o, "out", (B, HG, T, d), dt)
    lse = torch.empty((B, HG, T), dtype=torch.float32, device=v.device) if lse is None else lse
    _require(lse, "lse", (B, HG, T), torch.float32)
    if workspace is None:
        need = int(lib.nats_hybrid_attn_decode_tree_workspace_bytes(ctypes.byref(p)))
        workspace = torch.empty(need, dtype=torch.uint8, device=v.device)
    _require_workspace(workspace)
    _check(lib.nats_hybrid_attn_decode_tree(ctypes.byref(p), _ptr(state), _ptr(k_cache), _ptr(v_cache), _ptr(cache_len), _ptr(q),
                                            _ptr(k), _ptr(v), _ptr(alpha), _ptr(beta), _ptr(mask), _ptr(parent), _ptr(n_nodes),
                                            _ptr(w_nla), _ptr(w_la), _ptr(o), _ptr(lse), _ptr(workspace), workspace.numel(),
                                            _stream_ptr()))
    return o, lse


def hybrid_attn_tree_commit(state, k_cache, v_cache, cache_len, k, v, alpha, beta, mask, parent, node, *,
                            linear_op: int = NATS_LINEAR_GDN, freeze_on_softmax: bool = False, k_nla=None, group: int = 1,
                            err_flags=None, vis=None, n_nodes=None) -> torch.Tensor:
    """nats_hybrid_attn_tree_commit: the path to node [B] i32 (-1: nothing) is written into state, caches and cache_len, in place
    -> vis [B,H*G,T] i32, the rows of the cache that each node of the path saw (0: not on the path).  n_nodes [B] i32, for padded
    trees (nats_hybrid_attn_tree_commit_ex): a node from there on is none, like a number outside -1 .. T - 1 (err_flags: 2)."""
    lib = nb.load_library()
    r = nb._host.tree_commit(state, k_cache, v_cache, cache_len, k, v, alpha, beta, mask, parent, node, n_nodes, k_nla, vis, err_flags,
                             linear_op, freeze_on_softmax, group)
    if r is not None:
        if type(r) is int:
            _check(r)
        return r
    B, H, T, d, cap, HG = _tree_shape(k, k_cache, group)
    dt = k_cache.dtype
    _require(state, "state", (B, HG, d, d), torch.float32)
    _require(k_cache, "k_cache", (B, HG, cap, d), dt)
    _require(v_cache, "v_cache", (B, HG, cap, d), dt)
    _require(cache_len, "cache_len", (B, HG), torch.int32)
    _require(k, "k", (B, H, T, d), dt)
    _require(v, "v", (B, HG, T, d), dt)
    _require(alpha, "alpha", (B, H, T), torch.float32)
    _require(beta, "beta", (B, H, T), torch.float32)
    _require(mask, "mask", (B, H, T), torch.uint8)
    _require(parent, "parent", (B, T), torch.int32)
    _require(node, "node", (B,), torch.int32)
    _require(n_nodes, "n_nodes", (B,), torch.int32)
    _require(k_nla, "k_nla", (B, HG, T, d), dt)
    _require(err_flags, "err_flags", (B, HG), torch.int32)
    vis = torch.empty((B, HG, T), dtype=torch.int32, device=v.device) if vis is None else vis
    _require(vis, "vis", (B, HG, T), torch.int32)
    _require_here(state, k_cache, v_cache, cache_len, k, v, alpha, beta, mask, parent, node, n_nodes, k_nla, err_flags, vis)
    p = TreeParams(B, H, T, d, cap, _dtype_code(k_cache), 0.0, 0.0, 0, 0.0, linear_op, int(freeze_on_softmax), group, None,
                   k_nla.data_ptr() if k_nla is not None else None)
    _check(lib.nats_hybrid_attn_tree_commit_ex(ctypes.byref(p), _ptr(state), _ptr(k_cache), _ptr(v_cache), _ptr(cache_len), _ptr(k),
                                               _ptr(v), _ptr(alpha), _ptr(beta), _ptr(mask), _ptr(parent), _ptr(n_nodes), _ptr(node),
                                               _ptr(vis), _ptr(err_flags), _stream_ptr()))
    return vis


def cache_weights(weights, q, k_cache, cache_len, *, lse=None, vis=None, softmax_scale: float = 0.0, decay: float = 1.0,
                  workspace=None) -> torch.Tensor:
    """nats_cache_weights: weights [B,H,cap] f32 <- decay * weights + the attention weight that the queries q [B,Hq,T,d] give to the
    rows of the cache, in place.  Hq divides H (a query head serves H / Hq heads of the cache in a row), so does the number of heads
    of vis [B,Hv,T] i32 (rows that a query sees; None: all).  lse [B,H,T] f32: None: taken over the rows that a query sees.
    A row that is appended later starts with what stands in weights at its place: 0, in an array of zeros that evictions clear."""
    lib = nb.load_library()
    r = nb._host.cache_weights(weights, q, k_cache, cache_len, lse, vis, workspace, softmax_scale, decay)
    if r is not None:
        if type(r) is int:
            _check(r)
        return r
    B, H, cap, d = _cache_shape(k_cache)
    dt = k_cache.dtype
    if q.dim() != 4 or q.shape[1] == 0 or H % q.shape[1]:
        raise ValueError(f"q must have 4 dimensions and a number of heads that divides {H}, got {tuple(q.shape)}")
    Hq, T = q.shape[1], q.shape[2]
    Hv = H if vis is None else vis.shape[1] if vis.dim() == 3 else 0
    if Hv == 0 or H % Hv:
        raise ValueError(f"vis must have 3 dimensions and a number of heads that divides {H}, got {tuple(vis.shape)}")
    _require(weights, "weights", (B, H, cap), torch.float32)
    _require(q, "q", (B, Hq, T, d), dt)
    _require(k_cache, "k_cache", (B, H, cap, d), dt)
    _require(cache_len, "cache_len", (B, H), torch.int32)
    _require(vis, "vis", (B, Hv, T), torch.int32)
    _require(lse, "lse", (B, H, T), torch.float32)
    _require_here(weights, q, k_cache, cache_len, vis, lse, workspace)
    p = CacheWeightsParams(B, H, T, d, cap, _dtype_code(k_cache), H // Hq, H // Hv, softmax_scale, decay)
    if workspace is None:
        need = int(lib.nats_cache_weights_workspace_bytes(ctypes.byref(p), int(lse is not None)))
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    _require_workspace(workspace)
    _check(lib.nats_cache_weights(ctypes.byref(p), _ptr(weights), _ptr(q), _ptr(k_cache), _ptr(cache_len), _ptr(vis), _ptr(lse),
                                  _ptr(workspace), workspace.numel(), _stream_ptr()))
    return weights


def cache_evict(k_cache, v_cache, cache_len, weights, keep: int, recent: int = 0, *, kept=None,
                clear_weights: bool = False) -> torch.Tensor:
    """nats_cache_evict: caches of more than `keep` rows keep their last `recent` rows and the heaviest of the others, in order and in
    place (k_cache, v_cache, weights, cache_len) -> kept [B,H,keep] i32, the row that each row was before (-1: no row).

    clear_weights: the weights of the rows that are given up become 0 (nats_cache_evict_clear).  Wanted wherever weights go on being
    added up while rows are appended; without it a new row starts with the weight of the one that lay in its place."""
    lib = nb.load_library()
    r = nb._host.cache_evict(k_cache, v_cache, cache_len, weights, kept, keep, recent, clear_weights)
    if r is not None:
        if type(r) is int:
            _check(r)
        return r
    B, H, cap, d = _cache_shape(k_cache)
    dt = k_cache.dtype
    _require(k_cache, "k_cache", (B, H, cap, d), dt)
    _require(v_cache, "v_cache", (B, H, cap, d), dt)
    _require(cache_len, "cache_len", (B, H), torch.int32)
    _require(weights, "weights", (B, H, cap), torch.float32)
    keep, recent = (max(-1, min(n, cap + 1)) for n in (keep, recent))   # (what is out of range is so in 32 bits, too)
    rows = max(0, min(keep, cap))
    kept = torch.empty((B, H, rows), dtype=torch.int32, device=k_cache.device) if kept is None else kept
    _require(kept, "kept", (B, H, rows), torch.int32)
    _require_here(k_cache, v_cache, cache_len, weights, kept)
    p = CacheEvictParams(B, H, d, cap, _dtype_code(k_cache), keep, recent)
    evict = lib.nats_cache_evict_clear if clear_weights else lib.nats_cache_evict
    _check(evict(ctypes.byref(p), _ptr(k_cache), _ptr(v_cache), _ptr(cache_len), _ptr(weights), _ptr(kept), _stream_ptr()))
    return kept
