"""The calls of nats_serve.h refuse written arrays that share memory with anything else of the call, before anything is launched.
(Host-side checks on addresses; nothing is read there.)"""
import ctypes

import pytest

from paper_2602_03681_amd import binding as nb
from paper_2602_03681_amd import serve

E_SHAPE = -2
B, H, G, T, d, cap, keep = 2, 3, 2, 8, 64, 100, 20
HG = H * G
ROWS = dict(k_cache=2 * B * HG * cap * d, v_cache=2 * B * HG * cap * d, cache_len=4 * B * HG)
NODES = dict(q=2 * B * H * T * d, k=2 * B * H * T * d, v=2 * B * HG * T * d, alpha=4 * B * H * T, beta=4 * B * H * T, mask=B * H * T,
             parent=4 * B * T, n_nodes=4 * B, q_nla=2 * B * HG * T * d, k_nla=2 * B * HG * T * d)
TREE = dict(state=4 * B * HG * d * d, **ROWS, **NODES, w_nla=4 * B * HG * T, w_la=4 * B * HG * T, o=2 * B * HG * T * d, lse=4 * B * HG * T)
COMMIT = dict(state=4 * B * HG * d * d, **ROWS, **{k: n for k, n in NODES.items() if k not in ("q", "q_nla")}, node=4 * B,
              vis=4 * B * HG * T, err_flags=4 * B * HG)
WEIGHTS = dict(weights=4 * B * HG * cap, q=2 * B * H * T * d, k_cache=ROWS["k_cache"], cache_len=4 * B * HG, vis=4 * B * H * T,
               lse=4 * B * HG * T)
EVICT = dict(**ROWS, weights=4 * B * HG * cap, kept=4 * B * HG * keep)


def places(sizes, move):
    at = {k: (i + 1) << 28 for i, k in enumerate(list(sizes) + ["workspace"])}
    at.update({k: f(at) for k, f in move.items()})
    return at


def tree(move):
    lib, p = nb.load_library(), serve.TreeParams()
    at = places(TREE, move)
    for k, x in dict(B=B, H=H, T=T, d=d, cap=cap, dtype=nb.NATS_BF16, group=G, q_nla=at["q_nla"], k_nla=at["k_nla"]).items():
        setattr(p, k, x)
    n = lib.nats_hybrid_attn_decode_tree_workspace_bytes(ctypes.byref(p))
    args = ("state", "k_cache", "v_cache", "cache_len", "q", "k", "v", "alpha", "beta", "mask", "parent", "n_nodes", "w_nla", "w_la", "o",
            "lse", "workspace")
    return lib.nats_hybrid_attn_decode_tree(ctypes.byref(p), *(at[k] for k in args), n, None), lib.nats_last_error().decode()


def commit(move):
    lib, p = nb.load_library(), serve.TreeParams()
    at = places(COMMIT, move)
    for k, x in dict(B=B, H=H, T=T, d=d, cap=cap, dtype=nb.NATS_BF16, group=G, k_nla=at["k_nla"]).items():
        setattr(p, k, x)
    args = ("state", "k_cache", "v_cache", "cache_len", "k", "v", "alpha", "beta", "mask", "parent", "n_nodes", "node", "vis", "err_flags")
    return lib.nats_hybrid_attn_tree_commit_ex(ctypes.byref(p), *(at[k] for k in args), None), lib.nats_last_error().decode()


def weights(move):
    lib, p = nb.load_library(), serve.CacheWeightsParams(B, HG, T, d, cap, nb.NATS_BF16, G, G, 0.0, 1.0)
    at = places(WEIGHTS, move)
    return (lib.nats_cache_weights(ctypes.byref(p), *(at[k] for k in (*WEIGHTS, "workspace")), 1 << 20, None),
            lib.nats_last_error().decode())


def evict(move, clear=False):
    lib, p = nb.load_library(), serve.CacheEvictParams(B, HG, d, cap, nb.NATS_BF16, keep, 5)
    at = places(EVICT, move)
    call = lib.nats_cache_evict_clear if clear else lib.nats_cache_evict
    return call(ctypes.byref(p), *(at[k] for k in EVICT), None), lib.nats_last_error().decode()


def evict_clear(move):
    return evict(move, True)


WRITTEN = {tree: (TREE, ("o", "lse")), commit: (COMMIT, ("state", "k_cache", "v_cache", "cache_len", "vis", "err_flags")),
           weights: (WEIGHTS, ("weights",)), evict: (EVICT, tuple(EVICT)), evict_clear: (EVICT, tuple(EVICT))}
PAIRS = [(call, a, b) for call, (sizes, written) in WRITTEN.items() for a in written for b in sizes if a != b]


def up16(n):
    return (n + 15) // 16 * 16


@pytest.mark.parametrize("call,a,b", PAIRS)
def test_overlaps_are_refused(call, a, b):
    n = WRITTEN[call][0]
    # the same place; a's first bytes in b's last 16; b's first in a's last 16
    for shift in (0, up16(n[b]) - 16, 16 - up16(n[a])):
        st, msg = call({a: lambda at: at[b] + shift})
        assert st == E_SHAPE and ("share memory" in msg or "alias" in msg or "two arrays" in msg), (shift, st, msg)


@pytest.mark.parametrize("a", list(TREE))
def test_the_trees_workspace_is_an_array_of_its_own(a):
    for shift in (0, 4096, 16 - up16(TREE[a])):
        st, msg = tree({a: lambda at: at["workspace"] + shift})
        assert st == E_SHAPE and "workspace" in msg, (shift, st, msg)


@pytest.mark.parametrize("a", list(WEIGHTS))
def test_the_weights_workspace_is_an_array_of_its_own(a):
    """(as far as the call uses it: without lse its maxima, sums and logits)"""
    lib, p = nb.load_library(), serve.CacheWeightsParams(B, HG, T, d, cap, nb.NATS_BF16, G, G, 0.0, 1.0)
    n = lib.nats_cache_weights_workspace_bytes(ctypes.byref(p), 0)
    at = places(WEIGHTS, {a: lambda at: at["workspace"] + n - 16})
    if a == "lse":
        return
    at["lse"] = None
    st = lib.nats_cache_weights(ctypes.byref(p), *(at[k] for k in (*WEIGHTS, "workspace")), 1 << 20, None)
    assert st == E_SHAPE and b"workspace" in lib.nats_last_error()
