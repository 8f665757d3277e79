"""The operators of nats_serve.h from their definitions, on the CPU in 64 bits, and inputs for them."""
import math

import torch


def tree_inputs(B, H, T, d, cap, dtype, seed, G=1, p=0.3, tree="tree", own_qk=False, lens=None, weights=False, device="cpu"):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)                                        # noqa: E731
    unit = lambda *s: torch.nn.functional.normalize(rnd(*s), dim=-1).to(dtype)           # noqa: E731
    HG = H * G
    x = dict(state=0.3 * rnd(B, HG, d, d), k_cache=rnd(B, HG, cap, d).to(dtype), v_cache=rnd(B, HG, cap, d).to(dtype),
             cache_len=torch.randint(0, cap + 1, (B, HG), generator=g, dtype=torch.int32) if lens is None
             else torch.tensor(lens, dtype=torch.int32).expand(B, HG).contiguous(),
             q=unit(B, H, T, d), k=unit(B, H, T, d), v=rnd(B, HG, T, d).to(dtype), alpha=torch.sigmoid(2 + 0.5 * rnd(B, H, T)),
             beta=torch.sigmoid(rnd(B, H, T)), mask=(torch.rand(B, H, T, generator=g) < p).to(torch.uint8))
    at = torch.arange(T)
    if tree == "chain":
        parent = (at - 1).expand(B, T)
    elif tree == "star":
        parent = torch.full((B, T), -1)
    else:
        parent = (torch.rand(B, T, generator=g) * (at + 1)).floor() - 1
    x["parent"] = parent.to(torch.int32).contiguous()
    if own_qk:
        x["q_nla"], x["k_nla"] = rnd(B, HG, T, d).to(dtype), rnd(B, HG, T, d).to(dtype)
    if weights:
        x["w_nla"], x["w_la"] = torch.rand(B, HG, T, generator=g), torch.rand(B, HG, T, generator=g)
    return {k: v.to(device) for k, v in x.items()}


def path_of(parent, i):
    """From the first token behind the committed ones to node i; a parent that is no earlier node counts as -1."""
    path = []
    while i >= 0:
        path.insert(0, i)
        up = int(parent[i])
        i = up if 0 <= up < i else -1
    return path


def _step(S, a, b, k, v, linear_op):
    S = a * S
    if b != 0:
        S = S + b * torch.outer(v - (S @ k if linear_op == 0 else 0), k)
    return S


def _merge(o_la, o_nla, wn, wl, mode, eps):
    norm = lambda x: x / math.sqrt(float((x * x).mean()) + eps)   # noqa: E731
    if mode == 0:
        return o_la + o_nla
    return wn * norm(o_nla) + wl * norm(o_la) if mode == 1 else norm(wn * o_nla + wl * o_la)


def decode_tree(x, G=1, combine_mode=0, linear_op=0, freeze_on_softmax=False, softmax_scale=0.0, la_scale=0.0, rms_eps=0.0,
                n_nodes=None):
    """(o, lse) in 64 bits: every node on its own, from the tokens of its path alone."""
    x = {k: v.cpu() for k, v in x.items()}
    B, HG, cap, d = x["k_cache"].shape
    T = x["k"].shape[2]
    scale, la = softmax_scale or d ** -0.5, la_scale or 1.0
    o = torch.zeros(B, HG, T, d, dtype=torch.float64)
    lse = torch.full((B, HG, T), -math.inf, dtype=torch.float64)
    qn, kn = x.get("q_nla"), x.get("k_nla")
    for b in range(B):
        for h in range(HG):
            l = h // G
            n = min(max(int(x["cache_len"][b, h]), 0), cap)
            K, V = x["k_cache"][b, h, :n].double(), x["v_cache"][b, h, :n].double()
            states = {}
            for t in range(T):
                if n_nodes is not None and t >= int(n_nodes[b]):
                    continue
                path = path_of(x["parent"][b], t)
                soft = bool(x["mask"][b, l, t])
                a = 1.0 if soft and freeze_on_softmax else float(x["alpha"][b, l, t])
                S = states[path[-2]] if len(path) > 1 else x["state"][b, h].double()
                S = _step(S, a, 0.0 if soft else float(x["beta"][b, l, t]), x["k"][b, l, t].double(), x["v"][b, h, t].double(), linear_op)
                states[t] = S
                o_la = la * (S @ x["q"][b, l, t].double())
                seen = [j for j in path if x["mask"][b, l, j]]
                keys = (kn[b, h, seen] if kn is not None else x["k"][b, l, seen]).double()
                q = (qn[b, h, t] if qn is not None else x["q"][b, l, t]).double()
                logits = scale * torch.cat([K, keys]) @ q
                o_nla = torch.zeros(d, dtype=torch.float64)
                if len(logits):
                    lse[b, h, t] = torch.logsumexp(logits, 0)
                    o_nla = torch.softmax(logits, 0) @ torch.cat([V, x["v"][b, h, seen].double()])
                default = 0.5 if combine_mode == 1 else 1.0
                wn = float(x["w_nla"][b, h, t]) if "w_nla" in x else default
                wl = float(x["w_la"][b, h, t]) if "w_la" in x else default
                o[b, h, t] = _merge(o_la, o_nla, wn, wl, combine_mode, rms_eps or 1e-6)
    return o, lse


def tree_commit(x, node, G=1, linear_op=0, freeze_on_softmax=False):
    """dict of state (64 bits), k_cache, v_cache, cache_len, vis, err_flags behind the call."""
    x = {k: v.cpu().clone() for k, v in x.items()}
    B, HG, cap, d = x["k_cache"].shape
    T = x["k"].shape[2]
    state, vis = x["state"].double(), torch.zeros(B, HG, T, dtype=torch.int32)
    err = torch.zeros(B, HG, dtype=torch.int32)
    keys = x.get("k_nla")
    for b in range(B):
        bad = not -1 <= int(node[b]) < T
        err[b] = 2 if bad else 0
        for t in path_of(x["parent"][b], -1 if bad else int(node[b])):
            for h in range(HG):
                l = h // G
                soft = bool(x["mask"][b, l, t])
                a = 1.0 if soft and freeze_on_softmax else float(x["alpha"][b, l, t])
                state[b, h] = _step(state[b, h], a, 0.0 if soft else float(x["beta"][b, l, t]), x["k"][b, l, t].double(),
                                    x["v"][b, h, t].double(), linear_op)
                n = int(x["cache_len"][b, h])
                if soft and 0 <= n < cap:
                    x["k_cache"][b, h, n] = keys[b, h, t] if keys is not None else x["k"][b, l, t]
                    x["v_cache"][b, h, n] = x["v"][b, h, t]
                    x["cache_len"][b, h] += 1
                elif soft:
                    err[b, h] = 1
                vis[b, h, t] = min(max(int(x["cache_len"][b, h]), 0), cap)
    return dict(state=state, k_cache=x["k_cache"], v_cache=x["v_cache"], cache_len=x["cache_len"], vis=vis, err_flags=err)


def cache_weights(weights, q, k_cache, cache_len, lse=None, vis=None, softmax_scale=0.0, decay=1.0):
    """(weights in 64 bits, lse that was used)"""
    weights, q, k_cache, cache_len = weights.cpu().double(), q.cpu(), k_cache.cpu(), cache_len.cpu()
    B, H, cap, d = k_cache.shape
    T, gq = q.shape[2], H // q.shape[1]
    used = torch.full((B, H, T), -math.inf, dtype=torch.float64)
    for b in range(B):
        for h in range(H):
            n = min(max(int(cache_len[b, h]), 0), cap)
            x = (softmax_scale or d ** -0.5) * q[b, h // gq].double() @ k_cache[b, h, :n].double().t()
            if vis is not None:
                rows = vis[b, h // (H // vis.shape[1])].cpu().clamp(0, n)
                x = torch.where(torch.arange(n) < rows[:, None], x, -math.inf)
            used[b, h] = torch.logsumexp(x, 1) if lse is None else lse[b, h].cpu().double()
            p = torch.where((used[b, h] == -math.inf)[:, None] | (x == -math.inf), 0.0, (x - used[b, h][:, None]).exp())
            weights[b, h, :n] = decay * weights[b, h, :n] + p.sum(0)
    return weights, used


def cache_evict(k_cache, v_cache, cache_len, weights, keep, recent):
    k_cache, v_cache, cache_len, weights = (t.cpu().clone() for t in (k_cache, v_cache, cache_len, weights))
    B, H, cap, d = k_cache.shape
    kept = torch.full((B, H, keep), -1, dtype=torch.int32)
    for b in range(B):
        for h in range(H):
            n = min(max(int(cache_len[b, h]), 0), cap)
            rows = list(range(n))
            if n > keep:
                w = weights[b, h].tolist()
                order = sorted(rows[:n - recent], key=lambda r: (math.isnan(w[r]), -w[r] if w[r] == w[r] else 0.0, r))
                rows = sorted(order[:keep - recent]) + rows[n - recent:]
                for t in (k_cache, v_cache, weights):
                    t[b, h, :keep] = t[b, h, rows].clone()
                cache_len[b, h] = keep
            kept[b, h, :len(rows)] = torch.tensor(rows, dtype=torch.int32)
    return dict(k_cache=k_cache, v_cache=v_cache, cache_len=cache_len, weights=weights, kept=kept)
