"""cache_weights and cache_evict against their definitions in 64 bits.

A weight is a sum of exp(logit - lse): a logit is off by at most d 2^-24 of the sum of its products' sizes (128 * 0.64 * 0.0884 = 7.3),
5.5e-5, and so is, relative to itself, each term; the sum over T terms adds T 2^-24 at most, 1.2e-4 at T 2000."""
import math

import pytest
import torch

import paper_2602_03681_amd as nats
import serve_reference as ref

pytestmark = pytest.mark.gpu
TOL = 5.5e-5 + 1.2e-4
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def inputs(B, H, T, d, cap, dtype, seed, Hq=None, lens=None):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    lens = torch.randint(0, cap + 1, (B, H), generator=g, dtype=torch.int32) if lens is None else torch.tensor(lens, dtype=torch.int32).expand(B, H).contiguous()
    return dict(weights=torch.rand(B, H, cap, generator=g), q=rnd(B, Hq or H, T, d).to(dtype), k_cache=rnd(B, H, cap, d).to(dtype),
                cache_len=lens)


def check(x, **kw):
    g = {k: v.cuda() for k, v in x.items()}
    same = {k: g[k].clone() for k in ("q", "k_cache", "cache_len")}
    got = nats.cache_weights(g["weights"], g["q"], g["k_cache"], g["cache_len"],
                             **{k: v.cuda() if torch.is_tensor(v) else v for k, v in kw.items()})
    want, _ = ref.cache_weights(**x, **kw)
    assert got.data_ptr() == g["weights"].data_ptr()
    cap = x["k_cache"].shape[2]
    behind = torch.arange(cap) >= x["cache_len"][..., None]
    assert torch.equal(got.cpu()[behind], x["weights"][behind])          # rows behind the cache's end are left alone
    off = (got.cpu().double() - want).abs() / want.abs().clamp_min(1e-30)
    assert float(torch.where(behind, 0.0, off).max()) <= TOL
    assert all(torch.equal(g[k], same[k]) for k in same)
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 3, 16, 17, 64, 65, 130])
def test_sums_over_the_cache_taken_here(dtype, d, T):
    check(inputs(2, 3, T, d, 210, DT[dtype], seed=T), decay=0.9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 600])
@pytest.mark.parametrize("T", [1, 20])
def test_lengths_about_the_tiles(dtype, lens, T):
    check(inputs(1, 2, T, 128, 600, DT[dtype], seed=lens, lens=lens))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,p", [(5, 0.5), (127, 0.3), (300, 1.0), (900, 0.1), (2000, 0.2)])
def test_a_prompts_weights_with_the_forwards_lse(dtype, T, p):
    """lse covers keys that are not in the cache, too: weights then add up to less than one per query."""
    x = inputs(1, 2, T, 64, max(1, int(1.3 * p * T)), DT[dtype], seed=T)
    cap = x["k_cache"].shape[2]
    g = torch.Generator().manual_seed(T)
    vis = (torch.rand(1, 2, T, generator=g) < p).int().cumsum(-1, dtype=torch.int32).clamp_max(cap)
    x["cache_len"] = vis[..., -1].contiguous()
    _, lse = ref.cache_weights(**x, vis=vis)
    check(x, vis=vis, lse=(lse + 0.1).float())
    check(x, vis=vis)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_groups_of_heads(dtype):
    x = inputs(2, 6, 33, 64, 100, DT[dtype], seed=3, Hq=2)
    g = torch.Generator().manual_seed(3)
    check(x, vis=torch.randint(0, 101, (2, 3, 33), generator=g, dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [9, 80])
def test_queries_that_see_nothing_and_any_order_of_counts(dtype, T):
    x = inputs(2, 2, T, 64, 90, DT[dtype], seed=5)
    g = torch.Generator().manual_seed(5)
    vis = torch.randint(-3, 120, (2, 2, T), generator=g, dtype=torch.int32)
    vis[0, 0] = 0
    check(x, vis=vis)
    lse = torch.randn(2, 2, T, generator=g) + 4
    lse[1, 1, ::2] = -math.inf
    check(x, vis=vis, lse=lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [4, 100])
def test_what_a_query_does_not_see_has_no_influence(dtype, T):
    """A query with vis 0 may hold anything, and rows behind the cache's end too."""
    x = inputs(1, 2, T, 64, 120, DT[dtype], seed=7, lens=77)
    vis = torch.full((1, 2, T), 60, dtype=torch.int32)
    vis[:, :, 1::2] = 0
    x["q"][:, :, 1::2] = math.nan
    x["k_cache"][:, :, 77:] = math.nan
    x["k_cache"][:, :, 60:77] = math.inf
    g = {k: v.cuda() for k, v in x.items()}
    got = nats.cache_weights(g["weights"].clone(), g["q"], g["k_cache"], g["cache_len"], vis=vis.cuda())
    y = {k: torch.nan_to_num(v, 0.0, 0.0) if v.is_floating_point() else v for k, v in x.items()}
    want, _ = ref.cache_weights(**y, vis=vis)
    assert float(((got.cpu().double() - want).abs() / want)[:, :, :77].max()) <= TOL
    lse = torch.full((1, 2, T), 4.0)
    lse[:, :, 1::2] = math.nan
    got = nats.cache_weights(g["weights"].clone(), g["q"], g["k_cache"], g["cache_len"], vis=vis.cuda(), lse=lse.cuda())
    want, _ = ref.cache_weights(**y, vis=vis, lse=torch.nan_to_num(lse))
    assert float(((got.cpu().double() - want).abs() / want)[:, :, :77].max()) <= TOL


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits(dtype):
    x = inputs(1, 2, 40, 64, 300, DT[dtype], seed=9, lens=300)
    g = {k: v.cuda() for k, v in x.items()}
    got = nats.cache_weights(g["weights"].zero_(), g["q"], g["k_cache"], g["cache_len"], softmax_scale=10.0)
    x["weights"].zero_()
    want, _ = ref.cache_weights(**x, softmax_scale=10.0)
    # logits of size 10 * 64 * 0.64 = 410 in sums of 64 products: off by up to 64 2^-24 * 410 = 1.6e-3, and so each weight, twice
    assert float(((got.cpu().double() - want).abs() / (want + 1e-6)).max()) <= 3.2e-3


def test_same_bits_each_time():
    g = {k: v.cuda() for k, v in inputs(2, 8, 700, 128, 500, torch.bfloat16, seed=10).items()}
    runs = [nats.cache_weights(g["weights"].clone(), g["q"], g["k_cache"], g["cache_len"]) for _ in range(3)]
    assert all(torch.equal(runs[0], r) for r in runs)


# ---- eviction -------------------------------------------------------------------------------------------------------------------
def check_evict(k_cache, v_cache, cache_len, weights, keep, recent):
    g = [t.cuda() for t in (k_cache, v_cache, cache_len, weights)]
    kept = nats.cache_evict(*g, keep, recent)
    want = ref.cache_evict(k_cache, v_cache, cache_len, weights, keep, recent)
    for name, got in zip(("k_cache", "v_cache", "cache_len", "weights", "kept"), (*g, kept)):
        got, w = got.cpu(), want[name]
        assert torch.equal(got.view(torch.int16 if got.dtype == torch.bfloat16 else torch.int32),
                           w.view(torch.int16 if w.dtype == torch.bfloat16 else torch.int32)), name


def evict_inputs(B, H, d, cap, dtype, seed, lens=None):
    x = inputs(B, H, 1, d, cap, dtype, seed, lens=lens)
    g = torch.Generator().manual_seed(seed + 1000)
    return x["k_cache"], torch.randn(B, H, cap, d, generator=g).to(dtype), x["cache_len"], x["weights"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,keep,recent", [(1, 1, 0), (2, 1, 1), (70, 64, 0), (70, 64, 64), (300, 17, 5), (500, 257, 100), (1500, 1024, 1),
                                             (3100, 1100, 128), (5000, 4999, 7)])
def test_evict(dtype, d, cap, keep, recent):
    check_evict(*evict_inputs(2, 2, d, cap, DT[dtype], seed=cap), keep, recent)
    check_evict(*evict_inputs(1, 2, d, cap, DT[dtype], seed=cap, lens=cap), keep, recent)


@pytest.mark.parametrize("lens", [-3, 0, 1, 63, 64, 65, 100, 5000])
def test_evict_about_the_budget(lens):
    check_evict(*evict_inputs(1, 2, 64, 100, torch.bfloat16, seed=1, lens=lens), 64, 16)


@pytest.mark.parametrize("levels", [1, 2, 5])
def test_evict_equal_weights_keep_the_lower_rows(levels):
    k, v, n, w = evict_inputs(2, 2, 64, 2500, torch.bfloat16, seed=2, lens=2400)
    w = (w * levels).floor()
    for keep, recent in ((1000, 0), (1500, 300), (7, 3)):
        check_evict(k, v, n, w, keep, recent)


def test_evict_signs_infinities_and_nans():
    k, v, n, w = evict_inputs(1, 3, 64, 400, torch.float32, seed=3, lens=390)
    w = w - 0.5
    w[:, 0, ::3], w[:, 0, 1::3] = 0.0, -0.0
    w[:, 1, ::5], w[:, 1, 1::5], w[:, 1, 2::5] = math.nan, math.inf, -math.inf
    w[:, 2] = math.nan
    w[:, 2, 300] = -3e38
    for keep, recent in ((300, 10), (100, 0), (1, 0), (390, 20)):
        check_evict(k, v, n, w, keep, recent)


def test_evict_weights_that_differ_in_their_last_bits():
    k, v, n, w = evict_inputs(1, 2, 64, 700, torch.bfloat16, seed=4, lens=700)
    w = (torch.full((1, 2, 700), 1.0).view(torch.int32) + torch.randperm(1400, generator=torch.Generator().manual_seed(4)).view(1, 2, 700).int()).view(torch.float32)
    check_evict(k, v, n, w, 333, 10)


def test_a_captured_eviction_replays():
    k, v, n, w = (t.cuda() for t in evict_inputs(2, 2, 128, 900, torch.bfloat16, seed=5, lens=900))
    first = [t.clone() for t in (k, v, n, w)]
    kept = torch.empty(2, 2, 400, dtype=torch.int32, device="cuda")
    want = ref.cache_evict(k, v, n, w, 400, 50)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nats.cache_evict(k, v, n, w, 400, 50, kept=kept)
    for _ in range(3):
        for t, f in zip((k, v, n, w), first):
            t.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        for name, got in zip(("k_cache", "v_cache", "cache_len", "weights", "kept"), (k, v, n, w, kept)):
            assert torch.equal(got.cpu(), want[name]), name


# ---- together -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_drafts_weights_and_eviction_together(dtype):
    """A prompt's forward hands over state, cache, counts and lse; its rows get their weights; then rounds of drafts, a tree read, a
    path committed, its weights added, the cache cut down; every step against the definition on what the step before left."""
    from nats_inputs import make_fwd_inputs
    dt = DT[dtype]
    B, H, L, d, T, cap, keep = 2, 2, 256, 64, 8, 160, 40
    x = make_fwd_inputs(B, H, L, d, dtype, 0.3, seed=71)
    g = {k: torch.from_numpy(v).cuda() for k, v in x.items()}
    Q, K, V = (g[k].to(dt) for k in ("Q", "K", "V"))
    r = nats.hybrid_attn_fwd_ex(Q, K, V, g["alpha"], g["beta"], g["mask"], 64, want=("final_state", "Kc", "Vc", "n_s", "cnt", "lse"), cap=cap)
    weights = torch.zeros(B, H, cap, device="cuda")
    nats.cache_weights(weights, Q, r["Kc"], r["n_s"], lse=r["lse"], vis=r["cnt"])
    # every query that sees a row hands out a weight of one (the forward's lse of bf16 tensors: logits to 2^-8)
    some = (r["cnt"] > 0).sum(-1).float()
    assert float((weights.sum(-1) / some - 1).abs().max()) <= 8e-3
    st = dict(state=r["final_state"], k_cache=r["Kc"], v_cache=r["Vc"], cache_len=r["n_s"])
    for turn in range(4):
        t = ref.tree_inputs(B, H, T, d, cap, dt, seed=80 + turn)
        t = {**{k: v.cuda() for k, v in t.items()}, **st}
        o, lse = nats.hybrid_attn_decode_tree(*(t[k] for k in ("state", "k_cache", "v_cache", "cache_len", "q", "k", "v", "alpha", "beta", "mask", "parent")))
        want_o, want_lse = ref.decode_tree(t)
        from gpu_util import host, rel_err
        assert rel_err(host(o), want_o.numpy(), "bf16" if dtype == "bf16" else None) <= 2.4e-4
        node = torch.tensor([turn, 7 - turn], dtype=torch.int32, device="cuda")
        want = ref.tree_commit(t, node)
        vis = nats.hybrid_attn_tree_commit(*(t[k] for k in ("state", "k_cache", "v_cache", "cache_len", "k", "v", "alpha", "beta", "mask", "parent")), node)
        assert torch.equal(vis.cpu(), want["vis"]) and torch.equal(t["cache_len"].cpu(), want["cache_len"])
        assert rel_err(host(t["state"]), want["state"].numpy()) <= 8e-5
        want_w, _ = ref.cache_weights(weights, t["q"], t["k_cache"], t["cache_len"], lse=lse, vis=vis, decay=0.95)
        nats.cache_weights(weights, t["q"], t["k_cache"], t["cache_len"], lse=lse, vis=vis, decay=0.95)
        assert float(((weights.cpu().double() - want_w).abs() / (want_w + 1e-6)).max()) <= TOL
        want = ref.cache_evict(t["k_cache"], t["v_cache"], t["cache_len"], weights, keep, 10)
        kept = nats.cache_evict(t["k_cache"], t["v_cache"], t["cache_len"], weights, keep, 10)
        for name, got in (("k_cache", t["k_cache"]), ("v_cache", t["v_cache"]), ("cache_len", t["cache_len"]), ("weights", weights), ("kept", kept)):
            assert torch.equal(got.cpu(), want[name]), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [1, 16, 20, 33, 64, 70, 129, 260, 530])
@pytest.mark.parametrize("T", [65, 200])
def test_many_queries_over_caches_of_every_width(dtype, d, cap, T):
    """Every number of wavefronts side by side on the rows, queries in one step and in several."""
    x = inputs(1, 3, T, d, cap, DT[dtype], seed=cap + T)
    g = torch.Generator().manual_seed(cap)
    vis = torch.randint(0, cap + 1, (1, 3, T), generator=g, dtype=torch.int32).sort(-1).values
    vis[:, :, -1] = cap
    x["cache_len"][0, 0] = cap
    check(x, vis=vis)
    _, lse = ref.cache_weights(**x, vis=vis)
    check(x, vis=vis, lse=lse.float())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_heads_and_queries(dtype):
    """Enough blocks that the queries go 256 and more at a time, several steps to a block."""
    x = inputs(2, 16, 1500, 64, 300, DT[dtype], seed=77)
    g = torch.Generator().manual_seed(77)
    vis = torch.randint(0, 301, (2, 16, 1500), generator=g, dtype=torch.int32).sort(-1).values
    _, lse = ref.cache_weights(**x, vis=vis)
    check(x, vis=vis, lse=lse.float(), decay=0.5)


def test_evict_from_a_cache_of_several_steps():
    """More rows than a block keeps in its registers; many equal weights, so that ranks go on from step to step."""
    k, v, n, w = evict_inputs(1, 2, 64, 70000, torch.bfloat16, seed=6, lens=69999)
    check_evict(k, v, n, w, 40000, 1500)
    check_evict(k, v, n, (w * 3).floor(), 50000, 0)
    check_evict(k, v, n, w, 33000, 33000)
    n[0, 1] = 32769
    check_evict(k, v, n, (w * 3).floor(), 300, 10)


@pytest.mark.parametrize("T", [66000, 70001])
def test_more_queries_than_a_block_takes_at_once(T):
    x = inputs(1, 2, T, 64, 40, torch.bfloat16, seed=T, lens=40)
    g = torch.Generator().manual_seed(T)
    vis = torch.randint(0, 41, (1, 2, T), generator=g, dtype=torch.int32).sort(-1).values
    _, lse = ref.cache_weights(**x, vis=vis)
    # the sums of T terms: by lanes, wavefronts and blocks, none of more than 1100 terms in a row
    check(x, vis=vis, lse=lse.float())


def test_captured_weights_and_a_stream_of_the_callers_own():
    """Few queries, more than keep their logits, and a prompt's; each with the sums taken here."""
    cases = [inputs(2, 3, T, 64, 700, DT["bf16"], seed=91 + T) for T in (3, 40, 200)]
    gs = [{k: v.cuda() for k, v in x.items()} for x in cases]
    names = ("weights", "q", "k_cache", "cache_len")
    first = [g["weights"].clone() for g in gs]
    wants = []
    for x in cases:
        w = dict(x)
        for _ in range(3):
            w["weights"] = ref.cache_weights(**w, decay=0.5)[0]
        wants.append(w["weights"])
    eager = [[nats.cache_weights(*(g[n] for n in names), decay=0.5).clone() for _ in range(3)] for g in gs]
    for x, e, want in zip(cases, eager, wants):
        there = torch.arange(700) < x["cache_len"][..., None]
        assert float(((e[2].cpu().double() - want).abs() / want.clamp_min(1e-30))[there].max()) <= 4 * TOL   # three calls, two of them decayed
    for g, f in zip(gs, first):
        g["weights"].copy_(f)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for g in gs:
            nats.cache_weights(*(g[n] for n in names), decay=0.5)
    for repeat in range(2):
        for g, f in zip(gs, first):
            g["weights"].copy_(f)
        for step in range(3):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(g["weights"], e[step]) for g, e in zip(gs, eager))
            torch.zeros(1 << 20, device="cuda").sum().item()
    for g, f in zip(gs, first):
        g["weights"].copy_(f)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for step in range(3):
            for g, e in zip(gs, eager):
                assert torch.equal(nats.cache_weights(*(g[n] for n in names), decay=0.5), e[step])


def test_evict_sizes_that_do_not_fit_32_bits():
    k, v, n, w = (t.cuda() for t in evict_inputs(1, 2, 64, 40, torch.bfloat16, seed=8, lens=40))
    before = [t.clone() for t in (k, v, n, w)]
    for keep, recent in (((1 << 32) + 5, 0), (41, 0), (0, 0), (-(1 << 32) + 5, 0), (5, 1 << 32), (5, -(1 << 32))):
        with pytest.raises(nats.NatsError, match="keep must be"):
            nats.cache_evict(k, v, n, w, keep, recent)
    assert all(torch.equal(a, b) for a, b in zip(before, (k, v, n, w)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_of_more_rows(dtype):
    """More than 64 queries of many heads over long caches: parts of up to 8192 rows (512 terms of a lane's sum in a row: 3.1e-5 more)."""
    x = inputs(1, 48, 100, 64, 9000, DT[dtype], seed=95)
    check(x)
    x = inputs(1, 3, 3000, 64, 9000, DT[dtype], seed=96)
    check(x)


@pytest.mark.parametrize("cap,lens", [(1000, [[256, 511, 512, 513, 767]]), (4000, [[512, 513, 1023, 1025, 3585]]),
                                      (9000, [[2047, 2048, 2049, 4097, 8193]]), (32800, [[32767, 32768, 32769, 2100, 28673]])])
def test_evict_lengths_about_a_threads_rows(cap, lens):
    """The rows of a cache are spread over the threads two by two each; the caches with and without a last share that is not whole."""
    k, v, n, w = evict_inputs(1, 5, 64, cap, torch.bfloat16, seed=cap, lens=lens)
    for keep, recent in ((200, 0), (200, 199), (200, 1), (255, 100)):
        check_evict(k, v, n, w, keep, recent)
    check_evict(k, v, n, torch.where(w < 0.5, w * 1e-30, (w * 4).floor()), 200, 7)     # a wide range of weights, many equal ones
    check_evict(k, v, n, torch.full_like(w, 0.25), 200, 7)
