"""hybrid_attn_decode_tree and hybrid_attn_tree_commit against their definitions in 64 bits, token by token along every path.

Tolerances (largest error over the RMS of the result).  fp32: sums of d products, n rows and up to 64 nodes, each with a rounding
of 2^-24: (128 + 1100 + 64) 2^-24 = 8e-5.  bf16 tensors: what is stored rounded to bf16 is off by half a step of that, which is
taken off first; the rest is fp32 arithmetic and operands held to 16 bits (2^-17 of each of d products whose sizes add up to about
0.64 sqrt(128) = 7 times the sum's RMS, in three products of that kind): 21 2^-17 = 1.6e-4, and the fp32 share.
lse: a logit is a sum of d products of size 0.64 scale each, 128 * 128 * 0.64 * 0.0884 * 2^-24 = 5.5e-5 at most."""
import math

import pytest
import torch

import paper_2602_03681_amd as nats
import serve_reference as ref
from gpu_util import host, rel_err
from paper_2602_03681_amd import binding as nb

pytestmark = pytest.mark.gpu
TOL = {torch.float32: 8e-5, torch.bfloat16: 2.4e-4}
TOL_LSE = 6e-5
STATE_ARGS = ("state", "k_cache", "v_cache", "cache_len")
NODE_ARGS = ("q", "k", "v", "alpha", "beta", "mask", "parent")
OPTIONAL = ("q_nla", "k_nla", "w_nla", "w_la")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def cuda(x):
    return {k: v.cuda() for k, v in x.items()}


def read(x, G=1, **kw):
    return nats.hybrid_attn_decode_tree(*(x[k] for k in STATE_ARGS + NODE_ARGS), group=G, **{k: x[k] for k in OPTIONAL if k in x}, **kw)


def check(x, G=1, out=None, **kw):
    g = cuda(x)
    before = {k: v.clone() for k, v in g.items()}
    o, lse = read(g, G, **kw) if out is None else out
    want_o, want_lse = ref.decode_tree(x, G, **kw)
    stored = "bf16" if o.dtype == torch.bfloat16 else None
    assert rel_err(host(o), want_o.numpy(), stored) <= TOL[o.dtype]
    got = lse.double().cpu()
    assert torch.equal(torch.isinf(got), torch.isinf(want_lse))
    fin = torch.isfinite(want_lse)
    assert float((got - want_lse)[fin].abs().max() if fin.any() else 0.0) <= TOL_LSE
    for k, v in g.items():
        assert torch.equal(v.view(torch.uint8), before[k].view(torch.uint8)), k        # nothing was changed
    return o, lse


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,tree", [(1, "tree"), (2, "chain"), (7, "tree"), (16, "chain"), (17, "tree"), (31, "star"), (33, "tree"),
                                    (48, "chain"), (64, "tree"), (64, "chain")])
def test_tree_against_each_path_alone(dtype, d, T, tree):
    check(ref.tree_inputs(2, 2, T, d, 300, DT[dtype], seed=T * d, tree=tree, own_qk=T % 2 == 0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("linear_op,freeze", [(0, False), (0, True), (1, False), (1, True)])
def test_merges_and_linear_operations(dtype, mode, linear_op, freeze):
    x = ref.tree_inputs(2, 2, 19, 128, 90, DT[dtype], seed=5 + mode, own_qk=True, weights=mode > 0 and not freeze)
    check(x, combine_mode=mode, linear_op=linear_op, freeze_on_softmax=freeze)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales_and_eps(dtype):
    x = ref.tree_inputs(1, 3, 9, 64, 70, DT[dtype], seed=11)
    check(x, softmax_scale=0.5, la_scale=0.7, combine_mode=1, rms_eps=1e-3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G,own_qk", [(2, False), (2, True), (3, False)])
def test_head_groups(dtype, G, own_qk):
    x = ref.tree_inputs(2, 2, 21, 64, 150, DT[dtype], seed=17 + G, G=G, own_qk=own_qk, weights=True)
    check(x, G=G, combine_mode=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1023, 1100])
def test_cache_lengths_about_the_tiles(dtype, lens):
    check(ref.tree_inputs(1, 2, 18, 128, 1100, DT[dtype], seed=lens, lens=lens, own_qk=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths_beyond_the_cache_and_below_zero(dtype):
    x = ref.tree_inputs(2, 2, 5, 64, 40, DT[dtype], seed=3)
    x["cache_len"] = torch.tensor([[41, 1 << 30], [-1, -(1 << 31)]], dtype=torch.int32)
    check(x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [0.0, 1.0])
def test_all_linear_and_all_softmax_over_an_empty_cache(dtype, p):
    """p = 0: no node sees a key."""
    for T in (1, 20):
        x = ref.tree_inputs(1, 2, T, 64, 8, DT[dtype], seed=7, p=p, lens=0)
        o, lse = check(x)
        assert torch.isinf(lse).all() == (p == 0.0)
        check(x, combine_mode=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parents_that_are_no_earlier_node_count_as_the_root(dtype):
    x = ref.tree_inputs(1, 2, 9, 64, 30, DT[dtype], seed=23)
    x["parent"] = torch.tensor([[0, 5, 1, 3, 100, -7, 5, 1 << 30, -(1 << 31)]], dtype=torch.int32)
    check(x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [6, 40])
def test_nodes_that_are_not_there(dtype, T):
    """Padded trees: rows of 0, lse -inf, and nothing of what stands there."""
    x = ref.tree_inputs(4, 2, T, 128, 60, DT[dtype], seed=29, own_qk=True)
    n = torch.tensor([T, 0, T // 2, T + 5], dtype=torch.int32)
    for k in ("q", "k", "v", "q_nla", "k_nla", "alpha", "beta"):
        x[k][1] = math.nan
        x[k][2, :, T // 2:] = math.nan
    g = cuda(x)
    o, lse = read(g, n_nodes=n.cuda(), combine_mode=1)
    clean = {k: torch.nan_to_num(v) if v.is_floating_point() else v for k, v in x.items()}
    check(clean, out=(o, lse), n_nodes=n, combine_mode=1)
    assert not o[1].any() and not o[2, :, T // 2:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, 3e38])
@pytest.mark.parametrize("T", [12, 50])
def test_what_is_not_finite_acts_on_its_descendants_alone(dtype, bad, T):
    x = ref.tree_inputs(1, 2, T, 64, 40, DT[dtype], seed=31, own_qk=True, p=0.4)
    x["parent"][0, 1:] = torch.tensor([max(-1, i - 3) for i in range(1, T)], dtype=torch.int32)
    at = 4
    below = [t for t in range(T) if at in ref.path_of(x["parent"][0], t)]
    others = [t for t in range(T) if t not in below]
    want_o, want_lse = ref.decode_tree(x)
    for key in ("k", "v", "k_nla", "q", "q_nla", "alpha", "beta"):
        y = {k: v.clone() for k, v in x.items()}
        y[key][0, :, at] = bad
        o, lse = read(cuda(y))
        assert torch.isfinite(o[:, :, others]).all(), key
        assert rel_err(host(o[:, :, others]), want_o[:, :, others].numpy(), "bf16" if dtype == "bf16" else None) <= TOL[DT[dtype]], key
        assert float((lse.cpu().double() - want_lse)[:, :, others].abs().max()) <= TOL_LSE, key
        if math.isnan(bad) and key in ("v", "q"):
            assert torch.isnan(o[:, :, at]).all() or key == "q_nla"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_behind_the_cache_are_not_read_into_the_result(dtype):
    x = ref.tree_inputs(1, 2, 10, 128, 200, DT[dtype], seed=37, lens=131)
    x["k_cache"][:, :, 131:] = math.nan
    x["v_cache"][:, :, 131:] = math.inf
    check(x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_infinity_in_a_cached_row_stays_one(dtype):
    x = ref.tree_inputs(1, 1, 10, 64, 200, DT[dtype], seed=41, lens=150)
    for row in (0, 77, 149):
        y = {k: v.clone() for k, v in x.items()}
        y["v_cache"][:, :, row, 5] = math.inf
        o, _ = read(cuda(y))
        assert (o[..., 5] == math.inf).all() and torch.isfinite(o[..., :5]).all() and torch.isfinite(o[..., 6:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits(dtype):
    """Logits of some hundreds: weights by the running maximum."""
    x = ref.tree_inputs(1, 2, 16, 64, 600, DT[dtype], seed=43, own_qk=True, lens=600)
    g = cuda(x)
    o, lse = read(g, softmax_scale=12.0)
    want_o, want_lse = ref.decode_tree(x, softmax_scale=12.0)
    # a logit of 12 x 64 products is off by up to 64 2^-24 of their sizes' sum (12 * 64 * 0.64 = 490): 1.9e-3, and so is a weight
    assert rel_err(host(o), want_o.numpy(), "bf16" if dtype == "bf16" else None) <= 2.5e-3
    assert float((lse.cpu().double() - want_lse).abs().max()) <= 2e-3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_node_is_the_decode_step(dtype):
    x = cuda(ref.tree_inputs(3, 2, 1, 128, 90, DT[dtype], seed=47, lens=80))
    o, _ = read(x)
    st = {k: x[k].clone() for k in STATE_ARGS}
    want = nats.hybrid_attn_decode(*(st[k] for k in STATE_ARGS), *(x[k][:, :, 0].contiguous() for k in ("q", "k", "v", "alpha", "beta", "mask")))
    assert rel_err(host(o[:, :, 0]), host(want)) <= 2 * TOL[DT[dtype]] + (2.0 ** -6 if dtype == "bf16" else 0)
    nats.hybrid_attn_tree_commit(*(x[k] for k in STATE_ARGS + NODE_ARGS[1:]), torch.zeros(3, dtype=torch.int32, device="cuda"))
    for k in ("k_cache", "v_cache", "cache_len"):
        assert torch.equal(x[k], st[k]), k
    assert rel_err(host(x["state"]), host(st["state"])) <= 8e-5


# ---- commit -------------------------------------------------------------------------------------------------------------------
def check_commit(x, node, G=1, **kw):
    g = cuda(x)
    B, HG = g["cache_len"].shape
    err = torch.full((B, HG), 9, dtype=torch.int32, device="cuda")
    vis = nats.hybrid_attn_tree_commit(*(g[k] for k in STATE_ARGS + NODE_ARGS[1:]), node.cuda(), group=G, err_flags=err,
                                       k_nla=g.get("k_nla"), **kw)
    want = ref.tree_commit(x, node, G, **kw)
    for k in ("k_cache", "v_cache", "cache_len"):
        assert torch.equal(g[k].cpu(), want[k]), k
    assert torch.equal(vis.cpu(), want["vis"]) and torch.equal(err.cpu(), want["err_flags"])
    assert rel_err(host(g["state"]), want["state"].numpy()) <= 8e-5
    return g


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,tree,G", [(1, "tree", 1), (5, "chain", 1), (16, "tree", 2), (33, "tree", 1), (64, "chain", 1), (64, "tree", 3)])
def test_commit(dtype, d, T, tree, G):
    x = ref.tree_inputs(4, 2, T, d, 100, DT[dtype], seed=T + d, tree=tree, G=G, own_qk=T % 2 == 0)
    check_commit(x, torch.tensor([T - 1, -1, T // 2, 0], dtype=torch.int32), G)


@pytest.mark.parametrize("linear_op,freeze", [(0, True), (1, False), (1, True)])
def test_commit_variants(linear_op, freeze):
    x = ref.tree_inputs(2, 2, 12, 64, 50, torch.bfloat16, seed=2, tree="chain")
    check_commit(x, torch.tensor([11, 6], dtype=torch.int32), linear_op=linear_op, freeze_on_softmax=freeze)


def test_commit_of_nodes_that_are_none():
    x = ref.tree_inputs(4, 2, 6, 64, 30, torch.float32, seed=3)
    g = check_commit(x, torch.tensor([6, -2, 1 << 30, -(1 << 31)], dtype=torch.int32))
    assert torch.equal(g["state"].cpu(), x["state"])


@pytest.mark.parametrize("lens", [-5, 0, 26, 28, 29, 30, 31])
def test_commit_into_a_cache_that_fills_up(lens):
    x = ref.tree_inputs(1, 2, 9, 64, 30, torch.bfloat16, seed=4, tree="chain", p=0.7, lens=lens)
    check_commit(x, torch.tensor([8], dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_committed_path_is_what_the_tree_read(dtype):
    """Round after round: a node's row, then the same token decoded on the committed state."""
    x = cuda(ref.tree_inputs(2, 2, 8, 64, 64, DT[dtype], seed=53, lens=10, tree="tree"))
    o, _ = read(x)
    node = torch.tensor([7, 4], dtype=torch.int32, device="cuda")
    parents = x["parent"].cpu()
    before = torch.tensor([ref.path_of(parents[b], int(node[b]))[-2] if len(ref.path_of(parents[b], int(node[b]))) > 1 else -1
                           for b in range(2)], dtype=torch.int32, device="cuda")
    nats.hybrid_attn_tree_commit(*(x[k] for k in STATE_ARGS + NODE_ARGS[1:]), before)
    token = {k: torch.stack([x[k][b, :, int(node[b])] for b in range(2)]).contiguous() for k in ("q", "k", "v", "alpha", "beta", "mask")}
    want = nats.hybrid_attn_decode(*(x[k] for k in STATE_ARGS), *(token[k] for k in ("q", "k", "v", "alpha", "beta", "mask")))
    got = torch.stack([o[b, :, int(node[b])] for b in range(2)])
    assert rel_err(host(got), host(want)) <= 2 * TOL[DT[dtype]] + (2.0 ** -6 if dtype == "bf16" else 0)


# ---- streams, graphs, two at once ---------------------------------------------------------------------------------------------
def test_a_captured_round_replays_to_the_eager_results():
    x = cuda(ref.tree_inputs(2, 4, 16, 128, 200, torch.bfloat16, seed=59, lens=100))
    node = torch.tensor([5, 9], dtype=torch.int32, device="cuda")
    first = {k: x[k].clone() for k in STATE_ARGS}
    ws = torch.empty(nats.decode_tree_workspace_bytes(2, 4, 16, 128, 200, nb.NATS_BF16), dtype=torch.uint8, device="cuda")
    out, lse, vis = torch.empty_like(x["v"]), torch.empty(2, 4, 16, device="cuda"), torch.empty(2, 4, 16, dtype=torch.int32, device="cuda")

    def round_():
        read(x, out=out, lse=lse, workspace=ws)
        nats.hybrid_attn_tree_commit(*(x[k] for k in STATE_ARGS + NODE_ARGS[1:]), node, vis=vis)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (out, lse, vis, *(x[k] for k in STATE_ARGS))]

    def restore():
        for k in STATE_ARGS:
            x[k].copy_(first[k])
    wants = []
    for _ in range(3):
        round_()
        wants.append(results())
    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_()
    for repeat in range(2):
        restore()
        for want in wants:
            graph.replay()
            for got, w in zip(results(), want):
                assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))
            torch.zeros(1 << 20, device="cuda").sum().item()


def test_two_streams_at_once():
    xs = [cuda(ref.tree_inputs(2, 4, 16, 128, 700, torch.bfloat16, seed=61 + i, lens=650)) for i in range(2)]
    want = [read(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for s, x in zip(streams, xs):
        with torch.cuda.stream(s):
            got.append([read(x) for _ in range(5)])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for o, lse in g:
            assert torch.equal(o, w[0]) and torch.equal(lse, w[1])


def test_offsets_beyond_32_bits():
    """Caches of 4.3 GB each; the last heads' rows are beyond 2^32 bytes, and 2^31 elements."""
    B, H, d, cap = 1, 66, 128, 1 << 18
    x = cuda(ref.tree_inputs(B, H, 6, d, 300, torch.bfloat16, seed=67, lens=290))
    k, v = (torch.zeros(B, H, cap, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[:, :, :300], v[:, :, :300] = x["k_cache"], x["v_cache"]
    want = read(x)
    node = torch.tensor([5], dtype=torch.int32, device="cuda")
    y = dict(x, state=x["state"].clone(), k_cache=k, v_cache=v, cache_len=x["cache_len"].clone())
    got = read(y)
    assert torch.equal(got[1][..., 0].isfinite(), want[1][..., 0].isfinite())
    assert rel_err(host(got[0]), host(want[0])) <= 2.0 ** -6 and float((got[1] - want[1]).abs().max()) <= TOL_LSE
    nats.hybrid_attn_tree_commit(*(x[n] for n in STATE_ARGS + NODE_ARGS[1:]), node)
    nats.hybrid_attn_tree_commit(*(y[n] for n in STATE_ARGS + NODE_ARGS[1:]), node)
    assert torch.equal(y["k_cache"][:, :, :300], x["k_cache"]) and torch.equal(y["v_cache"][:, :, :300], x["v_cache"])
    assert torch.equal(y["cache_len"], x["cache_len"]) and torch.equal(y["state"], x["state"])
    # and a cache that is long: its last rows count
    y["cache_len"][0, H - 1] = cap
    y["v_cache"][0, H - 1, cap - 1] = math.inf
    assert torch.isinf(read(y)[0][0, H - 1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,T", [(64, 5), (128, 3), (64, 20), (128, 40), (64, 60)])
def test_many_caches_in_equal_shares(dtype, d, T):
    """More than 128 caches of very different lengths, empty ones among them: blocks that begin and end inside a cache and take several."""
    B, H, cap = 11, 13, 1900
    g = torch.Generator().manual_seed(d + T)
    lens = (torch.rand(B, H, generator=g).pow(3) * (cap + 1)).int()
    lens[2, 3:] = 0
    lens[3, :9] = 0
    lens[10, 12] = cap
    x = ref.tree_inputs(B, H, T, d, cap, DT[dtype], seed=d + T, own_qk=True)
    x["cache_len"] = lens
    check(x)
    x["cache_len"] = torch.zeros_like(lens)
    x["cache_len"][5, 5] = 33
    check(x)


def test_captured_equal_shares_follow_the_lengths():
    """One workspace, lengths that change between the replays: what the shares of one call left behind is of no use to the next."""
    B, H, T, d, cap = 11, 13, 12, 128, 1900
    x = cuda(ref.tree_inputs(B, H, T, d, cap, torch.bfloat16, seed=83))
    g = torch.Generator().manual_seed(83)
    lens = [torch.randint(0, cap + 1, (B, H), generator=g, dtype=torch.int32).cuda(),
            torch.full((B, H), cap, dtype=torch.int32, device="cuda"), torch.zeros(B, H, dtype=torch.int32, device="cuda"),
            (torch.arange(B * H, dtype=torch.int32, device="cuda") % 67).view(B, H)]
    ws = torch.empty(nats.decode_tree_workspace_bytes(B, H, T, d, cap, nb.NATS_BF16), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(x["v"]), torch.empty(B, H, T, device="cuda")
    wants = []
    for n in lens:
        x["cache_len"].copy_(n)
        o, z = read(x)
        wants.append((o.clone(), z.clone()))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        read(x, out=out, lse=lse, workspace=ws)
    for repeat in range(2):
        for n, (o, z) in zip(lens, wants):
            x["cache_len"].copy_(n)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, o) and torch.equal(lse, z)
            torch.zeros(1 << 20, device="cuda").sum().item()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [16, 64])
def test_keys_longer_than_one(dtype, T):
    """Keys of length 2: a token's write overshoots, and the states grow along the path as they do token by token."""
    x = ref.tree_inputs(1, 4, T, 128, 50, torch.float32, seed=89, p=0.0, tree="chain", lens=0)
    x = {k: v.to(DT[dtype]) if k in ("k_cache", "v_cache", "q", "k", "v") else v for k, v in dict(x, k=2 * x["k"]).items()}
    check(x)
