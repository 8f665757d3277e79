"""Eviction with clear_weights: the weights behind the rows that stay become 0, so that a row that is appended later starts with nothing,
and a cache's rows are ranked by what queries gave them, round after round."""
import pytest
import torch

import paper_2602_03681_amd as nats
import serve_reference as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("k_cache", "v_cache", "cache_len", "weights", "kept")


def bits(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def check(B, H, d, cap, dtype, lens, keep, recent, seed):
    g = torch.Generator().manual_seed(seed)
    x = [torch.randn(B, H, cap, d, generator=g).to(dtype), torch.randn(B, H, cap, d, generator=g).to(dtype),
         torch.tensor(lens, dtype=torch.int32).expand(B, H).contiguous(), torch.rand(B, H, cap, generator=g)]
    want = ref.cache_evict(*x, keep, recent)
    n = x[2].clamp(0, cap)[..., None]
    at = torch.arange(cap)
    want["weights"] = torch.where((n > keep) & (at >= keep) & (at < n), 0.0, want["weights"])
    g = [t.cuda() for t in x]
    kept = nats.cache_evict(*g, keep, recent, clear_weights=True)
    for name, got in zip(NAMES, (*g, kept)):
        assert torch.equal(bits(got.cpu()), bits(want[name])), name


# caches that one launch takes and two, of one step and of several, within the budget and beyond; all, some and none of the rows recent ones
@pytest.mark.parametrize("cap,lens,keep,recent", [
    (1, [[1, 0, 1]], 1, 0), (70, [[64, 65, 70]], 64, 64), (300, [[300, 18, 17]], 17, 5), (1500, [[1500, 1200, 3]], 1024, 1),
    (3100, [[3100, 40, 1101]], 1100, 128), (5000, [[5000, 4999, 4998]], 4998, 4998), (5000, [[5000, 4100, -1]], 200, 199),
    (40000, [[40000, 33000, 50000]], 300, 10), (40000, [[40000, 32769, 39000]], 32768, 32768), (40000, [[40000, 35000, 39000]], 34000, 0)])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f32", 128)])
def test_the_weights_behind_the_rows_that_stay(dtype, d, cap, lens, keep, recent):
    check(1, 3, d, cap, DT[dtype], lens, keep, recent, seed=cap)


@pytest.mark.parametrize("cap,keep", [(600, 300), (1100, 300)])
def test_many_caches(cap, keep):
    g = torch.Generator().manual_seed(cap)
    lens = torch.randint(0, cap + 1, (27, 19), generator=g).tolist()
    check(27, 19, 64, cap, torch.bfloat16, lens, keep, 20, seed=cap)


@pytest.mark.parametrize("append", ["commit", "decode"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_new_row_has_what_queries_gave_it(dtype, append):
    """Rounds of four tokens, all softmax tokens, into caches cut down to 24 rows: every row's weight is the sum of what the queries
    since it was appended gave it, kept apart by the row's number over all rounds."""
    dt, B, H, d, cap, keep, T = DT[dtype], 1, 2, 64, 40, 24, 4
    st = {k: v.cuda() for k, v in ref.tree_inputs(B, H, T, d, cap, dt, seed=1, lens=cap - 4).items()}
    cache = [st[k] for k in ("state", "k_cache", "v_cache", "cache_len")]
    weights = torch.zeros(B, H, cap, device="cuda")
    number = [[list(range(cap - 4)) for _ in range(H)]]          # of the row that lies in each place
    given = {}                                                   # (head, row's number) -> weight
    new = cap - 4
    for turn in range(5):
        x = {k: v.cuda() for k, v in ref.tree_inputs(B, H, T, d, cap, dt, seed=20 + turn, p=1.0, tree="chain").items()}
        tokens = [x[k] for k in ("k", "v", "alpha", "beta", "mask")]
        if append == "commit":
            nats.hybrid_attn_tree_commit(*cache, *tokens, x["parent"], torch.full((B,), T - 1, dtype=torch.int32, device="cuda"))
        else:
            for t in range(T):
                nats.hybrid_attn_decode(*cache, *(z[:, :, t].contiguous() for z in [x["q"], *tokens]))
        for h in range(H):
            number[0][h] += range(new, new + T)
        new += T
        queries = torch.randn(B, H, T, d, generator=torch.Generator().manual_seed(turn)).to(dt).cuda()
        add, _ = ref.cache_weights(torch.zeros(B, H, cap), queries, cache[1], cache[3])
        nats.cache_weights(weights, queries, cache[1], cache[3], decay=0.5)
        for h in range(H):
            assert int(cache[3][0, h]) == len(number[0][h])
            for r, i in enumerate(number[0][h]):
                given[h, i] = 0.5 * given.get((h, i), 0.0) + float(add[0, h, r])
                assert abs(float(weights[0, h, r]) - given[h, i]) <= 1e-4 * given[h, i], (turn, h, r, i)
        kept = nats.cache_evict(cache[1], cache[2], cache[3], weights, keep, 4, clear_weights=True).cpu()
        for h in range(H):
            by = [given[h, i] for i in number[0][h]]
            best = sorted(sorted(range(len(by) - 4), key=lambda r: -by[r])[:keep - 4]) + list(range(len(by) - 4, len(by)))
            assert kept[0, h].tolist() == best
            number[0][h] = [number[0][h][r] for r in best]
        assert not weights[:, :, keep:].any()


def test_a_captured_eviction_replays():
    g = torch.Generator().manual_seed(7)
    x = [torch.randn(2, 2, 900, 128, generator=g).bfloat16().cuda(), torch.randn(2, 2, 900, 128, generator=g).bfloat16().cuda(),
         torch.tensor([[900, 300], [401, 700]], dtype=torch.int32, device="cuda"), torch.rand(2, 2, 900, generator=g).cuda()]
    first = [t.clone() for t in x]
    kept = torch.empty(2, 2, 400, dtype=torch.int32, device="cuda")
    nats.cache_evict(*x, 400, 50, kept=kept, clear_weights=True)
    want = [t.clone() for t in (*x, kept)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nats.cache_evict(*x, 400, 50, kept=kept, clear_weights=True)
    for _ in range(3):
        for t, f in zip(x, first):
            t.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*x, kept), want))
        torch.zeros(1 << 20, device="cuda").sum().item()
