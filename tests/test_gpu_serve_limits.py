"""The calls of nats_serve.h at the largest sizes that they take: 2^20 rows of a cache, 2^20 queries, 65535 (batch, head) pairs.  References
in 64 bits on the GPU; with 65535 pairs a call on a few of them alone."""
import math

import pytest
import torch

import paper_2602_03681_amd as nats

pytestmark = pytest.mark.gpu
ROWS = 1 << 20


def draws(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (lambda *s, dtype=torch.float32: torch.randn(*s, generator=g, device="cuda").to(dtype),
            lambda *s: torch.rand(*s, generator=g, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_longest_cache_read_by_a_tree(dtype):
    H, T, d = 2, 5, 64
    rnd, _ = draws(1)
    k, v, q = rnd(1, H, ROWS, d, dtype=dtype), rnd(1, H, ROWS, d, dtype=dtype), rnd(1, H, T, d, dtype=dtype)
    n = torch.tensor([[ROWS, ROWS - 31]], dtype=torch.int32, device="cuda")
    zero = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")   # noqa: E731
    o, lse = nats.hybrid_attn_decode_tree(zero(1, H, d, d), k, v, n, zero(1, H, T, d, dtype=dtype), zero(1, H, T, d, dtype=dtype),
                                          zero(1, H, T, d, dtype=dtype), zero(1, H, T), zero(1, H, T), zero(1, H, T, dtype=torch.uint8),
                                          torch.full((1, T), -1, dtype=torch.int32, device="cuda"), q_nla=q, k_nla=zero(1, H, T, d, dtype=dtype))
    for h in range(H):
        m = int(n[0, h])
        x = (q[0, h].double() @ k[0, h, :m].double().t()) / 8.0
        want = torch.softmax(x, 1) @ v[0, h, :m].double()
        # (64 products, 128 tiles of a wavefront, 512 parts) 2^-24 of sum p |v| / sum p = 0.8; bf16: half a step of what is stored
        off = (o[0, h].double() - want).abs() - (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0)
        assert float(off.max()) <= 5e-5 * 0.8
        assert float((lse[0, h].double() - torch.logsumexp(x, 1)).abs().max()) <= 6e-5


@pytest.mark.parametrize("T", [3, 40, 70])
def test_the_longest_caches_weights(T):
    rnd, uni = draws(2)
    k, q, w = rnd(1, 2, ROWS, 64, dtype=torch.bfloat16), rnd(1, 2, T, 64, dtype=torch.bfloat16), uni(1, 2, ROWS)
    n = torch.tensor([[ROWS - 5, ROWS]], dtype=torch.int32, device="cuda")
    before = w.double()
    nats.cache_weights(w, q, k, n, decay=1e-6)        # (weights of a row are about T 2^-20)
    for h in range(2):
        m = int(n[0, h])
        p = torch.softmax((q[0, h].double() @ k[0, h, :m].double().t()) / 8.0, 1).sum(0)
        want = 1e-6 * before[0, h, :m] + p
        # a logit and a log-sum-exp of 14 (2^-24 of it, twice): 5.5e-5 + 2e-6; the sum over the queries
        assert float(((w[0, h, :m].double() - want).abs() / want).max()) <= 6.5e-5
        assert torch.equal(w[0, h, m:].double(), before[0, h, m:])


@pytest.mark.parametrize("clear", [False, True])
def test_the_longest_cache_cut_down(clear):
    keep, recent = (1 << 19) + 7, 1000
    rnd, uni = draws(3)
    k, v = rnd(1, 2, ROWS, 64, dtype=torch.bfloat16), rnd(1, 2, ROWS, 64, dtype=torch.bfloat16)
    w = (uni(1, 2, ROWS) * 100).floor()                # equal weights by the thousand: ties go to the lower row
    n = torch.tensor([[ROWS, keep]], dtype=torch.int32, device="cuda")
    was = [t.clone() for t in (k, v, w)]
    kept = nats.cache_evict(k, v, n, w, keep, recent, clear_weights=clear)
    order = torch.sort(was[2][0, 0, :ROWS - recent], descending=True, stable=True).indices[:keep - recent].sort().values
    rows = torch.cat([order, torch.arange(ROWS - recent, ROWS, device="cuda")])
    assert torch.equal(kept[0, 0].long(), rows) and torch.equal(kept[0, 1].long(), torch.arange(keep, device="cuda"))
    for t, old in zip((k, v, w), was):
        assert torch.equal(t[0, 0, :keep], old[0, 0][rows]) and torch.equal(t[0, 1], old[0, 1])
        assert torch.equal(t[0, 0, keep:], old[0, 0, keep:]) if t is not w or not clear else not t[0, 0, keep:].any()
    assert n.tolist() == [[keep, keep]]


def test_the_most_queries():
    T, cap = 1 << 20, 40
    rnd, uni = draws(4)
    q, k, w = rnd(1, 2, T, 64, dtype=torch.bfloat16), rnd(1, 2, cap, 64, dtype=torch.bfloat16), uni(1, 2, cap)
    n = torch.tensor([[cap, 17]], dtype=torch.int32, device="cuda")
    vis = torch.randint(0, cap + 1, (1, 2, T), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    before = w.double()
    nats.cache_weights(w, q, k, n, vis=vis)
    for h in range(2):
        m = int(n[0, h])
        x = (q[0, h].double() @ k[0, h, :m].double().t()) / 8.0
        x = torch.where(torch.arange(m, device="cuda") < vis[0, h, :, None], x, -math.inf)
        want = before[0, h, :m] + torch.nan_to_num(torch.softmax(x, 1), 0.0).sum(0)
        # launches of 64 blocks' queries each add to the weights: 2^20 / (64 * 64) of them, and up to 64 sums of 64 terms in each
        assert float(((w[0, h, :m].double() - want).abs() / want).max()) <= 5.5e-5 + (256 + 64 + 64) * 2.0 ** -24
        assert torch.equal(w[0, h, m:].double(), before[0, h, m:])


def test_the_most_heads():
    """65535 pairs in each call; every 13107th of them in calls of their own, to the same bits (a row's weight: the same sums)."""
    H, T, d, cap, keep = 65535, 3, 64, 5, 3
    rnd, uni = draws(5)
    bf = torch.bfloat16
    x = dict(state=0.1 * rnd(1, H, d, d), k_cache=rnd(1, H, cap, d, dtype=bf), v_cache=rnd(1, H, cap, d, dtype=bf),
             cache_len=(uni(1, H) * 3).int(), q=0.1 * rnd(1, H, T, d, dtype=bf), k=0.1 * rnd(1, H, T, d, dtype=bf),
             v=rnd(1, H, T, d, dtype=bf), alpha=uni(1, H, T), beta=uni(1, H, T), mask=(uni(1, H, T) < 0.5).to(torch.uint8))
    parent = torch.tensor([[-1, 0, 1]], dtype=torch.int32, device="cuda")
    node = torch.tensor([2], dtype=torch.int32, device="cuda")
    few = torch.arange(0, H, 13107, device="cuda").tolist() + [H - 1]
    y = {n: t[:, few].contiguous() for n, t in x.items()}

    def round_(z):
        w = torch.zeros(1, z["k_cache"].shape[1], cap, device="cuda")
        o, lse = nats.hybrid_attn_decode_tree(*z.values(), parent)
        vis = nats.hybrid_attn_tree_commit(*(t for n, t in z.items() if n != "q"), parent, node)
        nats.cache_weights(w, z["q"], z["k_cache"], z["cache_len"], lse=lse, vis=vis)
        own = w.clone()
        kept = nats.cache_evict(z["k_cache"], z["v_cache"], z["cache_len"], w, keep, 1, clear_weights=True)
        return dict(o=o, lse=lse, vis=vis, own=own, w=w, kept=kept, **z)
    all_, alone = round_(x), round_(y)
    for n, t in all_.items():
        if n == "o":   # (another number of heads, other blocks of the linear branch)
            assert float((t[:, few].float() - alone[n].float()).abs().max()) <= 2.0 ** -7 * float(alone[n].float().abs().max())
        elif n in ("lse", "own", "w"):
            got, want = t[:, few], alone[n]
            fin = torch.isfinite(want)
            assert torch.equal(torch.isfinite(got), fin) and float((got - want)[fin].abs().max()) <= 1e-5
        else:
            assert torch.equal(t[:, few], alone[n]), n
    assert torch.isfinite(all_["o"].float()).all() and int(all_["cache_len"].max()) <= keep
