"""The forms that the host rules of tree_read.hip and cache_budget.hip choose by sizes, each at sizes that reach it, against the
definition in 64 bits (on the GPU where the sizes are large).  What a size is for stands beside it; where it hangs on a rule, the rule is
worked out again here, so that a test says when it has lost its form."""
import math

import pytest
import torch

import paper_2602_03681_amd as nats
import serve_reference as ref
from gpu_util import bf16_half_ulp, host, rel_err

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ARGS = ("state", "k_cache", "v_cache", "cache_len", "q", "k", "v", "alpha", "beta", "mask", "parent")


# ---- weights of many queries ----------------------------------------------------------------------------------------------------
def many_form(heads, T, cap, d, dtype):
    """(wavefronts that take rows side by side, a block's queries) for more than 64 queries"""
    tiles = 64 if dtype == "bf16" or d == 64 else 32
    least = 2 if dtype == "f32" and d == 128 else 1
    waves, chunk = (least if cap <= tiles else 2 if cap <= 2 * tiles else 4), 1024
    blocks = lambda: heads * -(-cap // (waves * tiles)) * -(-T // chunk)   # noqa: E731
    while chunk > 128 and blocks() < 1024:
        chunk //= 2
    while waves > least and blocks() < 256:
        waves //= 2
    return waves, 64 if blocks() < 256 else chunk


def weights_in_64_bits(weights, q, k, n, vis, lse, decay):
    """One head at a time on the GPU; lse None: taken over the rows that a query sees."""
    B, H, cap, d = k.shape
    out = weights.double()
    for b in range(B):
        for h in range(H):
            m = int(n[b, h])
            x = (q[b, h].double() @ k[b, h, :m].double().t()) * d ** -0.5
            x = torch.where(torch.arange(m, device="cuda") < vis[b, h, :, None], x, -math.inf)
            L = torch.logsumexp(x, 1) if lse is None else lse[b, h].double()
            p = torch.where((L == -math.inf)[:, None], 0.0, (x - L[:, None]).exp())
            out[b, h, :m] = decay * out[b, h, :m] + p.sum(0)
    return out


# a logit: 5.5e-5 (test_gpu_cache_budget.py); a lane adds up at most 256 of a block's 1024 queries one after the other, then the lanes', the
# wavefronts' and up to 64 blocks' sums are added: (256 + 2 + 4 + 64) 2^-24 = 2e-5
WEIGHTS_TOL = 5.5e-5 + 2e-5


@pytest.mark.parametrize("dtype,d,cap,waves", [("bf16", 128, 550, 4), ("bf16", 64, 300, 4), ("f32", 64, 260, 4), ("f32", 128, 300, 4),
                                               ("bf16", 128, 100, 2), ("bf16", 64, 128, 2), ("f32", 64, 65, 2), ("f32", 128, 60, 2),
                                               ("bf16", 128, 64, 1), ("bf16", 64, 33, 1), ("f32", 64, 50, 1)])
@pytest.mark.parametrize("with_lse", [True, False])
def test_many_queries(dtype, d, cap, waves, with_lse):
    """One, two and four wavefronts side by side on the rows, several steps of queries to a block; counts that rise as a prompt's do, so that
    blocks of later rows begin some steps in, and the last rows belong to no query at all."""
    B, H, T = 3, 16, 5500
    form = many_form(B * H, T, cap, d, dtype)
    assert form[0] == waves and form[1] >= 256
    g = torch.Generator(device="cuda").manual_seed(cap + d)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(DT[dtype])   # noqa: E731
    q, k = rnd(B, H, T, d), rnd(B, H, cap, d)
    vis = (torch.rand(B, H, T, generator=g, device="cuda") < cap / T).int().cumsum(-1, dtype=torch.int32).clamp_max(cap)
    n = torch.minimum(vis[..., -1] + 3, torch.tensor(cap)).int().contiguous()
    n[0, 0] = 0
    n[1, 5] = cap // 2
    weights = torch.rand(B, H, cap, generator=g, device="cuda")
    lse = None
    if with_lse:
        lse = torch.stack([torch.stack([torch.logsumexp(torch.where(torch.arange(cap, device="cuda") < vis[b, h, :, None],
                                                                    (q[b, h].double() @ k[b, h].double().t()) * d ** -0.5, -math.inf), 1)
                                        for h in range(H)]) for b in range(B)]).float() + 0.25
    want = weights_in_64_bits(weights, q, k, n, vis, lse, 0.75)
    before = weights.clone()
    nats.cache_weights(weights, q, k, n, lse=lse, vis=vis, decay=0.75)
    behind = torch.arange(cap, device="cuda") >= n[..., None]
    assert torch.equal(weights[behind], before[behind])
    assert float(((weights.double() - want).abs() / want)[~behind].max()) <= WEIGHTS_TOL


# ---- evictions ------------------------------------------------------------------------------------------------------------------
def check_evict(heads, cap, d, dtype, keep, recent, lens, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = lambda: torch.randint(-1 << 14, 1 << 14, (1, heads, cap, d * (2 if dtype == "f32" else 1)), generator=g, device="cuda",   # noqa: E731
                                 dtype=torch.int16)
    # bits of any kind, moved as they are
    k, v = (rows().view(torch.float32 if dtype == "f32" else torch.bfloat16) for _ in range(2))
    n = torch.randint(lens[0], lens[1] + 1, (1, heads), generator=g, device="cuda", dtype=torch.int32)
    w = torch.rand(1, heads, cap, generator=g, device="cuda")
    w[:, ::3] = (w[:, ::3] * 50).floor()                                                       # many equal ones
    x = [k, v, n, w]
    kept = torch.full((1, heads, keep), -1, dtype=torch.int32)
    for h, m in enumerate(n[0].tolist()):
        m = min(max(m, 0), cap)
        at = list(range(m))
        if m > keep:
            old = torch.argsort(-w[0, h, :m - recent].cpu(), stable=True)[:keep - recent]
            at = sorted(old.tolist()) + at[m - recent:]
        kept[0, h, :len(at)] = torch.tensor(at, dtype=torch.int32)
    want = [t.clone() for t in x]
    source = torch.arange(cap).expand(heads, cap).clone()
    over = n[0].cpu() > keep
    source[over, :keep] = kept[0, over].long()
    for h in range(heads):
        if over[h]:
            for t, y in zip(x, want):
                if t.dim() > 2:
                    y[0, h] = t[0, h][source[h].cuda()]
    want[2] = torch.where(n > keep, keep, n)
    got = nats.cache_evict(*x, keep, recent)
    bits = lambda t: t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)   # noqa: E731
    assert torch.equal(got.cpu(), kept)
    for name, a, b in zip(("k_cache", "v_cache", "cache_len", "weights"), x, want):
        assert torch.equal(bits(a), bits(b)), name


# Two launches (caches of more than 4096 rows): rows of 128, 256 and 512 bytes; heads that are no multiple of 4, nor are their arrays of 8.
# The slice and the block's threads go by the bytes of a row of all caches: 2 heads row_bytes.
@pytest.mark.parametrize("dtype,d,heads,form", [
    ("bf16", 64, 17, "32 x 1024"), ("bf16", 64, 70, "64 x 1024"), ("bf16", 64, 141, "64 x 256"), ("bf16", 64, 301, "128 x 256"),
    ("bf16", 128, 13, "32 x 1024"), ("bf16", 128, 37, "64 x 1024"), ("bf16", 128, 70, "64 x 256"), ("bf16", 128, 141, "128 x 256"),
    ("bf16", 128, 261, "256 x 256"), ("f32", 128, 7, "32 x 1024"), ("f32", 128, 18, "64 x 1024"), ("f32", 128, 35, "64 x 256"),
    ("f32", 128, 70, "128 x 256"), ("f32", 128, 141, "256 x 256"), ("f32", 64, 70, "64 x 256")])
@pytest.mark.parametrize("keep,recent", [(1100, 130), (2000, 2000), (3999, 0)])
def test_moves_in_slices(dtype, d, heads, form, keep, recent):
    row = d * (4 if dtype == "f32" else 2)
    total = 2 * heads * row
    by_rule = ("256 x 256" if row >= 256 and total >= 512 * 256 else "128 x 256" if total >= 512 * 128 else "64 x 256" if total >= 512 * 64
               else "64 x 1024" if total >= 256 * 64 else "32 x 1024")
    assert by_rule == form
    check_evict(heads, 4200, d, dtype, keep, recent, (keep - 200, 4200), seed=heads)


# One launch: 512 heads and more of up to 1024 and of up to 4096 rows; and few heads with little to move
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("heads,cap,keep,recent", [(515, 1030, 700, 33), (515, 600, 257, 0), (515, 1500, 900, 900), (9, 3000, 200, 50)])
def test_one_launch(dtype, d, heads, cap, keep, recent):
    check_evict(heads, cap, d, dtype, keep, recent, (keep - 100, cap), seed=cap + d)


# ---- trees ----------------------------------------------------------------------------------------------------------------------
# Logits, sums of d products, weights and the parts' sums in fp32: (128 + 256 + 129 + 64) 2^-24 = 3.4e-5 of the sizes of what is added,
# which for these inputs are about twice the result's RMS.  What bf16 tensors are stored with is taken off first.
TREE_TOL = 8e-5


def read(x, **kw):
    g = {k: v.cuda() for k, v in x.items()}
    return nats.hybrid_attn_decode_tree(*(g[k] for k in ARGS), **{k: g[k] for k in ("q_nla", "k_nla") if k in g}, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [5, 20, 33, 60])
@pytest.mark.parametrize("d", [64, 128])
def test_many_caches_in_parts(dtype, T, d):
    """More than 128 caches of at most 1024 rows: no equal shares, a head's linear branch in one block of two turns (d 128)."""
    x = ref.tree_inputs(11, 13, T, d, 900, DT[dtype], seed=T + d, own_qk=True)
    x["cache_len"][2, 3:7] = 0
    x["cache_len"][10, 12] = 900
    o, lse = read(x)
    want_o, want_lse = ref.decode_tree(x)
    assert rel_err(host(o), want_o.numpy(), "bf16" if dtype == "bf16" else None) <= TREE_TOL
    some = torch.isfinite(want_lse)
    assert torch.equal(torch.isfinite(lse.cpu()), some)
    assert float((lse.cpu().double() - want_lse)[some].abs().max()) <= 6e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_more_caches_than_equal_shares_are_made_for(dtype, d):
    """2050 caches and more than 1024 rows: parts again."""
    x = ref.tree_inputs(41, 50, 2, d, 70, DT[dtype], seed=d, own_qk=True)
    want_o, want_lse = ref.decode_tree(x)
    for name in ("k_cache", "v_cache"):   # the same rows in caches that could hold more
        rows = torch.zeros(41, 50, 1100, d, dtype=DT[dtype])
        rows[:, :, :70] = x[name]
        x[name] = rows
    o, lse = read(x)
    assert rel_err(host(o), want_o.numpy(), "bf16" if dtype == "bf16" else None) <= TREE_TOL
    some = torch.isfinite(want_lse)
    assert float((lse.cpu().double() - want_lse)[some].abs().max()) <= 6e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [3, 16, 40, 64])
@pytest.mark.parametrize("lens", [[[8191, 8192]], [[8193, 33000]], [[16640, 257]]])
def test_more_parts_than_the_merge_takes_at_once(dtype, d, T, lens):
    """Two caches of up to 33000 rows in 129 parts of 256, which the merge joins 32 at a time.  The linear branch brings 0, so that a part that is
    missing or counted twice shows: it moves an output by some 1e-3 and the lse by 1/129."""
    x = ref.tree_inputs(1, 2, T, d, 33000, DT[dtype], seed=T + d, own_qk=True, lens=lens)
    x["state"].zero_()
    x["beta"].zero_()
    o, lse = read(x)
    want_o, want_lse = ref.decode_tree(x)
    off = abs(host(o) - want_o.numpy()) - (bf16_half_ulp(want_o.numpy()) if dtype == "bf16" else 0.0)
    # relative to sum p |v| / sum p, about E|v| = 0.8
    assert float(off.max()) <= 8e-5 * 0.8
    assert float((lse.cpu().double() - want_lse).abs().max()) <= 6e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,T", [(64, 40), (128, 20), (128, 60)])
def test_equal_shares_of_every_width(dtype, d, T):
    """More than 128 caches of more than 1024 rows, up to four tiles of nodes."""
    x = ref.tree_inputs(10, 13, T, d, 1100, DT[dtype], seed=T + d, own_qk=True)
    x["cache_len"][2, 3:7] = 0
    x["cache_len"][9, 12] = 1100
    o, lse = read(x)
    want_o, want_lse = ref.decode_tree(x)
    assert rel_err(host(o), want_o.numpy(), "bf16" if dtype == "bf16" else None) <= TREE_TOL
    some = torch.isfinite(want_lse)
    assert float((lse.cpu().double() - want_lse)[some].abs().max()) <= 6e-5
