"""An infinity, or a number next to fp32's largest, in the state: nodes that write nothing before them (softmax tokens) and the gated
operation read it as the recurrence does, an infinity of the right sign, not a NaN; rows of the state without one are not touched by it.
Tolerances as in test_gpu_tree.py."""
import math

import pytest
import torch

import paper_2602_03681_amd as nats
import serve_reference as ref
from gpu_util import bf16_half_ulp, host

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ARGS = ("state", "k_cache", "v_cache", "cache_len", "q", "k", "v", "alpha", "beta", "mask", "parent")


def read(x, linear_op):
    g = {k: v.cuda() for k, v in x.items()}
    o, _ = nats.hybrid_attn_decode_tree(*(g[k] for k in ARGS), q_nla=g["q_nla"], k_nla=g["k_nla"], linear_op=linear_op)
    return o.float().cpu(), ref.decode_tree(x, linear_op=linear_op)[0]


def same(o, want, dtype):
    """Infinities and NaN where the definition has them; the rest to fp32 accuracy (and what storing in bf16 takes)."""
    assert torch.equal(torch.isnan(o), torch.isnan(want))
    assert torch.equal(torch.isposinf(o), torch.isposinf(want)) and torch.equal(torch.isneginf(o), torch.isneginf(want))
    return torch.isfinite(want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 9, 20, 60])
@pytest.mark.parametrize("linear_op,p", [(0, 1.0), (1, 0.3)])
def test_an_infinity(dtype, d, T, linear_op, p):
    x = ref.tree_inputs(1, 2, T, d, 30, DT[dtype], seed=d + T, own_qk=True, p=p)
    x["q"][0, 0] = x["q"][0, 0].abs()                   # of one sign in one head, of both in the other
    clean, _ = read(x, linear_op)
    for h in range(2):
        x["state"][0, h, 5, 9] = math.inf
        x["state"][0, h, 50, 60] = -math.inf
        x["state"][0, h, 33, 1:3] = math.inf            # both: of one sign, or NaN where the query's signs differ
    o, want = read(x, linear_op)
    fin = same(o, want, dtype)
    assert torch.isposinf(want[0, 0, :, 5]).all() and torch.isneginf(want[0, 0, :, 50]).all()
    assert not fin[0, 0, :, [5, 33, 50]].any()
    assert fin[0, :, :, [c for c in range(d) if c not in (5, 33, 50)]].all()
    # what does not read it: to what it is without (the same products, by another instruction where a neighbour has one)
    off = (o - clean).abs()[fin].double()
    rms = float(clean.double().square().mean().sqrt())
    step = torch.from_numpy(2 * bf16_half_ulp(clean[fin].numpy())) if dtype == "bf16" else 0.0
    assert float((off - step).max()) <= 1.6e-4 * rms


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [30, 1100])
def test_an_infinity_in_many_heads(dtype, cap):
    """More than 128 heads: a block takes 64 rows of the state, and then the others."""
    x = ref.tree_inputs(10, 13, 5, 128, 30, DT[dtype], seed=7, own_qk=True, p=0.3)
    for name in ("k_cache", "v_cache"):
        rows = torch.zeros(10, 13, cap, 128, dtype=DT[dtype])
        rows[:, :, :30] = x[name]
        x[name] = rows
    for h, row in enumerate((3, 40, 63, 64, 70, 100, 127)):
        x["state"][h, 2 * h - 1, row, 17] = -math.inf
    o, want = read(x, 1)
    assert torch.isinf(want).sum() == 7 * 5
    same(o, want, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("linear_op,p", [(0, 1.0), (1, 0.3)])
def test_numbers_that_bf16_rounds_to_an_infinity(dtype, linear_op, p):
    """3.4e38, alone in its row: the product with the query is finite, and off by a few roundings of it."""
    x = ref.tree_inputs(1, 2, 20, 64, 30, DT[dtype], seed=3, own_qk=True, p=p)
    x["alpha"].fill_(0.75)
    x["state"][:, :, 12] = 0.0
    x["state"][:, :, 12, 40] = 3.4e38
    o, want = read(x, linear_op)
    assert torch.isfinite(want).all() and torch.isfinite(o).all()
    got, want = o[..., 12].double(), want[..., 12]
    off = (got - want).abs() - (torch.from_numpy(bf16_half_ulp(want.numpy())) if dtype == "bf16" else 0.0)
    # 64 products of which one counts, the decays of up to 20 nodes
    assert float((off / want.abs().clamp_min(1e30)).max()) <= (64 + 40) * 2.0 ** -24


def test_an_infinite_query_of_a_root():
    """fp32 tensors: a softmax token that follows the last committed one reads the state alone."""
    x = ref.tree_inputs(1, 2, 7, 64, 30, torch.float32, seed=9, own_qk=True, p=1.0, tree="star")
    x["state"].clamp_(-0.9, 0.9)
    x["q"][:, :, 3, 8] = math.inf
    x["q"][:, :, 5, 8] = -3.4e38
    o, want = read(x, 0)
    same(o, want, "f32")
    assert torch.isinf(o[:, :, 3]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("linear_op,p", [(0, 1.0), (1, 0.3)])
def test_an_infinity_beside_nodes_that_are_not_there(dtype, linear_op, p):
    """The nodes behind n_nodes hold NaN; those before read the state's infinities as ever."""
    x = ref.tree_inputs(3, 2, 24, 64, 30, DT[dtype], seed=13, own_qk=True, p=p)
    nodes = torch.tensor([24, 11, 0], dtype=torch.int32)
    x["state"][:, 0, 5, 9] = math.inf
    x["state"][:, 1, 63, 0] = -math.inf
    want, _ = ref.decode_tree(x, linear_op=linear_op, n_nodes=nodes)
    for b in (1, 2):
        for k in ("q", "k", "v", "q_nla", "k_nla", "alpha", "beta"):
            x[k][b, :, int(nodes[b]):] = math.nan
    g = {k: v.cuda() for k, v in x.items()}
    o, _ = nats.hybrid_attn_decode_tree(*(g[k] for k in ARGS), q_nla=g["q_nla"], k_nla=g["k_nla"], linear_op=linear_op, n_nodes=nodes.cuda())
    o = o.float().cpu()
    fin = same(o, want, dtype)
    assert torch.isinf(want[0, 0, :, 5]).all() and torch.isinf(want[1, 1, :11, 63]).all() and not o[2].any()
    off = (o.double() - want)[fin].abs() - (torch.from_numpy(bf16_half_ulp(want[fin].numpy())) if dtype == "bf16" else 0.0)
    assert float(off.max()) <= 8e-5 * float(want[fin].square().mean().sqrt())
