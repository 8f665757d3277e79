"""The commit of a path over the whole range of fp32: what the recurrence, token by token, keeps finite is finite and right however far the
decays have fallen, and what it does not is infinite in the rows concerned alone.

Tolerance: as in test_gpu_tree.py, sums of d products and of up to 64 tokens in fp32, (128 + 64) 2^-24 of sizes a few times the
result's RMS: 8e-5."""
import math

import pytest
import torch

import paper_2602_03681_amd as nats
import serve_reference as ref
from gpu_util import host, rel_err

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ARGS = ("state", "k_cache", "v_cache", "cache_len", "k", "v", "alpha", "beta", "mask", "parent")


def commit(x, linear_op):
    g = {k: v.cuda() for k, v in x.items()}
    T = x["k"].shape[2]
    node = torch.full((x["k"].shape[0],), T - 1, dtype=torch.int32, device="cuda")
    nats.hybrid_attn_tree_commit(*(g[k] for k in ARGS), node, linear_op=linear_op)
    return g["state"], ref.tree_commit(x, node.cpu(), linear_op=linear_op)["state"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("linear_op", [0, 1])
@pytest.mark.parametrize("size,decay", [(1e30, 0.6), (1e36, 0.9), (2e37, 0.3), (1.0, 1.5)])
def test_large_writes_behind_small_decays(dtype, d, linear_op, size, decay):
    x = ref.tree_inputs(1, 3, 50, d, 4, DT[dtype], seed=d, p=0.0, tree="chain", lens=0)
    x["alpha"] = torch.full_like(x["alpha"], decay)
    x["v"][:, :, 30:] = (x["v"][:, :, 30:].float() * size).to(DT[dtype])     # the decays' product is 2^-22, 2^-5, 2^-52, 2^18 by then
    got, want = commit(x, linear_op)
    assert float(want.abs().max()) < 3e38
    assert torch.isfinite(got).all()
    assert rel_err(host(got), want.numpy()) <= 8e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_overflows_does_so_in_its_own_rows(dtype):
    """The gated operation: a row of S with an infinite value is infinite wherever its key is not 0, the others are as they would be."""
    x = ref.tree_inputs(1, 3, 40, 64, 4, DT[dtype], seed=5, p=0.0, tree="chain", lens=0)
    x["alpha"].fill_(0.5)
    want = ref.tree_commit(x, torch.tensor([39]), linear_op=1)["state"]
    x["v"][0, 1, 35, 7] = math.inf
    x["v"][0, 2, 3, 11] = -math.inf
    got, bad = commit(x, 1)
    assert torch.equal(torch.isposinf(got.cpu()), torch.isposinf(bad)) and torch.equal(torch.isneginf(got.cpu()), torch.isneginf(bad))
    assert torch.isinf(bad[0, 1, 7]).all() and torch.isinf(bad[0, 2, 11]).all()
    fin = torch.isfinite(bad)
    assert not torch.isnan(got).any()
    assert float((got.cpu().double() - want)[fin].abs().max()) <= 8e-5 * float(want.square().mean().sqrt())
