"""The commit of a padded tree: with n_nodes a node that is not there is refused like any other number that is no node."""
import pytest
import torch

import paper_2602_03681_amd as nats
import serve_reference as ref
from gpu_util import host, rel_err

pytestmark = pytest.mark.gpu
ARGS = ("state", "k_cache", "v_cache", "cache_len", "k", "v", "alpha", "beta", "mask", "parent")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G", [1, 2])
def test_a_node_that_is_not_there(dtype, G):
    B, T = 8, 9
    x = ref.tree_inputs(B, 2, T, 64, 30, dtype, seed=3, G=G, p=0.5, lens=12)
    nodes = torch.tensor([9, 5, 5, 0, -4, 1 << 30, 1, 0], dtype=torch.int32)
    node = torch.tensor([8, 4, 5, 0, -1, 9, 0, -1], dtype=torch.int32)
    there = node < nodes.clamp(0, T)
    want = ref.tree_commit(x, torch.where(there, node, 1 << 20), G)
    g = {k: v.cuda() for k, v in x.items()}
    err = torch.full((B, 2 * G), 9, dtype=torch.int32, device="cuda")
    vis = nats.hybrid_attn_tree_commit(*(g[k] for k in ARGS), node.cuda(), n_nodes=nodes.cuda(), group=G, err_flags=err)
    assert torch.equal(err.cpu(), want["err_flags"]) and torch.equal(vis.cpu(), want["vis"])
    assert err.cpu()[:, 0].tolist() == [0, 0, 2, 2, 0, 2, 0, 0]
    for k in ("k_cache", "v_cache", "cache_len"):
        assert torch.equal(g[k].cpu(), want[k]), k
    assert rel_err(host(g["state"]), want["state"].numpy()) <= 8e-5
    assert torch.equal(g["state"].cpu()[~there | (node < 0)], x["state"][~there | (node < 0)])


def test_without_the_number_of_nodes_all_are_there():
    x = ref.tree_inputs(2, 2, 6, 64, 30, torch.float32, seed=4, lens=3)
    node = torch.tensor([5, 3], dtype=torch.int32)
    want = ref.tree_commit(x, node)
    g = {k: v.cuda() for k, v in x.items()}
    vis = nats.hybrid_attn_tree_commit(*(g[k] for k in ARGS), node.cuda(), n_nodes=None)
    assert torch.equal(vis.cpu(), want["vis"]) and rel_err(host(g["state"]), want["state"].numpy()) <= 8e-5
