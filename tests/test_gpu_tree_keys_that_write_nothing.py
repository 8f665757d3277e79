"""The linear branch does not read the key of a softmax token: with softmax keys of its own (k_nla) what stands there in k, an infinity or
a NaN included, has no influence on the token's own row nor on its descendants'.  Tolerances as in test_gpu_tree.py."""
import math

import pytest
import torch

import paper_2602_03681_amd as nats
import serve_reference as ref
from gpu_util import host, rel_err

pytestmark = pytest.mark.gpu
TOL = {torch.float32: 8e-5, torch.bfloat16: 2.4e-4}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ARGS = ("state", "k_cache", "v_cache", "cache_len", "q", "k", "v", "alpha", "beta", "mask", "parent")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("linear_op", [0, 1])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("T,tree", [(1, "chain"), (12, "chain"), (12, "star"), (50, "tree")])
def test_a_softmax_tokens_linear_key(dtype, linear_op, bad, T, tree):
    x = ref.tree_inputs(2, 2, T, 64, 40, DT[dtype], seed=31 + T, own_qk=True, p=0.4, tree=tree)
    x["mask"][:, :, 0] = 1                                        # a root
    want_o, want_lse = ref.decode_tree(x, linear_op=linear_op)
    x["k"][x["mask"] != 0] = bad
    g = {k: v.cuda() for k, v in x.items()}
    o, lse = nats.hybrid_attn_decode_tree(*(g[k] for k in ARGS), q_nla=g["q_nla"], k_nla=g["k_nla"], linear_op=linear_op)
    assert torch.isfinite(o).all()
    assert rel_err(host(o), want_o.numpy(), "bf16" if dtype == "bf16" else None) <= TOL[DT[dtype]]
    assert float((lse.cpu().double() - want_lse).abs().max()) <= 6e-5
