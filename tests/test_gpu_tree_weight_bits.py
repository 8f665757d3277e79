"""The softmax weights of a tree over bf16 caches hold fp32's bits.

Two cached rows whose logits are one product each and whose values cancel: row 1's value is what takes row 0's share back, to bf16's
rounding.  What is left is about 2^-10 of the shares' sizes, so an error in a weight shows that an output of bf16 would hide.

Tolerance, relative to the shares' sizes A = sum p |v| / sum p.  A logit in powers of two, at most 4 in size, is off by 4 roundings of
it (the factor three, the product one), both of them and their difference: (2 * 4 * 4 + 4) 2^-24, times ln 2 is 25 2^-24 of the weight;
the exponential, two terms' sums and the division bring 7 2^-24 more: 2^-19.  A weight held to 17 bits is off by up to 2^-16."""
import pytest
import torch

import paper_2602_03681_amd as nats
from gpu_util import bf16_half_ulp, host

pytestmark = pytest.mark.gpu
TOL = 2.0 ** -19


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 20, 64])
@pytest.mark.parametrize("H", [96, 160])
def test_a_weights_bits(d, T, H):
    g = torch.Generator().manual_seed(d + T)
    bf = torch.bfloat16
    scale = d ** -0.5
    q, k = torch.zeros(1, H, T, d, dtype=bf), torch.zeros(1, H, 2, d, dtype=bf)
    q[..., 0] = (scale ** -0.5 * (1 + torch.rand(1, H, 1, generator=g))).to(bf)      # the same for all nodes of a head
    k[..., 0] = (scale ** -0.5 * (torch.rand(1, H, 2, generator=g) * 2 - 1) * 0.69).to(bf)
    z = scale * q[:, :, :1, 0].double() * k[..., 0].double()                                 # [1,H,2]
    assert float(z.abs().max()) / 0.6931 <= 4
    p = torch.exp(z - z.amax(-1, keepdim=True))
    v = torch.randn(1, H, 2, d, generator=g).to(bf)
    v[:, :, 1] = (-p[..., :1] * v[:, :, 0].double() / p[..., 1:]).to(bf)
    share = p[..., None] * v.double() / p.sum(-1)[..., None, None]
    want, size = share.sum(2), share.abs().sum(2)                                             # [1,H,d]
    zero = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype).cuda()   # noqa: E731
    cap = 2 if H < 128 else 1100      # more heads and longer caches: the caches in equal shares
    kc, vc = zero(1, H, cap, d, dtype=bf), zero(1, H, cap, d, dtype=bf)
    kc[:, :, :2], vc[:, :, :2] = k.cuda(), v.cuda()
    o, _ = nats.hybrid_attn_decode_tree(zero(1, H, d, d), kc, vc, torch.full((1, H), 2, dtype=torch.int32, device="cuda"),
                                        zero(1, H, T, d, dtype=bf), zero(1, H, T, d, dtype=bf), zero(1, H, T, d, dtype=bf),
                                        zero(1, H, T), zero(1, H, T), zero(1, H, T, dtype=torch.uint8),
                                        torch.full((1, T), -1, dtype=torch.int32, device="cuda"), q_nla=q.cuda(),
                                        k_nla=zero(1, H, T, d, dtype=bf))
    off = abs(host(o) - want[:, :, None].numpy()) - bf16_half_ulp(want[:, :, None].numpy())
    assert float((off / size[:, :, None].numpy()).max()) <= TOL
