"""A query adds to the rows that it sees, whatever its logits are: a NaN or an infinity in it, or in a row that it sees, stays out of
the others.  Tolerance as in test_gpu_cache_budget.py: 5.5e-5 of a logit, T 2^-24 of a sum."""
import math

import pytest
import torch

import paper_2602_03681_amd as nats
import serve_reference as ref

pytestmark = pytest.mark.gpu
TOL = 5.5e-5 + 1.2e-5
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def inputs(T, dtype, d=64, n=90, cap=100):
    g = torch.Generator().manual_seed(T)
    rnd = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    return dict(weights=torch.rand(1, 2, cap, generator=g), q=rnd(1, 2, T, d).to(dtype), k_cache=rnd(1, 2, cap, d).to(dtype),
                cache_len=torch.full((1, 2), n, dtype=torch.int32))


def close(got, want):
    return float(((got.cpu().double() - want).abs() / want).max()) <= TOL


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 5, 16, 17, 64, 65, 200])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("with_lse", [False, True])
def test_a_querys_nan_stays_in_the_rows_that_it_sees(dtype, T, bad, with_lse):
    x = inputs(T, DT[dtype])
    vis = torch.full((1, 2, T), 90, dtype=torch.int32)
    vis[:, :, T // 2] = 37
    lse = None
    if with_lse:
        _, lse = ref.cache_weights(**x, vis=vis)
        lse = lse.float()
    # the same without that query
    none = vis.clone()
    none[:, :, T // 2] = 0
    want, _ = ref.cache_weights(**x, vis=none, lse=lse, decay=0.5)
    x["q"][:, :, T // 2, 3] = bad
    g = {k: v.cuda() for k, v in x.items()}
    got = nats.cache_weights(*(g[k] for k in ("weights", "q", "k_cache", "cache_len")), vis=vis.cuda(), decay=0.5,
                             lse=None if lse is None else lse.cuda())
    if math.isnan(bad):
        assert torch.isnan(got[:, :, :37]).all()
    assert close(got[:, :, 37:90], want[:, :, 37:90])
    assert torch.equal(got[:, :, 90:].cpu(), x["weights"][:, :, 90:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [2, 16, 40, 100])
def test_a_rows_nan_stays_with_the_queries_that_see_it(dtype, T):
    """Row 50 is NaN: every other query sees it, and rows up to 80; the rest see 50 rows."""
    x = inputs(T, DT[dtype])
    vis = torch.full((1, 2, T), 50, dtype=torch.int32)
    vis[:, :, 1::2] = 80
    want, _ = ref.cache_weights(**x, vis=torch.zeros_like(vis), decay=0.25)
    x["k_cache"][:, :, 50] = math.nan
    g = {k: v.cuda() for k, v in x.items()}
    got = nats.cache_weights(*(g[k] for k in ("weights", "q", "k_cache", "cache_len")), vis=vis.cuda(), decay=0.25)
    assert torch.isnan(got[:, :, :80]).all()
    assert close(got[:, :, 80:90], want[:, :, 80:90])
