"""Host-side checks of nats_serve.h and its binding that need no GPU: what is refused is refused before anything is launched."""
import ctypes
import os

import pytest
import torch

import paper_2602_03681_amd as nats
from paper_2602_03681_amd import binding as nb
from paper_2602_03681_amd import serve

OK, E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_WS = 0, -1, -2, -3, -4, -5
FAKE = 0x10000  # an aligned non-NULL "device pointer"; validation fails before it is ever used
F32, BF16 = nb.NATS_F32, nb.NATS_BF16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(nb.library_path()):
        from paper_2602_03681_amd.build import build_library
        build_library()
    return nb.load_library()


def tree_params(**over):
    kw = dict(B=2, H=2, T=8, d=128, cap=512, dtype=BF16, group=1)
    kw.update(over)
    p = serve.TreeParams()
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def ptrs(n, **over):
    a = [FAKE + 256 * i for i in range(n)]
    for i, v in over.items():
        a[int(i[1:])] = v
    return a


def tree(lib, p, a=None, ws=FAKE + 65536, size=1 << 40):
    return lib.nats_hybrid_attn_decode_tree(None if p is None else ctypes.byref(p), *(a or ptrs(16)), ws, size, None)


def commit(lib, p, a=None):
    return lib.nats_hybrid_attn_tree_commit(None if p is None else ctypes.byref(p), *(a or ptrs(13)), None)


BAD_TREES = [(dict(T=0), E_SHAPE), (dict(T=65), E_SHAPE), (dict(T=-1), E_SHAPE), (dict(B=0), E_SHAPE), (dict(H=-2), E_SHAPE),
             (dict(d=96), E_SHAPE), (dict(cap=0), E_SHAPE), (dict(cap=(1 << 20) + 1), E_SHAPE), (dict(dtype=2), E_DTYPE),
             (dict(group=9), E_SHAPE), (dict(group=-1), E_SHAPE), (dict(B=40000, group=1), E_SHAPE), (dict(B=9000, group=8), E_SHAPE),
             (dict(combine_mode=3), E_SHAPE), (dict(linear_op=2), E_SHAPE), (dict(freeze_on_softmax=2), E_SHAPE)]


@pytest.mark.parametrize("over,code", BAD_TREES)
def test_tree_params(lib, over, code):
    p = tree_params(**over)
    assert tree(lib, p) == code and lib.nats_last_error() != b""
    assert commit(lib, p) == code
    assert lib.nats_hybrid_attn_decode_tree_workspace_bytes(ctypes.byref(p)) == 0


def test_tree_pointers(lib):
    p = tree_params()
    assert tree(lib, None) == E_NULL and commit(lib, None) == E_NULL
    need = lib.nats_hybrid_attn_decode_tree_workspace_bytes(ctypes.byref(p))
    assert need > 2 * 2 * 8 * 128 * 4
    for i in range(11):                       # state .. parent
        assert tree(lib, p, ptrs(16, **{f"p{i}": None})) == E_NULL, i
    assert tree(lib, p, ptrs(16, p14=None)) == E_NULL             # o
    for i in (0, 1, 2, 4, 5, 6, 14):
        assert tree(lib, p, ptrs(16, **{f"p{i}": FAKE + 2})) == E_ALIGN, i
    assert tree(lib, p, ws=None) == E_WS and tree(lib, p, size=need - 1) == E_WS and b"needed" in lib.nats_last_error()
    assert tree(lib, p, ws=FAKE + 4) == E_ALIGN
    for i in (0, 1, 2, 4, 5, 6):              # outputs that are inputs
        assert tree(lib, p, ptrs(16, p14=FAKE + 256 * i)) == E_SHAPE, i
        assert tree(lib, p, ptrs(16, p15=FAKE + 256 * i)) == E_SHAPE, i
    assert tree(lib, tree_params(q_nla=FAKE)) == E_NULL and tree(lib, tree_params(k_nla=FAKE)) == E_NULL
    assert tree(lib, tree_params(q_nla=FAKE, k_nla=FAKE + 8)) == E_ALIGN
    assert tree(lib, p, ptrs(16, p15=FAKE + 256 * 14)) == E_SHAPE  # o and lse
    for i in range(11):                       # state .. node
        assert commit(lib, p, ptrs(13, **{f"p{i}": None})) == E_NULL, i
    assert commit(lib, p, ptrs(13, p2=FAKE + 256)) == E_SHAPE      # k_cache and v_cache
    for i in (0, 1, 2):
        assert commit(lib, p, ptrs(13, p4=FAKE + 256 * i)) == E_SHAPE, i
        assert commit(lib, p, ptrs(13, p5=FAKE + 256 * i)) == E_SHAPE, i
    for i in (0, 1, 2, 4, 5):
        assert commit(lib, p, ptrs(13, **{f"p{i}": FAKE + 8})) == E_ALIGN, i
    assert commit(lib, tree_params(k_nla=FAKE + 8)) == E_ALIGN


def weights_params(**over):
    kw = dict(B=2, H=6, T=8, d=64, cap=512, dtype=F32, q_group=1, vis_group=1, softmax_scale=0.0, decay=1.0)
    kw.update(over)
    return serve.CacheWeightsParams(*(kw[f[0]] for f in serve.CacheWeightsParams._fields_))


def weights(lib, p, a=None, ws=FAKE + 65536, size=1 << 40):
    return lib.nats_cache_weights(None if p is None else ctypes.byref(p), *(a or ptrs(6)), ws, size, None)


@pytest.mark.parametrize("over,code", [(dict(T=0), E_SHAPE), (dict(d=80), E_SHAPE), (dict(cap=0), E_SHAPE), (dict(dtype=7), E_DTYPE),
                                       (dict(B=0), E_SHAPE), (dict(q_group=4), E_SHAPE), (dict(vis_group=5), E_SHAPE),
                                       (dict(q_group=-1), E_SHAPE), (dict(B=1, H=1, T=(1 << 20) + 1), E_SHAPE), (dict(B=20000), E_SHAPE)])
def test_weights_params(lib, over, code):
    assert weights(lib, weights_params(**over)) == code
    assert lib.nats_cache_weights_workspace_bytes(ctypes.byref(weights_params(**over)), 0) == 0


def test_weights_pointers(lib):
    p = weights_params()
    assert weights(lib, None) == E_NULL
    for i in range(4):
        assert weights(lib, p, ptrs(6, **{f"p{i}": None})) == E_NULL, i
    for i in (0, 1, 2):
        assert weights(lib, p, ptrs(6, **{f"p{i}": FAKE + 4})) == E_ALIGN, i
    for i in (1, 2, 5):
        assert weights(lib, p, ptrs(6, p0=FAKE + 256 * i)) == E_SHAPE, i
    need = lib.nats_cache_weights_workspace_bytes(ctypes.byref(p), 0)
    assert need >= 2 * 6 * 8 * 4
    no_lse = ptrs(6, p5=None)
    assert weights(lib, p, no_lse, ws=None) == E_WS and weights(lib, p, no_lse, size=need - 1) == E_WS


def evict(lib, a=None, **over):
    kw = dict(B=2, H=2, d=64, cap=512, dtype=F32, keep=100, recent=10)
    kw.update(over)
    p = serve.CacheEvictParams(*(kw[f[0]] for f in serve.CacheEvictParams._fields_))
    return lib.nats_cache_evict(ctypes.byref(p), *(a or ptrs(5)), None)


@pytest.mark.parametrize("over,code", [(dict(keep=0), E_SHAPE), (dict(keep=513), E_SHAPE), (dict(recent=-1), E_SHAPE),
                                       (dict(recent=101), E_SHAPE), (dict(d=32), E_SHAPE), (dict(dtype=3), E_DTYPE),
                                       (dict(cap=-1), E_SHAPE), (dict(H=0), E_SHAPE)])
def test_evict_params(lib, over, code):
    assert evict(lib, **over) == code


def test_evict_pointers(lib):
    assert lib.nats_cache_evict(None, *ptrs(5), None) == E_NULL
    for i in range(5):
        assert evict(lib, ptrs(5, **{f"p{i}": None})) == E_NULL, i
    for i in (0, 1, 3):
        assert evict(lib, ptrs(5, **{f"p{i}": FAKE + 8})) == E_ALIGN, i
    assert evict(lib, ptrs(5, p1=FAKE)) == E_SHAPE


def test_tensors_that_are_not_on_the_gpu_or_of_another_shape(lib):
    """The binding's own checks, before a pointer is taken."""
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)   # noqa: E731
    i = lambda *s: z(*s, dtype=torch.int32)                            # noqa: E731
    st = (z(1, 2, 64, 64), z(1, 2, 16, 64), z(1, 2, 16, 64), i(1, 2))
    node = (z(1, 2, 4, 64), z(1, 2, 4, 64), z(1, 2, 4), z(1, 2, 4), z(1, 2, 4, dtype=torch.uint8), i(1, 4))
    with pytest.raises(ValueError, match="GPU tensor"):
        nats.hybrid_attn_decode_tree(*st, node[0], *node)
    with pytest.raises(ValueError, match="GPU tensor"):
        nats.hybrid_attn_tree_commit(*st, *node, i(1))
    with pytest.raises(ValueError, match="group"):
        nats.hybrid_attn_decode_tree(*st, node[0], *node, group=2)
    with pytest.raises(ValueError, match="4 dimensions"):
        nats.hybrid_attn_tree_commit(*st, z(1, 2, 64), *node[1:], i(1))
    with pytest.raises(ValueError, match="GPU tensor"):
        nats.cache_weights(z(1, 2, 16), z(1, 2, 3, 64), st[1], st[3])
    with pytest.raises(ValueError, match="divides"):
        nats.cache_weights(z(1, 2, 16), z(1, 3, 3, 64), st[1], st[3])
    with pytest.raises(ValueError, match="divides"):
        nats.cache_weights(z(1, 2, 16), z(1, 2, 3, 64), st[1], st[3], vis=i(1, 4, 3))
    with pytest.raises(ValueError, match="GPU tensor"):
        nats.cache_evict(st[1], st[2], st[3], z(1, 2, 16), 8)


def test_sizes_whose_product_passes_64_bits(lib):
    big = dict(B=1 << 30, H=1 << 30)
    assert tree(lib, tree_params(**big, group=8)) == E_SHAPE and commit(lib, tree_params(**big, group=8)) == E_SHAPE
    assert evict(lib, B=(1 << 31) - 1, H=(1 << 31) - 1) == E_SHAPE
