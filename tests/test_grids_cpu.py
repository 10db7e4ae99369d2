"""Sizes whose launches would take 2^32 threads along a grid's x (which wrap
without an error) are refused before anything is launched."""
import pytest

from paper_2007_00072_amd import lib

PTR = 0x10000


def attn(B, J, K, H, G, P, **kw):
    d = lib.AttnDesc(B, J, K, H, G, P, lib.DM_BF16, 0.0, 0.0, 0)
    d.q = d.out = lib.AttnStride(J * H * P, P, H * P)
    d.k = d.v = lib.AttnStride(K * G * P, P, G * P)
    for n, x in kw.items():
        setattr(d, n, x)
    return d


@pytest.mark.parametrize("B,J,K,H,G", [(2 ** 21, 1, 1, 8, 8), (2 ** 24, 1, 1, 1, 1), (1, 100, 1, 2 ** 24, 2 ** 24),
                                       (1, 127, 1, 16909320, 1), (2 ** 23, 33, 1, 1, 1)])
def test_attention_blocks(B, J, K, H, G):
    with pytest.raises(lib.DmError) as e:
        lib.attn_sizes(attn(B, J, K, H, G, 8))
    assert e.value.code == lib.DM_ERR_UNSUPPORTED and "blocks" in str(e.value)


@pytest.mark.parametrize("B,J,K,H,G", [(2 ** 31 - 1,) * 5, (2 ** 31 - 1, 2 ** 31 - 1, 1, 2 ** 30, 1),
                                       (1, 1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)])
def test_sizes_whose_products_pass_64_bits(B, J, K, H, G):
    d = attn(1, 1, 1, 1, 1, 8)
    d.B, d.J, d.K, d.H, d.G = B, J, K, H, G
    with pytest.raises(lib.DmError) as e:
        lib.attn_sizes(d)
    assert e.value.code == lib.DM_ERR_UNSUPPORTED and "rows" in str(e.value)


def test_attention_blocks_that_fit():
    for B, J, K, H, G in ((2 ** 21 - 1, 1, 1, 8, 8), (2 ** 24 - 1, 1, 1, 1, 1), (1, 2 ** 30, 1, 1, 1), (8, 512, 512, 16, 16)):
        lib.attn_sizes(attn(B, J, K, H, G, 8))


@pytest.mark.parametrize("P,K,ok", [(64, 2 ** 30 - 1024, True), (64, 2 ** 30 - 64, False), (128, 2 ** 29, False)])
def test_attention_backward_blocks(P, K, ok):
    d = attn(2, 1, K, 1, 1, P)
    bwd = lib.attn_sizes(d)[2]
    with pytest.raises(lib.DmError) as e:
        lib.attn_bwd(d, *[PTR] * 9, PTR, bwd - 1, stream=0)
    assert e.value.code == (lib.DM_ERR_WORKSPACE if ok else lib.DM_ERR_UNSUPPORTED)


@pytest.mark.parametrize("n", [2 ** 36 - 4095, 2 ** 42, 2 ** 63 - 1])
def test_optimizer_blocks(n):
    a = lib.AdamwDesc(lib.DM_BF16, 8, 1e-3, 0.9, 0.999, 1e-8, 1.0, 1, None)
    t = (lib.AdamwTensor * 1)(lib.AdamwTensor(PTR, None, PTR, PTR, PTR, PTR, PTR, n, 0.0))
    with pytest.raises(lib.DmError) as e:
        lib.adamw_step(a, t, 1, stream=0)
    assert e.value.code == lib.DM_ERR_UNSUPPORTED and "n=" in str(e.value)
