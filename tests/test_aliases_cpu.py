"""Outputs that alias inputs or one another are refused where host code can see
it (nothing is launched)."""
import itertools

import pytest
import torch

from paper_2007_00072_amd import lib, runner

PTR = 0x10000


@pytest.fixture(autouse=True)
def float32_by_default():
    # (other test modules may have set another default type)
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def desc(J=64, K=96):
    d = lib.AttnDesc(2, J, K, 8, 8, 64, lib.DM_BF16, 0.0, 0.0, 0)
    d.q = d.out = lib.AttnStride(J * 512, 64, 512)
    d.k = d.v = lib.AttnStride(K * 512, 64, 512)
    return d


def test_attention():
    d = desc()
    _, fwd, bwd = lib.attn_sizes(d)
    own = {n: PTR * (i + 1) for i, n in enumerate(("q", "k", "v", "out", "saved", "dout", "dq", "dk", "dv"))}
    for other in ("q", "k", "v", "saved"):
        p = dict(own, out=own[other])
        with pytest.raises(lib.DmError) as e:
            lib.attn_fwd(d, p["q"], p["k"], p["v"], p["out"], p["saved"], PTR * 100, fwd, stream=0)
        assert e.value.code == lib.DM_ERR_ARG and "out aliases" in str(e.value)
    for name, other in itertools.product(("dq", "dk", "dv"), own):
        if name == other:
            continue
        p = dict(own)
        p[name] = own[other]
        with pytest.raises(lib.DmError) as e:
            lib.attn_bwd(d, *p.values(), PTR * 100, bwd, stream=0)
        assert e.value.code == lib.DM_ERR_ARG and "aliases" in str(e.value)


def test_embedding():
    for y in (PTR, 2 * PTR):
        with pytest.raises(lib.DmError) as e:
            lib.embed_fwd(1, 4, 10, 64, PTR, 2 * PTR, 1.0, y, stream=0)
        assert e.value.code == lib.DM_ERR_ARG and "aliases" in str(e.value)
        with pytest.raises(lib.DmError) as e:
            lib.embed_bwd(1, 4, 10, 64, PTR, -1, 2 * PTR, 1.0, y, 3 * PTR, 1 << 40, stream=0)
        assert e.value.code == lib.DM_ERR_ARG and "aliases" in str(e.value)


def test_optimizer_owner():
    x = torch.zeros(4000)
    with pytest.raises(ValueError, match="share memory"):
        runner.AdamW([x[:1000], x[996:1996]])
    with pytest.raises(ValueError, match="share memory"):
        runner.AdamW([x[:1000], x[1000:2000]], m=[torch.zeros(1000)] * 2)
    with pytest.raises(ValueError, match="share memory"):
        runner.AdamW([x[:16].half()], master=[x[:16]], m=[x[8:24]], v=[torch.zeros(16)])
    runner.AdamW([x[:1000], x[1000:2000], x[:0]], m=[x[2000:3000], x[3000:], torch.zeros(0)])
