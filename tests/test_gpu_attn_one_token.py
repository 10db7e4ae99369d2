"""Attention where an axis has one token: its stride is never taken, so what a
descriptor holds there (0, a large number) changes nothing."""
import pytest
import torch

from _attention import check, reference
from paper_2007_00072_amd import lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def float32_by_default():
    # (other test modules may have set another default type)
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("J,K", [(1, 1), (70, 1), (1, 130), (200, 1)])
@pytest.mark.parametrize("t", [0, 8, 2 ** 20, 2 ** 31, 2 ** 32 + 64])
def test_stride_of_one_token(dt, J, K, t):
    B, H, G, P = 2, 4, 2, 64
    g = torch.Generator().manual_seed(J + K)
    q, k, v, dout = (torch.randn(B, L, n, P, generator=g).to(T[dt]) for L, n in ((J, H), (K, G), (K, G), (J, H)))
    d = lib.AttnDesc(B, J, K, H, G, P, lib.DTYPE_CODES[dt], 0.0, 0.0, 0)
    d.q = d.out = lib.AttnStride(J * H * P, P, H * P if J > 1 else t)
    d.k = d.v = lib.AttnStride(K * G * P, P, G * P if K > 1 else t)
    saved_bytes, fwd, bwd = lib.attn_sizes(d)
    ws = torch.empty(max(fwd, bwd, 1), dtype=torch.uint8, device=DEV)
    saved = torch.empty(saved_bytes, dtype=torch.uint8, device=DEV)
    qd, kd, vd, gd = (x.to(DEV) for x in (q, k, v, dout))
    out, dq, dk, dv = (torch.full_like(x, float("nan")) for x in (qd, qd, kd, vd))
    lib.attn_fwd(d, qd, kd, vd, out, saved, ws, ws.numel())
    lib.attn_bwd(d, qd, kd, vd, out, saved, gd, dq, dk, dv, ws, ws.numel())
    torch.cuda.synchronize()
    want = reference(q, k, v, dout)
    for n, x in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
        check(f"{n} {dt}", x, want[n])
