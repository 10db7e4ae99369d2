"""Scores far above what a trained model has, up to the bound that the header
states: every query's first key takes all."""
import pytest
import torch

from paper_2007_00072_amd import runner

pytestmark = pytest.mark.gpu
DEV = "cuda"
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(autouse=True)
def float32_by_default():
    # (other test modules may have set another default type)
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("J", [3, 300])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("log", [10, 14, 18, 24])
def test_one_key_takes_all(dt, J, sign, log):
    # all products are exact; the largest score 2^log and the others half of it, or -2^(log - 1) and -2^log
    B, K, H, P, scaler = 2, 520, 8, 64, 0.125
    first, others = (2.0 ** log, 2.0 ** (log - 1)) if sign > 0 else (-2.0 ** (log - 1), -2.0 ** log)
    a = 2.0 ** (log // 2 - 1)
    at = torch.arange(H) * 60
    q = torch.full((B, J, H, P), a).to(T[dt])
    k = torch.full((B, K, H, P), others / (8 * a))
    for h in range(H):
        k[:, at[h], h] = first / (8 * a)
    k = k.to(T[dt])
    assert float(q[0, 0, 0].double() @ k[0, 0, 0].double()) * scaler == first
    g = torch.Generator().manual_seed(log)
    v, dout = (torch.randn(B, L, H, P, generator=g).to(T[dt]) for L in (K, J))
    d = [x.to(DEV) for x in (q, k, v)]
    att = runner.Attention(*d, scaler=scaler)
    out = att.forward(*d)
    dq, dk, dv = att.backward(*d, out, dout.to(DEV))
    torch.cuda.synchronize()
    want = torch.stack([v[:, at[h], h] for h in range(H)], 1)[:, None].double()
    # one probability of 1, the others 0: it is rounded for the product and not in the sum, then the quotient is
    assert ((out.cpu().double() - want).abs() <= (8 * 2.0 ** -24 + 2.02 * U[dt]) * want.abs() + 1e-30).all()
    assert all(torch.isfinite(t).all() for t in (dq, dk, dv))
    got = torch.stack([dv[:, at[h], h] for h in range(H)], 1).cpu().double()
    if log <= 18:
        sums, size = dout.double().sum(1), dout.double().abs().sum(1)
        # the log-sum, 2^log / ln 2, is off by half a step of float32: 2^(log - 24) of the probability (2 % for higher
        # orders), which is rounded; sums of J terms in float32, rounded
        room = (2.0 ** (log - 24) * 1.02 + 1.01 * U[dt] + (J + 8) * 2.0 ** -24) * size + U[dt] * 1.01 * sums.abs()
        assert ((got - sums).abs() <= room).all()
        rest = dv.clone()
        for h in range(H):
            rest[:, at[h], h] = 0
        assert not rest.any()
