"""fp16 gradients where the values are large: a score's gradient p (dout . v -
D) passes the type's largest number although dq, dk and dv do not."""
import pytest
import torch

from _attention import check, reference
from paper_2007_00072_amd import runner

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(autouse=True)
def float32_by_default():
    # (other test modules may have set another default type)
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.mark.parametrize("J,K,H,G,P,size", [(40, 2, 2, 2, 128, 3000.0), (300, 3, 4, 2, 128, 60000.0),
                                            (129, 2, 2, 1, 64, 20000.0), (33, 40, 1, 1, 128, 4000.0),
                                            (300, 301, 8, 2, 128, 3000.0)])
@pytest.mark.parametrize("cap", [0.0, 4.0])
def test_values_of_one_sign_over_a_head(J, K, H, G, P, size, cap):
    B, half = 2, torch.float16
    g = torch.Generator().manual_seed(K)
    q, k, v, dout = (torch.randn(B, L, n, P, generator=g) for L, n in ((J, H), (K, G), (K, G), (J, H)))
    # (values and gradients agree in sign over the head, two or three keys share what a query sees)
    sign = torch.where(torch.arange(K) % 2 == 0, 1.0, -1.0)[None, :, None, None]
    q, k = (q * 0.5).to(half), k.to(half)
    v = (sign * size * (1 - 0.1 * v.abs().clamp_max(5))).to(half)
    dout = ((1 - 0.1 * dout.abs().clamp_max(5)) * 16 / (P * size)).to(half)
    doc = (torch.arange(K) // 2).int().expand(B, K).contiguous()
    pad = torch.zeros(B, K, dtype=torch.int32)
    for kw in (dict(), dict(doc=doc, causal=True) if J == K - 1 else dict(k_len=pad[:, 0] + K)):
        kw["cap"] = cap
        want = reference(q, k, v, dout, **kw)
        # A score gradient is held as 2^e p (dout . v - D) (capped scores: a quarter of its slope's share), with 2^e
        # from 1 / (4 top) to 1 / (2 top) for the largest |dout| top, less 2^s where P |v| is 2^(15 + s) to 2^(16 + s).
        # Under fp16's normal numbers it is off by 2^-25; the reference has room for that at s = 0 without a cap.
        s = max(0.0, float(torch.floor(torch.log2(P * v.double().abs().max()))) - 15)
        more = 2.0 ** -24 * float(dout.double().abs().max()) * (2 ** s * (4 if cap else 1) - 1) / P ** 0.5
        rows = {"dq": k.double().abs().sum(1, keepdim=True).repeat_interleave(H // G, 2),
                "dk": q.double().abs().sum(1, keepdim=True).view(B, 1, G, H // G, P).sum(3)}
        for n, r in rows.items():
            want[n] = (want[n][0], want[n][1] + more * r)
        on = {n: x.to(DEV) if isinstance(x, torch.Tensor) else x for n, x in kw.items()}
        d = [x.to(DEV) for x in (q, k, v)]
        a = runner.Attention(*d, **on)
        out = a.forward(*d)
        grads = a.backward(*d, out, dout.to(DEV))
        torch.cuda.synchronize()
        for n, x in zip(("out", "dq", "dk", "dv"), (out, *grads)):
            check(n, x, want[n])
