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


def test_a_large_value_behind_a_long_sequence():
    # (the largest |v| is looked for in groups of keys, which grow with the sequence)
    J, K, P, half = 5, 70001, 16, torch.float16
    g = torch.Generator().manual_seed(2)
    q, v, dout = torch.randn(1, J, 1, P, generator=g), torch.randn(1, K, 1, P, generator=g), torch.ones(1, J, 1, P)
    k = torch.zeros(1, K, 1, P)
    k[:, -2:] = 4.0 * q.mean(1, keepdim=True)
    v[:, -1], v[:, -2] = 50000.0, -50000.0
    q, k, v, dout = q.to(half), k.to(half), v.to(half), (dout * 2.0 ** -12).to(half)
    want = reference(q, k, v, dout, scaler=8.0)
    d = [x.to(DEV) for x in (q, k, v)]
    a = runner.Attention(*d, scaler=8.0)
    out = a.forward(*d)
    grads = a.backward(*d, out, dout.to(DEV))
    torch.cuda.synchronize()
    # (as above: 2^s more under fp16's normal numbers)
    s = float(torch.floor(torch.log2(P * v.double().abs().max()))) - 15
    more = 2.0 ** -24 * 2.0 ** -12 * (2 ** s - 1) * 8.0
    want["dq"] = (want["dq"][0], want["dq"][1] + more * k.double().abs().sum(1, keepdim=True))
    want["dk"] = (want["dk"][0], want["dk"][1] + more * q.double().abs().sum(1, keepdim=True))
    for n, x in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        check(n, x, want[n])


def test_graph_replays():
    # the step's largest |dout| and |v| are found anew in every replay
    B, L, H, G, P = 2, 300, 4, 2, 64
    g = torch.Generator().manual_seed(3)
    sets = [[(torch.randn(B, L, n, P, generator=g) * std).half().to(DEV) for n, std in ((H, 1), (G, 1), (G, sv), (H, sd))]
            for sv, sd in ((1.0, 1.0), (5000.0, 1e-3), (1e-3, 100.0))]
    a = runner.Attention(*sets[0][:3], causal=True)

    def step(q, k, v, dout):
        out = a.forward(q, k, v)
        return (out, *a.backward(q, k, v, out, dout))

    want = [[t.clone() for t in step(*s)] for s in sets]
    held = [t.clone() for t in sets[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*held)
    for i in (1, 0, 2, 1):
        for x, y in zip(held, sets[i]):
            x.copy_(y)
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want[i]))
        assert all(torch.equal(x, y) for x, y in zip(step(*sets[i]), want[i]))
