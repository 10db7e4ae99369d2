"""The operators as a program uses them together: ids to embeddings, a layer,
gradients back to the table, an optimiser step on all of it; attention on
packed documents between the library's own contractions; single tokens over a
cache that a prompt has filled."""
import pytest
import torch

from _attention import check, reference
from paper_2007_00072_amd import lib, runner
from paper_2007_00072_amd.inputs import WORKLOADS, Shape, make_activation, make_params

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(autouse=True)
def float32_by_default():
    # (other test modules may have set another default type)
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def train_step(emb, layer, opt, ids, dy, step):
    x = emb.forward(ids)
    y = layer.forward(x)
    dx = layer.backward(x, dy)
    emb.backward(ids, dx)
    opt.step([layer.grads[n] for n in layer.params] + [emb.grad], step)
    return y


@pytest.mark.parametrize("bits", [32, 8])
def test_a_training_step_of_a_layer(bits):
    wl = WORKLOADS["bert_large_f16"].with_(shape=Shape(B=2, J=64, K=64, H=4, P=64, W=64, I=256, F=1024))
    g = torch.Generator().manual_seed(5)
    table = (torch.randn(1000, 256, generator=g) * 0.1).half().to(DEV)
    ids = torch.randint(0, 1000, (2, 64), generator=g).int().to(DEV)
    dy = make_activation(wl, 1).to(DEV)

    def made():
        emb = runner.Embedding(table.clone(), scale=16.0, pad_id=0)
        layer = runner.EncoderLayer(runner.desc_for(wl), make_params(wl), DEV)
        opt = runner.AdamW([*layer.params.values(), emb.table], lr=1e-3, decay=0.01, state_bits=bits)
        return emb, layer, opt

    a, b = made(), made()
    before = {n: t.clone() for n, t in a[1].params.items()}
    y1 = train_step(*a, ids, dy, 1)
    torch.cuda.synchronize()
    # the first step: m = (1 - b1) g, v = (1 - b2) g^2, so a step of lr sign(g) but for eps
    for n, t in a[1].params.items():
        gr = a[1].grads[n].double()
        want = before[n].double() * (1 - 1e-3 * 0.01) - 1e-3 * gr / (gr.abs() + 1e-8)
        # (the quotient's roundings in float32, and the weight's in half precision)
        room = 1e-3 * 32 * 2.0 ** -24 + 2.0 ** -11 * 1.01 * want.abs() + 2.0 ** -24
        big = gr.abs() > 1e-12  # (squares of smaller ones leave float32's normal numbers)
        assert ((t.double() - want).abs() <= room)[big].all(), n
    y2 = train_step(*a, ids, dy, 2)
    torch.cuda.synchronize()
    assert not torch.equal(y1, y2)
    # the same two steps, the second as a graph
    train_step(*b, ids, dy, 1)
    torch.cuda.synchronize()
    sc = torch.tensor([1e-3, 1 / (1 - 0.9 ** 2), 1 / (1 - 0.999 ** 2), 1.0], device=DEV)
    emb, layer, opt = b
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x = emb.forward(ids)
        y = layer.forward(x)
        emb.backward(ids, layer.backward(x, dy))
        grads = [layer.grads[n] for n in layer.params] + [emb.grad]
        opt.step(grads, 2, scalars=sc)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, y2)
    for p, q in zip(a[2].master, b[2].master):
        assert ((p - q).abs() <= 4 * 2.0 ** -24 * (p.abs() + 1)).all()


def test_packed_documents_between_contractions():
    # x -> [q k v] = x w -> attention -> o; back through both, all in float32
    B, L, H, G, P, I = 2, 96, 4, 2, 32, 64
    g = torch.Generator().manual_seed(3)
    n = (H + 2 * G) * P
    x, w = torch.randn(B * L, I, generator=g), torch.randn(I, n, generator=g) * 0.2
    dout = torch.randn(B, L, H, P, generator=g)
    doc = torch.stack([(torch.arange(L) // 30).int(), (torch.arange(L) // 50).int()])
    dx, dw = (torch.empty(B * L, I, device=DEV), torch.empty(I, n, device=DEV))
    xd, wd = x.to(DEV), w.to(DEV)
    qkv, dqkv = torch.empty(B, L, H + 2 * G, P, device=DEV), torch.empty(B, L, H + 2 * G, P, device=DEV)
    f = lib.DM_F32
    lib.contract(f, 1, B * L, n, I, 1.0, xd, 0, 0, wd, 0, 0, None, qkv, 1, 0)
    parts = lambda t: (t[:, :, :H], t[:, :, H:H + G], t[:, :, H + G:])  # noqa: E731
    a = runner.Attention(*parts(qkv), causal=True, doc=doc.to(DEV), cap=8.0)
    out = a.forward(*parts(qkv))
    a.backward(*parts(qkv), out, dout.to(DEV), *parts(dqkv))
    lib.contract(f, 1, B * L, I, n, 1.0, dqkv, 0, 0, wd, 1, 0, None, dx, 1, 0)
    lib.contract(f, 1, I, n, B * L, 1.0, xd, 1, 0, dqkv, 0, 0, None, dw, 1, 0)
    torch.cuda.synchronize()
    X, W = x.double().requires_grad_(), w.double().requires_grad_()
    q, k, v = parts((X @ W).view(B, L, H + 2 * G, P))
    k, v = k.repeat_interleave(H // G, 2), v.repeat_interleave(H // G, 2)
    s = 8 * torch.tanh(torch.einsum("bjhp,bkhp->bhjk", q, k) / P ** 0.5 / 8)
    see = (doc[:, :, None] == doc[:, None, :]) & torch.ones(L, L, dtype=torch.bool).tril()
    y = torch.einsum("bhjk,bkhp->bjhp", torch.softmax(s.masked_fill(~see[:, None], float("-inf")), -1), v)
    y.backward(dout.double())
    # sums of up to 256 terms in float32 after sums of 64 and 96: far under 2^-12 of the largest element
    for name, got, want in (("out", out, y), ("dx", dx, X.grad), ("dw", dw, W.grad)):
        err = (got.cpu().double().view(want.shape) - want).abs().max() / want.abs().max()
        assert float(err.detach()) < 2.0 ** -14, name


def test_a_prompt_then_single_tokens():
    B, H, G, P, cap_len, prompt = 2, 8, 2, 64, 400, 290
    g = torch.Generator().manual_seed(8)
    q, k, v = (torch.randn(B, prompt + 6, n, P, generator=g).bfloat16() for n in (H, G, G))
    slopes = torch.exp2(-torch.arange(1, H + 1).double()).float()
    want = reference(q, k, v, causal=True, slopes=slopes)["out"]
    cache = [torch.full((B, G, cap_len, P), float("nan"), dtype=torch.bfloat16, device=DEV).transpose(1, 2) for _ in "kv"]
    n = torch.full((B,), prompt, dtype=torch.int32, device=DEV)
    for c, t in zip(cache, (k, v)):
        c[:, :prompt] = t[:, :prompt].to(DEV)
    qd = q.to(DEV)
    kw = dict(causal=True, k_len=n, slopes=slopes.to(DEV), train=False)
    out = [runner.Attention(qd[:, :prompt], *cache, **kw).forward(qd[:, :prompt], *cache)]
    one = runner.Attention(qd[:, :1], *cache, **kw)
    for i in range(prompt, prompt + 6):
        for c, t in zip(cache, (k, v)):
            c[:, i] = t[:, i].to(DEV)
        n += 1
        out.append(one.forward(qd[:, i:i + 1], *cache))
    torch.cuda.synchronize()
    check("out", torch.cat(out, 1), want)
