"""Embedding lookup and gradient against their definition in 64 bits."""
import pytest
import torch

from paper_2007_00072_amd import lib, runner

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


def make(dt, tokens, V, I, kind="even", seed=1):
    g = torch.Generator().manual_seed(seed)
    table = torch.randn(V, I, generator=g).to(T[dt])
    dy = torch.randn(tokens, I, generator=g).to(T[dt])
    if kind == "even":
        ids = torch.randint(0, V, (tokens,), generator=g)
    elif kind == "one":  # every token the same word
        ids = torch.full((tokens,), V // 2)
    elif kind == "words":  # as words are: uniform in the logarithm of the rank
        ids = (V ** torch.rand(tokens, generator=g, dtype=torch.float64)).long() - 1
    else:  # descending, the last word first
        ids = (V - 1 - torch.arange(tokens)).clamp_min(0)
    return table, dy, ids.clamp(0, V - 1).int()


def check_step(dt, table, dy, ids, scale, pad=-1):
    V, I = table.shape
    e = runner.Embedding(table.to(DEV), scale=scale, pad_id=pad)
    e.grad.fill_(float("nan"))
    y = e.forward(ids.to(DEV))
    d = e.backward(ids.to(DEV), dy.to(DEV))
    torch.cuda.synchronize()
    inside = (ids >= 0) & (ids < V)
    want = torch.where(inside[..., None], table.double()[ids.long().clamp(0, V - 1)], 0.0) * scale
    # one product in float32, then the storage type (fp16: its smallest numbers)
    room = (U[dt] * 1.01 + 2.0 ** -24) * want.abs() + (2.0 ** -25 if dt == "f16" else 0.0)
    assert ((y.cpu().double() - want).abs() <= room).all()
    use = inside & (ids != pad)
    at = ids[use].long()
    want = torch.zeros(V, I, dtype=torch.float64).index_add_(0, at, dy[use].double()) * scale
    size = torch.zeros(V, I, dtype=torch.float64).index_add_(0, at, dy[use].double().abs()) * scale
    n = torch.bincount(at, minlength=V).double()[:, None]
    # a sum of n terms in float32 in any order, one product
    assert ((d.cpu().double() - want).abs() <= (n + 1) * 2.0 ** -24 * abs(size) + 1e-40).all()
    assert (d.cpu()[n[:, 0] == 0] == 0).all()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("tokens,V,I", [(1, 1, 8), (1, 5000, 64), (3, 17, 1032), (255, 40, 72), (256, 1000, 768),
                                        (257, 1000, 8), (2049, 300, 136), (5000, 33000, 64), (20000, 70, 264)])
@pytest.mark.parametrize("kind", ["even", "one", "words", "down"])
def test_lookup_and_gradient(dt, tokens, V, I, kind):
    check_step(dt, *make(dt, tokens, V, I, kind), scale=1.5)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_many_tokens(dt):
    check_step(dt, *make(dt, 70001, 30522, 128, "words"), scale=0.37, pad=0)
    check_step(dt, *make(dt, 65536, 100001, 16, "even"), scale=2.0, pad=100000)


def test_wide_rows():
    check_step("bf16", *make("bf16", 300, 50, 16384, "words"), scale=1.0)


@pytest.mark.parametrize("tokens", [200, 9000])
def test_padding_and_ids_outside(tokens):
    table, dy, ids = make("bf16", tokens, 500, 128, "words")
    ids[::7] = 3
    ids[1::11], ids[2::13], ids[5::17] = -1, 500, 2 ** 31 - 1
    dy[ids == 3] = float("nan")  # padding's gradients are not looked at
    dy[(ids < 0) | (ids >= 500)] = float("inf")
    check_step("bf16", table, dy, ids, 1.0, pad=3)


def test_no_tokens():
    table, dy, ids = make("f16", 0, 40, 64)
    check_step("f16", table, dy, ids, 1.0)


def test_ids_of_any_shape_and_same_bits():
    table, dy, ids = make("f16", 6000, 3000, 96, "words")
    e = runner.Embedding(table.to(DEV))
    shaped = ids.view(3, 50, 40).to(DEV)
    y = e.forward(shaped)
    assert y.shape == (3, 50, 40, 96)
    d1 = e.backward(shaped, dy.view(3, 50, 40, 96).to(DEV)).clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        d2 = e.backward(shaped, dy.view(3, 50, 40, 96).to(DEV)).clone()
    torch.cuda.synchronize()
    assert torch.equal(d1, d2)


@pytest.mark.parametrize("tokens", [100, 20000])
def test_graph_replays(tokens):
    table, dy, ids = make("bf16", tokens, 2000, 64, "words")
    e = runner.Embedding(table.to(DEV))
    ids, dy = ids.to(DEV), dy.to(DEV)
    e.backward(ids, dy)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        e.backward(ids, dy)
    other = make("bf16", tokens, 2000, 64, "words", seed=2)
    for which in (other, make("bf16", tokens, 2000, 64, "one"), other):
        dy.copy_(which[1])
        ids.copy_(which[2])
        e.grad.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        got = e.grad.clone()
        assert torch.equal(got, e.backward(ids, dy))


@pytest.mark.parametrize("tokens", [37, 12345])
def test_writes_stay_inside(tokens):
    V, I, band = 91, 40, 4096
    table, dy, ids = (t.to(DEV) for t in make("f16", tokens, V, I, "words"))
    need = lib.embed_ws_bytes(tokens, V, I)
    bufs = [torch.full((n + 2 * band,), 0xA5, dtype=torch.uint8, device=DEV) for n in (tokens * I * 2, V * I * 4, need)]
    y, d, ws = (b[band:b.numel() - band] for b in bufs)
    lib.embed_fwd(lib.DM_F16, tokens, V, I, ids, table, 1.0, y)
    lib.embed_bwd(lib.DM_F16, tokens, V, I, ids, -1, dy, 1.0, d, ws, need)
    torch.cuda.synchronize()
    for b in bufs:
        assert bool((b[:band] == 0xA5).all()) and bool((b[b.numel() - band:] == 0xA5).all())


def test_a_captured_backward_outlives_a_larger_one():
    # (the larger one needs another workspace; the graph keeps its own)
    table, dy, ids = (t.to(DEV) for t in make("f16", 2000, 2000, 64, "words"))
    e = runner.Embedding(table)
    want = e.backward(ids, dy).clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        e.backward(ids, dy)
    big = [t.to(DEV) for t in make("f16", 30000, 2000, 64, "words", seed=3)]
    large = e.backward(big[2], big[1]).clone()
    others = [torch.full((1 << 20,), -1, dtype=torch.int32, device=DEV) for _ in range(8)]
    for _ in range(2):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(e.grad, want)
        assert torch.equal(e.backward(big[2], big[1]), large)
    assert all((t == -1).all() for t in others)
