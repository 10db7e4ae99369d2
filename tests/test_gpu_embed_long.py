"""Embedding lookup and gradient over more tokens than one row of a grid holds
threads for (2^32), against values that are exact in every type."""
import pytest
import torch

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


def room(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GB")


def test_lookup_of_many_wide_tokens():
    # 64 lanes a token: 2^32 threads and a few more
    tokens, V, I = 2 ** 26 + 13, 251, 264
    room(45)
    table = (torch.arange(V, device=DEV)[:, None] + torch.arange(I, device=DEV) % 5).bfloat16() / 256
    ids = (torch.arange(tokens, device=DEV, dtype=torch.int64) * 7 % V).int()
    e = runner.Embedding(table)
    y = torch.full((tokens, I), float("nan"), dtype=torch.bfloat16, device=DEV)
    e.forward(ids, y)
    torch.cuda.synchronize()
    step = 1 << 22
    for t in range(0, tokens, step):
        assert torch.equal(y[t:t + step], table[ids[t:t + step].long()]), t


def test_gradient_of_many_tokens():
    # 2^29 tokens and some: id v has the tokens v, v + V, ...; sums of small
    # whole numbers, exact in any order
    V, I, n = 2 ** 20, 8, 513
    tokens = V * n
    room(60)
    ids = (torch.arange(tokens, device=DEV, dtype=torch.int32) & (V - 1))
    dy = torch.empty(n, V, I, dtype=torch.bfloat16, device=DEV)
    want = torch.zeros(V, I, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    for i in range(n):
        dy[i] = torch.randint(-8, 9, (V, I), generator=g, device=DEV).bfloat16()
        want += dy[i].float()
    table = torch.zeros(V, I, dtype=torch.bfloat16, device=DEV)
    e = runner.Embedding(table)
    e.grad.fill_(float("nan"))
    e.backward(ids, dy.view(tokens, I))
    torch.cuda.synchronize()
    assert torch.equal(e.grad, want)


@pytest.mark.parametrize("V", [2 ** 18 - 1, 2 ** 18, 300007, 2 ** 24 + 5])
@pytest.mark.parametrize("tokens", [1, 300, 1025, 5000])
def test_large_vocabularies(V, tokens):
    # (ids past the bits that the sort of lists has)
    I = 8
    g = torch.Generator(device=DEV).manual_seed(V % 1000 + tokens)
    ids = torch.randint(0, V, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    ids[::3] = V - 1
    ids[1::7] = V
    dy = torch.randint(-8, 9, (tokens, I), generator=g, device=DEV).half()
    table = (torch.arange(V, device=DEV, dtype=torch.int32)[:, None] % 2048 + torch.zeros(I, device=DEV)).half()
    e = runner.Embedding(table)
    inside = (ids < V)[:, None]
    assert torch.equal(e.forward(ids), torch.where(inside, table[ids.long().clamp(max=V - 1)], torch.zeros((), device=DEV).half()))
    e.grad.fill_(float("nan"))
    want = torch.zeros(V, I, device=DEV).index_add_(0, ids.long().clamp(max=V - 1), torch.where(inside, dy.float(), 0.0))
    assert torch.equal(e.backward(ids, dy), want)
