"""The embedding owner's workspace: what it outgrows is given back, but for what
a captured backward uses."""
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


def batch(tokens, V, I, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randint(0, V, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    return ids, torch.randint(-8, 9, (tokens, I), generator=g, device=DEV).half()


def plain(ids, dy, V):
    return torch.zeros(V, dy.shape[1], device=DEV).index_add_(0, ids.long(), dy.float())  # (whole numbers: exact)


@pytest.mark.parametrize("where", ["side", "default", "both"])
def test_outgrown_workspaces_are_given_back(where):
    V, I = 1000, 256
    runs = [batch(n, V, I, n) for n in (20000, 50000, 120000)]
    want = [plain(*r, V) for r in runs]
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    e = runner.Embedding(torch.zeros(V, I, dtype=torch.float16, device=DEV))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    streams = {"side": [side], "default": [torch.cuda.current_stream()], "both": [side, torch.cuda.current_stream()]}
    for (ids, dy), w in zip(runs, want):
        for s in streams[where]:
            with torch.cuda.stream(s):
                got = e.backward(ids, dy).clone()
            torch.cuda.synchronize()
        assert torch.equal(got, w)
        del got
    torch.cuda.empty_cache()  # (blocks that wait for another stream are looked at)
    held = torch.cuda.memory_allocated() - before
    assert held <= e.ws.numel() + 4 * V * I + 2 * V * I + (1 << 20)


def test_a_workspace_grown_in_a_capture():
    V, I = 500, 64
    small, big, bigger = batch(3000, V, I, 1), batch(30000, V, I, 2), batch(200000, V, I, 3)
    e = runner.Embedding(torch.zeros(V, I, dtype=torch.float16, device=DEV))
    want = [plain(*r, V) for r in (small, big, bigger)]
    assert torch.equal(e.backward(*small), want[0])
    graphs = []
    for r in (small, big):  # (the second finds too little and makes another)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            e.backward(*r)
        graphs.append(g)
    assert torch.equal(e.backward(*bigger), want[2])
    others = [torch.full((1 << 22,), -1, dtype=torch.int32, device=DEV) for _ in range(16)]
    for _ in range(3):
        for g, r, w in zip(graphs, (small, big), want):
            e.grad.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(e.grad, w)
            assert torch.equal(e.backward(*bigger), want[2])
    assert all((t == -1).all() for t in others)
