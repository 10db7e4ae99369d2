"""Streaming attention (attn_fwd, attn_bwd) against its definition in 64 bits:
masks, caps, distance bias, shared heads, lengths, strides, refusals of nothing
but what the CPU tests name; streams, graphs and large offsets."""
import pytest
import torch

from _attention import check, reference
from paper_2007_00072_amd import lib, runner

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


def normal(seed, *shape, std=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * std


def aux_on(aux, dev):
    return {n: t.to(dev) if isinstance(t, torch.Tensor) else t for n, t in aux.items()}


def inputs(dt, B, J, K, H, G, P, seed=1):
    q, k, v, g = (normal(seed + i, B, L, n, P).to(T[dt]) for i, (L, n) in enumerate([(J, H), (K, G), (K, G), (J, H)]))
    return q, k, v, g


def run(q, k, v, g=None, **kw):
    d = [t.to(DEV) for t in (q, k, v)]
    a = runner.Attention(*d, train=g is not None, **aux_on(kw, DEV))
    out = a.forward(*d)
    r = {"out": out}
    if g is not None:
        r["dq"], r["dk"], r["dv"] = a.backward(*d, out, g.to(DEV))
    torch.cuda.synchronize()
    return r


def compare(dt, B, J, K, H, G, P, seed=1, grads=True, **kw):
    q, k, v, g = inputs(dt, B, J, K, H, G, P, seed)
    g = g if grads else None
    got, want = run(q, k, v, g, **kw), reference(q, k, v, g, **kw)
    assert sorted(got) == sorted(want)
    for n in want:
        check(f"{n} {dt}", got[n], want[n])


def i32(*x):
    return torch.tensor(x, dtype=torch.int32)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("J,K,P", [(1, 1, 64), (3, 2, 8), (33, 65, 32), (64, 64, 64), (129, 257, 128), (70, 300, 96),
                                   (200, 31, 40)])
def test_plain(dt, J, K, P):
    compare(dt, 2, J, K, 2, 2, P)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("H,G", [(4, 2), (6, 1), (3, 3)])
@pytest.mark.parametrize("J,K", [(150, 150), (130, 201)])
def test_causal_shared_heads(dt, H, G, J, K):
    compare(dt, 2, J, K, H, G, 64, causal=True)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("P", [32, 64, 128])
@pytest.mark.parametrize("cap,alibi", [(5.0, False), (0.0, True), (2.0, True)])
def test_cap_and_distance(dt, P, cap, alibi):
    s = torch.exp2(-torch.arange(1, 4).double()).float() if alibi else None
    compare(dt, 1, 100, 100, 3, 3, P, cap=cap, slopes=s, scaler=0.3)
    compare(dt, 1, 70, 140, 3, 3, P, cap=cap, slopes=s, causal=True)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("P", [72, 96, 128])
def test_many_blocks_of_wide_heads(dt, P):
    # more blocks than one launch of the backward takes both kernels for
    B, K, H, G = 12, 301, 16, 8
    doc = (torch.arange(K) // 140).int().expand(B, K).contiguous()
    doc[3, 60:75] = -1
    n = torch.randint(1, K + 1, (B,), generator=torch.Generator().manual_seed(9)).int()
    compare(dt, B, K, K, H, G, P, causal=True, cap=6.0)
    compare(dt, B, K, K, H, G, P, doc=doc, k_len=n, q_len=n, slopes=torch.full((H,), 0.05))
    # sequences without queries: their keys have no gradient
    q, k, v, g = inputs(dt, B, K, K, H, G, P)
    got = run(q, k, v, g, q_len=torch.zeros(B, dtype=torch.int32))
    assert not any(t.any() for t in got.values())


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_documents(dt, causal):
    # documents of 1 to 130 keys, padding inside and behind, ids in no order
    B, K = 3, 333
    doc = torch.full((B, K), -1, dtype=torch.int32)
    doc[0] = torch.bucketize(torch.arange(K), torch.tensor([1, 2, 64, 65, 195, 256, 300]), right=True).int()
    doc[1, 10:200] = 7
    doc[1, 200:201] = 2 ** 31 - 1
    doc[1, 220:] = (torch.arange(K - 220) % 3).int()
    compare(dt, B, K, K, 2, 1, 64, doc=doc, causal=causal)
    # queries behind a cache: positions with documents of their own
    compare(dt, B, 40, K, 4, 2, 32, doc=doc, causal=causal)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("J", [1, 90, 200])
def test_lengths_and_prefixes(dt, J):
    K = 200
    k_len = i32(200, 0, 1, 77)
    q_len = i32(min(J, 200), min(J, 5), 1, min(J, 77))
    for kw in (dict(), dict(causal=True), dict(causal=True, prefix=i32(0, 3, 200, 64))):
        compare(dt, 4, J, K, 2, 2, 64, k_len=k_len, q_len=q_len, **kw)
        compare(dt, 4, J, K, 2, 1, 64, k_len=k_len, **kw)  # q_len = J: rows before the first key see none


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,J,K,H,G,P", [(1, 1, 331, 12, 12, 64), (3, 1, 3000, 8, 2, 128), (2, 2, 5000, 8, 1, 96),
                                         (1, 1, 20000, 4, 4, 32), (2, 1, 129, 40, 8, 80), (1, 7, 1025, 5, 1, 64),
                                         (2, 130, 2100, 2, 1, 64)])
def test_few_queries_over_a_cache(dt, B, J, K, H, G, P):
    k_len = torch.randint(J, K + 1, (B,), generator=torch.Generator().manual_seed(3)).int()
    compare(dt, B, J, K, H, G, P, causal=True, k_len=k_len, grads=False)
    compare(dt, B, J, K, H, G, P, cap=20.0, slopes=torch.full((H,), 0.01), grads=False)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_what_is_outside_is_not_read(dt):
    # NaN and infinities behind the lengths and in padding documents
    B, K, H, P = 2, 190, 2, 64
    q, k, v, g = inputs(dt, B, K, K, H, H, P)
    n = i32(100, 190)
    doc = torch.zeros(B, K, dtype=torch.int32)
    doc[1, 50:70] = -1
    clean = run(q, k, v, g, k_len=n, q_len=n, doc=doc, causal=True)
    for t, bad in ((q, float("nan")), (k, float("inf")), (v, float("nan")), (g, float("-inf"))):
        t[0, 100:] = bad
        t[1, 50:70] = bad
    dirty = run(q, k, v, g, k_len=n, q_len=n, doc=doc, causal=True)
    for name in clean:
        assert torch.equal(clean[name], dirty[name]), name
        assert not clean[name][0, 100:].any() and not clean[name][1, 50:70].any(), name


def test_scores_of_any_size():
    # large scores of both signs: one key takes all, no overflow
    for dt in ("f16", "bf16", "f32"):
        q, k, v, g = inputs(dt, 1, 65, 130, 1, 1, 64)
        q, k = (q * 30).to(T[dt]), (k * 30).to(T[dt])
        got, want = run(q, k, v), reference(q, k, v)
        check("out", got["out"], want["out"])
        same = torch.zeros_like(k)
        got, want = run(q, same, v, g), reference(q, same, v, g)
        for n in want:
            check(n, got[n], want[n])


@pytest.mark.parametrize("scale", [2.0 ** -12, 2.0 ** 12])
def test_small_and_large_gradients_in_half_precision(scale):
    q, k, v, g = inputs("f16", 1, 300, 300, 2, 1, 64)
    g = (g.double() * scale).half()
    got, want = run(q, k, v, g, causal=True), reference(q, k, v, g, causal=True)
    for n in want:
        check(n, got[n], want[n])


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_gradients_against_differences(dt):
    # along a direction, central differences of the definition in 64 bits
    q, k, v, g = inputs(dt, 1, 40, 40, 4, 2, 32)
    kw = dict(causal=True, cap=3.0, slopes=torch.tensor([0.5, 0.25, 0.125, 0.0]))
    got = run(q, k, v, g, **kw)
    dirs = [normal(50 + i, *t.shape) for i, t in enumerate((q, k, v))]
    h = 1e-5

    def loss(sign):
        # (the reference takes the types' values: float64 copies moved along the directions)
        moved = [t.double() + sign * h * d for t, d in zip((q, k, v), dirs)]
        from _attention import U
        U[torch.float64] = 0.0
        return float((reference(*moved, **kw)["out"][0] * g.double()).sum())

    num = (loss(1) - loss(-1)) / (2 * h)
    want = reference(q, k, v, g, **kw)
    ana = sum(float((got[n].cpu().double() * d).sum()) for n, d in zip(("dq", "dk", "dv"), dirs))
    room = sum(float((want[n][1] * d.abs()).sum()) for n, d in zip(("dq", "dk", "dv"), dirs))
    assert abs(num - ana) <= room + 1e-6 * abs(num)


def test_strides_and_layouts():
    # a fused projection's views, head-major caches, padded rows, broadcast keys
    B, L, H, G, P = 2, 75, 4, 2, 64
    q, k, v, g = inputs("bf16", B, L, L, H, G, P)
    want = run(q, k, v, g, causal=True)
    qkv = torch.cat([q, k, v], 2).to(DEV)
    dqkv = torch.zeros_like(qkv)
    parts = [qkv[:, :, :H], qkv[:, :, H:H + G], qkv[:, :, H + G:]]
    grads = [dqkv[:, :, :H], dqkv[:, :, H:H + G], dqkv[:, :, H + G:]]
    a = runner.Attention(*parts, causal=True)
    out = torch.empty(B, H, L + 3, P + 8, device=DEV, dtype=q.dtype).transpose(1, 2)[:, :L, :, :P]
    a.forward(*parts, out=out)
    dout = torch.empty_strided(out.shape, out.stride(), dtype=out.dtype, device=DEV)
    dout.copy_(g)
    a.backward(*parts, out, dout, *grads)
    torch.cuda.synchronize()
    for n, t in zip(("out", "dq", "dk", "dv"), [out, *grads]):
        assert torch.equal(t, want[n]), n
    one = [t[:1].expand(B, -1, -1, -1) for t in (k.to(DEV), v.to(DEV))]
    b = runner.Attention(q.to(DEV), *one, causal=True, train=False)
    both = b.forward(q.to(DEV), *one)
    ref = run(q, k[:1].expand(B, -1, -1, -1).contiguous(), v[:1].expand(B, -1, -1, -1).contiguous(), causal=True)
    assert torch.equal(both, ref["out"])


def test_offsets_past_32_bits():
    # the second sequence's rows begin 2^32 elements behind the first's
    B, K, P, far = 2, 100, 64, 2 ** 32 + 64
    q, k, v, g = inputs("bf16", B, K, K, 1, 1, P)
    want = run(q, k, v, g, causal=True)
    store = torch.empty(far + 3 * K * P, dtype=torch.bfloat16, device=DEV)
    parts = [store.as_strided((B, K, 1, P), (far, P, P, 1), i * K * P) for i in range(3)]
    for t, x in zip(parts, (q, k, v)):
        t.copy_(x)
    a = runner.Attention(*parts, causal=True)
    out = a.forward(*parts)
    grads = [torch.empty_strided(t.shape, (K * P, P, P, 1), dtype=t.dtype, device=DEV) for t in parts]
    del store
    with pytest.raises(ValueError):
        a.backward(*parts, out, g.to(DEV), *grads)
    assert torch.equal(out, want["out"])


def test_no_keys_and_no_queries():
    q, k, v, g = inputs("f16", 2, 5, 0, 2, 2, 64)
    got = run(q, k, v, g)
    assert not got["out"].any() and not got["dq"].any() and got["dk"].numel() == 0
    q, k, v, g = inputs("f16", 2, 0, 40, 2, 2, 64)
    got = run(q, k, v, g)
    assert got["out"].numel() == 0 and not got["dk"].any() and not got["dv"].any()


def test_writes_stay_inside():
    B, J, K, H, G, P = 2, 37, 91, 4, 2, 40
    for dt in ("f32", "f16"):
        q, k, v, g = (t.to(DEV) for t in inputs(dt, B, J, K, H, G, P))
        a = runner.Attention(q, k, v, causal=True, doc=torch.zeros(B, K, dtype=torch.int32, device=DEV))
        band, bufs = 4096, []

        def guarded(n, a=None):
            t = torch.full((n + 2 * band,), 0xA5, dtype=torch.uint8, device=DEV)
            bufs.append((t, n))
            return t[band:band + n]

        def like(t):
            return guarded(t.numel() * t.element_size()).view(t.dtype).view(t.shape)

        a.saved, a.ws = guarded(a.saved_bytes), guarded(a.ws_bytes)
        out = like(q)
        a.forward(q, k, v, out=out)
        a.backward(q, k, v, out, g, like(q), like(k), like(v))
        torch.cuda.synchronize()
        for t, n in bufs:
            assert bool((t[:band] == 0xA5).all()) and bool((t[band + n:] == 0xA5).all())


def test_same_bits_every_time_on_any_stream_and_in_graphs():
    B, J, K, H, G, P = 2, 260, 260, 4, 2, 64
    q, k, v, g = (t.to(DEV) for t in inputs("bf16", B, J, K, H, G, P))
    doc = (torch.arange(K) // 60).int().expand(B, K).contiguous().to(DEV)
    token = (torch.arange(J, device=DEV) >= J - 1)
    objs = [runner.Attention(q, k, v, doc=doc, causal=True), runner.Attention(q, k, v, cap=4.0)]
    few = runner.Attention(q[:, -1:], k, v, causal=True, train=False)
    del token

    def step(a):
        out = a.forward(q, k, v)
        return (out, *a.backward(q, k, v, out, g))

    want = [step(a) for a in objs] + [(few.forward(q[:, -1:], k, v),)]
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for a, s in zip(objs, side):
        with torch.cuda.stream(s):
            got.append(step(a))
    torch.cuda.synchronize()
    for x, y in zip(want, got):
        assert all(torch.equal(s, t) for s, t in zip(x, y))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = [step(a) for a in objs] + [(few.forward(q[:, -1:], k, v),)]
    for _ in range(3):
        for x in held:
            for t in x:
                t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, held):
            assert all(torch.equal(s, t) for s, t in zip(x, y))
        step(objs[0])
        torch.cuda.synchronize()


def test_entry_points_take_plain_pointers():
    q, k, v, _ = (t.to(DEV) for t in inputs("f16", 1, 10, 20, 2, 2, 64))
    d = lib.AttnDesc(1, 10, 20, 2, 2, 64, lib.DM_F16, 0.0, 0.0, 0)
    d.q = d.out = lib.AttnStride(10 * 128, 64, 128)
    d.k = d.v = lib.AttnStride(20 * 128, 64, 128)
    out = torch.empty_like(q)
    _, need, _ = lib.attn_sizes(d)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    lib.attn_fwd(d, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), None, ws.data_ptr(), need)
    torch.cuda.synchronize()
    check("out", out, reference(q.cpu(), k.cpu(), v.cpu())["out"])
