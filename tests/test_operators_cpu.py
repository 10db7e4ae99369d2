"""Refusals of the attention, embedding and optimiser entry points (host code,
nothing is launched), their sizes, and the Python owners' own checks."""
import ctypes as C

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


def desc(**kw):
    d = lib.AttnDesc(2, 64, 96, 8, 2, 64, lib.DM_BF16, 0.0, 0.0, 0)
    d.q = d.out = lib.AttnStride(64 * 512, 64, 512)
    d.k = d.v = lib.AttnStride(96 * 128, 64, 128)
    for n, x in kw.items():
        setattr(d, n, x)
    return d


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=9), 2, "dtype"), (dict(B=-1), 1, "negative"), (dict(H=7), 1, "multiple"), (dict(G=0), 1, "multiple"),
    (dict(P=60), 2, "head size"), (dict(P=136), 2, "head size"), (dict(cap=-1.0), 1, "cap"),
    (dict(cap=float("nan")), 1, "cap"), (dict(cap=1e-4), 1, "cap"), (dict(cap=2000.0), 1, "cap"),
    (dict(doc=PTR + 2), 1, "doc"), (dict(slopes=PTR + 1), 1, "slopes"),
    (dict(v=lib.AttnStride(96 * 128, 64, 2 ** 22 + 8)), 2, "v: token"), (dict(k=lib.AttnStride(0, 64, 0)), 2, "k: token"), (dict(scaler=float("inf")), 1, "scaler"), (dict(causal=2), 1, "causal"),
    (dict(prefix=PTR), 1, "prefix"), (dict(J=2 ** 30), 2, "rows"), (dict(K=2 ** 30 + 1), 2, "rows"),
    (dict(k=lib.AttnStride(96 * 128, 64, 132)), 2, "k: strides"), (dict(q=lib.AttnStride(-8, 64, 512)), 2, "negative"),
    (dict(out=lib.AttnStride(0, 64, 512)), 2, "out"), (dict(out=lib.AttnStride(64 * 512, 56, 512)), 2, "overlap"),
    (dict(out=lib.AttnStride(64 * 512, 64, 256)), 2, "overlap")])
def test_attention_descriptors(kw, code, word):
    with pytest.raises(lib.DmError) as e:
        lib.attn_sizes(desc(**kw))
    assert e.value.code == code and word in str(e.value)


def test_attention_sizes():
    saved, fwd, bwd = lib.attn_sizes(desc())
    rows = 2 * 8 * 64
    assert saved >= rows * (4 + 64 * 2) and bwd >= rows * 4
    assert lib.attn_sizes(desc(dtype=lib.DM_F32))[0] < saved       # nothing was rounded off
    assert lib.attn_sizes(desc(doc=PTR))[1] >= fwd + 2 * 2 * 8     # ranges of document ids
    # one token over a long cache: parts to join
    long = desc(B=1, J=1, K=100000, H=8, G=8)
    assert lib.attn_sizes(long)[1] >= 2 * 8 * (64 + 2) * 4


def test_attention_buffers():
    d = desc()
    saved, fwd, bwd = lib.attn_sizes(d)
    ok = [PTR] * 4
    for i, name in enumerate(("q", "k", "v", "out")):
        for bad in (None, PTR + 8):
            p = list(ok)
            p[i] = bad
            with pytest.raises(lib.DmError) as e:
                lib.attn_fwd(d, *p, None, PTR, fwd, stream=0)
            assert e.value.code == lib.DM_ERR_ARG and name in str(e.value)
    with pytest.raises(lib.DmError) as e:
        lib.attn_fwd(desc(doc=PTR), *ok, None, PTR, 8, stream=0)
    assert e.value.code == lib.DM_ERR_WORKSPACE
    with pytest.raises(lib.DmError) as e:
        lib.attn_bwd(d, *ok, PTR, PTR, PTR, PTR, PTR, PTR, bwd - 1, stream=0)
    assert e.value.code == lib.DM_ERR_WORKSPACE
    with pytest.raises(lib.DmError) as e:
        lib.attn_bwd(d, *ok, None, PTR, PTR, PTR, PTR, PTR, bwd, stream=0)
    assert "saved" in str(e.value)
    # keys that sequences share are read, but have no gradient of their own
    shared = desc(k=lib.AttnStride(0, 64, 128))
    lib.attn_sizes(shared)
    with pytest.raises(lib.DmError) as e:
        lib.attn_bwd(shared, *ok, PTR, PTR, PTR, PTR, PTR, PTR, bwd, stream=0)
    assert e.value.code == lib.DM_ERR_UNSUPPORTED and "dk" in str(e.value)
    lib.attn_fwd(desc(B=0), None, None, None, None, None, None, 0, stream=0)  # nothing to do


@pytest.mark.parametrize("args,code", [
    ((9, 4, 10, 64), 2), ((1, -1, 10, 64), 1), ((1, 4, 0, 64), 1), ((1, 4, 10, 60), 2), ((1, 4, 10, 16392), 2),
    ((1, 2 ** 31, 10, 64), 2)])
def test_embedding_shapes(args, code):
    for call in (lambda: lib.embed_fwd(*args, PTR, PTR, 1.0, PTR, stream=0),
                 lambda: lib.embed_bwd(*args, PTR, -1, PTR, 1.0, PTR, PTR, 1 << 40, stream=0)):
        with pytest.raises(lib.DmError) as e:
            call()
        assert e.value.code == code


def test_embedding_buffers():
    for i in range(3):
        p = [PTR, PTR, PTR]
        p[i] = None
        with pytest.raises(lib.DmError) as e:
            lib.embed_fwd(1, 4, 10, 64, p[0], p[1], 1.0, p[2], stream=0)
        assert e.value.code == lib.DM_ERR_ARG
        with pytest.raises(lib.DmError) as e:
            lib.embed_bwd(1, 4, 10, 64, p[0], -1, p[1], 1.0, p[2], PTR, 1 << 40, stream=0)
        assert e.value.code == lib.DM_ERR_ARG
    with pytest.raises(lib.DmError):
        lib.embed_fwd(1, 4, 10, 64, PTR, PTR, float("nan"), PTR, stream=0)
    lib.embed_fwd(1, 0, 10, 64, None, None, 1.0, None, stream=0)
    need = lib.embed_ws_bytes(1 << 20, 30522, 1024)
    if need:
        with pytest.raises(lib.DmError) as e:
            lib.embed_bwd(1, 1 << 20, 30522, 1024, PTR, -1, PTR, 1.0, PTR, PTR, need - 1, stream=0)
        assert e.value.code == lib.DM_ERR_WORKSPACE


def adamw(bits=32, dtype=lib.DM_BF16, **kw):
    d = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1, scalars=None)
    d.update(kw)
    return lib.AdamwDesc(dtype, bits, *d.values())


def tensor(bits=32, **kw):
    d = dict(param=PTR, master=PTR, grad=PTR, m=PTR, v=PTR, m_scale=PTR if bits == 8 else None,
             v_scale=PTR if bits == 8 else None, n=10, decay=0.0)
    d.update(kw)
    return lib.AdamwTensor(*d.values())


@pytest.mark.parametrize("d,t,word", [
    (dict(dtype=7), {}, "dtype"), (dict(bits=16), {}, "bits"), (dict(beta1=1.0), {}, "beta1"),
    (dict(beta2=-0.1), {}, "beta2"), (dict(eps=0.0), {}, "eps"), (dict(step=0), {}, "step"),
    (dict(lr=float("nan")), {}, "lr"), (dict(lr=-1.0), {}, "lr"), (dict(grad_scale=float("inf")), {}, "grad_scale"),
    (dict(scalars=PTR + 4), {}, "scalars"), ({}, dict(n=-1), "n="), ({}, dict(grad=None), "grad"),
    ({}, dict(m=PTR + 4), "m is"), ({}, dict(master=PTR + 2), "master"), ({}, dict(decay=-1.0), "decay"),
    (dict(dtype=lib.DM_F32), {}, "master"), ({}, dict(m_scale=PTR), "scales"),
    (dict(bits=8), {}, "scale"), (dict(bits=8), dict(m_scale=PTR, v_scale=PTR + 2), "scale")])
def test_optimizer_arguments(d, t, word):
    arr = (lib.AdamwTensor * 2)(tensor(n=0, param=None, master=None), tensor(**t))
    with pytest.raises(lib.DmError) as e:
        lib.adamw_step(adamw(**d), arr, 2, stream=0)
    assert word in str(e.value)


def test_optimizer_lists():
    with pytest.raises(lib.DmError):
        lib.adamw_step(adamw(), None, 1, stream=0)
    with pytest.raises(lib.DmError):
        lib.adamw_step(adamw(), (lib.AdamwTensor * 1)(), -1, stream=0)
    with pytest.raises(lib.DmError) as e:
        lib.adamw_step(adamw(), (lib.AdamwTensor * 2)(tensor(), tensor(master=None)), 2, stream=0)
    assert "all tensors" in str(e.value)
    lib.adamw_step(adamw(), None, 0, stream=0)
    lib.adamw_step(adamw(), (lib.AdamwTensor * 1)(lib.AdamwTensor()), 1, stream=0)  # an empty tensor


def test_owners_check_their_tensors():
    f = torch.float16
    q, k = torch.zeros(2, 5, 4, 64, dtype=f), torch.zeros(2, 7, 2, 64, dtype=f)
    a = runner.Attention(q, k, k)
    for bad in (q.float(), q[:1], q[:, :, :, :32]):
        with pytest.raises(ValueError):
            a.forward(bad, k, k)
    with pytest.raises(ValueError):
        a.forward(q, k, k.transpose(2, 3).contiguous().transpose(2, 3))
    with pytest.raises(ValueError):
        a.backward(q, k, k, q, q, torch.zeros(2, 4, 5, 64, dtype=f).transpose(1, 2))
    for kw in (dict(q_len=torch.zeros(3, dtype=torch.int32)), dict(doc=torch.zeros(2, 7)),
               dict(slopes=torch.zeros(4, dtype=torch.float64))):
        with pytest.raises(ValueError):
            runner.Attention(q, k, k, **kw)
    with pytest.raises(ValueError):
        runner.Attention(q, k, k, train=False).backward(q, k, k, q, q)
    e = runner.Embedding(torch.zeros(10, 64, dtype=f))
    with pytest.raises(ValueError):
        e.forward(torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        e.backward(torch.zeros(3, dtype=torch.int32), torch.zeros(4, 64, dtype=f))
    p = [torch.zeros(3, 4, dtype=f), torch.zeros(5, dtype=f)]
    with pytest.raises(ValueError):
        runner.AdamW([p[0], p[1].float()])
    with pytest.raises(ValueError):
        runner.AdamW([p[0], p[1], p[0]])
    with pytest.raises(ValueError):
        runner.AdamW(p).step([torch.zeros(3, 4)], 1)
    with pytest.raises(ValueError):
        runner.AdamW(p).step([torch.zeros(3, 4), torch.zeros(6)], 1)
    assert C.sizeof(lib.AttnDesc) == 10 * 4 + 12 * 8 + 5 * 8


def test_strides_of_axes_of_one_element_are_free():
    x = torch.zeros(4096, dtype=torch.bfloat16)
    q = x.as_strided((1, 1, 4, 64), (3, 5, 64, 1))
    k = x.as_strided((1, 7, 1, 64), (1, 64, 1, 1))
    runner.Attention(q, k, k)
    two = x.as_strided((2, 7, 1, 64), (3, 64, 1, 1))
    with pytest.raises(lib.DmError):
        runner.Attention(q.expand(2, 1, 4, 64), two, two)
