"""The optimiser step against its definition in 64 bits, its 8-bit states code
by code, and its use in graphs."""
import math

import pytest
import torch

from paper_2007_00072_amd import runner

pytestmark = pytest.mark.gpu
DEV = "cuda"
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
F = 2.0 ** -24
HP = dict(lr=2e-3, beta1=0.9, beta2=0.99, eps=1e-8)
SIZES = [1, 3, 255, 256, 257, 4095, 4096, 4097, 10000, 70001]


@pytest.fixture(autouse=True)
def float32_by_default():
    # (other test modules may have set another default type)
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def tensors(sizes, seed, std):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, generator=g) * std for n in sizes]


def e4m3(x):
    """Nearest e4m3 values, ties to even (64 bits)."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def blocks(x):
    n = -(-x.numel() // 256)
    out = torch.zeros(n * 256, dtype=torch.float64)
    out[:x.numel()] = x.double()
    return out.view(n, 256)


def step64(w, g, m, v, decay, step, gs=1.0, lr=None):
    lr = HP["lr"] if lr is None else lr
    w, g, m, v = w.double(), g.double() * gs, m.double(), v.double()
    m = HP["beta1"] * m + (1 - HP["beta1"]) * g
    v = HP["beta2"] * v + (1 - HP["beta2"]) * g * g
    u = (m / (1 - HP["beta1"] ** step)) / (torch.sqrt(v / (1 - HP["beta2"] ** step)) + HP["eps"])
    return w * (1 - lr * decay) - lr * u, m, v, u


def close(got, want, room):
    err = (got.cpu().double() - want).abs()
    assert (err <= room).all(), float((err / room.clamp_min(1e-300)).max())


@pytest.mark.parametrize("dt,master", [("f32", False), ("f16", True), ("f16", False), ("bf16", True), ("bf16", False)])
@pytest.mark.parametrize("step", [1, 1000])
def test_states_in_32_bits(dt, master, step):
    w = [t.to(T[dt]) for t in tensors(SIZES, 1, 0.05)]
    g, m = tensors(SIZES, 2, 0.1), tensors(SIZES, 3, 0.01)
    v = [t * t for t in tensors(SIZES, 4, 0.1)]
    decay = [0.1 * (i % 2) for i in range(len(SIZES))]
    wm = [t.float() + 1e-4 * torch.sin(torch.arange(t.numel())) for t in w] if master else None
    on = lambda ts: None if ts is None else [t.to(DEV) for t in ts]  # noqa: E731
    o = runner.AdamW(on(w), master=on(wm), m=on(m), v=on(v), decay=decay, **HP)
    o.step(on(g), step, grad_scale=0.5)
    torch.cuda.synchronize()
    for i in range(len(SIZES)):
        w0 = wm[i] if master else w[i]
        we, me, ve, u = step64(w0, g[i], m[i], v[i], decay[i], step, 0.5)
        # each operation rounds once in float32
        m_size = m[i].double().abs() + g[i].double().abs()
        close(o.m[i], me, 4 * F * m_size)
        close(o.v[i], ve, 6 * F * ve)
        room_u = 16 * F * u.abs() + 4 * F * m_size / (torch.sqrt(ve) + HP["eps"]) / (1 - HP["beta1"] ** step)
        room = 4 * F * w0.double().abs() + HP["lr"] * room_u + 2 * F * we.abs()
        if master:
            close(o.master[i], we, room)
        small = 2.0 ** -25 if dt == "f16" else 0.0
        close(o.params[i], we, room + (U[dt] * 1.01 * we.abs() + small if dt != "f32" else 0.0))
        if master:
            assert torch.equal(o.params[i], o.master[i].to(T[dt]))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_states_in_8_bits(dt):
    w, sizes = [t.to(T[dt]) for t in tensors(SIZES, 1, 0.05)], SIZES
    o = runner.AdamW([t.to(DEV) for t in w], decay=0.01, state_bits=8, **HP)
    w0 = [t.double() for t in w]
    for step in (1, 2, 3):
        old = [[t.cpu().double() if t.dtype == torch.float32 else t.cpu().float().double() for t in x]
               for x in (o.m, o.m_scale, o.v, o.v_scale)]
        g = tensors(sizes, 10 + step, 0.1 ** step)
        for t in g:
            t[::5] *= 1e-4  # the codes' whole range
            t[::97] = 0.0
        if step == 3:
            g[8][256:512] = 0.0
        o.step([t.to(DEV) for t in g], step)
        torch.cuda.synchronize()
        for i, n in enumerate(sizes):
            m0 = (blocks(old[0][i]) * old[1][i][:, None]).view(-1)[:n]
            r0 = (blocks(old[2][i]) * old[3][i][:, None]).view(-1)[:n]
            we, me, ve, _ = step64(w0[i], g[i], m0, r0 * r0, 0.01, step)
            got = (o.master[i] if dt != "f32" else o.params[i]).cpu().double()
            # the step's size is lr times a quotient of up to a few units
            assert ((got - we).abs() <= 4 * F * w0[i].abs() + 64 * F * HP["lr"] * 10 + 2 * F * we.abs()).all()
            w0[i] = got
            for x, code, scale, root in ((me, o.m[i], o.m_scale[i], False), (torch.sqrt(ve), o.v[i], o.v_scale[i], True)):
                xb, sc = blocks(x), scale.cpu().double()
                top = xb.abs().amax(1)
                # sums that nearly cancel have 32-bit errors of their terms' size
                slack = 8 * F * (blocks(m0).abs() + blocks(g[i]).abs()) if not root else 8 * F * xb
                assert ((sc - top / 448).abs() <= 2 * F * top / 448 + slack.amax(1) / 448).all()
                c = blocks(code.cpu().float())
                exact = xb / sc.clamp_min(1e-300)[:, None]
                near = (c - exact).abs()
                step_size = torch.exp2(torch.floor(torch.log2(exact.abs().clamp_min(2.0 ** -6))) - 3)
                ok = near <= step_size / 2 * (1 + 1e-4) + slack / sc.clamp_min(1e-300)[:, None] + 1e-4 * step_size
                if root:
                    ok |= (c == 2.0 ** -9) & (xb > 0) & (exact < 2.0 ** -9)
                    assert ((c > 0) | (xb == 0)).all()  # what is not zero stays above zero
                assert ok.all()
                assert torch.equal(c, e4m3(c))


def test_blocks_of_zeros_and_tiny_values():
    p = [torch.ones(700, device=DEV)]
    o = runner.AdamW(p, state_bits=8, **HP)
    g = torch.zeros(700, device=DEV)
    g[300:310] = 1e-35  # squares vanish, the first moment is under 2^-100
    o.step([g], 1)
    torch.cuda.synchronize()
    assert torch.isfinite(p[0]).all() and (p[0][:256] == 1).all()
    assert not o.m[0].float().any() and not o.m_scale[0].any() and not o.v_scale[0].any()


def test_many_tensors_in_groups():
    # more than a launch holds, of many sizes, some empty: the same as one by one
    sizes = [(i * 37) % 1500 for i in range(150)]
    w, g = tensors(sizes, 1, 0.1), tensors(sizes, 2, 0.1)
    both = []
    for group in (sizes, None):
        ps = [t.to(DEV).to(torch.bfloat16) for t in w]
        gs = [t.to(DEV) for t in g]
        if group:
            o = runner.AdamW(ps, decay=0.1, **HP)
            o.step(gs, 1)
            o.step(gs, 2)
        else:
            for p, x in zip(ps, gs):
                o = runner.AdamW([p], decay=0.1, **HP)
                o.step([x], 1)
                o.step([x], 2)
        both.append(ps)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*both))


def test_overflowed_gradients_show():
    p = [torch.ones(600, device=DEV, dtype=torch.float16)]
    o = runner.AdamW(p, **HP)
    g = torch.full((600,), 0.1, device=DEV)
    g[5], g[300] = float("inf"), float("nan")
    o.step([g], 1)
    torch.cuda.synchronize()
    bad = ~torch.isfinite(p[0])
    assert bad[5] and bad[300] and int(bad.sum()) == 2


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step_with_new_scalars(bits):
    sizes = [5000, 300]
    w, g = tensors(sizes, 1, 0.1), [t.to(DEV) for t in tensors(sizes, 2, 0.1)]

    def made():
        return runner.AdamW([t.to(DEV).half() for t in w], decay=0.1, state_bits=bits, **HP)

    def scalars(step):
        return torch.tensor([HP["lr"] / step, 1 / (1 - HP["beta1"] ** step), 1 / (1 - HP["beta2"] ** step), 0.25])

    eager, held = made(), made()
    sc = scalars(1).to(DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held.step(g, 1, scalars=sc)
    for step in (1, 2, 3):
        sc.copy_(scalars(step))
        graph.replay()
        eager.step(g, step, lr=HP["lr"] / step, grad_scale=0.25)
        torch.cuda.synchronize()
        for a, b in zip(eager.master, held.master):
            # 1 - lr decay is formed in 64 bits by the host, in 32 by the kernel
            assert ((a - b).abs() <= 4 * step * F * (a.abs() + 1)).all()


def test_writes_stay_inside():
    band, sizes = 1024, [1, 255, 4097]
    bufs = []

    def guarded(t):
        n = t.numel() * t.element_size()
        room = -(-n // 16) * 16
        b = torch.full((room + 2 * band,), 0xA5, dtype=torch.uint8, device=DEV)
        x = b[band:band + n]
        x.copy_(t.to(DEV).contiguous().view(-1).view(torch.uint8))
        bufs.append((b, n))
        return x.view(t.dtype)

    for bits in (32, 8):
        o = runner.AdamW([guarded(t.half()) for t in tensors(sizes, 1, 1.0)],
                         master=[guarded(t) for t in tensors(sizes, 1, 1.0)],
                         m=[guarded(torch.zeros(n) if bits == 32 else torch.zeros(n, dtype=torch.uint8).view(torch.float8_e4m3fn)) for n in sizes],
                         v=[guarded(torch.zeros(n) if bits == 32 else torch.zeros(n, dtype=torch.uint8).view(torch.float8_e4m3fn)) for n in sizes],
                         m_scale=[guarded(torch.zeros(math.ceil(n / 256))) for n in sizes] if bits == 8 else None,
                         v_scale=[guarded(torch.zeros(math.ceil(n / 256))) for n in sizes] if bits == 8 else None, **HP)
        o.step([t.to(DEV) for t in tensors(sizes, 2, 1.0)], 1)
    torch.cuda.synchronize()
    for b, n in bufs:
        assert bool((b[:band] == 0xA5).all()) and bool((b[band + n:] == 0xA5).all())


def test_8_bit_states_are_the_plain_forms_bit_for_bit():
    # every operation rounds by itself in float32, the scale by a reciprocal:
    # several steps of the same operations by torch give the same codes
    n, c1, c2 = 256 * 1600, 1 - HP["beta1"], 1 - HP["beta2"]
    w, m, r, *grads = (t.to(DEV) for t in tensors([n] * 6, 31, 0.02))

    def pack(x, root):
        top = x.view(-1, 256).abs().amax(1)
        y = x.view(-1, 256) * (torch.reciprocal(top) * 448.0)[:, None]
        code = y.to(torch.float8_e4m3fn)
        if root:
            code = torch.where((y > 0) & (code.float() == 0), 2.0 ** -9, code.float()).to(torch.float8_e4m3fn)
        return code.view(-1), top * torch.tensor(1 / 448.0, dtype=torch.float32)

    def value(code, scale):
        return (code.float().view(-1, 256) * scale[:, None]).view(-1)

    mc, ms = pack(m, False)
    vc, vs = pack(r.abs(), True)
    own = [t.clone() for t in (w, mc, vc, ms, vs)]
    o = runner.AdamW([own[0]], m=[own[1]], v=[own[2]], m_scale=[own[3]], v_scale=[own[4]], decay=[0.0], **HP)
    for s, g in enumerate(grads):
        step = 50 + s
        o.step([g], step)
        m = value(mc, ms) * HP["beta1"] + g * c1
        v = value(vc, vs) ** 2 * HP["beta2"] + (g * g) * c2
        u = (m * (1.0 / (1.0 - HP["beta1"] ** step))) / (torch.sqrt(v * (1.0 / (1.0 - HP["beta2"] ** step))) + HP["eps"])
        w = w - u * HP["lr"]
        (mc, ms), (vc, vs) = pack(m, False), pack(torch.sqrt(v), True)
        for a, b in zip(own, (w, mc, vc, ms, vs)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_learning_rate_of_one_step():
    w = tensors([300], 7, 0.1)[0].to(DEV)
    o = runner.AdamW([w], **HP)
    before, g = w.clone(), torch.ones(300, device=DEV)
    o.step([g], 1, lr=0.0)
    assert torch.equal(w, before)
    o.step([g], 2)
    # (the second of two equal gradients: a step of about lr)
    assert ((before - w) / HP["lr"] - 1).abs().max() < 1e-3
