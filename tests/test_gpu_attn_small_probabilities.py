"""fp16 attention where one key has nearly all of the softmax and a value of
zero (a sink), so that outputs and gradients are sums over many probabilities
below fp16's normal numbers."""
import math

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


def worst_score(steps, dt):
    """A score, exact in the type, whose probability is next to `steps` and a half of fp16's smallest numbers."""
    n = 8 if dt == "bf16" else 64
    return min((-i / n for i in range(8 * n, 16 * n)), key=lambda s: abs(math.exp(s) * 2.0 ** 24 - (steps + 0.45)))


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("J", [1, 200])
@pytest.mark.parametrize("steps", [2, 5, 9])
@pytest.mark.parametrize("sink", [0, 20000])
def test_a_sink_and_many_small_ones(dt, J, steps, sink):
    K, H, P = 32768, 2, 32
    s = worst_score(steps, dt)
    q, k, v = torch.zeros(1, J, H, P), torch.zeros(1, K, H, P), torch.zeros(1, K, H, P)
    q[..., 0] = 1.0
    k[..., 0] = s
    k[:, sink, :, 0] = 0.0
    v[...] = torch.linspace(0.5, 1.0, P)
    v[:, sink] = 0.0
    q, k, v = (t.to(T[dt]) for t in (q, k, v))
    d = [t.to(DEV) for t in (q, k, v)]
    a = runner.Attention(*d, scaler=1.0, train=False)
    assert lib.attn_form(a.desc)[0] == (32 if J == 1 else 128)
    out = a.forward(*d).cpu().double()
    p = math.exp(s)
    want = v[:, 1].double()[:, None] * ((K - 1) * p / (1 + (K - 1) * p))
    # a probability (its exponential to 2^-20 at this score) and the result are rounded to the type; K terms in float32
    # in lanes, waves and parts (64 at the least of them, sums of up to K / 64 terms)
    room = 2.02 * U[dt] + 2.0 ** -20 + (K / 64 + 64) * 2.0 ** -24
    assert ((out - want).abs() <= room * want).all(), float(((out - want).abs() / want).max())


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("J", [1, 200])
@pytest.mark.parametrize("P", [32, 128])
@pytest.mark.parametrize("steps", [2, 9])
def test_gradients_of_a_row_with_small_ones(dt, J, P, steps):
    # one element of dout is 64 times the others, and no value answers to it
    K, H = 8192, 2
    s = worst_score(steps, dt)
    q, k, v, dout = torch.zeros(1, J, H, P), torch.zeros(1, K, H, P), torch.zeros(1, K, H, P), torch.zeros(1, J, H, P)
    q[..., 0] = 1.0
    k[:, 1:, :, 0] = s
    v[:, 1:, :, 1:] = 0.75
    dout[...] = 2.0 ** -6
    dout[..., 0] = 1.0
    d = [t.to(T[dt]).to(DEV) for t in (q, k, v)]
    a = runner.Attention(*d, scaler=1.0)
    out = a.forward(*d)
    dq, _, _ = a.backward(*d, out, dout.to(T[dt]).to(DEV))
    p, c = math.exp(s), (P - 1) * 0.75 * 2.0 ** -6
    one, rest = p / (1 + (K - 1) * p), (K - 1) * p / (1 + (K - 1) * p)
    want = rest * (1 - rest) * c * s
    # a score's gradient is held times 2^e: |dout| 2^e is 2^-1 for the largest, times 2^15 over the power of two below
    # P |v|; half of fp16's smallest number of that
    held = one * c * (1 - rest) * 2.0 ** (14 - math.floor(math.log2(P * 0.75)))
    room = (2.0 ** -25 / held if dt == "f16" else 0.0) + 3.1 * U[dt] + 2.0 ** -14 + K / 2 * 2.0 ** -24
    got = dq[..., 0].cpu().double()
    assert ((got - want).abs() <= room * abs(want)).all(), (float(got[0, 0, 0]), want, room)
    assert not dq[..., 1:].any()
