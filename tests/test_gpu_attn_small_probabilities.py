"""fp16 attention where one key has nearly all of the softmax and a value of
zero (a sink), so that the output is a sum of many probabilities below fp16's
normal numbers."""
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
