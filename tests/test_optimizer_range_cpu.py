"""The optimiser step computes in float32: numbers of its descriptor that are
zero or infinite there are refused (host code, nothing is launched)."""
import pytest

from paper_2007_00072_amd import lib

PTR = 0x10000


def step(decay=0.0, **kw):
    d = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1, scalars=None)
    d.update(kw)
    t = (lib.AdamwTensor * 1)(lib.AdamwTensor(PTR, None, PTR, PTR, PTR, None, None, 10, decay))
    lib.adamw_step(lib.AdamwDesc(lib.DM_F32, 32, *d.values()), t, 1, stream=0)


@pytest.mark.parametrize("kw,word", [(dict(eps=1e-46), "eps"), (dict(eps=1e-40), "eps"), (dict(eps=1e39), "eps"),
                                     (dict(eps=float("nan")), "eps"), (dict(eps=1e-46, scalars=PTR), "eps"),
                                     (dict(lr=1e39), "lr"), (dict(grad_scale=1e39), "grad_scale"),
                                     (dict(grad_scale=-1e39), "grad_scale"), (dict(decay=1e39), "decay")])
def test_numbers_outside_float32(kw, word):
    with pytest.raises(lib.DmError) as e:
        step(**kw)
    assert e.value.code == lib.DM_ERR_ARG and word in str(e.value)
