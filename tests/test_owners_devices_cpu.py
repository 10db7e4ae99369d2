"""The Python owners refuse host tensors before a kernel would read them."""
import pytest
import torch

from paper_2007_00072_amd import runner


@pytest.fixture(autouse=True)
def float32_by_default():
    # (other test modules may have set another default type)
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def test_host_tensors_are_refused():
    f = torch.float16
    q, k = torch.zeros(2, 5, 4, 64, dtype=f), torch.zeros(2, 7, 2, 64, dtype=f)
    a = runner.Attention(q, k, k)
    out = torch.zeros_like(q)
    e = runner.Embedding(torch.zeros(10, 64, dtype=f))
    ids = torch.zeros(3, dtype=torch.int32)
    o = runner.AdamW([torch.zeros(16)])
    for call in (lambda: a.forward(q, k, k), lambda: a.backward(q, k, k, out, out), lambda: e.forward(ids),
                 lambda: e.backward(ids, torch.zeros(3, 64, dtype=f)), lambda: o.step([torch.zeros(16)], 1)):
        with pytest.raises(ValueError, match="cpu"):
            call()
