"""Refusals of the speculative calls' marshalling, host only: tensors without memory stand
for those of a GPU."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode


@pytest.fixture(scope="module")
def E():
    from paper_2607_21475_gb300.build import build
    build()
    from paper_2607_21475_gb300 import ebd
    return ebd


def on_gpu(*shape, dtype=torch.bfloat16, device="cuda:0"):
    """A tensor that says it is on that GPU; an address is not to be had from it."""
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device=device)


@pytest.mark.parametrize("shape", [(2 ** 31, 1, 1), (1, 2 ** 31, 1), (1, 1, 2 ** 31)])
def test_sizes_past_31_bits_are_refused(E, shape):
    x, w = on_gpu(*shape), on_gpu(shape[2])
    with pytest.raises(ValueError, match="out of range"):
        E.ebd_norm_rotary(x, w, out=x)
    with pytest.raises(ValueError, match="out of range"):
        E.ebd_norm_rotary_backward(x, x, w, dx=x, dweight=on_gpu(shape[2], dtype=torch.float32))
