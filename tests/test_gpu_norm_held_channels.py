"""Layer norm's backward pass from checkpoints of more channels than maps may have."""
import pytest
import torch

from tests import test_gpu_norm as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [4097, 9001])
def test_backward_from_a_checkpoint_alone(c, dtype):
    """An object that has seen no x: its strides are not used, whatever the number of channels."""
    from paper_2409_09083_amd import tokens
    x, dy, gamma, beta = N._make(2, 3, c, dtype)
    n = tokens.Norm(2, 3, c, dtype)
    n.forward(x, gamma, beta)
    kept = tokens.Checkpoint(6, c, dtype, 64).pack(x.reshape(-1, c))
    want = [t.clone() for t in n.backward(dy, kept, gamma)]
    got = tokens.Norm(2, 3, c, dtype).backward(dy, kept, gamma, n.mean, n.rstd)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_channel_at_any_stride(dtype):
    """The stride of an axis of one is any number: dy as a map's view, x as a checkpoint or a view like it."""
    from paper_2409_09083_amd import tokens
    x, dy, gamma, beta = N._make(4, 5, 1, dtype)
    x = x + torch.arange(20, device="cuda").view(4, 5, 1)
    kept = tokens.Checkpoint(20, 1, dtype, 32).pack(x.reshape(-1, 1))
    n = tokens.Norm(4, 5, 1, dtype)
    n.forward(x, gamma, beta)
    want = [t.clone() for t in n.backward(dy, kept, gamma)]
    view = dy.reshape(4, 1, 5).transpose(1, 2)
    assert view.stride(2) != 1
    assert all(torch.equal(a, b) for a, b in zip(n.backward(view, kept, gamma), want))
    want = [t.clone() for t in n.backward(dy, x, gamma)]
    assert all(torch.equal(a, b) for a, b in zip(n.backward(view, x.reshape(4, 1, 5).transpose(1, 2), gamma), want))
