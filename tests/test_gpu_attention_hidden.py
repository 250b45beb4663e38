"""Causal attention where what a query does not see holds the type's largest numbers."""
import pytest
import torch

from tests import test_gpu_attention as A

pytestmark = pytest.mark.gpu
LARGEST = float(torch.finfo(torch.bfloat16).max)                # (the largest bfloat: what fp32 inputs may hold, too)


# workgroups of 64 rows and of 128, shared heads, heads of 128
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 80, 80, 64), (800, 1, 1, 80, 80, 64), (2, 4, 2, 80, 80, 128), (1, 2, 1, 300, 300, 32)])
@pytest.mark.parametrize("at", [40, 70])
def test_hidden_keys_of_the_largest_numbers(shape, at, dtype):
    """The score of key `at` would be just below the largest fp32 number, for rows that do not see it: the rows before it get equal bits with any other key there."""
    q, k, v, do = A._make(*shape, dtype)
    q[..., 0] = torch.linspace(0.9, 1.0, shape[3], device="cuda").to(q.dtype)[None, :, None]
    q[:, ::2] *= -1
    want = A._run(q, k, v, do, dtype, True)
    for sign in (1, -1):
        k2, v2 = k.clone(), v.clone()
        k2[:, at] = 0
        k2[:, at, :, 0] = sign * LARGEST
        v2[:, at] = LARGEST
        got = A._run(q, k2, v2, do, dtype, True)
        assert torch.equal(got.out[:, :at], want.out[:, :at])
        assert torch.equal(got.lse[:, :, :at], want.lse[:, :, :at])
        assert torch.equal(got.dq[:, :at], want.dq[:, :at])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 80, 80, 64), (2, 4, 2, 80, 80, 128), (1, 2, 1, 300, 300, 32)])
def test_hidden_queries_of_the_largest_numbers(shape, dtype):
    """Query 5 is hidden from the keys behind it, whose scores with it would be the largest there are: their gradients keep their bits."""
    q, k, v, do = A._make(*shape, dtype)
    k[..., 0] = 1.0
    k[:, :6, :, 0] = 0.01
    want = A._run(q, k, v, do, dtype, True)
    q2, do2 = q.clone(), do.clone()
    q2[:, 5] = 0
    q2[:, 5, :, 0] = LARGEST
    do2[:, 5] = LARGEST
    got = A._run(q2, k, v, do2, dtype, True)
    assert torch.equal(got.dk[:, 6:], want.dk[:, 6:])
    assert torch.equal(got.dv[:, 6:], want.dv[:, 6:])
