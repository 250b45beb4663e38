"""What the token block holds between its passes: checkpoints and what it says besides, no tensor that a checkpoint stands for."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _asked_for():
    """Bytes of the tensors there are (torch.cuda.memory_allocated() counts their blocks, up to 1 MB larger each)."""
    return torch.cuda.memory_stats()["requested_bytes.all.current"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,side,channels,heads,kv", [(4, 40, 128, 4, 2), (3, 37, 96, 3, 1)])
def test_memory_between_the_passes(batch, side, channels, heads, kv, dtype):
    from paper_2409_09083_amd.token_step import TokenBlock
    rows, c, hidden, es = batch * side * side, channels, 4 * channels, 4 if dtype == "f32" else 2
    width = (heads + 2 * kv) * (c // heads)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    y = torch.randn((batch, c, side, side), device="cuda").to(t)
    dz = torch.randn((rows, c), device="cuda").to(t)
    torch.cuda.synchronize()
    before = _asked_for()
    block = TokenBlock(batch, side * side, c, heads, kv, hidden, dtype, block=64)
    for _ in range(2):                                          # (what the first step makes stays)
        z = block.forward(y)
        held = _asked_for() - before - z.nbytes
        block.backward(dz)
        del z
    cols = 3 * c + 2 * hidden                                   # n1, x2, n2 and the hidden layer before and after its activation
    checkpoints = rows * (cols + sum(-(-n // 64) for n in (c, c, c, hidden, hidden)))
    tensors = rows * ((width + c) * es + 4 * heads + 16)        # q, k, v, out; log-sums, means and deviations
    gradients = rows * ((width + 2 * c) * es + c + -(-c // 64))  # dq, dk, dv, dx of the norms, out in 8 bits for a weight gradient
    weights = c * (width + c + 2 * hidden) + 4 * c
    scratch = sum(o._ws.nbytes for o in (block.norm1, block.norm2, block.attention, block.kept_n1, block.kept_n2, block.kept_a, block.out8))
    assert held <= checkpoints + tensors + gradients + weights * (es + 4) + scratch + 60 * 512          # (room for 60 tensors that are not named here)
    assert block.kept_bytes() == (checkpoints, rows * cols * es)
    assert block.other_bytes() == (tensors, gradients + 4 * weights + scratch)


def test_norm_into_a_caller_s_tensor():
    """Rows and maps of any strides; the object's own buffer is made when it is asked for, and keeps its layout."""
    from paper_2409_09083_amd import tokens
    x = torch.randn((3, 50, 48), device="cuda")
    n = tokens.Norm(3, 50, 48, "f32", y_layout="map")
    wide = torch.full((3, 50, 64), float("nan"), device="cuda")
    assert n.forward(x, out=wide[:, :, :48]).data_ptr() == wide.data_ptr()
    assert n._y is None and wide[:, :, 48:].isnan().all()
    mean = n.mean.clone()
    y = n.forward(x)
    assert y.data_ptr() == n.y_buffer.data_ptr() and n.y_buffer.shape == (3, 48, 50)
    # (rows and maps are added up in different orders: 128 roundings of numbers up to 5 either way)
    assert (n.mean - mean).abs().max() <= 1e-4 and (y - wide[:, :, :48]).abs().max() <= 1e-4
    n.forward(x, out=wide[:, :, :48])
    assert torch.equal(n.forward(x + 1), n.y) and n.y_buffer.is_contiguous()
    with pytest.raises(ValueError):
        n.forward(x, out=wide)
    with pytest.raises(TypeError):
        n.forward(x, out=wide[:, :, :48].bfloat16())
