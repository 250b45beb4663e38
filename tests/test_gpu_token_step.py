"""The token block behind the early layers: its gradients against torch's automatic ones in 64 bits, a few training steps, its command.

The block keeps what its backward pass needs in 8 bits: a value is off by at most half a step, 2^-7 of its block's largest, uniformly
so by 2^-7 / sqrt(3) * largest / 2 in the mean; with the largest of 64 normal numbers at 2.5 times their size that is below 1 % of a
tensor's norm.  A gradient meets at most three such tensors one after the other: 3 % of its norm; bfloat adds 8 roundings of 2^-8 each: 6 %."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _reference(block, y, dz):
    b, n, c = block.shape
    p = {k: v.double().requires_grad_(True) for k, v in block.params.items()}
    y = y.double().requires_grad_(True)
    x = y.view(b, c, n).transpose(1, 2)

    def norm(t, g, s):
        m = t.mean(2, keepdim=True)
        return (t - m) * (((t - m) ** 2).mean(2, keepdim=True) + 1e-5) ** -0.5 * g + s
    h, kv, d = block.heads, block.kv_heads, block.hd
    q, k, v = (norm(x, p["g1"], p["b1"]) @ p["wqkv"].t()).view(b, n, -1, d).split((h, kv, kv), 2)
    k, v = (t.repeat_interleave(h // kv, 2).transpose(1, 2) for t in (k, v))
    pr = torch.softmax(q.transpose(1, 2) @ k.transpose(2, 3).contiguous() * d ** -0.5, 3)
    x2 = x + (pr @ v.contiguous()).transpose(1, 2).reshape(b, n, c) @ p["wo"].t()
    u = norm(x2, p["g2"], p["b2"]) @ p["w1"].t()
    z = x2 + (u * torch.special.ndtr(u)) @ p["w2"].t()
    names = list(p)
    grads = torch.autograd.grad(z, [y] + [p[k] for k in names], dz.double().view(z.shape))
    return z.detach().reshape(-1, c), grads[0], dict(zip(names, grads[1:]))


@pytest.mark.parametrize("dtype,bound", [("f32", 0.03), ("bf16", 0.06)])
@pytest.mark.parametrize("batch,side,channels,heads,kv", [(2, 9, 32, 4, 2), (1, 13, 64, 2, 2), (3, 5, 48, 6, 1)])
def test_gradients(batch, side, channels, heads, kv, dtype, bound):
    from paper_2409_09083_amd.token_step import TokenBlock
    block = TokenBlock(batch, side * side, channels, heads, kv, 3 * channels, dtype, block=32)
    g = torch.Generator(device="cuda").manual_seed(4)
    t = block.params["wo"].dtype
    y = torch.randn((batch, channels, side, side), generator=g, device="cuda").to(t)
    dz = torch.randn((batch * side * side, channels), generator=g, device="cuda").to(t)
    z = block.forward(y)
    dy = block.backward(dz)
    want_z, want_dy, want = _reference(block, y, dz)

    def off(a, b):
        return float((a.double().reshape(-1) - b.reshape(-1)).norm() / b.norm())
    assert off(z, want_z) <= bound
    assert off(dy, want_dy) <= bound
    for name, w in want.items():
        assert off(block.grads[name], w) <= bound, name
    held, plain = block.kept_bytes()
    assert held <= (0.27 if dtype == "f32" else 0.54) * plain


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_approach_the_target(dtype):
    from paper_2409_09083_amd.token_step import TokenStep
    s = TokenStep(images=2, size=72, dtype=dtype, channels=32)
    before = [w.clone() for w in s.early.weights if w is not None]
    losses = [float(s.step(0.05)) for _ in range(8)]
    assert all(x == x for x in losses) and losses[-1] < 0.9 * losses[0], losses
    assert all(not torch.equal(a, b) for a, b in zip(before, [w for w in s.early.weights if w is not None]))


def test_command(capsys):
    from paper_2409_09083_amd import token_step
    token_step.main(["--images", "1", "--size", "64", "--steps", "2", "--dtype", "f32"])
    out = capsys.readouterr().out
    assert "64 tokens an image" in out and "step 1: loss" in out and "in 8 bits" in out
