"""The token block trained on codes: known codes entering as embedding rows, the loss over the vocabulary with the same table, gradients through all of it
against torch's automatic ones in 64 bits, orthogonal updates, the command.

Bounds as for the token block itself (its 8-bit checkpoints are most of the error): 3 % of a gradient's norm, 6 % in bfloats; the loss, which sees
one rounded block output, 1 %."""
import pytest
import torch

from tests.test_gpu_token_step import _reference

pytestmark = pytest.mark.gpu


def _codes(places, vocabulary, missing=0.2):
    g = torch.Generator(device="cuda").manual_seed(11)
    codes = torch.randint(0, vocabulary, (places,), generator=g, device="cuda")
    u = torch.rand(places, generator=g, device="cuda")
    return torch.where(u < 0.4, codes, -1), torch.where((u >= 0.4) & (u < 1 - missing), codes, -1)          # known, to be told; some are neither


@pytest.mark.parametrize("dtype,bound", [("f32", 0.03), ("bf16", 0.06)])
@pytest.mark.parametrize("batch,side,channels,heads,kv,vocabulary", [(2, 9, 32, 4, 2, 100), (1, 13, 64, 2, 2, 777), (3, 5, 48, 6, 1, 40)])
def test_gradients(batch, side, channels, heads, kv, vocabulary, dtype, bound):
    from paper_2409_09083_amd.token_step import Codes, TokenBlock
    n = side * side
    block = TokenBlock(batch, n, channels, heads, kv, 3 * channels, dtype, block=32)
    codes = Codes(*_codes(batch * n, vocabulary), channels, vocabulary, dtype)
    t = codes.table.dtype
    y = torch.randn((batch, channels, side, side), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(t)
    x = codes.enter(y)
    loss = codes.forward(block.forward(x)).clone()
    dmap = block.backward(codes.backward())
    codes.entered(dmap)
    # in 64 bits: the block's own reference, with the embedding before it and the loss behind it
    table = codes.table.double().requires_grad_(True)
    there = codes.ids >= 0
    rows = torch.where(there[:, None], table[codes.ids.clamp(min=0)] * channels ** 0.5, 0.0)
    inner = (y.double().view(batch, channels, n) + rows.view(batch, n, channels).transpose(1, 2)).detach()
    z = _reference(block, inner, torch.zeros((batch * n, channels), device="cuda"))[0].requires_grad_(True)
    told = codes.labels >= 0
    s = z[told] @ table.t().contiguous()
    want = (torch.logsumexp(s, 1) - s.gather(1, codes.labels[told][:, None]).squeeze(1)).mean()
    dz, dhead = torch.autograd.grad(want, [z, table])
    _, dy, grads = _reference(block, inner, dz)
    dtable = torch.autograd.grad(rows, table, dy.reshape(batch, channels, n).transpose(1, 2).reshape(-1, channels))[0] + dhead

    def off(a, b):
        return float((a.double().reshape(-1) - b.reshape(-1)).norm() / b.norm())
    assert abs(float(loss) - float(want.detach())) <= 0.01 * float(want.detach())
    assert off(dmap, dy) <= bound and off(codes.grad, dtable) <= bound
    for name, w in grads.items():
        assert off(block.grads[name], w) <= bound, name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("orthogonal", [False, True])
def test_steps_run_and_move_everything(dtype, orthogonal):
    from paper_2409_09083_amd.token_step import TokenStep
    s = TokenStep(images=2, size=72, dtype=dtype, channels=32, vocabulary=500, orthogonal=orthogonal)
    tensors = [w for w in s.early.weights if w is not None] + list(s.block.params.values()) + [s.codes.table]
    before = [w.clone() for w in tensors]
    losses = [float(s.step(0.02)) for _ in range(3)]
    assert all(x == x and x < 50 for x in losses)
    assert all(not torch.equal(a, b) for a, b in zip(before, tensors))


def test_orthogonal_update_is_a_step_in_every_direction():
    from paper_2409_09083_amd.token_step import OrthogonalUpdate
    w = {"w": torch.zeros((48, 20), device="cuda")}
    u = OrthogonalUpdate(w, momentum=0.5)
    g = torch.randn((48, 20), generator=torch.Generator().manual_seed(1)).cuda()
    u.update({"w": g}, 1.0)
    values = torch.linalg.svdvals(w["w"].double().cpu()) / (48 / 20) ** 0.5
    assert 0.6 <= float(values.min()) and float(values.max()) <= 1.3
    assert float((w["w"].double() * g.double()).sum()) < 0
    u.update({"w": -0.5 * g}, 1.0)
    assert not u.sums["w"].any()                                # 0.5 g - 0.5 g: no direction, no step
    once = w["w"].clone()
    u.update({"w": torch.zeros_like(g)}, 1.0)
    assert torch.equal(w["w"], once)


def test_command(capsys):
    from paper_2409_09083_amd import token_step
    token_step.main(["--images", "1", "--size", "64", "--steps", "2", "--vocabulary", "300", "--orthogonal"])
    out = capsys.readouterr().out
    assert "300 codes" in out and "step 1: loss" in out


def test_a_run_of_them_captured():
    """The operators one after the other, captured once and replayed with other inputs and eager work between, every replay equal to the eager run."""
    from paper_2409_09083_amd import orthogonal, vocabulary
    rows, vocab, c = 130, 210, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    ids, labels = _codes(rows, vocab)
    table = torch.randn((vocab, c), generator=g, device="cuda").bfloat16()
    e, head = vocabulary.Embedding(rows, vocab, c, "bf16"), vocabulary.TokenLoss(rows, vocab, c, "bf16")
    o = orthogonal.Orthogonal(vocab, c)

    def run():
        x = e.forward(ids, table)
        head.forward(x, table, labels)
        dx, dw = head.backward(x, table, labels)
        e.backward(ids, dx)
        o.forward(e.dtable)
        return [e.out, head.mean, head.losses, dx, dw, e.dtable, o.out]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        outs = run()
    for k in range(4):
        table.copy_(torch.randn((vocab, c), generator=g, device="cuda"))
        ids.copy_(ids.roll(k))
        labels.copy_(labels.roll(2 * k))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert all(torch.equal(a, b) for a, b in zip(run(), got))
        torch.cuda.synchronize()
