"""What the block trained on codes holds between its passes is what it says: nothing else stays, and the loss' scratch is part of it."""
import pytest
import torch

from tests.test_gpu_code_step import _codes
from tests.test_gpu_token_step_memory import _asked_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,side,channels,vocabulary", [(4, 40, 128, 3000), (3, 37, 96, 517)])
def test_memory_between_the_passes(batch, side, channels, vocabulary, dtype):
    from paper_2409_09083_amd.token_step import Codes, OrthogonalUpdate, TokenBlock
    n, es = batch * side * side, 4 if dtype == "f32" else 2
    y = torch.randn((batch, channels, side, side), device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    ids = _codes(n, vocabulary)
    y.view(-1, channels).t() @ y.view(-1, channels)             # (a process' first product makes the library's own workspace, 76 MB here, through the same allocator)
    torch.cuda.synchronize()
    before = _asked_for()
    block = TokenBlock(batch, side * side, channels, 4 if channels == 128 else 3, 1, 4 * channels, dtype, block=64)
    codes = Codes(*ids, channels, vocabulary, dtype)
    update = OrthogonalUpdate(block.matrices())
    for _ in range(2):                                          # (what the first step makes stays)
        codes.forward(block.forward(codes.enter(y)))
        held = _asked_for() - before
        codes.entered(block.backward(codes.backward()))
        update.update(block.grads, 0.01)
    weights = sum(w.numel() for w in block.params.values())
    said = block.kept_bytes()[0] + sum(sum(p.other_bytes()) for p in (block, codes, update))
    assert 0 <= held - said - weights * es - codes.table.nbytes <= 60 * 512          # (room for 60 tensors that are not named here)
    assert codes.other_bytes()[1] >= codes.head._ws.nbytes > 4 * n * vocabulary         # G as two bfloats or three


@pytest.mark.parametrize("orthogonal", [False, True])
def test_command_says_it(capsys, orthogonal):
    from paper_2409_09083_amd import token_step
    token_step.main(["--images", "2", "--size", "96", "--steps", "1", "--vocabulary", "2000"] + ["--orthogonal"] * orthogonal)
    out = capsys.readouterr().out
    s = token_step.TokenStep(2, 96, "bf16", vocabulary=2000, orthogonal=orthogonal)
    s.step()
    tensors, buffers = s.other_bytes()
    assert "and %.1f MB of q, k, v" % (tensors / 1e6) in out and "scratch: %.1f MB" % (buffers / 1e6) in out
    places = s.codes.ids.shape[0]
    assert buffers > s.block.other_bytes()[1] + 4 * places * 2000
    assert tensors >= s.block.other_bytes()[0] + 2 * 2 * places * 64


def test_command_without_a_vocabulary(capsys):
    from paper_2409_09083_amd import token_step
    token_step.main(["--images", "2", "--size", "96", "--steps", "1"])
    out = capsys.readouterr().out
    s = token_step.TokenStep(2, 96, "bf16")
    s.step()
    assert s.other_bytes() == s.block.other_bytes()
    assert "%.1f MB of q, k, v, attention's output and statistics\n" % (s.block.other_bytes()[0] / 1e6) in out
