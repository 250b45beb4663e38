"""The loss' gradients where G does not fit its 1 GiB (or a piece's 2^20 ids), so that the vocabulary goes in several pieces: dx is added up over them, dweight and the labels are a piece's.  The scratch asked for shows that
there are several: with one, it would hold G whole beside x and the weight as bfloats.  Bounds as in test_gpu_token_loss.py and, where sums cancel, test_gpu_token_gradients.py."""
import pytest
import torch

from tests import test_gpu_token_gradients as gradients
from tests.test_gpu_token_loss import _case, _check

pytestmark = pytest.mark.gpu


def _up(n, to):
    return (n + to - 1) // to * to


def _several(head, rows, vocab, channels, dtype):
    planes, of_g = (3, 3) if dtype == "f32" else (1, 2)
    rows, channels = _up(rows, 64), _up(channels, 64)
    return head._ws.numel() < 2 * planes * channels * (rows + _up(vocab, 64)) + 2 * of_g * rows * _up(vocab, 256)


# planes laid out; the weight as it lies; few rows, pieces of 2^20 ids
SIZES = [(6000, 33000, 64, "f32"), (9000, 34000, 72, "bf16"), (3000, 100000, 64, "bf16"), (1500, 125000, 40, "f32"), (10, 1100000, 64, "bf16"), (40, 1100000, 8, "f32")]


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("rows,vocab,channels,dtype", SIZES)
def test_pieces(rows, vocab, channels, dtype, weighted):
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(rows, vocab, channels, dtype, 0.3, seed=rows, label=torch.int32 if weighted else torch.int64)
    labels[0], labels[1], labels[2] = vocab - 1, 0, -1
    dloss = torch.randn(rows, generator=torch.Generator().manual_seed(2)).cuda() if weighted else None
    scale = torch.tensor(-0.7).item() if weighted else 1.0
    head = vocabulary.TokenLoss(rows, vocab, channels, dtype, scale=scale)
    assert _several(head, rows, vocab, channels, dtype)
    _check(head, x, w, labels, scale, dtype, dloss)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,vocab,channels", [(9000, 34000, 64), (3000, 100000, 64)])
def test_pieces_that_cancel(rows, vocab, channels):
    from paper_2409_09083_amd import vocabulary
    x, w, labels = gradients._case(rows, vocab, channels, "bf16", 0.1, seed=rows)
    head = vocabulary.TokenLoss(rows, vocab, channels, "bf16")
    assert _several(head, rows, vocab, channels, "bf16")
    head.forward(x, w, labels)
    dx, dw = head.backward(x, w, labels)
    there, _, want_dx, want_dw = gradients._bounds(x, w, labels, "bf16", None)
    assert gradients._outside(dx[there], want_dx) == 0 and not dx[~there].any() and gradients._outside(dw, want_dw) == 0
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,vocab,channels,dtype", [(6000, 33000, 64, "f32"), (3000, 100000, 64, "bf16")])
def test_one_of_the_gradients(rows, vocab, channels, dtype):
    """dx alone and dweight alone, through the C entry, are what both together are."""
    from paper_2409_09083_amd import binding as B
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(rows, vocab, channels, dtype, 0.3, seed=5)
    head = vocabulary.TokenLoss(rows, vocab, channels, dtype)
    head.forward(x, w, labels)
    dx, dw = (t.clone() for t in head.backward(x, w, labels))
    for alone in range(2):
        head.dx.fill_(float("nan"))
        head.dweight.fill_(float("nan"))
        out = [head.dx.data_ptr(), head.dweight.data_ptr()]
        out[1 - alone] = 0
        B.ftp_token_loss_backward(head.desc, x.data_ptr(), w.data_ptr(), labels.data_ptr(), head.lse.data_ptr(), 0, *out, head._ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
        assert torch.equal((head.dx, head.dweight)[alone], (dx, dw)[alone]) and bool((head.dweight, head.dx)[alone].isnan().all())
    torch.cuda.empty_cache()
