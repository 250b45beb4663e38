"""The loss over a vocabulary with a scale of 0 or below what 32 bits hold as normal numbers, and products of x and the weight that are large; a single row whatever its stride.  Bounds as in test_gpu_token_loss.py."""
import math

import pytest
import torch

from tests.test_gpu_token_loss import U, _case, _check

pytestmark = pytest.mark.gpu
ROWS = [5, 40, 100, 700]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", ROWS)
def test_scale_of_zero(rows, dtype):
    """All logits are 0, however large the products: the losses are log(vocab), a sum of `vocab` ones (310 + vocab / 128 additions, the logarithm, log2(e) as a factor and back); no gradient."""
    from paper_2409_09083_amd import vocabulary
    vocab = 300
    x, w, labels = _case(rows, vocab, 64, dtype, 0.2, seed=31)
    labels[0] = 7
    x, w = x * 2.0 ** 60, w * 2.0 ** 62                         # (products up to some 1e37)
    assert 1e36 < float((x.double() @ w.double().t().contiguous()).abs().max()) < 1e38
    there = (labels >= 0) & (labels < vocab)
    for scale in (0.0, -0.0):
        head = vocabulary.TokenLoss(rows, vocab, 64, dtype, scale=scale)
        mean = float(head.forward(x, w, labels))
        tol = U * (8 * math.log(vocab) + 310 + vocab / 128)
        for got in (head.losses[there], head.lse[there]):
            assert float((got.double() - math.log(vocab)).abs().max()) <= tol
        assert abs(mean - math.log(vocab)) <= tol
        dx, dw = head.backward(x, w, labels)
        assert not dx.any() and not dw.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [2.0 ** -110, -3.0 * 2.0 ** -131, 5.0 * 2.0 ** -140])
@pytest.mark.parametrize("rows", ROWS)
def test_small_scales(rows, scale, dtype):
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(rows, 300, 64, dtype, 0.2, seed=32)
    labels[0] = 7
    x, w = x * 2.0 ** 59, w * 2.0 ** 60
    _check(vocabulary.TokenLoss(rows, 300, 64, dtype, scale=scale), x, w, labels, scale, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("channels", [64, 72])
def test_one_row_of_any_stride(channels, dtype):
    from paper_2409_09083_amd import binding as B
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(1, 333, channels, dtype, seed=33)
    head = vocabulary.TokenLoss(1, 333, channels, dtype)
    want = [t.clone() for t in (head.forward(x, w, labels), head.losses, head.lse, *head.backward(x, w, labels))]
    stream = torch.cuda.current_stream().cuda_stream
    for stride in (0, 1, 3, channels - 1, channels + 5, 1 << 40):
        head.desc.x_stride = stride
        B.ftp_token_loss_forward(head.desc, x.data_ptr(), w.data_ptr(), labels.data_ptr(), *head._outputs, head._ws.data_ptr(), stream)
        B.ftp_token_loss_backward(head.desc, x.data_ptr(), w.data_ptr(), labels.data_ptr(), head.lse.data_ptr(), 0, head.dx.data_ptr(), head.dweight.data_ptr(), head._ws.data_ptr(), stream)
        assert all(torch.equal(a, b) for a, b in zip((head.mean, head.losses, head.lse, head.dx, head.dweight), want)), stride
