"""The loss' gradients where rounding its gradient by the logits, G, would be seen: weights and inputs with a part that all rows share, which the sums over the vocabulary (G's rows add up to 0) and, of a
weight that has learned its labels, over the rows cancel.  What is left is small beside the sums of absolute values, and so is the rounding of the results.

Bounds as in test_gpu_token_loss.py, with u = 2^-24 and the operand G held to 2^-16 of itself where the tensors are bfloats (two of them: the second is what the first, off by at most 2^-8, leaves, to 2^-8
of that), 4 u in 32 bits, at any number of rows; a sum of n products of so many planes adds (planes n + 32) u of its absolute values."""
import pytest
import torch

from tests.test_gpu_token_loss import TYPES, U

pytestmark = pytest.mark.gpu
HELD = {"f32": 4 * U, "bf16": 2.0 ** -16}
PLANES = {"f32": 6, "bf16": 2}
LAST = {"f32": U, "bf16": 2.0 ** -8}


def _case(rows, vocab, channels, dtype, missing, seed):
    """x and w: a 64th of a random number; in 8 channels around 1, the part that all rows share; 4 more make the logits."""
    g = torch.Generator().manual_seed(seed)
    w, x = (torch.randn((n, channels), generator=g) / 64 for n in (vocab, rows))
    w[:, 4:12] += 1
    x[:, 4:12] += 1
    x[:, :4] *= 2048
    t = TYPES[dtype]
    x, w = x.to(t).cuda(), w.to(t).cuda()
    # labels drawn from the logits' own probabilities: dweight's sums over the rows nearly cancel
    p = torch.softmax(x.double() @ w.double().t().contiguous(), 1).float()
    labels = torch.multinomial(p.cpu(), 1, generator=g).squeeze(1)
    labels[torch.rand(rows, generator=g) < missing] = -1
    labels[0] = vocab - 1
    return x, w, labels.cuda()


def _bounds(x, w, labels, dtype, dloss):
    """(labelled rows, G, dx, dweight in 64 bits, their bounds)"""
    (vocab, c), wd = w.shape, w.double()
    there = (labels >= 0) & (labels < vocab)
    x, lab = x[there].double(), labels[there]
    n, at = len(lab), torch.arange(len(lab), device="cuda")
    s = x @ wd.t().contiguous()
    lse = torch.logsumexp(s, 1)
    big = ((c + 8) * U * (x.abs() @ wd.abs().t().contiguous())).amax(1) + U * (8 * s.abs().amax(1) + 8 * lse.abs() + 310 + vocab / 128)
    p = torch.exp(s - lse[:, None])
    weight = torch.full((n,), 1 / n, dtype=torch.float64, device="cuda") if dloss is None else dloss[there].double()
    g = p.clone()
    g[at, lab] -= 1
    dg = (2 * big[:, None] * p + (HELD[dtype] + 8 * U) * (g.abs() + 2 * big[:, None] * p)) * weight.abs()[:, None] + 2.0 ** -126 * (weight.abs() + 2)[:, None]
    g = g * weight[:, None]
    dx, dw = g @ wd, g.t().contiguous() @ x
    tx = dg @ wd.abs() + (PLANES[dtype] * vocab + 32) * U * (g.abs() @ wd.abs())
    tw = dg.t().contiguous() @ x.abs() + (PLANES[dtype] * n + 32) * U * (g.abs().t().contiguous() @ x.abs())
    return there, g, (dx, tx + LAST[dtype] * (dx.abs() + tx) + 1e-37), (dw, tw + LAST[dtype] * (dw.abs() + tw) + 1e-37)


def _outside(got, want_tol):
    want, tol = want_tol
    return int(((got.double() - want).abs() > tol).sum())


# a few rows; up to 64; blocks of 128, of 256 x 128; most rows without a label
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("rows,vocab,channels,missing", [(10, 300, 64, 0.0), (60, 200, 72, 0.0), (256, 300, 64, 0.1), (257, 300, 64, 0.1), (300, 300, 64, 0.97), (1100, 517, 96, 0.3), (2000, 2300, 192, 0.2),
                                                         (4100, 900, 320, 0.6)])
def test_gradients_that_cancel(rows, vocab, channels, missing, weighted, dtype):
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(rows, vocab, channels, dtype, missing, seed=rows)
    dloss = 0.5 + torch.rand(rows, generator=torch.Generator().manual_seed(1)).cuda() if weighted else None
    head = vocabulary.TokenLoss(rows, vocab, channels, dtype)
    head.forward(x, w, labels)
    dx, dw = head.backward(x, w, labels, dloss)
    there, g, want_dx, want_dw = _bounds(x, w, labels, dtype, dloss)
    assert _outside(dx[there], want_dx) == 0 and not dx[~there].any()
    assert _outside(dw, want_dw) == 0
    if dtype == "bf16":
        # (one bfloat of G is seen here, whatever else is exact)
        one = g.float().bfloat16().double()
        assert _outside((one @ w.double()).bfloat16(), want_dx) > 0
        assert _outside((one.t().contiguous() @ x[there].double()).bfloat16(), want_dw) > 0


def test_more_results_than_one_launch_sums():
    """2^21 rows of 8192 channels, one row of x for all of them, and 2^21 * 8192 / 4 = 2^32 threads that add up dx' shares: more than a launch has.  140 GB of dx and scratch.  Rows of one
    label are equal bit by bit, those of the first 256 are checked against the formula, those without a label are zeros."""
    from paper_2409_09083_amd import vocabulary
    rows, vocab, channels, none = 1 << 21, 256, 1 << 13, 7
    g = torch.Generator().manual_seed(3)
    x = torch.randn((1, channels), generator=g).bfloat16().cuda().expand(rows, channels)
    w = (torch.randn((vocab, channels), generator=g) * channels ** -0.5).bfloat16().cuda()
    labels = torch.arange(rows, device="cuda") % vocab
    labels[none::vocab] = -1
    head = vocabulary.TokenLoss(rows, vocab, channels, "bf16")
    try:
        head.forward(x, w, labels)
        for t in head.dx.split(1 << 18):
            t.fill_(float("nan"))
        dx, _ = head.backward(x, w, labels, torch.ones(rows, device="cuda"))
        first = dx[:vocab].clone()
        there, _, want, _ = _bounds(x[:vocab], w, labels[:vocab], "bf16", torch.ones(vocab, device="cuda"))
        assert _outside(first[there], want) == 0 and not first[none].any()
        for t in dx.view(-1, vocab, channels).split(256):
            assert bool((t == first).all())
    finally:
        del head
        torch.cuda.empty_cache()
