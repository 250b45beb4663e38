"""The loss over a vocabulary and its gradients against the formulas in 64 bits.

Bounds, with u = 2^-24.  A logit is a sum of C products: fp32 operands are three bfloats (what is left out is below 4 u of a product), bfloat products are exact; in any order the sum is off by
e = (C + 8) u |scale| sum|x w|.  A power's argument adds 4 u (max|s| + |log-sum|), the power 4 u; a sum of V positive numbers, in chains of at most 300 + V / 128 additions, that many u of
itself.  So a log-sum is off by E = e + u (8 max|s| + 8 |lse| + 310 + V / 128), a loss by twice that, a probability by 2 E of itself.  The gradients' operand g is rounded to a bfloat where the tensors are
(2^-8 of itself; three bfloats: 4 u), their sums over n terms are off by n u sum|terms|, and the results are rounded to the type.
What is below 2^-126 becomes 0: the power p, and either of the two lower bfloats of g = (p - [v = label]) dloss (dloss 1 where it is not given), so g is off by 2^-126 (|dloss| + 2) more before the scale."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def _case(rows, vocab, channels, dtype, missing=0.0, seed=0, label=torch.int64):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn((vocab, channels), generator=g) * channels ** -0.5
    labels = torch.randint(0, vocab, (rows,), generator=g)
    x = torch.randn((rows, channels), generator=g) + 8 * torch.rand((rows, 1), generator=g) * w[labels]
    if missing:
        labels[torch.rand(rows, generator=g) < missing] = -1
        labels[torch.rand(rows, generator=g) < missing / 4] = vocab
    t = TYPES[dtype]
    return x.to(t).cuda(), w.to(t).cuda(), labels.to(label).cuda()


def _reference(x, w, labels, scale, dtype, dloss=None):
    """Everything in 64 bits, with the bounds."""
    vocab, c = w.shape
    there = (labels >= 0) & (labels < vocab)
    x, w, lab = x[there].double(), w.double(), labels[there].long()
    at = torch.arange(len(lab), device="cuda")
    s = (x @ w.t().contiguous()) * scale
    e = ((c + 8) * U * abs(scale) * (x.abs() @ w.t().contiguous().abs())).amax(1) if len(lab) else s.new_zeros(0)
    lse = torch.logsumexp(s, 1)
    loss = lse - s[at, lab]
    top = s.abs().amax(1) if len(lab) else e
    big = e + U * (8 * top + 8 * lse.abs() + 310 + vocab / 128)
    p = torch.exp(s - lse[:, None])
    weight = (torch.full((len(lab),), 1 / max(1, len(lab)), dtype=torch.float64, device="cuda") if dloss is None else dloss[there].double()) * scale
    g = p.clone()
    g[at, lab] -= 1
    half = 2.0 ** -8 if dtype == "bf16" else 4 * U
    dg = (2 * big[:, None] * p + (half + 8 * U) * (g.abs() + 2 * big[:, None] * p)) * weight.abs()[:, None]
    outer = scale / max(1, len(lab)) if dloss is None else scale
    dg += 2.0 ** -126 * (weight.abs() + 2 * abs(outer))[:, None]
    g = g * weight[:, None]
    dx, dw = g @ w, g.t().contiguous() @ x
    last = 2.0 ** -8 if dtype == "bf16" else U
    tdx = dg @ w.abs() + (vocab + 32) * U * (g.abs() @ w.abs())
    tdw = dg.t().contiguous() @ x.abs() + (len(lab) + 32) * U * (g.abs().t().contiguous() @ x.abs())
    return {"there": there, "loss": (loss, 2 * big), "lse": (lse, big), "dx": (dx, tdx + last * (dx.abs() + tdx) + 1e-37), "dw": (dw, tdw + last * (dw.abs() + tdw) + 1e-37)}


def _near(got, want_tol):
    want, tol = want_tol
    return bool(((got.double() - want).abs() <= tol).all())


def _check(head, x, w, labels, scale, dtype, dloss=None):
    mean = head.forward(x, w, labels).clone()
    r = _reference(x, w, labels, scale, dtype, dloss)
    there = r["there"]
    assert _near(head.lse[there], r["lse"]) and _near(head.losses[there], r["loss"])
    assert not head.losses[~there].any() and not head.lse[~there].any()
    n = int(there.sum())
    want = float(r["loss"][0].mean()) if n else 0.0
    assert abs(float(mean) - want) <= (float(r["loss"][1].mean()) if n else 0) + 2 * U * abs(want)
    head.dx.fill_(math.nan)
    head.dweight.fill_(math.nan)
    dx, dw = (t.clone() for t in head.backward(x, w, labels, dloss))
    assert _near(dx[there], r["dx"]) and not dx[~there].any()
    assert _near(dw, r["dw"])
    head._ws.fill_(255)                                         # scratch need not be cleared: NaN everywhere
    again = head.backward(x, w, labels, dloss)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    lse, losses = head.lse.clone(), head.losses.clone()
    head._ws.fill_(255)
    assert torch.equal(head.forward(x, w, labels), mean) and torch.equal(head.lse, lse) and torch.equal(head.losses, losses)


SIZES = [(1, 1, 1), (1, 2, 3), (4, 1000, 64), (31, 129, 40), (32, 700, 128), (33, 257, 64), (64, 64, 250), (65, 1024, 72), (130, 5000, 33), (257, 300, 320), (600, 2049, 192), (1030, 515, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,channels", SIZES)
def test_all_labelled(rows, vocab, channels, dtype):
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(rows, vocab, channels, dtype)
    _check(vocabulary.TokenLoss(rows, vocab, channels, dtype), x, w, labels, 1.0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("missing", [0.0, 0.4])
@pytest.mark.parametrize("channels", [72, 128])
@pytest.mark.parametrize("rows", [4, 5, 16, 17, 32, 33, 63, 64, 65])
def test_few_rows(rows, channels, missing, dtype):
    """Around the numbers of rows where the blocks' sizes and the joins of their statistics change, with x as it lies and gathered."""
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(rows, 700, channels, dtype, missing, seed=5)
    _check(vocabulary.TokenLoss(rows, 700, channels, dtype), x, w, labels, 1.0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("missing", [0.3, 0.95, 1.1])
@pytest.mark.parametrize("rows,vocab,channels", [(3, 50, 64), (20, 300, 96), (64, 513, 64), (200, 1000, 130), (1500, 260, 64)])
def test_some_labelled(rows, vocab, channels, missing, dtype):
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(rows, vocab, channels, dtype, missing, seed=1, label=torch.int32)
    dloss = torch.randn(rows, generator=torch.Generator().manual_seed(2)).cuda()
    scale = torch.tensor(-0.7).item()
    _check(vocabulary.TokenLoss(rows, vocab, channels, dtype, scale=-0.7), x, w, labels, scale, dtype, dloss)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_rows_without_a_label_hold_reaches_nothing(dtype):
    from paper_2409_09083_amd import vocabulary
    for rows in (9, 300):
        x, w, labels = _case(rows, 400, 64, dtype, 0.4, seed=3)
        labels[0], labels[1] = 5, -1
        there = (labels >= 0) & (labels < 400)
        dloss = torch.rand(rows, device="cuda")
        head = vocabulary.TokenLoss(rows, 400, 64, dtype)
        want = [t.clone() for t in (head.forward(x, w, labels), head.losses, head.lse, *head.backward(x, w, labels, dloss))]
        for bad in (math.nan, math.inf, -math.inf):
            x[~there] = bad
            dloss[~there] = bad
            got = head.forward(x, w, labels), head.losses, head.lse, *head.backward(x, w, labels, dloss)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), bad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_bad_row_spoils_itself_and_the_weight(dtype):
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(150, 300, 64, dtype, seed=4)
    head = vocabulary.TokenLoss(150, 300, 64, dtype)
    head.forward(x, w, labels)
    losses, dx = head.losses.clone(), head.backward(x, w, labels, torch.ones(150, device="cuda"))[0].clone()
    x[70, 3] = math.nan
    mean = head.forward(x, w, labels)
    other = torch.arange(150, device="cuda") != 70
    assert mean.isnan() and head.losses[70].isnan() and torch.equal(head.losses[other], losses[other])
    got, dw = head.backward(x, w, labels, torch.ones(150, device="cuda"))
    assert got[70].isnan().all() and torch.equal(got[other], dx[other]) and dw.isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_and_equal_logits(dtype):
    """Logits of +-2e4, of one value all, and a vocabulary of one word (loss 0 and no gradient)."""
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(100, 500, 64, dtype, seed=5)
    _check(vocabulary.TokenLoss(100, 500, 64, dtype, scale=2000.0), x, w, labels, 2000.0, dtype)
    head = vocabulary.TokenLoss(100, 500, 64, dtype)
    zero = torch.zeros_like(x)
    assert abs(float(head.forward(zero, w, labels)) - math.log(500)) <= 1e-5
    one = vocabulary.TokenLoss(100, 1, 64, dtype)
    # the one logit, |s| < 64, and the log-sum are the same number but for 4 u |s|
    assert abs(float(one.forward(x, w[:1], torch.zeros_like(labels)))) <= 256 * U
    dx, dw = one.backward(x, w[:1], torch.zeros_like(labels))
    # exp(s - lse) of the one word is 1 up to the rounding of lse's product with log2(e)
    assert float(dx.abs().max()) <= 1e-4 and float(dw.abs().max()) <= 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 1)])
def test_rows_inside_wider_ones(pad, offset, dtype):
    from paper_2409_09083_amd import vocabulary
    for rows in (6, 90):
        x, w, labels = _case(rows, 333, 64, dtype, 0.2, seed=6)
        head = vocabulary.TokenLoss(rows, 333, 64, dtype)
        want = [t.clone() for t in (head.forward(x, w, labels), head.losses, *head.backward(x, w, labels))]

        def wide(t):
            b = torch.full((t.shape[0] * (64 + pad) + offset,), math.nan, dtype=t.dtype, device="cuda")
            v = b[offset:].view(t.shape[0], 64 + pad)[:, :64]
            v.copy_(t)
            return v
        got = head.forward(wide(x), wide(w), labels), head.losses, *head.backward(wide(x), wide(w), labels)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_gradients_by_differences():
    from paper_2409_09083_amd import vocabulary
    x, w, labels = _case(40, 70, 24, "f32", 0.2, seed=7)
    head = vocabulary.TokenLoss(40, 70, 24)
    head.forward(x, w, labels)
    dx, dw = (t.double().clone() for t in head.backward(x, w, labels))

    def mean(x, w):
        there = (labels >= 0) & (labels < 70)
        s = x.double()[there] @ w.double().t().contiguous()
        return float((torch.logsumexp(s, 1) - s.gather(1, labels[there].long()[:, None]).squeeze(1)).mean())
    g = torch.Generator().manual_seed(8)
    for _ in range(4):
        ux, uw = torch.randn(x.shape, generator=g).cuda().double(), torch.randn(w.shape, generator=g).cuda().double()
        h = 1e-4
        d = (mean(x.double() + h * ux, w.double() + h * uw) - mean(x.double() - h * ux, w.double() - h * uw)) / (2 * h)
        got = float((dx * ux).sum() + (dw * uw).sum())
        assert abs(d - got) <= 1e-5 * (1 + abs(d))              # (a third derivative of about 100 times h^2, and 32-bit gradients)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pieces_of_the_vocabulary_and_splits(dtype, monkeypatch):
    """Sizes whose gradients go in several pieces of the vocabulary, and in shares of a contraction."""
    from paper_2409_09083_amd import vocabulary
    for rows, vocab, channels in ((40, 30000, 64), (4100, 640, 64)) + (((9000, 34000, 64),) if dtype == "bf16" else ((3000, 33000, 64),)):
        x, w, labels = _case(rows, vocab, channels, dtype, 0.1, seed=9)
        _check(vocabulary.TokenLoss(rows, vocab, channels, dtype), x, w, labels, 1.0, dtype)


@pytest.mark.parametrize("rows,dtype", [(4100, "bf16"), (70, "bf16"), (33, "f32")])
def test_offsets_of_more_than_31_bits(rows, dtype):
    """A weight of 2.4 GB (its planes 7.4), G of 1.2 GB where there are many rows; labels at both ends of it."""
    from paper_2409_09083_amd import vocabulary
    vocab, channels = 150000, 8192
    g = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.randn((vocab, channels), generator=g, device="cuda") * channels ** -0.5).to(TYPES[dtype])
    labels = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    labels[0], labels[1], labels[2] = vocab - 1, 0, -1
    x = (torch.randn((rows, channels), generator=g, device="cuda") + 8 * w[labels.clamp(min=0)].float()).to(TYPES[dtype])
    head = vocabulary.TokenLoss(rows, vocab, channels, dtype)
    mean = float(head.forward(x, w, labels))
    r = _reference(x, w, labels, 1.0, dtype)
    there = r["there"]
    assert _near(head.lse[there], r["lse"]) and _near(head.losses[there], r["loss"])
    assert abs(mean - float(r["loss"][0].mean())) <= float(r["loss"][1].mean()) + 2 * U * abs(mean)
    dx, dw = head.backward(x, w, labels)
    assert _near(dx[there], r["dx"]) and not dx[~there].any() and _near(dw, r["dw"])


def test_empty_refusals_streams_and_graph():
    from paper_2409_09083_amd import vocabulary
    e = vocabulary.TokenLoss(0, 50, 8)
    none, x0, w0 = torch.empty((0,), dtype=torch.int64, device="cuda"), torch.empty((0, 8), device="cuda"), torch.randn((50, 8), device="cuda")
    assert float(e.forward(x0, w0, none)) == 0
    e.dweight.fill_(1)
    assert e.backward(x0, w0, none)[0].shape == (0, 8) and not e.dweight.any()
    x, w, labels = _case(100, 220, 64, "bf16", 0.2, seed=10)
    head = vocabulary.TokenLoss(100, 220, 64, "bf16")
    for bad in (lambda: head.forward(x.float(), w, labels), lambda: head.forward(x, w.float(), labels), lambda: head.forward(x, w, labels.short()),
                lambda: head.backward(x, w, labels, torch.ones(100, device="cuda").double())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: head.forward(x[:-1], w, labels), lambda: head.forward(x, w[:, :-1], labels), lambda: head.forward(x, w, labels[:-1]), lambda: head.forward(x, w.t().contiguous().t(), labels),
                lambda: head.backward(x, w, labels, torch.ones(1, device="cuda").expand(100)), lambda: vocabulary.TokenLoss(100, 220, 64, training=False).backward(x.float(), w.float(), labels)):
        with pytest.raises(ValueError):
            bad()
    few = vocabulary.TokenLoss(3, 220, 64, "bf16")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())

    def all_of():
        head.forward(x, w, labels)
        head.backward(x, w, labels)
        few.forward(x[:3], w, labels[:3])
        return [t for o in (head, few) for t in (o.mean, o.losses, o.lse)] + [head.dx, head.dweight]
    with torch.cuda.stream(side):
        all_of()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        outs = all_of()
    for k in range(4):
        a, b, c = _case(100, 220, 64, "bf16", 0.1 * k, seed=20 + k)
        x.copy_(a), w.copy_(b), labels.copy_(c)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert all(torch.equal(p, q) for p, q in zip(all_of(), got))
        torch.cuda.synchronize()
