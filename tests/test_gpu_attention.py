"""Softmax attention, forward and backward, against the formulas in 64 bits, element by element.

Bounds, u = 2^-24: a score is a sum of D products, off by at most D u * scale * sum|q||k|, so a probability is off by the factor
1 + r with r = 2 D u * max(scale sum|q||k|) + 16 u (exponent's argument, exponential, sum).  A result is a sum of n terms one after the
other: (n + 16) u + r, and with bfloats another 2^-8 for each of: the probability (or its gradient) as an operand, the result, and in the
backward pass out, from which delta is computed - of the sum of the terms' magnitudes.  ds = p (dp - delta) has the error of both
parts: its magnitude is taken as p (|dp| sums + |delta| sums)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _make(b, h, kv, ql, kl, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(TYPES[dtype])    # noqa: E731
    return new(b, ql, h, d), new(b, kl, kv, d), new(b, kl, kv, d), new(b, ql, h, d)


def _reference(q, k, v, do, causal, scale, q_lens, kv_lens):
    b, ql, h, d = q.shape
    kl, kv = k.shape[1], k.shape[2]
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device="cuda")    # noqa: E731
    r = {n: z(b, ql, h, d) for n in ("out", "dq", "out_abs", "dq_abs")}
    r.update({n: z(b, kl, kv, d) for n in ("dk", "dv", "dk_abs", "dv_abs")})
    r["lse"] = z(b, h, ql) - math.inf
    r["smax"] = 0.0
    for n in range(b):
        qn = ql if q_lens is None else min(max(int(q_lens[n]), 0), ql)
        kn = kl if kv_lens is None else min(max(int(kv_lens[n]), 0), kl)
        if qn == 0 or kn == 0:
            continue
        see = torch.ones((qn, kn), dtype=torch.bool, device="cuda")
        if causal:
            see = torch.arange(kn, device="cuda")[None] <= torch.arange(qn, device="cuda")[:, None] + kn - qn
        any_ = see.any(1)
        for j in range(h):
            c = j // (h // kv)
            Q, K, V, G = q[n, :qn, j].double(), k[n, :kn, c].double(), v[n, :kn, c].double(), do[n, :qn, j].double()
            s = torch.where(see, Q @ K.t().contiguous() * scale, -math.inf)
            lse = torch.logsumexp(s, 1)
            p = torch.where(see, torch.exp(s - torch.where(any_, lse, torch.zeros_like(lse))[:, None]), 0.0)
            o = p @ V
            dp = G @ V.t().contiguous()
            delta = (G * o).sum(1, keepdim=True)
            ds = p * (dp - delta) * scale
            o_abs = p @ V.abs()
            ds_abs = p * (G.abs() @ V.abs().t().contiguous() + (G.abs() * o_abs).sum(1, keepdim=True)) * abs(scale)
            r["out"][n, :qn, j], r["out_abs"][n, :qn, j] = o, o_abs
            r["lse"][n, j, :qn] = lse
            r["dq"][n, :qn, j], r["dq_abs"][n, :qn, j] = ds @ K, ds_abs @ K.abs()
            r["dv"][n, :kn, c] += p.t().contiguous() @ G
            r["dv_abs"][n, :kn, c] += p.t().contiguous() @ G.abs()
            r["dk"][n, :kn, c] += ds.t().contiguous() @ Q
            r["dk_abs"][n, :kn, c] += ds_abs.t().contiguous() @ Q.abs()
            r["smax"] = max(r["smax"], float((Q.abs() @ K.abs().t().contiguous()).max()) * abs(scale))
    return r


def _check(a, ref, dtype, d, terms):
    r = 2 * d * U * ref["smax"] + 16 * U
    exact = (terms + 16) * U + r
    op = 2.0 ** -8 if dtype == "bf16" else 0.0
    seen = ref["lse"] > -math.inf
    assert torch.equal(a.lse == -math.inf, ~seen)
    assert (a.lse.double() - ref["lse"])[seen].abs().le(r + 16 * U * (1 + ref["lse"][seen].abs())).all()
    for n, roundings in (("out", 2), ("dv", 2), ("dq", 3), ("dk", 3)):
        got = getattr(a, n).double()
        bound = (exact * (1 if n in ("out", "dv") else 3) + roundings * op) * ref[n + "_abs"] + 1e-36
        assert (got - ref[n]).abs().le(bound).all(), (n, float(((got - ref[n]).abs() / bound).max()))


def _run(q, k, v, do, dtype, causal=False, scale=None, q_lens=None, kv_lens=None):
    from paper_2409_09083_amd import tokens
    b, ql, h, d = q.shape
    a = tokens.Attention(b, h, k.shape[2], ql, k.shape[1], d, dtype, causal=causal, scale=scale)
    for t in (a.out, a.dq, a.dk, a.dv, a.lse):
        t.fill_(math.nan)                                       # everything has to be written
    a.forward(q, k, v, q_lens, kv_lens)
    a.backward(do, q, k, v, q_lens, kv_lens)
    torch.cuda.synchronize()
    return a


def _both(shape, dtype, causal=False, scale=None, q_lens=None, kv_lens=None, seed=0):
    b, h, kv, ql, kl, d = shape
    q, k, v, do = _make(b, h, kv, ql, kl, d, dtype, seed)
    lens = [None if n is None else torch.tensor(n, dtype=torch.int32, device="cuda") for n in (q_lens, kv_lens)]
    a = _run(q, k, v, do, dtype, causal, scale, *lens)
    ref = _reference(q, k, v, do, causal, d ** -0.5 if scale is None else scale, q_lens, kv_lens)
    _check(a, ref, dtype, d, max(kl, ql * (h // kv)))
    return a, (q, k, v, do)


# lengths around the tiles of 32 and 64 keys, the blocks of 128 rows and keys; one token; shared heads
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1, 8), (2, 2, 1, 1, 70, 64), (1, 4, 4, 31, 33, 32), (2, 6, 2, 64, 64, 128), (1, 2, 2, 65, 129, 40),
                                   (1, 8, 1, 17, 300, 64), (2, 3, 3, 257, 257, 16), (1, 5, 1, 128, 64, 96), (1, 2, 1, 200, 513, 128), (3, 2, 2, 5, 1, 24)])
def test_lengths_heads_and_sizes(shape, causal, dtype):
    _both(shape, dtype, causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 2, 7, 8, 24, 33, 63, 72, 120, 127])
def test_head_sizes(d, dtype):
    _both((1, 2, 1, 70, 90, d), dtype, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_ragged_lengths_and_rows_that_see_nothing(causal, dtype):
    """Lengths of 0 and 1, lengths outside the tensors (cut), more queries than keys (the first ones see nothing when causal)."""
    _both((8, 4, 2, 150, 130, 64), dtype, causal, q_lens=[150, 0, 1, 97, 140, 9, 500, -3], kv_lens=[130, 60, 1, 128, 0, 70, 900, 20])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ql,kl,group", [(1, 4000, 1), (1, 4000, 8), (3, 1500, 4), (1, 700, 40)])
def test_few_queries_of_a_long_cache(ql, kl, group, dtype):
    """The keys are split over workgroups; ragged, so that some splits are empty."""
    _both((3, 2 * group, 2, ql, kl, 64), dtype, True, q_lens=[ql, ql, 1], kv_lens=[kl, 65, kl - 129])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_keys_of_many_queries(dtype):
    """The rows are split in the gradients of keys and values."""
    _both((1, 4, 1, 900, 20, 32), dtype)
    _both((1, 2, 2, 1500, 100, 64), dtype)


# enough of them that a workgroup takes 128 rows, a wavefront each: bfloats with heads of up to 64 and of up to 128
@pytest.mark.parametrize("shape,causal", [((40, 20, 20, 70, 130, 64), True), ((40, 20, 20, 129, 33, 40), True), ((20, 20, 20, 100, 65, 31), False),
                                          ((20, 20, 20, 70, 100, 128), False), ((20, 40, 20, 65, 97, 100), True)])
def test_many_images_and_heads(shape, causal):
    b, ql, kl = shape[0], shape[3], shape[4]
    _both(shape, "bf16", causal, q_lens=[(17 * n) % (ql + 1) for n in range(b)], kv_lens=[kl - (13 * n) % (kl + 1) for n in range(b)])


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("images", [1, 800])
def test_hidden_values_in_either_half_of_a_tile(images, bad):
    """Key and value 40 or 70 (the second 32 of their tile of 64, the first of the next): the queries before them are as without."""
    q, k, v, do = _make(images, 1, 1, 80, 80, 64, "bf16")
    want = _run(q, k, v, do, "bf16", True)
    for at in (40, 70):
        k2, v2 = k.clone(), v.clone()
        k2[0, at, 0], v2[0, at, 0, 1] = bad, bad
        got = _run(q, k2, v2, do, "bf16", True)
        for x, y in ((got.out, want.out), (got.dq, want.dq)):
            assert (x[0, :at] - y[0, :at]).abs().max() <= 3e-2 * y[0, :at].abs().max()
            assert torch.equal(x[1:], y[1:])
        assert not got.out[0, at:].isfinite().all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_hidden_values_of_wide_heads(bad):
    """fp32 heads of 128: the gradients of a key's first and last 64 channels are two wavefronts' work."""
    q, k, v, do = _make(1, 2, 1, 90, 90, 100, "f32")
    want = _run(q, k, v, do, "f32", True)
    for c in (3, 97):
        do2 = do.clone()
        do2[0, 40, 1, c] = bad                                  # seen by the keys up to 40
        got = _run(q, k, v, do2, "f32", True)
        for t in ("dk", "dv"):
            x, y = getattr(got, t)[0, 41:], getattr(want, t)[0, 41:]
            assert (x - y).abs().max() <= 1e-5 * y.abs().max(), t
        assert not got.dv[0, :41, :, c].isfinite().any()
        k2, v2 = k.clone(), v.clone()
        k2[0, 70, 0, c], v2[0, 70, 0, c] = bad, bad             # only the queries from 70 on see them
        got = _run(q, k2, v2, do, "f32", True)
        for t in ("out", "dq"):
            x, y = getattr(got, t)[0, :70], getattr(want, t)[0, :70]
            assert (x - y).abs().max() <= 1e-5 * y.abs().max(), t


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.0])
def test_other_scales(scale):
    _both((1, 2, 2, 70, 70, 32), "f32", True, scale=scale)
    _both((1, 2, 2, 70, 70, 32), "bf16", True, scale=scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    """Slices of one projection, a cache with room behind its tokens, heads before tokens, an odd address, broadcast keys and dout."""
    d, h, kv, b, n = 64, 4, 2, 2, 90
    q, k, v, do = _make(b, h, kv, n, n, d, dtype)
    want = _run(q, k, v, do, dtype, True)
    packed = torch.cat([q, k, v], 2)
    a = _run(packed[:, :, :h], packed[:, :, h:h + kv], packed[:, :, h + kv:], do, dtype, True)
    cache = torch.full((b, kv, 500, d), math.nan, dtype=TYPES[dtype], device="cuda")
    cache[:, :, :n] = k.transpose(1, 2)
    first = torch.empty((b, h, n, d), dtype=TYPES[dtype], device="cuda").copy_(q.transpose(1, 2)).transpose(1, 2)
    c = _run(first, cache[:, :, :n].transpose(1, 2), v, do, dtype, True)
    odd = torch.zeros(do.numel() + 1, dtype=TYPES[dtype], device="cuda")[1:].view(do.shape)
    odd.copy_(do)
    e = _run(q, k, v, odd, dtype, True)
    for t in ("out", "lse", "dq", "dk", "dv"):
        for x in (a, c, e):
            assert torch.equal(getattr(x, t), getattr(want, t)), t
    k1, do1 = k[:1].expand(b, n, kv, d), do[:, :1].expand(b, n, h, d)
    f = _run(q, k1, v, do1, dtype, True)
    g = _run(q, k1.contiguous(), v, do1.contiguous(), dtype, True)
    for t in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(f, t), getattr(g, t)), t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_hidden_values_reach_nothing(bad, dtype):
    """What lies past the lengths, in keys, values, queries and dout, and what a causal query does not see."""
    b, h, kv, n, d = 2, 4, 2, 150, 64
    q, k, v, do = _make(b, h, kv, n, n, d, dtype)
    lens = torch.tensor([97, 150], dtype=torch.int32, device="cuda")
    want = _run(q, k, v, do, dtype, True, q_lens=lens, kv_lens=lens)
    for t in (q, k, v, do):
        t[0, 97:] = bad
    got = _run(q, k, v, do, dtype, True, q_lens=lens, kv_lens=lens)
    for t in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(got, t), getattr(want, t)), t
    # the last key and value of image 1: only the last query sees them
    k2, v2 = k.clone(), v.clone()
    k2[1, -1, 0], v2[1, -1, 1] = bad, bad
    got = _run(q, k2, v2, do, dtype, True, q_lens=lens, kv_lens=lens)
    tol = 1e-5 if dtype == "f32" else 3e-2
    for t in ("out", "dq"):
        x, y = getattr(got, t)[1, :-1], getattr(want, t)[1, :-1]
        assert x.isfinite().all() and (x - y).abs().max() <= tol * y.abs().max(), t
    assert not got.out[1, -1].isfinite().all()
    # the first query's dout: it reaches the first key alone
    do2 = do.clone()
    do2[1, 0] = bad
    got = _run(q, k, v, do2, dtype, True, q_lens=lens, kv_lens=lens)
    for t in ("dk", "dv"):
        x, y = getattr(got, t)[1, 1:], getattr(want, t)[1, 1:]
        assert x.isfinite().all() and (x - y).abs().max() <= tol * y.abs().max(), t
    assert not got.dv[1, 0].isfinite().any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(dtype):
    """One key far above the others, scores beyond the exponential's range either way: finite, and the one key's value."""
    q, k, v, do = _make(1, 1, 1, 40, 80, 64, dtype)
    q.fill_(8.0)
    k.fill_(-8.0)
    k[0, 50] = 8.0
    a = _run(q, k, v, do, dtype, scale=1.0)                     # scores -4096 and 4096
    assert torch.equal(a.out, v[:, 50:51].expand_as(a.out)) and a.lse.eq(4096).all()
    assert a.dq.abs().max() <= 1e-3 and a.dk.abs().max() <= 1e-3
    want = do.double().sum(1)[0, 0]
    assert (a.dv[0, 50, 0].double() - want).abs().le(2.0 ** -8 * want.abs() + 1e-5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,causal,lens", [((2, 4, 2, 1, 1, 64), True, None), ((1, 2, 1, 70, 1, 40), False, None), ((2, 6, 2, 90, 90, 64), True, None),
                                               ((2, 2, 2, 60, 50, 128), True, None), ((3, 4, 1, 33, 500, 32), False, [1, 500, 1]),
                                               ((1, 80, 1, 3, 3, 16), True, None), ((1, 2, 2, 1500, 1, 64), True, None)])
def test_rows_that_see_one_key(shape, causal, lens, dtype):
    """Probability 1 whatever the score: dq exactly 0, nothing of them in dk, their dout in dv."""
    a, (q, k, v, do) = _both(shape, dtype, causal, kv_lens=lens)
    b, h, kv, ql, kl, d = shape
    for n in range(b):
        kn = kl if lens is None else lens[n]
        seen = [min(max(i + kn - ql + 1, 0), kn) if causal else kn for i in range(ql)]
        one = [i for i in range(ql) if seen[i] == 1]
        assert a.dq[n, one].abs().sum() == 0
        if kn == 1:
            assert a.dk[n].abs().sum() == 0


def test_gradient_by_differences():
    """Against central differences in 64 bits, with shared heads."""
    q, k, v, do = _make(1, 4, 2, 9, 12, 16, "f32")
    a = _run(q, k, v, do, "f32", True)

    def loss(q, k, v):
        k, v = (t.repeat_interleave(2, 2).transpose(1, 2) for t in (k, v))
        s = q.transpose(1, 2) @ k.transpose(2, 3).contiguous() / 4
        hide = torch.arange(12, device="cuda")[None] > torch.arange(9, device="cuda")[:, None] + 3
        return float((torch.softmax(s.masked_fill(hide, -math.inf), 3) @ v.contiguous() * do.double().transpose(1, 2)).sum())
    base = [t.double() for t in (q, k, v)]
    for which, got in enumerate((a.dq, a.dk, a.dv)):
        for at in ((0, 0, 0, 0), (0, 5, 1, 3), (0, 8, 1, 15)):
            step = torch.zeros_like(base[which])
            step[at] = 1e-5
            ends = []
            for sign in (1, -1):
                t = list(base)
                t[which] = t[which] + sign * step
                ends.append(loss(*t))
            want = (ends[0] - ends[1]) / 2e-5
            assert abs(float(got[at]) - want) <= 2e-5 * (1 + abs(want))


def test_equal_bits_empty_calls_and_refusals():
    from paper_2409_09083_amd import binding as B
    from paper_2409_09083_amd import tokens
    for shape in ((2, 8, 2, 333, 500, 64), (1, 2, 1, 1, 3000, 128)):
        a, (q, k, v, do) = _both(shape, "bf16", True)
        c = _run(q, k, v, do, "bf16", True)
        for t in ("out", "lse", "dq", "dk", "dv"):
            assert torch.equal(getattr(a, t), getattr(c, t))
    for ql, kl in ((0, 5), (5, 0), (0, 0)):
        q, k, v, do = _make(2, 2, 1, ql, kl, 32, "f32")
        a = _run(q, k, v, do, "f32")
        assert all(float(t.abs().sum()) == 0 for t in (a.out, a.dq, a.dk, a.dv))
    for bad in (dict(heads=3, kv_heads=2), dict(head_dim=136), dict(head_dim=0), dict(q_len=-1)):
        args = dict(batch=1, heads=2, kv_heads=2, q_len=4, kv_len=4, head_dim=32)
        args.update(bad)
        with pytest.raises(B.FtpError):
            tokens.Attention(**args, dtype="f32")
    a = tokens.Attention(1, 2, 2, 4, 4, 32, "f32", training=False)
    q, k, v, do = _make(1, 2, 2, 4, 4, 32, "f32")
    with pytest.raises(ValueError):
        a.forward(q, k[:, :3], v)
    with pytest.raises(ValueError):
        a.forward(q.transpose(2, 3).contiguous().transpose(2, 3), k, v)
    with pytest.raises(TypeError):
        a.forward(q, k, v.bfloat16())
    with pytest.raises(TypeError):
        a.forward(q, k, v, kv_lens=torch.tensor([4], device="cuda"))
    with pytest.raises(ValueError):
        a.backward(do, q, k, v)


def test_graph_replays():
    """One token against a growing cache: the lengths change on the device between the replays."""
    from paper_2409_09083_amd import tokens
    q, k, v, _ = _make(2, 8, 2, 1, 1000, 64, "bf16")
    lens = torch.tensor([10, 300], dtype=torch.int32, device="cuda")
    a = tokens.Attention(2, 8, 2, 1, 1000, 64, "bf16", causal=True, training=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.forward(q, k, v, kv_lens=lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.forward(q, k, v, kv_lens=lens)
    for step in range(3):
        lens += 123
        q.copy_(torch.randn_like(q))
        graph.replay()
        torch.cuda.synchronize()
        got = a.out.clone()
        a.forward(q, k, v, kv_lens=lens)
        assert torch.equal(a.out, got)
