"""Causal attention where what a query does not see holds the type's largest numbers, infinities or NaN."""
import math

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


def _times(call, n):
    call()
    torch.cuda.synchronize()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        call()
    b.record()
    b.synchronize()
    return a.elapsed_time(b) / n


@pytest.mark.parametrize("what", ["all", "keys and values", "one channel of the values", "query 500's dout"])
def test_time_where_numbers_are_not_finite(what):
    """A call on NaN takes a bounded multiple of one on numbers: one more walk over the tiles at most, and up to 192 keys (queries) of a row (key) that some of its neighbours do not see, one by
    one: 5 products of 64 channels each, about 50 cycles a channel, 3 million cycles or 1.5 ms; 1024 workgroups are two to a CU, in two rounds: 3 ms a kernel.  One kernel
    forward, two backward; and 2.5 times the finite call."""
    from paper_2409_09083_amd import tokens
    q, k, v, do = A._make(4, 4, 4, 4096, 4096, 64, "bf16")
    a = tokens.Attention(4, 4, 4, 4096, 4096, 64, "bf16", causal=True)
    forward, backward = _times(lambda: a.forward(q, k, v), 5), _times(lambda: a.backward(do, q, k, v), 5)
    if what == "query 500's dout":
        do[:, 500] = math.nan
    else:
        for t in (q, k, v, do)[slice(0, 4) if what == "all" else slice(1, 3) if what == "keys and values" else slice(2, 3)]:
            if what == "one channel of the values":
                t[..., 7] = math.nan
            else:
                t.fill_(math.nan)
    f2, b2 = _times(lambda: a.forward(q, k, v), 1), _times(lambda: a.backward(do, q, k, v), 1)
    print(what, forward, f2, backward, b2)
    assert f2 <= 2.5 * forward + 3 and b2 <= 2.5 * backward + 6


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("shape", [(1, 2, 2, 400, 400, 64), (2, 6, 2, 333, 333, 128), (300, 2, 1, 150, 150, 32), (1, 1, 1, 300, 700, 40), (1, 2, 1, 500, 300, 64)])
def test_one_bad_token_in_the_middle(shape, bad, dtype):
    """Queries before it and keys behind it are as without it; queries behind it have its value's channel spoiled and the others right."""
    b, h, kv, ql, kl, d = shape
    q, k, v, do = A._make(*shape, dtype)
    want = A._run(q, k, v, do, dtype, True)
    at = kl // 2
    first = max(0, at - (kl - ql))                              # the first query that sees key `at`
    tol = 2e-5 if dtype == "f32" else 3e-2

    def near(x, y):
        return x.numel() == 0 or (x.isfinite().all() and (x - y).abs().max() <= tol * y.abs().max())
    v2 = v.clone()
    v2[:, at, :, 3] = bad
    got = A._run(q, k, v2, do, dtype, True)
    others = [c for c in range(d) if c != 3]
    assert near(got.out[:, :first], want.out[:, :first])
    assert near(got.out[:, first:][..., others], want.out[:, first:][..., others])
    assert not got.out[:, first:, :, 3].isfinite().any()
    assert torch.equal(got.lse, want.lse)
    assert near(got.dq[:, :first], want.dq[:, :first])
    assert not got.dq[:, first + 1:].isfinite().any()
    k2 = k.clone()
    k2[:, at, :, 3] = math.nan
    got = A._run(q, k2, v, do, dtype, True)
    assert near(got.out[:, :first], want.out[:, :first]) and not got.out[:, first:].isfinite().any()
    do2, q2 = do.clone(), q.clone()
    do2[:, first + 9] = bad
    q2[:, first + 9] = math.nan
    last = first + 9 + kl - ql                                  # the last key that this query sees
    for got in (A._run(q, k, v, do2, dtype, True), A._run(q2, k, v, do, dtype, True)):
        for t in ("dk", "dv"):
            assert near(getattr(got, t)[:, last + 1:], getattr(want, t)[:, last + 1:]), t
        assert not got.dv[:, :last + 1].isfinite().any()
        assert torch.equal(got.dq[:, :first + 9], want.dq[:, :first + 9]) and torch.equal(got.dq[:, first + 10:], want.dq[:, first + 10:])


@pytest.mark.parametrize("c", [3, 97])
@pytest.mark.parametrize("shape", [(8, 8, 8, 300, 300, 128), (4, 12, 4, 260, 260, 100)])
def test_one_channel_of_wide_fp32_heads(shape, c):
    """Gradients of a key's first and last 64 channels are two wavefronts' work, of which one bad channel of a query or of its dout spoils one: the scores are both's all the same."""
    q, k, v, do = A._make(*shape, "f32")
    want = A._run(q, k, v, do, "f32", True)
    for which in ("dout", "query"):
        q2, do2 = q.clone(), do.clone()
        (do2 if which == "dout" else q2)[:, 70, ::2, c] = math.nan
        got = A._run(q2, k, v, do2, "f32", True)
        for t in ("dk", "dv"):
            x, y = getattr(got, t)[:, 71:], getattr(want, t)[:, 71:]
            assert x.isfinite().all() and (x - y).abs().max() <= 2e-5 * y.abs().max(), (which, t)


# (rows split over workgroups in the last one's dq, keys' gradients of many rows in the one before)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,causal", [((2, 4, 2, 90, 90, 64), True), ((1, 2, 2, 60, 50, 128), True), ((2, 2, 1, 70, 1, 40), False), ((1, 2, 2, 1500, 1, 64), False),
                                          ((1, 2, 2, 40, 1500, 32), True)])
def test_one_key_of_a_score_that_is_not_finite(shape, causal, dtype):
    """A query that sees one key: probability 1 whatever the score, but NaN if it is none, forward and backward."""
    b, h, kv, ql, kl, d = shape
    q, k, v, do = A._make(*shape, dtype)
    lens = torch.tensor([ql] * b, dtype=torch.int32, device="cuda"), torch.tensor([1 if kl == 1500 else kl] * b, dtype=torch.int32, device="cuda")
    want = A._run(q, k, v, do, dtype, causal, None, *lens)
    row = max(0, ql - int(lens[1][0])) if causal else 7         # (the first one that sees a key; not causal: any)
    for bad in (math.nan, math.inf):
        q2 = q.clone()
        q2[:, row, 0, 3] = bad
        got = A._run(q2, k, v, do, dtype, causal, None, *lens)
        for t in ("out", "dq"):
            x, y = getattr(got, t), getattr(want, t)
            assert x[:, row, 0].isnan().all(), t
            assert torch.equal(x[:, row, 1:], y[:, row, 1:]) and torch.equal(x[:, :row], y[:, :row]) and torch.equal(x[:, row + 1:], y[:, row + 1:]), t
        for t in ("dk", "dv"):
            x, y = getattr(got, t), getattr(want, t)
            assert x[:, 0, 0].isnan().all() and torch.equal(x[:, 0, 1:], y[:, 0, 1:]), t
            assert x[:, 1:].isfinite().all() and (x[:, 1:] - y[:, 1:]).abs().sum() <= 0.03 * y[:, 1:].abs().sum(), t


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(2, 3, 1, 50, 50, 64), (1, 2, 2, 200, 300, 128), (40, 6, 6, 100, 90, 40)])
def test_bfloat_keys_at_minus_infinity(shape, causal):
    """A key whose scores all are -infinity has probability 0: it is as a key that nobody sees, its own gradients 0 (lengths and groups leave rows of tiles empty)."""
    b, h, kv, ql, kl, d = shape
    q, k, v, do = A._make(*shape, "bf16")
    q[..., 5] = q[..., 5].abs() + 0.5
    lens = torch.tensor([ql - 7] * b, dtype=torch.int32, device="cuda"), torch.tensor([kl - 3] * b, dtype=torch.int32, device="cuda")
    far = k.clone()
    far[:, 10, :, 5] = -1e30                                    # (as good as -infinity)
    want = A._run(q, far, v, do, "bf16", causal, None, *lens)
    k[:, 10, :, 5] = -math.inf
    got = A._run(q, k, v, do, "bf16", causal, None, *lens)
    for t in ("out", "lse"):
        assert torch.equal(getattr(got, t), getattr(want, t)), t
    assert torch.equal(got.dv, want.dv)
    others = [j for j in range(kl) if j != 10]
    assert torch.equal(got.dk[:, others], want.dk[:, others]) and (got.dk[:, 10] == 0).all()
