"""Embedding rows and their gradient against the formulas in 64 bits.

Bounds: the forward pass is one product rounded to fp32 and then to the type, as torch's.  The backward pass adds n rows in some fixed order and multiplies by the
scale: (n + 1) 2^-24 sum|terms|."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _ids(rows, vocab, how, dtype=torch.int64, seed=0):
    g = torch.Generator().manual_seed(seed)
    if how == "one":
        ids = torch.full((rows,), vocab - 1)
    elif how == "none":
        ids = torch.full((rows,), -1)
    elif how == "skewed":
        ids = (torch.rand(rows, generator=g) ** 4 * vocab).long().clamp(max=vocab - 1)
        ids[torch.rand(rows, generator=g) < 0.2] = -1
        ids[torch.rand(rows, generator=g) < 0.05] = vocab
    else:
        ids = torch.randint(0, vocab, (rows,), generator=g)
    return ids.to(dtype).cuda()


def _normal(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(TYPES[dtype]).cuda()


def _backward64(ids, dy, vocab, scale):
    there = (ids >= 0) & (ids < vocab)
    want = torch.zeros((vocab, dy.shape[1]), dtype=torch.float64, device="cuda")
    sums = torch.zeros_like(want)
    n = torch.zeros(vocab, dtype=torch.float64, device="cuda")
    want.index_add_(0, ids[there].long(), dy[there].double() * scale)
    sums.index_add_(0, ids[there].long(), dy[there].double().abs() * abs(scale))
    n.index_add_(0, ids[there].long(), torch.ones(int(there.sum()), dtype=torch.float64, device="cuda"))
    return want, (n[:, None] + 1) * 2.0 ** -24 * sums


SIZES = [(1, 1, 1), (3, 7, 5), (31, 2, 8), (32, 40, 64), (33, 1, 250), (64, 300, 16), (1000, 255, 96), (1025, 256, 33), (4995, 1001, 250), (2049, 65536, 40), (5000, 70000, 8), (700, 90, 1100)]


@pytest.mark.parametrize("how", ["skewed", "one"])
@pytest.mark.parametrize("rows", [8192, 8193, 32768, 32769])
def test_gradient_around_changes_of_plan(rows, how):
    """Where the list leaves one workgroup's LDS, and where its pieces become longer."""
    from paper_2409_09083_amd import vocabulary
    ids, dy = _ids(rows, 1500, how, torch.int64), _normal((rows, 40), "bf16", 3)
    e = vocabulary.Embedding(rows, 1500, 40, "bf16", scale=1.7)
    got = e.backward(ids, dy)
    want, tol = _backward64(ids, dy, 1500, torch.tensor(1.7).double().item())
    assert ((got.double() - want).abs() <= tol * 1.01 + 1e-7 * want.abs()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["any", "skewed", "one", "none"])
@pytest.mark.parametrize("rows,vocab,channels", SIZES)
def test_both_passes(rows, vocab, channels, how, dtype):
    from paper_2409_09083_amd import vocabulary
    ids = _ids(rows, vocab, how, torch.int32 if rows % 2 else torch.int64)
    table, dy = _normal((vocab, channels), dtype, 1), _normal((rows, channels), dtype, 2)
    e = vocabulary.Embedding(rows, vocab, channels, dtype, scale=1.7)
    got = e.forward(ids, table)
    there = (ids >= 0) & (ids < vocab)
    want = (table[torch.where(there, ids, 0).long()].float() * 1.7).to(TYPES[dtype])
    assert torch.equal(got, torch.where(there[:, None], want, torch.zeros_like(want)))
    e.dtable.fill_(math.nan)
    got = e.backward(ids, dy).clone()
    want, tol = _backward64(ids, dy, vocab, torch.tensor(1.7).double().item())
    assert ((got.double() - want).abs() <= tol * 1.01 + 1e-7 * want.abs()).all()
    e._ws.fill_(255)
    assert torch.equal(e.backward(ids, dy), got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_of_few_ids(dtype):
    """Runs over many pieces, several workgroups of the sort, three passes of it."""
    from paper_2409_09083_amd import vocabulary
    for rows, vocab, how in ((70000, 3, "any"), (40000, 200000, "skewed"), (300000, 17, "skewed")):
        ids, dy = _ids(rows, vocab, how), _normal((rows, 24), dtype, 3)
        e = vocabulary.Embedding(rows, vocab, 24, dtype)
        want, tol = _backward64(ids, dy, vocab, 1.0)
        assert ((e.backward(ids, dy).double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(3, 1), (8, 0)])
def test_rows_inside_wider_ones(pad, offset, dtype):
    from paper_2409_09083_amd import vocabulary
    rows, vocab, c = 77, 50, 36
    t = TYPES[dtype]

    def wide(x):
        w = torch.full((x.shape[0] * (c + pad) + offset,), math.nan, dtype=t, device="cuda")
        v = w[offset:].view(x.shape[0], c + pad)[:, :c]
        v.copy_(x)
        return w, v
    ids, table, dy = _ids(rows, vocab, "skewed"), _normal((vocab, c), dtype, 4), _normal((rows, c), dtype, 5)
    e = vocabulary.Embedding(rows, vocab, c, dtype, scale=0.25)
    want, grad = e.forward(ids, table).clone(), e.backward(ids, dy).clone()
    around, out = wide(torch.zeros_like(dy))
    assert e.forward(ids, wide(table)[1], out=out) is out and torch.equal(out, want)
    assert around[:offset].isnan().all() and around[offset:].view(rows, c + pad)[:, c:].isnan().all()
    assert torch.equal(e.backward(ids, wide(dy)[1]), grad)
    assert torch.equal(e.backward(ids, dy[:1].expand(rows, c)), e.backward(ids, dy[:1].repeat(rows, 1)))       # a broadcast gradient
    strided = torch.stack((ids, ids), 1)[:, 0]
    with pytest.raises(ValueError):
        e.forward(strided, table)


def test_what_rows_without_an_id_hold_reaches_nothing():
    from paper_2409_09083_amd import vocabulary
    ids = _ids(500, 30, "skewed")
    dy = _normal((500, 20), "f32", 6)
    e = vocabulary.Embedding(500, 30, 20)
    want = e.backward(ids, dy).clone()
    dy[(ids < 0) | (ids >= 30)] = math.nan
    assert torch.equal(e.backward(ids, dy), want)
    dy[ids == 4] = math.inf
    got = e.backward(ids, dy)
    assert got[4].isinf().all() and torch.equal(got[:4], want[:4]) and torch.equal(got[5:], want[5:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_of_more_than_31_bits(dtype):
    """A table of 2.9 billion elements, ids at both ends of it."""
    from paper_2409_09083_amd import vocabulary
    vocab, c = 700000, 4104
    ids = torch.tensor([vocab - 1, 0, vocab - 1, 523300, -1, vocab - 2, 0], device="cuda")
    dy = _normal((7, c), dtype, 1)
    e = vocabulary.Embedding(7, vocab, c, dtype)
    table = torch.empty((vocab, c), dtype=TYPES[dtype], device="cuda")
    for r in (vocab - 1, vocab - 2, 523300, 0):
        table[r] = r % 97
    assert e.forward(ids, table)[:, -1].tolist() == [float((r % 97) if r >= 0 else 0) for r in ids.tolist()]
    del table
    d = e.backward(ids, dy)
    assert sorted(torch.count_nonzero(d, dim=1).nonzero().squeeze(1).tolist()) == [0, 523300, vocab - 2, vocab - 1]
    assert torch.equal(d[vocab - 1], dy[0].float() + dy[2].float()) and torch.equal(d[0], dy[1].float() + dy[6].float()) and torch.equal(d[523300], dy[3].float())


def test_gradient_by_differences():
    from paper_2409_09083_amd import vocabulary
    ids, g = _ids(40, 9, "skewed"), _normal((40, 6), "f32", 7)
    table = _normal((9, 6), "f32", 8)
    e = vocabulary.Embedding(40, 9, 6, scale=2.0)
    got = e.backward(ids, g).double()
    for v, c in ((0, 0), (3, 5), (8, 2)):
        # the output is linear in the table: a difference of 1 is exact but for its 40 products' rounding
        one = table.clone()
        one[v, c] += 1
        up, down = e.forward(ids, one).double().clone(), e.forward(ids, table).double()
        d = ((up - down) * g.double()).sum()
        assert abs(d - got[v, c]) <= 40 * 2.0 ** -22 * (g.double().abs().sum(0)[c] * 4)


def test_empty_refusals_and_graph():
    from paper_2409_09083_amd import vocabulary
    e = vocabulary.Embedding(0, 5, 4)
    none = torch.empty((0,), dtype=torch.int64, device="cuda")
    assert e.forward(none, torch.zeros((5, 4), device="cuda")).shape == (0, 4)
    e.dtable.fill_(1)
    assert float(e.backward(none, torch.empty((0, 4), device="cuda")).abs().max()) == 0
    ids, table, dy = _ids(90, 12, "skewed"), _normal((12, 16), "bf16", 1), _normal((90, 16), "bf16", 2)
    e = vocabulary.Embedding(90, 12, 16, "bf16")
    for bad in (lambda: e.forward(ids.float(), table), lambda: e.forward(ids, table.float()), lambda: e.backward(ids, dy.float())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: e.forward(ids[:-1], table), lambda: e.forward(ids, table[:-1]), lambda: e.forward(ids, table.t().contiguous().t()), lambda: e.forward(ids.cpu(), table),
                lambda: vocabulary.Embedding(90, 12, 16, "bf16", training=False).backward(ids, dy), lambda: e.forward(ids, table, out=table.new_empty((90, 17))),
                lambda: vocabulary.Embedding(90, 12, 16, "f16")):
        with pytest.raises(ValueError):
            bad()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        e.forward(ids, table)
        e.backward(ids, dy)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        e.forward(ids, table)
        e.backward(ids, dy)
    for k in range(4):
        ids.copy_(_ids(90, 12, "any", seed=k))
        dy.copy_(_normal((90, 16), "bf16", 10 + k))
        graph.replay()
        torch.cuda.synchronize()
        out, grad = e.out.clone(), e.dtable.clone()
        assert torch.equal(e.forward(ids, table), out) and torch.equal(e.backward(ids, dy), grad)
        torch.cuda.synchronize()
