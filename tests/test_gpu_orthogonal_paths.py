"""Orthogonal updates on each of the ways that a size may take: all steps in one launch (a side of at most 64, the other at most 256; one, two or four blocks of 64), a launch a step (longer ones, where their blocks
are few, or many and long; several blocks a workgroup above 2048), three products a step (the others).  What the header promises holds on all of them.  Bounds as in test_gpu_orthogonal.py."""
import math
import os
import re

import pytest
import torch

from tests.test_gpu_orthogonal import ABC, HELD, LAST, TYPES, U, _matrix, _one_step_bound, _steps

pytestmark = pytest.mark.gpu
ONE = [(40, 50), (64, 128), (117, 33), (50, 190), (64, 256), (256, 64), (193, 64)]
EACH = [(64, 257), (576, 50), (64, 2049), (4608, 64), (20, 9000)]
GENERAL = [(65, 65), (133, 307), (307, 133), (640, 200)]
PATHS = [(40, 70), (64, 256), (256, 60), (64, 576), (576, 50), (33, 2500), (133, 307), (307, 133)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", ONE + EACH + GENERAL + [(32768, 64), (7, 32768)])
def test_one_step(rows, cols, dtype):
    from paper_2409_09083_amd import orthogonal
    x = _matrix(2, rows, cols, dtype, seed=21)
    got = orthogonal.Orthogonal(rows, cols, dtype, count=2, steps=1).forward(x)
    for m in range(2):
        want, tol = _steps(x[m], 1), _one_step_bound(x[m], dtype)
        assert ((got[m].double() - want).abs() <= tol + LAST[dtype] * (want.abs() + tol) + 1e-37).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", ONE + EACH + GENERAL)
def test_several_steps(rows, cols, dtype):
    from paper_2409_09083_amd import orthogonal
    x = _matrix(2, rows, cols, dtype, seed=22)
    h = HELD[dtype]
    for steps in (2, 5):
        o = orthogonal.Orthogonal(rows, cols, dtype, count=2, steps=steps)
        got = o.forward(x).clone()
        o._ws.fill_(255)                                        # scratch need not be cleared
        assert torch.equal(o.forward(x), got)
        for m in range(2):
            g = torch.Generator(device="cuda").manual_seed(m)

            def some(v):
                return 2 * torch.rand(v.shape, generator=g, device="cuda", dtype=torch.float64) - 1

            def noise(v, k=0, size=None):
                if size is not None:
                    v = v + some(v) * (math.sqrt(k) * U + 2 * h) * size
                return v * (1 + (h + U) * some(v))
            want = _steps(x[m], steps)
            off = max(float((_steps(x[m], steps, noise=noise) - want).norm()) for _ in range(3))
            assert float((got[m].double() - want).norm()) <= 8 * off + LAST[dtype] * float(want.norm())


# a launch a step: few blocks in all, up to three a workgroup; many and long, 6 and 16 a workgroup.  Beside them those that go as three products instead
NUMBERS = [(1, 64, 4608), (1, 6144, 64), (1, 64, 6145), (2, 30, 3072), (2, 3073, 64), (16, 64, 384), (17, 64, 384), (22, 64, 12000), (21, 64, 12000), (8, 32768, 50), (7, 32768, 50)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,rows,cols", NUMBERS)
def test_numbers_of_matrices_where_the_way_turns(count, rows, cols, dtype):
    from paper_2409_09083_amd import orthogonal
    x = _matrix(count, rows, cols, dtype, seed=26)
    one = orthogonal.Orthogonal(rows, cols, dtype, count=count, steps=1).forward(x).clone()
    o = orthogonal.Orthogonal(rows, cols, dtype, count=count)
    got = o.forward(x).clone()
    o._ws.fill_(255)
    assert torch.equal(o.forward(x), got)
    x[count - 1, 3, 5] = math.nan
    o._ws.fill_(255)
    bad = o.forward(x)
    assert bad[count - 1].isnan().all() and (count == 1 or torch.equal(bad[:-1], got[:-1]))
    for m in sorted({0, (count - 1) // 2, max(count - 2, 0)}):
        y = _matrix(count, rows, cols, dtype, seed=26)[m]
        want, tol = _steps(y, 1), _one_step_bound(y, dtype)
        assert ((one[m].double() - want).abs() <= tol + LAST[dtype] * (want.abs() + tol) + 1e-37).all()
        h, g = HELD[dtype], torch.Generator(device="cuda").manual_seed(m)

        def some(v):
            return 2 * torch.rand(v.shape, generator=g, device="cuda", dtype=torch.float64) - 1

        def noise(v, k=0, size=None):
            if size is not None:
                v = v + some(v) * (math.sqrt(k) * U + 2 * h) * size
            return v * (1 + (h + U) * some(v))
        want = _steps(y, 5)
        off = max(float((_steps(y, 5, noise=noise) - want).norm()) for _ in range(3))
        assert float((got[m].double() - want).norm()) <= 8 * off + LAST[dtype] * float(want.norm())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", PATHS)
def test_special_matrices(rows, cols, dtype):
    """A zero matrix, one with a NaN, one with an infinity among others of a call; scales whose squares 32 bits do not hold."""
    from paper_2409_09083_amd import orthogonal
    x = _matrix(5, rows, cols, dtype, seed=23)
    o = orthogonal.Orthogonal(rows, cols, dtype, count=5)
    want = o.forward(x).clone()
    x[1] = 0
    x[2, rows - 1, cols // 2] = math.nan
    x[3, 0, cols - 1] = -math.inf
    got = o.forward(x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[4], want[4]) and not got[1].any() and got[2].isnan().all() and got[3].isnan().all()
    one = orthogonal.Orthogonal(rows, cols, dtype, eps=0.0)
    y = _matrix(1, rows, cols, dtype, seed=24)[0]
    want = one.forward(y).clone()
    for scale in (2.0 ** 100, 2.0 ** -90):
        assert torch.equal(one.forward(y * scale), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", PATHS)
def test_strides_in_place_and_graph(rows, cols, dtype):
    from paper_2409_09083_amd import binding as B
    from paper_2409_09083_amd import orthogonal
    x = _matrix(3, rows, cols, dtype, seed=25)
    o = orthogonal.Orthogonal(rows, cols, dtype, count=3)
    want = o.forward(x).clone()
    around = torch.full((3 * (rows + 3) * (cols + 7) + 1,), math.nan, dtype=x.dtype, device="cuda")
    v = around[1:].view(3, rows + 3, cols + 7)[:, :rows, :cols]
    v.copy_(x)
    assert torch.equal(o.forward(v), want)
    assert torch.equal(o.forward(x[1:2].expand(3, rows, cols))[2], want[1])
    same = x[:, :1].expand(3, rows, cols)                       # all rows of a matrix one row of memory
    assert torch.equal(o.forward(same).clone(), o.forward(same.contiguous()))
    y = x.clone()
    B.ftp_orthogonal(o.desc, y.data_ptr(), y.data_ptr(), o._ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert torch.equal(y, want)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o.forward(x)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        o.forward(x)
    for k in range(4):
        x.copy_(_matrix(3, rows, cols, dtype, seed=30 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = o.out.clone()
        assert torch.equal(o.forward(x), got)
        torch.cuda.synchronize()


def _promise():
    """The header's words on where singular values end: (smallest share of |x|, least, most)."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "include", "ftp.h")) as f:
        return tuple(map(float, re.search(r"singular values from ([\d.]+) of \|x\| on end between ([\d.]+) and ([\d.]+)\.\s", f.read()).groups()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(40, 70), (64, 576), (133, 307), (307, 133)])
def test_singular_values_at_the_stated_limit(rows, cols, dtype):
    """One entry a row and column: the singular values are those, down to the smallest number of the type that is not below the limit."""
    from paper_2409_09083_amd import orthogonal
    limit, least, most = _promise()
    n = min(rows, cols)
    values = torch.logspace(0, -2, n, dtype=torch.float64).to(TYPES[dtype])
    values[-1] = 0
    low = (limit * values.double().norm() / math.sqrt(1 - limit ** 2)).to(TYPES[dtype])
    while float(low) < limit * float(torch.cat((values.double(), low.double()[None])).norm()):
        low = torch.nextafter(low, torch.tensor(1.0, dtype=TYPES[dtype]))
    values[-1] = low
    g = torch.Generator().manual_seed(4)
    at, to = torch.randperm(rows, generator=g)[:n], torch.randperm(cols, generator=g)[:n]
    x = torch.zeros((rows, cols), dtype=TYPES[dtype])
    x[at, to] = values
    got = orthogonal.Orthogonal(rows, cols, dtype).forward(x.cuda()).double().cpu()
    ends = got[at, to]
    rest = got.clone()
    rest[at, to] = 0
    assert not rest.any() and least <= float(ends.min()) and float(ends.max()) <= most
    # and the limit is one: what the polynomial makes of it and of a tenth less
    a, b, c = ABC

    def end(v):
        for _ in range(5):
            v = a * v + b * v ** 3 + c * v ** 5
        return v
    assert least <= end(limit) and min(end(limit * 10 ** (k / 1000)) for k in range(2853)) >= least > end(0.9 * limit)
