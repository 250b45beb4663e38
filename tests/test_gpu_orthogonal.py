"""Newton-Schulz steps against the formula in 64 bits.

Bounds of one step, element by element, u = 2^-24: a number between two products is held to h of itself (three bfloats h = u, two 2^-16), products of such numbers are off by 3 h each beside the sum's
(K + 8) u, whatever its order; the bound follows the formula from X (3 u for the norm and the product with its inverse) over S and Q = a I + b S + c S^2 to the result Q X, each absolute value in the place of its number.

Bound of several steps: such errors go through the steps that follow, by factors that depend on the matrix.  So the formula runs in 64 bits with every held number and every product's result changed by random parts of
that size (uniform within +-h, the sums' by +-sqrt(K) u of their absolute values' sum), which makes an error of the size that the kernel's roundings make; the kernel's norm of the error may be 8 times that, and the type's rounding."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HELD = {"f32": 2.0 ** -24, "bf16": 2.0 ** -16}
LAST = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U = 2.0 ** -24
ABC = (3.4445, -4.775, 2.0315)


def _mm(a, b):
    return a @ b.contiguous()


def _matrix(count, rows, cols, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((count, rows, cols), generator=g) * torch.exp(torch.randn((count, rows, 1), generator=g) * 0.5)
    return (0.01 * x).to(TYPES[dtype]).cuda()


def _wide(x):
    """Its smaller side first: x x^T x = (x^T (x^T)^T x^T)^T."""
    return (x, False) if x.shape[0] <= x.shape[1] else (x.t().contiguous(), True)


def _steps(x, steps, eps=1e-7, abc=ABC, noise=None):
    a, b, c = (torch.tensor(v, dtype=torch.float32).double().item() for v in abc)
    x, turned = _wide(x.double())
    keep = noise or (lambda v, k=0, size=None: v)
    x = keep(x / (torch.linalg.vector_norm(x) + eps))
    for _ in range(steps):
        s = keep(_mm(x, x.t()), x.shape[1], _mm(x.abs(), x.t().abs()))
        q = keep(a * torch.eye(len(s), dtype=s.dtype, device=s.device) + b * s + c * _mm(s, s), s.shape[0], abs(c) * _mm(s.abs(), s.abs()))
        x = keep(_mm(q, x), s.shape[0], _mm(q.abs(), x.abs()))
    return x.t().contiguous() if turned else x


def _one_step_bound(x, dtype, eps=1e-7):
    a, b, c = (abs(v) for v in ABC)
    h = HELD[dtype]
    x, turned = _wide(x.double())
    x = x / (torch.linalg.vector_norm(x) + eps)
    n, k = x.shape
    ax = x.abs()
    ex = (3 * U + h) * ax
    p = _mm(ax, ax.t())
    es = ((k + 8) * U + 3 * h) * p + _mm(ex, ax.t()) + _mm(ax, ex.t())
    s = _mm(x, x.t()).abs()
    es = es + (h + U) * (s + es)
    ss = _mm(s, s)
    q = b * s + c * ss + a * torch.eye(n, dtype=torch.float64, device=x.device)
    eq = b * es + c * (_mm(es, s) + _mm(s, es) + _mm(es, es)) + (c * ((n + 8) * U + 3 * h)) * _mm(s + es, s + es) + (h + 4 * U) * (q + b * es)
    e = _mm(eq, ax + ex) + _mm(q, ex) + ((n + 8) * U + 3 * h) * _mm(q + eq, ax + ex)
    return e.t().contiguous() if turned else e


SIZES = [(1, 1, 1), (2, 1, 7), (1, 5, 3), (3, 8, 8), (1, 64, 64), (2, 63, 65), (1, 64, 576), (2, 133, 307), (2, 307, 133), (1, 300, 300), (1, 1, 2000), (1, 2000, 3), (1, 513, 129), (1, 257, 1100), (20, 32, 96)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,rows,cols", SIZES + [(1, 1030, 2100), (5, 640, 600)])
def test_one_step(count, rows, cols, dtype):
    from paper_2409_09083_amd import orthogonal
    x = _matrix(count, rows, cols, dtype)
    got = orthogonal.Orthogonal(rows, cols, dtype, count=count, steps=1).forward(x)
    assert got.shape == x.shape and got.dtype == x.dtype
    for m in range(count):
        want, tol = _steps(x[m], 1), _one_step_bound(x[m], dtype)
        assert ((got[m].double() - want).abs() <= tol + LAST[dtype] * (want.abs() + tol) + 1e-37).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,rows,cols", SIZES)
def test_several_steps(count, rows, cols, dtype):
    from paper_2409_09083_amd import orthogonal
    x = _matrix(count, rows, cols, dtype, seed=1)
    h = HELD[dtype]
    for steps in (2, 5):
        o = orthogonal.Orthogonal(rows, cols, dtype, count=count, steps=steps)
        got = o.forward(x).clone()
        o._ws.fill_(255)                                        # scratch need not be cleared
        assert torch.equal(o.forward(x), got)
        for m in range(count):
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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(96, 400), (400, 96)])
def test_singular_values_and_vectors(rows, cols, dtype):
    """Singular values from 1 to a hundredth of the largest end between 0.6 and 1.3, on the vectors they had: out x^T (x^T out) is symmetric."""
    from paper_2409_09083_amd import orthogonal
    x = _matrix(1, rows, cols, "f32", seed=2)[0].double().cpu()
    u, _, v = torch.linalg.svd(x, full_matrices=False)
    x = ((u * torch.logspace(0, -2, min(rows, cols), dtype=torch.float64)) @ v).to(TYPES[dtype]).cuda()
    out = orthogonal.Orthogonal(rows, cols, dtype).forward(x).double()
    values = torch.linalg.svdvals(out.cpu())
    assert 0.6 <= float(values.min()) and float(values.max()) <= 1.3
    p = _mm(out, x.double().t()) if rows <= cols else _mm(out.t(), x.double())
    # (a rounding of the result by `LAST` turns its vectors by that much; 1e-5 is 5 steps of 32-bit roundings)
    assert float((p - p.t()).norm()) <= (2 * LAST[dtype] + 1e-5) * float(p.norm()) * 2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("abc", [(1.5, -0.5, 0.0), (0.0, 1.0, 0.0), (2.0, 0.0, -1.0), (1.0, 0.0, 0.0), (0.0, 0.0, 1.0)])
def test_other_coefficients(abc, dtype):
    """Also those that are 0; x's largest singular value is below 1, so that no bound is larger than (1 + |a| + |b| + |c|) times what one step's operands are held to."""
    from paper_2409_09083_amd import orthogonal
    for rows, cols in ((30, 50), (90, 200), (200, 90)):
        x = _matrix(1, rows, cols, dtype, seed=9)[0]
        got = orthogonal.Orthogonal(rows, cols, dtype, steps=1, coefficients=abc).forward(x).double()
        want = _steps(x, 1, abc=abc)
        n = max(rows, cols)
        # norms: |X| = 1, |S| <= 1, |S^2| <= 1; each is off by (n + 8) u + 4 h of the absolute values' product, of norm at most |X|^2 = 1, at most 8 such errors behind each other
        assert float((got - want).norm()) <= 8 * (sum(map(abs, abc)) + 1) * ((n + 8) * U + 4 * HELD[dtype]) + LAST[dtype] * float(want.norm())


def test_special_matrices():
    from paper_2409_09083_amd import orthogonal
    x = _matrix(4, 40, 70, "f32", seed=3)
    o = orthogonal.Orthogonal(40, 70, count=4)
    want = o.forward(x).clone()
    x[1] = 0
    x[2, 5, 6] = math.nan
    x[3, 0, 0] = math.inf
    got = o.forward(x)
    assert torch.equal(got[0], want[0]) and not got[1].any() and got[2].isnan().all() and got[3].isnan().all()
    # the scale does not matter, down to numbers whose squares 32 bits do not hold
    y = _matrix(1, 40, 70, "f32", seed=4)[0]
    one = orthogonal.Orthogonal(40, 70, eps=0.0)
    want = one.forward(y).clone()
    for scale in (2.0 ** 100, 2.0 ** -90):
        assert torch.equal(one.forward(y * scale), want)
    # one row is divided by its norm; the polynomial of 1 five times is a number
    v = 1.0
    a, b, c = (torch.tensor(k, dtype=torch.float32).double().item() for k in ABC)
    for _ in range(5):
        v = a * v + b * v ** 3 + c * v ** 5
    r = torch.randn((1, 300), device="cuda")
    got = orthogonal.Orthogonal(1, 300).forward(r).double()
    assert (got - v * r.double() / r.double().norm()).abs().max() <= 1e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_shapes(dtype):
    from paper_2409_09083_amd import orthogonal
    x = _matrix(3, 50, 90, dtype, seed=5)
    o = orthogonal.Orthogonal(50, 90, dtype, count=3)
    want = o.forward(x).clone()
    around = torch.full((3 * 53 * 97 + 1,), math.nan, dtype=x.dtype, device="cuda")
    v = around[1:].view(3, 53, 97)[:, :50, :90]
    v.copy_(x)
    assert torch.equal(o.forward(v), want)
    assert torch.equal(o.forward(x[:1].expand(3, 50, 90))[2], want[0])
    one = orthogonal.Orthogonal(50, 90, dtype)
    assert one.forward(x[0]).shape == (50, 90) and torch.equal(one.forward(x[0]), one.forward(x[:1])[0])
    filters = orthogonal.Orthogonal(16, 27, dtype)              # a filter's gradient as a matrix
    f = _matrix(1, 16, 27, dtype, seed=6).view(16, 3, 3, 3)
    assert filters.forward(f.view(16, -1)).view(f.shape).shape == f.shape


def test_in_place_empty_refusals_and_graph():
    from paper_2409_09083_amd import binding as B
    from paper_2409_09083_amd import orthogonal
    x = _matrix(2, 70, 64, "f32", seed=7)
    o = orthogonal.Orthogonal(70, 64, count=2)
    want = o.forward(x).clone()
    y = x.clone()
    B.ftp_orthogonal(o.desc, y.data_ptr(), y.data_ptr(), o._ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert torch.equal(y, want)
    assert orthogonal.Orthogonal(4, 5, count=0).forward(torch.empty((0, 4, 5), device="cuda")).shape == (0, 4, 5)
    with pytest.raises(TypeError):
        o.forward(x.bfloat16())
    for bad in (lambda: o.forward(x[:1]), lambda: o.forward(x[0]), lambda: o.forward(x.transpose(1, 2).contiguous().transpose(1, 2)), lambda: o.forward(x.cpu()),
                lambda: orthogonal.Orthogonal(4, 4, "f16")):
        with pytest.raises(ValueError):
            bad()
    for bad in (dict(rows=0), dict(cols=40000), dict(steps=0), dict(count=-1), dict(eps=-1.0), dict(coefficients=(1.0, math.nan, 0.0))):
        with pytest.raises(B.FtpError):
            orthogonal.Orthogonal(**{"rows": 4, "cols": 4, **bad})
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o.forward(x)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        o.forward(x)
    for k in range(4):
        x.copy_(_matrix(2, 70, 64, "f32", seed=30 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = o.out.clone()
        assert torch.equal(o.forward(x), got)
        torch.cuda.synchronize()
