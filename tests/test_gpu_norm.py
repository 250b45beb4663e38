"""Layer norm, forward and backward, against the formulas in 64 bits.

Bounds, u = 2^-24 (2^-8 more for a result rounded to a bfloat, relative to it):
  mean, variance: a lane adds at most 64 terms one after the other, lanes meet in at most 10 further additions; with the divisions
  and the product behind them fewer than 128 roundings of numbers no larger than the token's largest, so h is off by at most
  128 u (1 + max|x - mean| / sigma + |mean| / sigma).
  dgamma, dbeta: at most 128 additions one after the other (rows of a workgroup, workgroups, lanes) up to 2^17 tokens, of terms
  that are themselves off by the bound above: 256 u sum|terms| (1 + the bracket).
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _make(outer, inner, c, dtype, x_layout="rows", dy_layout="rows", pad=0, offset=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[dtype]

    def tensor(layout, shift=0.0):
        t = (torch.randn((outer, inner, c), generator=g, device="cuda") * 1.5 + shift).to(dt)
        if layout == "map":
            return t.transpose(1, 2).contiguous().transpose(1, 2)
        if pad or offset:
            wide = torch.full((outer * inner * (c + pad) + offset,), float("nan"), device="cuda", dtype=dt)
            v = wide[offset:].view(outer, inner, c + pad)[:, :, :c]
            v.copy_(t)
            return v
        return t
    x, dy = tensor(x_layout, 0.7), tensor(dy_layout)
    gamma = (1 + 0.2 * torch.randn(c, generator=g, device="cuda")).to(dt)
    beta = (0.2 * torch.randn(c, generator=g, device="cuda")).to(dt)
    return x, dy, gamma, beta


def _reference(x, dy, gamma, beta, eps):
    x, dy = x.double(), dy.double()
    g = torch.ones(x.shape[2], device=x.device, dtype=torch.float64) if gamma is None else gamma.double()
    b = torch.zeros_like(g) if beta is None else beta.double()
    mean = x.mean(2, keepdim=True)
    sigma2 = ((x - mean) ** 2).mean(2, keepdim=True) + eps
    r = sigma2 ** -0.5
    h = (x - mean) * r
    a = dy * g
    dx = r * (a - a.mean(2, keepdim=True) - h * (a * h).mean(2, keepdim=True))
    size = 1 + h.abs().amax(2, keepdim=True) + mean.abs() * r
    return {"y": h * g + b, "mean": mean[..., 0], "rstd": r[..., 0], "dx": dx, "dgamma": (dy * h).sum((0, 1)), "dbeta": dy.sum((0, 1)),
            "h": h, "size": size, "g": g, "terms": ((dy * h).abs().sum((0, 1)), dy.abs().sum((0, 1))), "a": a, "r": r}


def _check(got, ref, dtype, gamma):
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    e = 128 * U * ref["size"]                                   # of h
    assert (got["mean"].double() - ref["mean"]).abs().le(128 * U * (ref["size"] / ref["r"])[..., 0]).all()
    assert (got["rstd"].double() / ref["rstd"] - 1).abs().le(256 * U * ref["size"][..., 0]).all()
    assert (got["y"].double() - ref["y"]).abs().le(half * ref["y"].abs() + e * (1 + ref["g"].abs()) + U * ref["y"].abs()).all()
    big = ref["a"].abs().amax(2, keepdim=True) * (1 + ref["h"].abs().amax(2, keepdim=True)) ** 2
    assert (got["dx"].double() - ref["dx"]).abs().le(half * ref["dx"].abs() + 2 * e * ref["r"] * big).all()
    worst = 256 * U * float(ref["size"].max())
    assert (got["dgamma"].double() - ref["dgamma"]).abs().le(worst * (ref["terms"][0] + ref["terms"][1]) + 1e-30).all()
    assert (got["dbeta"].double() - ref["dbeta"]).abs().le(256 * U * ref["terms"][1] + 1e-30).all()


def _run(x, dy, gamma, beta, dtype, x_layout="rows", y_layout="rows", eps=1e-5, norm=None):
    from paper_2409_09083_amd import tokens
    n = norm or tokens.Norm(*x.shape, dtype, eps=eps, x_layout=x_layout, y_layout=y_layout)
    n.forward(x, gamma, beta)
    n.backward(dy, x, gamma)
    torch.cuda.synchronize()
    return n, {k: getattr(n, k).clone() for k in ("y", "mean", "rstd", "dx", "dgamma", "dbeta")}


# channels around the powers of two, vector widths and the kernels' borders: 64 lanes x 8 values, a workgroup a row, rows beyond registers
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("outer,inner,c", [(1, 1, 1), (1, 1, 2), (3, 1, 7), (2, 5, 8), (1, 33, 31), (5, 13, 64), (2, 129, 100), (3, 67, 250),
                                           (1, 300, 256), (2, 77, 513), (2, 9, 1024), (1, 11, 2046), (1, 7, 2052), (1, 5, 4099), (1, 6, 8192),
                                           (2, 3, 8200), (1, 3, 20000)])
def test_rows(outer, inner, c, dtype):
    x, dy, gamma, beta = _make(outer, inner, c, dtype)
    _, got = _run(x, dy, gamma, beta, dtype)
    _check(got, _reference(x, dy, gamma, beta, 1e-5), dtype, gamma)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("x_layout,y_layout", [("map", "map"), ("map", "rows"), ("rows", "map")])
@pytest.mark.parametrize("outer,inner,c", [(1, 1, 1), (2, 1, 24), (3, 49, 16), (2, 361, 64), (1, 64, 32), (2, 100, 33), (1, 133, 250), (1, 70, 512),
                                           (1, 40, 1100), (1, 9, 4096)])
def test_maps(outer, inner, c, x_layout, y_layout, dtype):
    x, dy, gamma, beta = _make(outer, inner, c, dtype, x_layout, y_layout)
    n, got = _run(x, dy, gamma, beta, dtype, x_layout, y_layout)
    _check(got, _reference(x, dy, gamma, beta, 1e-5), dtype, gamma)
    assert n.y_buffer.shape == ((outer, c, inner) if y_layout == "map" else (outer, inner, c))
    assert n.dx_buffer.is_contiguous() and n.y_buffer.is_contiguous()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(8, 0), (24, 8), (1, 0), (3, 1), (64, 3)])
def test_strided_rows_and_odd_addresses(pad, offset, dtype):
    x, dy, gamma, beta = _make(4, 37, 96, dtype, pad=pad, offset=offset)
    _, got = _run(x, dy, gamma, beta, dtype)
    _check(got, _reference(x, dy, gamma, beta, 1e-5), dtype, gamma)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_images_apart_and_broadcast_inputs(dtype):
    """An image stride that is not the tokens' total; x the same for all images; dy one number (the gradient of a sum)."""
    x, dy, gamma, beta = _make(6, 20, 48, dtype)
    x, dy = x[::2], dy[::2]
    _, got = _run(x, dy, gamma, beta, dtype)
    _check(got, _reference(x, dy, gamma, beta, 1e-5), dtype, gamma)
    x = x[:1].expand(3, 20, 48)
    dy = torch.full((1, 1, 1), 0.5, device="cuda", dtype=TYPES[dtype]).expand(3, 20, 48)
    _, got = _run(x, dy, gamma, beta, dtype)
    _check(got, _reference(x, dy, gamma, beta, 1e-5), dtype, gamma)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_parameters_and_constant_tokens(dtype):
    x, dy, _, _ = _make(2, 30, 72, dtype)
    x[0, 3] = 2.0                                               # variance 0: rstd = eps^-1/2, h = 0
    _, got = _run(x, dy, None, None, dtype, eps=1e-3)
    ref = _reference(x, dy, None, None, 1e-3)
    _check(got, ref, dtype, None)
    assert got["y"][0, 3].abs().max() == 0


def test_many_tokens_and_equal_bits():
    x, dy, gamma, beta = _make(16, 4096, 40, "bf16")
    n, a = _run(x, dy, gamma, beta, "bf16")
    _check(a, _reference(x, dy, gamma, beta, 1e-5), "bf16", gamma)
    _, b = _run(x, dy, gamma, beta, "bf16", norm=n)
    assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_not_finite_values_stay_in_their_token(dtype):
    x, dy, gamma, beta = _make(2, 20, 64, dtype)
    x[0, 5, 7] = float("nan")
    x[1, 2, 0] = float("inf")
    _, got = _run(x, dy, gamma, beta, dtype)
    bad = torch.zeros(2, 20, dtype=torch.bool, device="cuda")
    bad[0, 5] = bad[1, 2] = True
    for k in ("y", "dx"):
        assert torch.equal(got[k].isfinite().all(2), ~bad)


def test_gradient_by_differences():
    """dx and dgamma against central differences of sum(w y) in 64 bits, through the framework's own gradients."""
    x, dy, gamma, beta = _make(1, 3, 24, "f32")
    _, got = _run(x, dy, gamma, beta, "f32")

    def loss(x, g):
        m = x.mean(2, keepdim=True)
        v = ((x - m) ** 2).mean(2, keepdim=True)
        return float(((x - m) * (v + 1e-5) ** -0.5 * g * dy.double()).sum())
    d = 1e-5
    for t, c in [(0, 0), (1, 7), (2, 23)]:
        e = torch.zeros_like(x, dtype=torch.float64)
        e[0, t, c] = d
        want = (loss(x.double() + e, gamma.double()) - loss(x.double() - e, gamma.double())) / (2 * d)
        assert abs(float(got["dx"][0, t, c]) - want) <= 1e-5 * (1 + abs(want))
    e = torch.zeros(24, dtype=torch.float64, device="cuda")
    e[5] = d
    want = (loss(x.double(), gamma.double() + e) - loss(x.double(), gamma.double() - e)) / (2 * d)
    assert abs(float(got["dgamma"][5]) - want) <= 1e-5 * (1 + abs(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("outer,inner,c,block", [(1, 1, 5, 32), (2, 31, 64, 64), (3, 17, 250, 64), (1, 90, 512, 128), (2, 5, 1000, 256), (1, 4, 2500, 32),
                                                 (1, 3, 9001, 32)])
def test_backward_from_a_checkpoint(outer, inner, c, block, dtype):
    from paper_2409_09083_amd import tokens
    x, dy, gamma, beta = _make(outer, inner, c, dtype)
    kept = tokens.Checkpoint(outer * inner, c, dtype, block)
    kept.pack(x.reshape(-1, c))
    n = tokens.Norm(outer, inner, c, dtype)
    n.forward(x, gamma, beta)
    held = kept.unpack().clone().view(x.shape)
    n.backward(dy, kept, gamma)
    got = {k: getattr(n, k).clone() for k in ("dx", "dgamma", "dbeta")}
    n.backward(dy, held, gamma)                                 # the values are exact in either type: the same numbers
    for k in got:
        assert torch.equal(got[k], getattr(n, k)), k


def test_in_place_empty_and_other_stream():
    from paper_2409_09083_amd import binding as B
    from paper_2409_09083_amd import tokens
    for c in (96, 20000):
        x, dy, gamma, beta = _make(2, 10, c, "bf16")
        n, want = _run(x, dy, gamma, beta, "bf16")
        n.dx = n.dx_buffer = dy                                 # dx over dy
        n.backward(dy, x, gamma)
        assert torch.equal(dy, want["dx"]) and torch.equal(n.dgamma, want["dgamma"])
    e = tokens.Norm(0, 5, 16, "f32")
    t = torch.empty((0, 5, 16), device="cuda")
    e.forward(t)
    assert float(e.backward(t, t)[1].abs().sum()) == 0          # sums of nothing are zero
    x, dy, gamma, beta = _make(8, 200, 128, "f32")
    _, want = _run(x, dy, gamma, beta, "f32")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        n = tokens.Norm(8, 200, 128, "f32")
        n.forward(x, gamma, beta)
        n.backward(dy, x, gamma)
    s.synchronize()
    assert torch.equal(n.dx, want["dx"]) and torch.equal(n.dgamma, want["dgamma"])
    with pytest.raises(B.FtpError):
        tokens.Norm(1, 1, 0, "f32")
    with pytest.raises(ValueError):
        n.forward(x[:, :, :64], gamma, beta)
    with pytest.raises(TypeError):
        n.forward(x.bfloat16(), gamma, beta)
    with pytest.raises(ValueError):
        n.forward(x, gamma[::2])
