"""8-bit activation checkpoints: codes and exponents bit for bit against a host implementation of the definition, what the backward
pass computes from them against 64 bits.

Bounds: GELU's formula 7.1.26 is within 1.5e-7 of erf and its evaluation (polynomial of five terms with a sum of magnitudes below 5)
within 5 * 4 * 2^-24 of that: 1.5e-6 (1 + |x|) for the value, the derivative alike; the sigmoid within 8 roundings.  A bfloat result adds 2^-8 of itself.
Weight gradient: products are exact (a code and its exponent are a bfloat; an fp32 dy is three bfloats), sums of n terms one after the
other: n 2^-24 sum|terms|, and 2^-24 more for three partial products each."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _host_pack(x, block):
    """The definition, value by value in 64 bits."""
    x = x.astype(np.float64)
    rows, cols = x.shape
    nb = -(-cols // block)
    codes, exps = np.zeros((rows, cols), np.int8), np.zeros((rows, nb), np.int8)
    for r in range(rows):
        for b in range(nb):
            v = x[r, b * block:(b + 1) * block]
            if not np.isfinite(v).all():
                exps[r, b] = 127
                continue
            top = np.max(np.abs(v))
            e = -126
            while top > 127.0 * 2.0 ** e:
                e += 1
            most = 63 if e == 122 else 127
            exps[r, b] = e
            codes[r, b * block:(b + 1) * block] = np.clip(np.rint(v / 2.0 ** e), -most, most)
    return codes, exps


def _held(codes, exps, block):
    unit = np.where(exps == 127, np.nan, 2.0 ** exps.astype(np.float64))
    return codes * np.repeat(unit, block, 1)[:, :codes.shape[1]]


def _values(rows, cols, dtype, seed=0, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * torch.exp(spread * torch.randn((rows, 1), generator=g))
    return x.to(TYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block", [32, 64, 128, 256])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 32), (4, 250), (7, 256), (2, 1031), (33, 64), (1, 4096), (64, 8)])
def test_codes_exponents_and_values(rows, cols, block, dtype):
    from paper_2409_09083_amd import tokens
    x = _values(rows, cols, dtype)
    kept = tokens.Checkpoint(rows, cols, dtype, block)
    got = kept.pack(x.cuda()).unpack()
    codes, exps = _host_pack(x.float().numpy(), block)
    assert np.array_equal(kept.exponents.cpu().numpy(), exps)
    assert np.array_equal(kept.codes.cpu().numpy(), codes)
    assert np.array_equal(got.float().cpu().numpy(), _held(codes, exps, block).astype(np.float32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_numbers(dtype):
    """Zeros, denormals, the borders of the exponent rule, the largest numbers, ties, infinities and NaN."""
    from paper_2409_09083_amd import tokens
    top = float(torch.finfo(TYPES[dtype]).max)
    tiny = 2.0 ** -126
    rows = [[0.0], [-0.0, 0.0], [tiny], [tiny / 64], [tiny / 2, tiny], [127.0], [127.5], [128.0], [127.0, 0.5, 1.5, 2.5, -0.5, -1.5], [127.0 * 2.0 ** -126],
            [128.0 * 2.0 ** -126], [top], [-top, top / 2], [2.0 ** 127], [1.984375 * 2.0 ** 127], [127.0 * 2.0 ** 121], [math.inf, 1.0], [1.0, -math.inf],
            [math.nan, 3.0], [254.0, 3.0, 5.0, -7.0], [1e-30, 1e30]]
    x = torch.zeros((len(rows), 70), dtype=TYPES[dtype])
    for i, v in enumerate(rows):
        for j, n in enumerate(v):
            x[i, (j * 13) % 32] = n
    kept = tokens.Checkpoint(len(rows), 70, dtype, 32)
    got = kept.pack(x.cuda()).unpack().float().cpu().numpy()
    codes, exps = _host_pack(x.float().numpy(), 32)
    assert np.array_equal(kept.exponents.cpu().numpy(), exps)
    assert np.array_equal(kept.codes.cpu().numpy(), codes)
    want = _held(codes, exps, 32)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isfinite(got[~np.isnan(want)]).all()
    assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)].astype(np.float32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(8, 0), (5, 0), (16, 3)])
def test_strided_rows(pad, offset, dtype):
    from paper_2409_09083_amd import tokens
    x = _values(9, 200, dtype)
    wide = torch.full((9 * (200 + pad) + offset,), math.nan, dtype=TYPES[dtype], device="cuda")
    v = wide[offset:].view(9, 200 + pad)[:, :200]
    v.copy_(x)
    kept = tokens.Checkpoint(9, 200, dtype, 64)
    kept.pack(v)
    codes, exps = _host_pack(x.float().numpy(), 64)
    assert np.array_equal(kept.codes.cpu().numpy(), codes) and np.array_equal(kept.exponents.cpu().numpy(), exps)
    kept.unpack(out=v)                                              # into the strided rows: nothing beside them is touched
    assert np.array_equal(v.float().cpu().numpy(), _held(codes, exps, 64).astype(np.float32))
    beside = wide[offset:].view(9, 200 + pad)[:, 200:]
    assert beside.isnan().all() and wide[:offset].isnan().all()


def _act64(x, act, slope):
    phi = 0.5 * torch.erfc(-x * math.sqrt(0.5))
    if act == "leaky":
        return torch.where(x > 0, x, x * slope), torch.where(x > 0, torch.ones_like(x), torch.full_like(x, slope))
    if act == "gelu":
        return x * phi, phi + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(x)
        return x * s, s + x * s * (1 - s)
    return x, torch.ones_like(x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "leaky", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (13, 77), (6, 512)])
def test_activations(rows, cols, act, dtype):
    from paper_2409_09083_amd import tokens
    x = _values(rows, cols, dtype, spread=1.0).cuda()
    x[0, 0] = 30.0                                                  # far out in the tails
    x[-1, -1] = -30.0
    kept = tokens.Checkpoint(rows, cols, dtype, 32).pack(x)
    held = kept.unpack().double().clone()
    dy = _values(rows, cols, dtype, seed=1, spread=0.1).cuda()
    value, slope = _act64(held, act, 0.1)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    far = 1.5e-6 * (1 + held.abs())
    got = kept.unpack(act=act).double()
    assert (got - value).abs().le(half * value.abs() + far).all()
    got = kept.act_backward(dy, act=act).double()
    want = dy.double() * slope
    assert (got - want).abs().le(half * want.abs() + far * dy.double().abs()).all()
    assert torch.equal(kept.act_backward(dy, act=act, out=dy).double(), got)       # in place


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_derivative_by_differences(dtype):
    from paper_2409_09083_amd import tokens
    x = torch.linspace(-4, 4, 64, device="cuda").to(TYPES[dtype])[None]
    kept = tokens.Checkpoint(1, 64, dtype, 64).pack(x)
    held = kept.unpack().double().clone()
    one = torch.ones_like(x)
    for act in ("gelu", "silu"):
        d = 1e-4
        want = (_act64(held + d, act, 0)[0] - _act64(held - d, act, 0)[0]) / (2 * d)
        assert (kept.act_backward(one, act=act).double() - want).abs().max() <= (2.0 ** -8 * 1.2 if dtype == "bf16" else 0) + 1e-5


@pytest.mark.parametrize("act", ["none", "leaky", "gelu", "silu"])
def test_a_bad_block_is_nan_everywhere_it_reaches(act):
    from paper_2409_09083_amd import tokens
    x = torch.ones((2, 96), device="cuda")
    x[1, 40] = math.inf
    kept = tokens.Checkpoint(2, 96, "f32", 32, outputs=5).pack(x)
    bad = torch.zeros((2, 96), dtype=torch.bool, device="cuda")
    bad[1, 32:64] = True
    assert torch.equal(kept.unpack(act=act).isnan(), bad)
    assert torch.equal(kept.act_backward(torch.ones_like(x), act=act).isnan(), bad)
    assert torch.equal(kept.wgrad(torch.ones((2, 5), device="cuda")).isnan(), bad[1][None].expand(5, 96))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block", [32, 128])
@pytest.mark.parametrize("rows,cols,n", [(1, 1, 1), (31, 16, 8), (32, 128, 128), (33, 129, 127), (100, 250, 33), (700, 64, 300), (2049, 202, 133), (5000, 96, 48)])
def test_weight_gradient(rows, cols, n, block, dtype):
    from paper_2409_09083_amd import tokens
    kept = tokens.Checkpoint(rows, cols, dtype, block, outputs=n).pack(_values(rows, cols, dtype, spread=1.0).cuda())
    dy = _values(rows, n, dtype, seed=2, spread=1.0).cuda()
    held = kept.unpack().double()
    got = kept.wgrad(dy).clone()
    want = dy.double().t().contiguous() @ held
    terms = dy.double().abs().t().contiguous() @ held.abs()
    assert (got.double() - want).abs().le((rows + 8) * 2.0 ** -24 * terms + 1e-37).all()
    assert torch.equal(kept.wgrad(dy), got)
    # ... and with dy inside wider rows at an odd address
    wide = torch.full((rows * (n + 3) + 1,), math.nan, dtype=dy.dtype, device="cuda")
    v = wide[1:].view(rows, n + 3)[:, :n]
    v.copy_(dy)
    assert torch.equal(kept.wgrad(v), got)


def test_weight_gradient_of_fp32_keeps_low_bits():
    """Numbers whose bfloat parts matter down to the last: 1 + 2^-23 against whole codes comes out exact."""
    from paper_2409_09083_amd import tokens
    kept = tokens.Checkpoint(64, 32, "f32", 32, outputs=32).pack(torch.eye(64, 32, device="cuda") * 64)
    dy = 1 + torch.arange(64 * 32, device="cuda").view(64, 32).float() * 2.0 ** -23
    assert torch.equal(kept.wgrad(dy), dy[:32].t() * 64)


def test_empty_refusals_and_graph():
    from paper_2409_09083_amd import binding as B
    from paper_2409_09083_amd import tokens
    e = tokens.Checkpoint(0, 64, "f32", 32, outputs=8)
    e.pack(torch.empty((0, 64), device="cuda")).unpack()
    assert float(e.wgrad(torch.empty((0, 8), device="cuda")).abs().max()) == 0
    with pytest.raises(B.FtpError):
        tokens.Checkpoint(4, 64, "f32", 48)
    kept = tokens.Checkpoint(300, 64, "bf16", 64, outputs=16)
    x = torch.randn((300, 64), device="cuda").bfloat16()
    with pytest.raises(TypeError):
        kept.pack(x.float())
    with pytest.raises(ValueError):
        kept.pack(x.t().contiguous().t())
    with pytest.raises(ValueError):
        kept.unpack(act="tanh")
    with pytest.raises(ValueError):
        tokens.Checkpoint(300, 64, "bf16", 64).wgrad(x)
    # captured once, replayed with other inputs and eager work between
    dy = torch.randn((300, 16), device="cuda").bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        kept.pack(x)
        kept.wgrad(dy)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        kept.pack(x)
        kept.wgrad(dy)
    for k in range(3):
        x.copy_(torch.randn((300, 64), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = kept.dw.clone()
        kept.pack(x)
        assert torch.equal(kept.wgrad(dy), got)
