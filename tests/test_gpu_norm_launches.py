"""Layer norm of more tokens than a launch has workgroups (2^24 of 256 threads).

Inputs are windows into one short buffer, so that only outputs take memory; tokens at the launches' borders and at the end are compared in 64 bits
within the bounds of tests/test_gpu_norm.py, nothing may be left unwritten."""
import pytest
import torch

from tests import test_gpu_norm as N

pytestmark = pytest.mark.gpu
MANY = 2 ** 24


def _windows(rows, c, stride, dtype):
    g = torch.Generator(device="cuda").manual_seed(0)
    base = torch.randn(rows + stride * c, generator=g, device="cuda").to(N.TYPES[dtype])
    return base.as_strided((rows, 1, c), (1, 1, stride))


def _compare(x, y, mean, rstd, dtype):
    rows = x.shape[0]
    for at in (0, MANY - 40, MANY // 2 - 20, rows - 40):
        part = x[at:at + 40]
        ref = N._reference(part, torch.ones_like(part), None, None, 1e-5)
        half = 2.0 ** -8 if dtype == "bf16" else 0.0
        e = 128 * N.U * ref["size"]
        assert (y[at:at + 40].double() - ref["y"]).abs().le(half * ref["y"].abs() + 2 * e + N.U * ref["y"].abs()).all()
        assert (mean[at:at + 40].double() - ref["mean"]).abs().le(128 * N.U * (ref["size"] / ref["r"])[..., 0]).all()
        assert (rstd[at:at + 40].double() / ref["rstd"] - 1).abs().le(256 * N.U * ref["size"][..., 0]).all()


def _written(t):
    for part in t.flatten().split(1 << 30):
        assert not part.isnan().any()


@pytest.mark.parametrize("dtype,c,stride", [("f32", 8, 2), ("bf16", 513, 1)])
def test_forward(dtype, c, stride):
    """A tile a token (strided channels), and a workgroup a row (an odd number of channels above 512)."""
    from paper_2409_09083_amd import tokens
    rows = MANY + 77
    x = _windows(rows, c, stride, dtype)
    n = tokens.Norm(rows, 1, c, dtype)
    for t in (n.y, n.mean, n.rstd):
        t.fill_(float("nan"))
    n.forward(x)
    _compare(x, n.y, n.mean, n.rstd, dtype)
    for t in (n.y, n.mean, n.rstd):
        _written(t)
    del n, t
    torch.cuda.empty_cache()


def test_rows_beyond_registers():
    """A workgroup a row in both passes: 69 GB of results, the backward pass over the forward one's."""
    from paper_2409_09083_amd import binding as B
    rows, c = MANY + 77, 2051
    x = _windows(rows, c, 1, "bf16")
    y = torch.empty((rows, 1, c), dtype=torch.bfloat16, device="cuda")
    mean, rstd = (torch.full((rows, 1), float("nan"), device="cuda") for _ in range(2))
    stream = torch.cuda.current_stream().cuda_stream
    s = B.ftp_norm_shape(outer=rows, inner=1, channels=c, dtype=B.FTP_BF16, eps=1e-5)
    s.x_stride[:] = s.dy_stride[:] = x.stride()
    s.y_stride[:] = s.dx_stride[:] = y.stride()
    y[-100:] = float("nan")
    B.ftp_norm_forward(s, x.data_ptr(), 0, 0, y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), stream)
    _compare(x, y, mean, rstd, "bf16")
    _written(mean)
    y[-100:] = float("nan")
    B.ftp_norm_backward(s, x.data_ptr(), x.data_ptr(), 0, 0, 0, 0, mean.data_ptr(), rstd.data_ptr(), y.data_ptr(), 0, 0, 0, stream)
    for at in (0, MANY - 40, rows - 40):
        part = x[at:at + 40]
        ref = N._reference(part, part, None, None, 1e-5)
        big = ref["a"].abs().amax(2, keepdim=True) * (1 + ref["h"].abs().amax(2, keepdim=True)) ** 2
        bound = 2.0 ** -8 * ref["dx"].abs() + 2 * 128 * N.U * ref["size"] * ref["r"] * big
        assert (y[at:at + 40].double() - ref["dx"]).abs().le(bound).all()
    del y
    torch.cuda.empty_cache()
