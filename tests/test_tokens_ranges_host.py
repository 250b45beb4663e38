"""Strides and sizes beyond what the token block's operators take are refused before anything is launched (no GPU needed)."""
import pytest

P = 4096                                                        # an address that nothing reads


@pytest.fixture(scope="module")
def B():
    import paper_2409_09083_amd as F
    return F.binding


def _attention(B, **k):
    strides = {n: k.pop(n + "_stride") for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv") if n + "_stride" in k}
    d = dict(batch=1, heads=4, kv_heads=2, q_len=5, kv_len=7, head_dim=32, dtype=B.FTP_BF16, causal=1, scale=0.5)
    d.update(k)
    s = B.ftp_attention_shape(**d)
    for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        getattr(s, n + "_stride")[:] = strides.get(n, (1024, 128, 32))
    return s


def _code(B, f, *args):
    with pytest.raises(B.FtpError) as e:
        f(*args)
    return e.value.code


@pytest.mark.parametrize("tensor", ["q", "k", "v", "out", "dout", "dq", "dk", "dv"])
@pytest.mark.parametrize("axis", [0, 1, 2])
def test_attention_refuses_negative_strides(B, tensor, axis):
    stride = [1024, 128, 32]
    stride[axis] *= -1
    s = _attention(B, **{tensor + "_stride": stride})
    if tensor in ("q", "k", "v", "out"):
        assert _code(B, B.ftp_attention_forward, s, P, P, P, 0, 0, P, P, P) == B.FTP_EINVAL
    assert _code(B, B.ftp_attention_backward, s, P, P, P, P, 0, 0, P, P, P, P, P, P) == B.FTP_EINVAL
