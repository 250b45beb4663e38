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


# workgroups of 128 rows or keys (64 where those are few, and of keys of wide fp32 heads); a launch has fewer than 2^24, counted with what rounds (image, key head) groups up to eights
@pytest.mark.parametrize("dtype", ["FTP_F32", "FTP_BF16"])
@pytest.mark.parametrize("size,fits", [(dict(batch=(1 << 24) - 8, heads=1, kv_heads=1, q_len=1, kv_len=1), True), (dict(batch=1 << 24, heads=1, kv_heads=1, q_len=1, kv_len=1), False),
                                       (dict(batch=1 << 21, heads=7, kv_heads=7, q_len=128, kv_len=128), True), (dict(batch=1 << 21, heads=8, kv_heads=8, q_len=128, kv_len=1), False),
                                       (dict(batch=1 << 21, heads=8, kv_heads=8, q_len=1, kv_len=1), False), (dict(batch=1 << 20, heads=8, kv_heads=8, q_len=1, kv_len=300), False),
                                       (dict(batch=1 << 20, heads=8, kv_heads=8, q_len=300, kv_len=1), False), (dict(batch=1, heads=1, kv_heads=1, q_len=1 << 30, kv_len=1), True),
                                       (dict(batch=1, heads=1, kv_heads=1, q_len=1, kv_len=1 << 30), True), (dict(batch=1, heads=4, kv_heads=4, q_len=5, kv_len=1 << 30), False)])
def test_attention_refuses_more_workgroups_than_a_launch_has(B, size, fits, dtype):
    s = _attention(B, dtype=getattr(B, dtype), head_dim=64, **size)
    if fits:
        assert B.ftp_attention_workspace(s) is not None
        return
    assert _code(B, B.ftp_attention_workspace, s) == B.FTP_EUNSUPPORTED
    assert _code(B, B.ftp_attention_forward, s, P, P, P, 0, 0, P, P, P) == B.FTP_EUNSUPPORTED
    assert _code(B, B.ftp_attention_backward, s, P, P, P, P, 0, 0, P, P, P, P, P, P) == B.FTP_EUNSUPPORTED


def test_weight_gradient_refuses_more_workgroups_than_a_launch_has(B):
    s = B.ftp_checkpoint_shape(rows=3, cols=1 << 30, stride=1 << 30, block=32, dtype=B.FTP_F32)
    assert _code(B, B.ftp_checkpoint_wgrad, s, P, P, P, 257, 257, P, P) == B.FTP_EUNSUPPORTED
