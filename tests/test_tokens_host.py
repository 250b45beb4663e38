"""The token block's entry points refuse what they cannot do, before anything is launched (no GPU needed)."""
import ctypes

import pytest

P = 4096                                                        # an address that nothing reads


@pytest.fixture(scope="module")
def B():
    import paper_2409_09083_amd as F
    return F.binding


def _norm(B, **k):
    d = dict(outer=2, inner=3, channels=8, dtype=B.FTP_F32, eps=1e-5)
    d.update(k)
    strides = {n: d.pop(n, (24, 8, 1)) for n in ("x_stride", "y_stride", "dy_stride", "dx_stride")}
    s = B.ftp_norm_shape(**d)
    for n, v in strides.items():
        getattr(s, n)[:] = v
    return s


def _attention(B, **k):
    d = dict(batch=1, heads=4, kv_heads=2, q_len=5, kv_len=7, head_dim=32, dtype=B.FTP_BF16, causal=1, scale=0.5)
    d.update(k)
    return B.ftp_attention_shape(**d)


def _checkpoint(B, **k):
    d = dict(rows=3, cols=40, stride=40, block=32, dtype=B.FTP_F32)
    d.update(k)
    return B.ftp_checkpoint_shape(**d)


def _code(B, f, *args):
    with pytest.raises(B.FtpError) as e:
        f(*args)
    return e.value.code


@pytest.mark.parametrize("bad,code", [(dict(channels=0), "FTP_EINVAL"), (dict(dtype=7), "FTP_EINVAL"), (dict(outer=-1), "FTP_EINVAL"),
                                      (dict(eps=-1.0), "FTP_EINVAL"), (dict(eps=float("nan")), "FTP_EINVAL"), (dict(x_stride=(-1, 8, 1)), "FTP_EINVAL"),
                                      (dict(outer=1 << 20, inner=1 << 20), "FTP_EUNSUPPORTED"),
                                      (dict(channels=5000, x_stride=(1, 1, 3)), "FTP_EUNSUPPORTED")])
def test_norm_shapes(B, bad, code):
    assert _code(B, B.ftp_norm_forward, _norm(B, **bad), P, P, P, P, P, P) == getattr(B, code)


def test_norm_pointers(B):
    s = _norm(B)
    assert _code(B, B.ftp_norm_forward, s, 0, P, P, P, P, P) == B.FTP_EINVAL
    back = [s, P, P, 0, 0, 0, P, P, P, P, P, P, P]
    for at in (1, 2, 7, 8, 9, 10, 11, 12):                      # dy, x, mean, rstd, dx, one of dgamma and dbeta, the scratch
        args = list(back)
        args[at] = 0
        assert _code(B, B.ftp_norm_backward, *args) == B.FTP_EINVAL
    both = list(back)
    both[3] = both[4] = P                                       # x and a checkpoint of it
    both[5] = 32
    assert _code(B, B.ftp_norm_backward, *both) == B.FTP_EINVAL
    both[2], both[5] = 0, 33
    assert _code(B, B.ftp_norm_backward, *both) == B.FTP_EUNSUPPORTED
    both[0], both[5] = _norm(B, dy_stride=(24, 1, 3)), 32
    assert _code(B, B.ftp_norm_backward, *both) == B.FTP_EUNSUPPORTED
    B.ftp_norm_forward(_norm(B, outer=0), 0, 0, 0, 0)           # nothing to do is no error
    assert B.ftp_norm_workspace(s) >= 2 * 8 * 4


@pytest.mark.parametrize("bad,code", [(dict(cols=0), "FTP_EINVAL"), (dict(rows=-1), "FTP_EINVAL"), (dict(stride=39), "FTP_EINVAL"), (dict(dtype=2), "FTP_EINVAL"),
                                      (dict(block=48), "FTP_EUNSUPPORTED"), (dict(block=0), "FTP_EUNSUPPORTED"),
                                      (dict(cols=(1 << 30) + 1, stride=1 << 31), "FTP_EUNSUPPORTED")])
def test_checkpoint_shapes(B, bad, code):
    s = _checkpoint(B, **bad)
    assert _code(B, B.ftp_checkpoint_pack, s, P, P, P) == getattr(B, code)
    assert _code(B, B.ftp_checkpoint_unpack, s, P, P, 0, 0.0, P) == getattr(B, code)
    assert _code(B, B.ftp_checkpoint_act_backward, s, P, P, 0, 0.0, P, P) == getattr(B, code)
    assert _code(B, B.ftp_checkpoint_workspace, s, 8) == getattr(B, code)
    assert _code(B, B.ftp_checkpoint_wgrad, s, P, P, P, 8, 8, P, P) == getattr(B, code)


def test_checkpoint_arguments(B):
    s = _checkpoint(B)
    assert _code(B, B.ftp_checkpoint_pack, s, 0, P, P) == B.FTP_EINVAL
    assert _code(B, B.ftp_checkpoint_unpack, s, P, P, 4, 0.0, P) == B.FTP_EINVAL
    assert _code(B, B.ftp_checkpoint_act_backward, s, P, P, -1, 0.0, P, P) == B.FTP_EINVAL
    assert _code(B, B.ftp_checkpoint_workspace, s, 0) == B.FTP_EINVAL
    assert _code(B, B.ftp_checkpoint_wgrad, s, P, P, P, 7, 8, P, P) == B.FTP_EINVAL         # rows of dy overlap
    assert _code(B, B.ftp_checkpoint_wgrad, s, P, P, 0, 8, 8, P, P) == B.FTP_EINVAL
    long = _checkpoint(B, rows=100000)
    assert B.ftp_checkpoint_workspace(long, 8) > 0
    assert _code(B, B.ftp_checkpoint_wgrad, long, P, P, P, 8, 8, P, 0) == B.FTP_EINVAL       # needs its scratch
    B.ftp_checkpoint_pack(_checkpoint(B, rows=0), 0, 0, 0)


@pytest.mark.parametrize("bad,code", [(dict(heads=3), "FTP_EINVAL"), (dict(kv_heads=0), "FTP_EINVAL"), (dict(batch=-1), "FTP_EINVAL"),
                                      (dict(q_len=-1), "FTP_EINVAL"), (dict(kv_len=-1), "FTP_EINVAL"), (dict(head_dim=0), "FTP_EINVAL"),
                                      (dict(dtype=-1), "FTP_EINVAL"), (dict(scale=float("inf")), "FTP_EINVAL"),
                                      (dict(scale=float("nan")), "FTP_EINVAL"), (dict(head_dim=129), "FTP_EUNSUPPORTED"),
                                      (dict(q_len=1 << 30, heads=64), "FTP_EUNSUPPORTED")])
def test_attention_shapes(B, bad, code):
    s = _attention(B, **bad)
    assert _code(B, B.ftp_attention_workspace, s) == getattr(B, code)
    assert _code(B, B.ftp_attention_forward, s, P, P, P, 0, 0, P, P, P) == getattr(B, code)
    assert _code(B, B.ftp_attention_backward, s, P, P, P, P, 0, 0, P, P, P, P, P, P) == getattr(B, code)


def test_attention_pointers(B):
    s = _attention(B)
    for at in (1, 2, 3, 6):                                     # q, k, v, out
        args = [s, P, P, P, 0, 0, P, P, P]
        args[at] = 0
        assert _code(B, B.ftp_attention_forward, *args) == B.FTP_EINVAL
    for at in (1, 2, 3, 4, 7, 8, 9, 10, 11, 12):
        args = [s, P, P, P, P, 0, 0, P, P, P, P, P, P]
        args[at] = 0
        assert _code(B, B.ftp_attention_backward, *args) == B.FTP_EINVAL
    long = _attention(B, q_len=1, kv_len=10000)
    assert B.ftp_attention_workspace(long)[0] > 0
    assert _code(B, B.ftp_attention_forward, long, P, P, P, 0, 0, P, P, 0) == B.FTP_EINVAL
    B.ftp_attention_forward(_attention(B, batch=0), 0, 0, 0, 0, 0, 0, 0, 0)
    for empty in (dict(batch=0), dict(q_len=0), dict(kv_len=0), dict(q_len=0, kv_len=0)):
        assert B.ftp_attention_workspace(_attention(B, **empty))[0] == 0
    null = ctypes.POINTER(B.ftp_attention_shape)()
    assert _code(B, B.ftp_attention_workspace, null) == B.FTP_EINVAL
