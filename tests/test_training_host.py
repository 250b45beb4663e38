"""The training operators' entry points refuse what they cannot do, before anything is launched, and their objects call the library on their own device (no GPU needed)."""
import contextlib
import ctypes
import inspect
import random
import re

import pytest
import torch

P = 4096                                                        # an address that nothing reads


@pytest.fixture(scope="module")
def B():
    import paper_2409_09083_amd as F
    return F.binding


def _embedding(B, **k):
    return B.ftp_embedding_shape(**{**dict(rows=3, vocab=10, channels=8, dtype=B.FTP_F32, id_type=B.FTP_I64, scale=1.0, table_stride=8, row_stride=8), **k})


def _loss(B, **k):
    return B.ftp_token_loss_shape(**{**dict(rows=3, vocab=10, channels=8, dtype=B.FTP_BF16, id_type=B.FTP_I32, scale=1.0, x_stride=8, w_stride=8, dx_stride=8, dw_stride=8), **k})


def _orthogonal(B, **k):
    return B.ftp_orthogonal_shape(**{**dict(count=2, rows=5, cols=7, dtype=B.FTP_F32, steps=5, a=3.4, b=-4.8, c=2.0, eps=1e-7, matrix_stride=35, row_stride=7), **k})


def _code(B, f, *args):
    with pytest.raises(B.FtpError) as e:
        f(*args)
    return e.value.code


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("bad,code", [(dict(rows=-1), "FTP_EINVAL"), (dict(vocab=0), "FTP_EINVAL"), (dict(channels=0), "FTP_EINVAL"), (dict(dtype=2), "FTP_EINVAL"), (dict(id_type=2), "FTP_EINVAL"),
                                      (dict(scale=NAN), "FTP_EINVAL"), (dict(scale=INF), "FTP_EINVAL"), (dict(table_stride=-1), "FTP_EINVAL"), (dict(row_stride=-8), "FTP_EINVAL"),
                                      (dict(rows=(1 << 26) + 1), "FTP_EUNSUPPORTED"), (dict(vocab=(1 << 26) + 1), "FTP_EUNSUPPORTED"), (dict(channels=(1 << 20) + 1), "FTP_EUNSUPPORTED")])
def test_embedding_shapes(B, bad, code):
    s = _embedding(B, **bad)
    assert _code(B, B.ftp_embedding_forward, s, P, P, P) == getattr(B, code)
    assert _code(B, B.ftp_embedding_workspace, s) == getattr(B, code)
    assert _code(B, B.ftp_embedding_backward, s, P, P, P, P) == getattr(B, code)


def test_embedding_pointers(B):
    for at in (1, 2, 3):
        args = [_embedding(B), P, P, P]
        args[at] = 0
        assert _code(B, B.ftp_embedding_forward, *args) == B.FTP_EINVAL
    for at in (1, 2, 3, 4):
        args = [_embedding(B), P, P, P, P]
        args[at] = 0
        assert _code(B, B.ftp_embedding_backward, *args) == B.FTP_EINVAL
    assert _code(B, B.ftp_embedding_forward, _embedding(B, row_stride=7), P, P, P) == B.FTP_EINVAL          # rows of the output overlap
    B.ftp_embedding_forward(_embedding(B, rows=0), 0, 0, 0)     # nothing to do is no error
    assert _code(B, B.ftp_embedding_workspace, ctypes.POINTER(B.ftp_embedding_shape)()) == B.FTP_EINVAL


@pytest.mark.parametrize("bad,code", [(dict(rows=-1), "FTP_EINVAL"), (dict(vocab=0), "FTP_EINVAL"), (dict(channels=-3), "FTP_EINVAL"), (dict(dtype=7), "FTP_EINVAL"), (dict(id_type=-1), "FTP_EINVAL"),
                                      (dict(scale=NAN), "FTP_EINVAL"), (dict(scale=-2e38), "FTP_EINVAL"), (dict(x_stride=-1), "FTP_EINVAL"), (dict(w_stride=-1), "FTP_EINVAL"),
                                      (dict(dx_stride=-1), "FTP_EINVAL"), (dict(dw_stride=-1), "FTP_EINVAL"), (dict(rows=(1 << 22) + 1), "FTP_EUNSUPPORTED"),
                                      (dict(vocab=(1 << 22) + 1), "FTP_EUNSUPPORTED"), (dict(channels=(1 << 14) + 1), "FTP_EUNSUPPORTED"), (dict(rows=1 << 20, vocab=1 << 20), "FTP_EUNSUPPORTED")])
def test_loss_shapes(B, bad, code):
    s = _loss(B, **bad)
    assert _code(B, B.ftp_token_loss_workspace, s) == getattr(B, code)
    assert _code(B, B.ftp_token_loss_forward, s, P, P, P, P, P, P, P) == getattr(B, code)
    assert _code(B, B.ftp_token_loss_backward, s, P, P, P, P, P, P, P, P) == getattr(B, code)


def test_loss_pointers(B):
    for at in (1, 2, 3, 7):                                     # x, weight, labels, the scratch
        args = [_loss(B), P, P, P, P, P, P, P]
        args[at] = 0
        assert _code(B, B.ftp_token_loss_forward, *args) == B.FTP_EINVAL
    for at in (1, 2, 3, 4, 8):                                  # ... and lse
        args = [_loss(B), P, P, P, P, P, P, P, P]
        args[at] = 0
        assert _code(B, B.ftp_token_loss_backward, *args) == B.FTP_EINVAL
    assert _code(B, B.ftp_token_loss_backward, _loss(B, dx_stride=7), P, P, P, P, P, P, P, P) == B.FTP_EINVAL
    assert _code(B, B.ftp_token_loss_backward, _loss(B, dw_stride=7), P, P, P, P, P, P, P, P) == B.FTP_EINVAL
    forward, backward = B.ftp_token_loss_workspace(_loss(B, rows=0))
    assert forward > 0 and backward > 0                         # a call without rows still writes the mean and the weight's gradient
    assert _code(B, B.ftp_token_loss_workspace, ctypes.POINTER(B.ftp_token_loss_shape)()) == B.FTP_EINVAL


@pytest.mark.parametrize("bad,code", [(dict(count=-1), "FTP_EINVAL"), (dict(rows=0), "FTP_EINVAL"), (dict(cols=0), "FTP_EINVAL"), (dict(dtype=3), "FTP_EINVAL"), (dict(steps=0), "FTP_EINVAL"),
                                      (dict(eps=-1.0), "FTP_EINVAL"), (dict(eps=NAN), "FTP_EINVAL"), (dict(eps=INF), "FTP_EINVAL"), (dict(a=INF), "FTP_EINVAL"), (dict(c=NAN), "FTP_EINVAL"),
                                      (dict(matrix_stride=-1), "FTP_EINVAL"), (dict(row_stride=-7), "FTP_EINVAL"), (dict(rows=32769), "FTP_EUNSUPPORTED"), (dict(cols=40000), "FTP_EUNSUPPORTED"),
                                      (dict(steps=65), "FTP_EUNSUPPORTED"), (dict(count=65536), "FTP_EUNSUPPORTED"), (dict(count=40000, rows=2000, cols=2000), "FTP_EUNSUPPORTED")])
def test_orthogonal_shapes(B, bad, code):
    s = _orthogonal(B, **bad)
    assert _code(B, B.ftp_orthogonal_workspace, s) == getattr(B, code)
    assert _code(B, B.ftp_orthogonal, s, P, P, P) == getattr(B, code)


def test_orthogonal_pointers(B):
    for at in (1, 2, 3):
        args = [_orthogonal(B), P, P, P]
        args[at] = 0
        assert _code(B, B.ftp_orthogonal, *args) == B.FTP_EINVAL
    B.ftp_orthogonal(_orthogonal(B, count=0), 0, 0, 0)
    assert _code(B, B.ftp_orthogonal_workspace, ctypes.POINTER(B.ftp_orthogonal_shape)()) == B.FTP_EINVAL


def test_embedding_gradients_of_too_many_threads(B):
    """2^19 rows (all the same in memory) of 2^20 channels are 2^14 pieces of 32 rows x 2^18 vectors of four numbers, 2^32 threads: refused before anything is launched.  The lookup has
    a loop for them."""
    s = _embedding(B, rows=1 << 19, channels=1 << 20, row_stride=0)
    assert _code(B, B.ftp_embedding_workspace, s) == B.FTP_EUNSUPPORTED
    assert _code(B, B.ftp_embedding_backward, s, P, P, P, P) == B.FTP_EUNSUPPORTED
    assert B.ftp_embedding_workspace(_embedding(B, rows=1 << 18, channels=1 << 20, row_stride=0)) > 0
    assert B.ftp_embedding_workspace(_embedding(B, rows=1 << 26, channels=1 << 12, row_stride=0)) > 0


def test_scratch_of_all_sizes(B):
    """The plans of sizes over the whole range come to an end and ask for scratch that a card has, for as much of it as grows with the sizes."""
    r = random.Random(1)

    def some(lo, hi):
        return int(round(lo * (hi / lo) ** r.random()))
    for _ in range(400):
        dtype = r.choice((B.FTP_F32, B.FTP_BF16))
        planes = 3 if dtype == B.FTP_F32 else 2
        rows, vocab, channels = some(1, 1 << 17), some(1, 1 << 17), some(1, 4096)
        forward, backward = B.ftp_token_loss_workspace(_loss(B, rows=rows, vocab=vocab, channels=channels, dtype=dtype))
        padded = (channels + 63) // 64 * 64
        held = (2 * planes + 8) * (rows + vocab + 320) * padded                 # the planes, and sums of both gradients
        assert 0 < forward <= held + 8 * (rows + 64) * (vocab // 128 + 2) + 64 * rows + 1e6
        assert 0 < backward <= 17 * held + (1 << 30) + 6 * 320 * (rows + 256) + 64 * rows + 1e6
        n, k, count = some(1, 8192), some(1, 8192), some(1, 64)
        need = B.ftp_orthogonal_workspace(_orthogonal(B, rows=n, cols=k, count=count, dtype=dtype))
        n, k = ((v + 63) // 64 * 64 for v in (n, k))
        assert 0 < need <= 2 * planes * count * (2 * n * k + 2 * min(n, k) ** 2) * 1.5 + 512 * 32 * 65536 * 4 + 1e6


def test_objects_call_on_their_own_device(monkeypatch):
    from paper_2409_09083_amd import orthogonal, tokens, vocabulary
    # everything but the questions that launch nothing goes through the call that makes the object's device current
    direct = set(re.findall(r"\bB\.(ftp_\w+)\(", inspect.getsource(vocabulary) + inspect.getsource(orthogonal)))
    assert direct == {"ftp_embedding_shape", "ftp_token_loss_shape", "ftp_orthogonal_shape", "ftp_embedding_workspace", "ftp_token_loss_workspace", "ftp_orthogonal_workspace"}
    now, seen = [0], []

    @contextlib.contextmanager
    def device(index):
        before, now[0] = now[0], index
        try:
            yield
        finally:
            now[0] = before
    monkeypatch.setattr(tokens, "_current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(tokens, "_current_stream", lambda index: 1000 + index)
    for kind in (vocabulary.Embedding, vocabulary.TokenLoss, orthogonal.Orthogonal):
        o = kind.__new__(kind)
        o.device = torch.device("cuda", 2)
        o._call(lambda *args: seen.append((now[0],) + args), "x")
        assert seen[-1] == (2, "x", 1002) and now[0] == 0
