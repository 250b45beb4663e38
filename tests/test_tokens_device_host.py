"""Calls of the token block's objects start on the object's device and its current stream, whichever device is current (no GPU needed)."""
import contextlib

import torch


def test_a_call_makes_its_device_current(monkeypatch):
    from paper_2409_09083_amd import tokens
    now = [0]

    @contextlib.contextmanager
    def device(index):
        before, now[0] = now[0], index
        try:
            yield
        finally:
            now[0] = before
    monkeypatch.setattr(tokens, "_current_device", lambda: now[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(tokens, "_current_stream", lambda index: 1000 + index, raising=False)
    seen = []
    for calls in range(2):
        for index in (0, 1, 3):
            op = tokens._Operator()
            op.device = torch.device("cuda", index)
            op._call(lambda *args: seen.append((now[0],) + args), "x", 7)
            assert seen[-1] == (index, "x", 7, 1000 + index)
            assert now[0] == 0                                  # as it was


def test_every_method_goes_that_way():
    """Nothing of the library is called past it but the questions that launch nothing."""
    import inspect
    import re
    from paper_2409_09083_amd import tokens
    direct = set(re.findall(r"\bB\.(ftp_\w+)\(", inspect.getsource(tokens)))
    assert direct == {"ftp_norm_shape", "ftp_checkpoint_shape", "ftp_attention_shape", "ftp_norm_workspace", "ftp_checkpoint_workspace", "ftp_attention_workspace"}
