"""Calls on tensors of a device that is not the current one, without a GPU."""
import pytest
import torch

replay = pytest.importorskip("paper_2608_11034_amd.replay")


class _Stream:
    def __init__(self, index):
        self.device, self.cuda_stream = torch.device("cuda", index), 77


def test_handle(monkeypatch):
    """Kernels run on the current device; its stream and its tensors go with it."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(replay, "_raw_stream", None)
    monkeypatch.setattr(replay, "_stream", lambda stream: 55 if stream is None else stream.cuda_stream)
    one, two = torch.device("cuda", 1), torch.device("cuda", 2)
    assert replay._handle(None, one) == 55 and replay._handle(_Stream(1), one) == 77
    for stream, device in ((None, two), (_Stream(2), two), (_Stream(2), one), (_Stream(1), two)):
        with pytest.raises(replay.C3Error):
            replay._handle(stream, device)


def test_every_call_asks():
    """No launch takes a stream that was not looked at."""
    src = open(replay.__file__).read()
    body = src[src.index("def rotary("):]
    assert "_stream(stream)" not in body and body.count("_handle(stream, ") >= 7


def test_workspace(monkeypatch):
    monkeypatch.setattr(replay, "_dev_tensor", lambda t, name: t)
    ws = torch.empty(512, dtype=torch.uint8)
    assert replay._workspace(256, ws, torch.device("cpu"), "attention", None) is ws
    with pytest.raises(replay.C3Error):
        replay._workspace(256, ws, torch.device("cuda", 0), "attention", None)
    with pytest.raises(replay.C3Error):
        replay._workspace(1024, ws, torch.device("cpu"), "attention", None)
