"""The workspaces that the bindings bring themselves, on the CPU: two calls that are under way at the same time do not
get the same memory."""
import torch

from paper_2602_06935_amd import binding


def test_every_call_has_its_own_workspace(monkeypatch):
    monkeypatch.setattr(binding, "_current_device", lambda: None)
    monkeypatch.setattr(binding, "_current_stream_handle", lambda device: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    like = torch.zeros(1)
    first, second = binding._workspace(like, 3000, 0), binding._workspace(like, 2000, 0)
    assert first.numel() >= 3000 and second.numel() >= 2000
    assert first.data_ptr() != second.data_ptr()


def test_the_stream_is_that_of_the_tensors_device(monkeypatch):
    """A call on another GPU than the current one goes to that GPU's current stream."""
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_current_stream_handle", lambda device: 100 + device)
    assert binding._stream_handle(None, torch.device("cuda", 1)) == 101
    assert binding._stream_handle(None, torch.device("cuda", 0)) == 100
    assert binding._stream_handle(77, torch.device("cuda", 1)) == 77
