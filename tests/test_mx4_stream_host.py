"""A stream of another device than the tensors' is refused (no GPU: neither is made current)."""
import pytest
import torch

from paper_2509_24416_amd import mx4


class _Stream:
    def __init__(self, index):
        self.device = torch.device("cuda", index)


def test_a_stream_of_another_device_is_refused(monkeypatch):
    current = []
    monkeypatch.setattr(torch.cuda, "stream", lambda s: current.append(s))
    monkeypatch.setattr(torch.cuda, "device", lambda d: current.append(d))
    with pytest.raises(ValueError, match="stream"):
        mx4._elsewhere(torch.device("cuda", 0), _Stream(1))
    assert not current
    s = _Stream(1)
    mx4._elsewhere(torch.device("cuda", 1), s)
    mx4._elsewhere(torch.device("cuda", 2), None)
    assert current == [s, torch.device("cuda", 2)]
