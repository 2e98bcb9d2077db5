"""Host logic of the expert layer's graph (no GPU: stand-ins for the operators and the graph)."""
import pytest
import torch

from paper_2509_24416_amd.experts import ExpertMLP


class _Graph:
    def __init__(self):
        self.replays = 0

    def replay(self):
        self.replays += 1


def _layer(tokens=None, hidden=64):
    """A layer without weights, as if captured for so many tokens."""
    m = object.__new__(ExpertMLP)
    m.router, m.graph = torch.zeros(4, hidden), None
    if tokens is not None:
        m.x_in, m.graph = torch.zeros(tokens, hidden, dtype=torch.float16), _Graph()
        m.x_out = m.x_in + 1
    return m


def test_replay_takes_the_captured_shape_and_type_only():
    m = _layer(5)
    x = torch.ones(5, 64, dtype=torch.float16)
    assert m.replay(x) is m.x_out and m.graph.replays == 1 and torch.equal(m.x_in, x)
    for bad in (x[:1] * 2, x[:4] * 2, x[0] * 2, torch.ones(1, 1).half(), x.float() * 2, x.bfloat16() * 2):
        with pytest.raises(ValueError, match="captured"):
            m.replay(bad)
    assert m.graph.replays == 1 and torch.equal(m.x_in, x)
