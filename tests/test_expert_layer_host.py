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


class _Recorder:
    """torch.cuda's device and graph contexts, in the order they are entered."""

    def __init__(self, monkeypatch):
        self.entered = []
        monkeypatch.setattr(torch.cuda, "device", lambda d: self._context(("device", d)))
        monkeypatch.setattr(torch.cuda, "graph", lambda g, stream=None: self._context(("graph", stream)))
        monkeypatch.setattr(torch.cuda, "Stream", lambda device: ("stream", device))
        monkeypatch.setattr(torch.cuda, "synchronize", lambda d=None: None)
        monkeypatch.setattr(torch.cuda, "CUDAGraph", _Graph)

    def _context(self, what):
        import contextlib

        @contextlib.contextmanager
        def run():
            self.entered.append(what)
            yield
        return run()


def test_a_capture_that_fails_leaves_the_one_before(monkeypatch):
    m = _layer(5)
    x_in, x_out, graph = m.x_in, m.x_out, m.graph
    _Recorder(monkeypatch)

    def fail(x):
        raise RuntimeError("no")

    m.forward = fail
    with pytest.raises(RuntimeError):
        m.capture(9)
    assert m.x_in is x_in and m.x_out is x_out and m.graph is graph
    m.replay(torch.ones(5, 64, dtype=torch.float16))
    assert graph.replays == 1


def test_capture_is_on_the_layers_device(monkeypatch):
    m, r = _layer(), _Recorder(monkeypatch)
    m.forward = lambda x: x + 1
    m.capture(3)
    # (a stream of its own: the graph context's may be another device's)
    assert r.entered == [("device", m.router.device), ("graph", ("stream", m.router.device))]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_process_without_tokens_gets_none_back(dtype):
    m = _layer()
    m.top_k, m.route = 2, {}
    y = m.forward(torch.zeros(0, 64, dtype=dtype))
    assert y.shape == (0, 64) and y.dtype == dtype
    for bad in (torch.zeros(0, 32, dtype=dtype), torch.zeros(0, 64), torch.zeros(0, dtype=dtype)):
        with pytest.raises(Exception):
            m.forward(bad)
