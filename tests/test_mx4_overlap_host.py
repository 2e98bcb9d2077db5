"""Outputs that a caller gives may lie beside the inputs, not in them (no GPU: what is accepted
ends where the launch's device is looked up)."""
import pytest
import torch

import paper_2509_24416_amd as clq


def _bytes(n=1 << 16):
    return torch.zeros(n, dtype=torch.uint8)


def _mx4(buf, at, rows=40, K=128):
    return clq.MX4(buf[at:at + 64 * 64 + 2 * 256], rows, K)


def _weight(codes, scales):
    return clq.MX4Weight(codes, scales, 128, 128)


def _calls(out, q, w, plan):
    yield lambda: clq.clq_mx4_linear_mx4(q, w, out=out)
    yield lambda: clq.clq_mx4_experts_mx4(q, plan, w, out=out)


def _plan():
    return clq.ExpertPlan(torch.zeros(4, dtype=torch.int32), 1, 1, None, 40, 0)


class _Accepted(Exception):
    pass


@pytest.fixture
def accepting(monkeypatch):
    def stop():
        raise _Accepted

    monkeypatch.setattr("paper_2509_24416_amd.mx4._current_device", stop)


def test_an_mx4_result_that_overlaps_its_operands_is_refused(accepting):
    size = 64 * 64 + 2 * 256
    buf, plan = _bytes(), _plan()
    q = _mx4(buf, 2 * size)
    w = _weight(buf[4 * size:4 * size + 128 * 64], buf[8 * size:8 * size + 4 * 256])
    for at, bad in ((0, False), (size, False), (size + 16, True), (2 * size - 16, True), (2 * size, True),
                    (2 * size + 16, True), (3 * size - 16, True), (3 * size, False), (3 * size + 16, True),
                    (4 * size + 64, True), (4 * size + 128 * 64, False), (7 * size + 16, True),
                    (8 * size + 4 * 256, False)):
        for call in _calls(_mx4(buf, at), q, w, plan):
            with pytest.raises(ValueError if bad else _Accepted, match="output" if bad else None):
                call()


def test_pieces_of_rows():
    from paper_2509_24416_amd.mx4 import _meet
    a = (1000, 5, 100, 40)                       # five pieces of 40 bytes, 100 apart
    for at, want in ((900, False), (960, False), (961, True), (1000, True), (1039, True), (1040, False), (1060, False), (1061, True),
                     (1440, False), (1439, True), (1500, False)):
        assert _meet(a, (at, 1, 40, 40)) == _meet((at, 1, 40, 40), a) == want, at
    assert _meet(a, (0, 1, 5000, 5000)) and _meet((1060, 3, 100, 41), a)
    assert not _meet(a, (1040, 5, 100, 60)) and not _meet((1040, 5, 100, 60), a)   # the other columns of one matrix
    assert not _meet(a, (1440, 7, 100, 60)) and not _meet(a, (640, 3, 100, 100)) and _meet(a, (640, 4, 100, 100))
    assert _meet((1000, 1, 512, 40), (1039, 1, 64, 40)) and not _meet((1000, 1, 512, 40), (1040, 1, 64, 40))
    # every placement of two small sets of pieces, byte by byte
    def covered(at, rows, pitch, width):
        return {at + r * pitch + i for r in range(rows) for i in range(width)}
    for at in range(0, 60):
        for rows, width in ((1, 3), (2, 7), (3, 10)):
            x, y = (20, 3, 10, 4), (at, rows, 10, width)
            assert _meet(x, y) == bool(covered(*x) & covered(*y)), (x, y)


def test_weights_reach_as_far_as_their_matrices(accepting):
    """What lies behind them in a larger buffer is the caller's."""
    buf, plan = _bytes(), _plan()
    q, size = _mx4(buf, 0), 64 * 64 + 2 * 256
    codes, scales = buf[16384:], buf[40960:]
    for at, bad in ((16384 + 128 * 64, False), (16384 + 128 * 64 - 16, True), (40960 + 4 * 256, False),
                    (40960 + 4 * 256 - 16, True), (40960 - size, False)):
        for call in _calls(_mx4(buf, at), q, _weight(codes, scales), plan):
            with pytest.raises(ValueError if bad else _Accepted):
                call()
    # several experts' matrices
    two = clq.MX4Weight(codes, scales, 100, 128, experts=2)
    plan.experts = 2
    for at, bad in ((16384 + 2 * 128 * 64 - 16, True), (16384 + 2 * 128 * 64, False), (40960 + 2 * 4 * 256 - 16, True),
                    (40960 + 2 * 4 * 256, False)):
        with pytest.raises(ValueError if bad else _Accepted):
            clq.clq_mx4_experts_mx4(q, plan, two, out=_mx4(buf, at))
