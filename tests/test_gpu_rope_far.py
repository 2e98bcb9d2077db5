"""Rotary positions as far as an int32 goes: the turn is that of position * freq itself, not of its fp64 rounding."""
import math
from fractions import Fraction

import pytest

torch = pytest.importorskip("torch")

from test_gpu_block import BF16, F16, F32, U, half_step

pytestmark = pytest.mark.gpu

# Machin's formula in whole numbers: pi to 100 digits
_ONE = 10 ** 110


def _arctan_inverse(n):
    total, term, k = 0, _ONE // n, 0
    while term:
        total += (-1) ** k * term // (2 * k + 1)
        term //= n * n
        k += 1
    return total


PI = Fraction(4 * (4 * _arctan_inverse(5) - _arctan_inverse(239)), _ONE)


@pytest.fixture(scope="module")
def clq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2509_24416_amd as m
    return m


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"\n[gpu case] {request.node.nodeid}", flush=True)
    yield


def near_whole_turns(p, n):
    """n frequencies (fp64) that take position p to within a ten-thousandth of a whole number of turns, and the
    angles that are left, exactly."""
    freqs, left = [], []
    for j in range(n):
        turns = int(Fraction(p) * Fraction(10 ** (-j / n)) / (2 * PI))
        f = float((turns * 2 * PI + Fraction(5 + j, 10 ** 5)) / Fraction(p))
        freqs.append(f)
        left.append(float(Fraction(p) * Fraction(f) - turns * 2 * PI))
    return freqs, left


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("inter", [True, False])
@pytest.mark.parametrize("p", [1, 1000003, 2 ** 31 - 1, 2.0 ** 31, 16777213.0])
def test_far_positions(clq, p, inter, t):
    """(1024, 0) turned by a small angle d: its second value is 1024 sin d, within the roundings of the argument (1 of
    it, 2 of its reduced form), the sine (4 units) and the product, relative to itself.  The angle that position * freq
    rounded to fp64 gives is off by up to 2^-53 of 2^31 and more, 2e-7: half a percent of the smallest value."""
    n = 32
    freqs, left = near_whole_turns(p, n)
    assert all(1e-5 < abs(d) < 1e-3 for d in left)
    pos = torch.tensor([[p], [-p]], dtype=F32 if isinstance(p, float) else torch.int32, device="cuda")
    x = torch.zeros(2, 1, 2 * n, dtype=t, device="cuda")
    first, second = (slice(0, None, 2), slice(1, None, 2)) if inter else (slice(0, n), slice(n, None))
    x[..., first] = 1024
    y = clq.clq_rope_axes(x, pos, torch.tensor(freqs, dtype=torch.float64, device="cuda"), (2 * n,), interleaved=inter)
    want = 1024 * torch.tensor([[math.sin(d) for d in left], [-math.sin(d) for d in left]], dtype=torch.float64)
    off = (y[:, 0, second].double().cpu() - want).abs()
    rel, _ = half_step(t)
    assert (off <= want.abs() * (rel + 8 * U)).all(), f"{float((off / want.abs()).max()):.3g}"
    assert (y[..., first] == 1024).all()   # (the cosine is 1 within 1e-6)
