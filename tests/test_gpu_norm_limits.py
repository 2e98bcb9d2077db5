"""The norm of rows as large as its fp32 sum of squares holds, and beyond."""
import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_block import BF16, F32, NORM, check_codes, close, gen, norm64

pytestmark = pytest.mark.gpu


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


def rows(g, K, t):
    """Four rows of one magnitude and random signs: an ordinary one, one whose squares add up to a little under 2^128 (by
    3%, type's rounding included less than 4), one a little over, and the type's largest numbers."""
    limit = 2.0 ** 64 / math.sqrt(K)
    size = torch.tensor([3.0, limit * (1 - 2.0 ** -6), limit * (1 + 2.0 ** -6), 0.0], device="cuda", dtype=torch.float64).to(t)
    size[3] = torch.finfo(t).max
    sums = K * size.double() ** 2
    assert 0.95 < sums[1] / 2.0 ** 128 < 0.99 and 1.01 < sums[2] / 2.0 ** 128 < 1.05
    sign = torch.randint(0, 2, (4, K), device="cuda", generator=g) * 2 - 1
    return size.unsqueeze(1) * sign.to(t)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("t", [BF16, F32])
@pytest.mark.parametrize("K", [64, 1152, 8256, 16384])
def test_sums_of_squares_up_to_2_128(clq, K, t, residual):
    g = gen(K)
    x = rows(g, K, t)
    r, x = (x, torch.zeros_like(x)) if residual else (None, x)
    want = norm64(x, r, None)[1]
    want[2:] = 0
    y = clq.clq_rms_norm(x, None, r, dtype=F32)
    if residual:
        y, s = y
        assert torch.equal(s, r)
    close(y, want, want.abs() * NORM)
    q, xs, *_ = clq.clq_rms_norm_act8(x, 64, None, r)
    # (the last row's rotation passes fp32's range: its scale is none)
    assert xs[2] == 0 and not xs[3] > 0
    check_codes(clq, q, xs[:2], want[:2], None, 64, K)
    assert (clq.clq_dequantize_act8(q, xs, K, dtype=F32)[2] == 0).all()


def test_heads(clq):
    """A head's norm ahead of its turn: the same limit over the head's columns."""
    g = gen(5)
    x = rows(g, 64, BF16).view(4, 1, 64)
    pos = torch.zeros(4, 1, dtype=torch.int32, device="cuda")   # (a turn by nothing)
    y = clq.clq_rope_axes(x, pos, clq.clq_rope_freqs((32,)), (32,), weight=torch.ones(64, device="cuda"))
    want = x.double().sign().flatten(1)
    want[2:] = 0
    close(y.flatten(1), want, want.abs() * NORM)
