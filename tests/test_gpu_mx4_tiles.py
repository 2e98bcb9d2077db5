"""The MX4 tile kernels themselves: every rest of the k loop, under load.

Sizes that few workgroups would do go to other kernels, so every test first counts the
workgroups that keep those away."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
UNIT = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 0.0}   # half a unit in the last place


@pytest.fixture(scope="module")
def clq():
    import paper_2509_24416_amd as m
    return m


def _units():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _div(a, b):
    return (a + b - 1) // b


def _rand(seed, *shape, dtype=F16, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(*shape, device="cuda", generator=g) * scale
    x[..., :: max(1, shape[-1] // 3)] *= 50.0
    return x.to(dtype)


def _values(clq, q):
    return clq.clq_mx4_dequantize(q, F32)


def _within(got, want, mass, K, dtype):
    """One rounding to dtype (of a result that may itself be a half unit of fp16's subnormals off)
    and at most K roundings of a 24-bit sum of `mass` = sum |terms|."""
    tol = UNIT[dtype] * want.abs() + K * 2.0 ** -24 * mass + (0.0 if dtype is F32 else 2.0 ** -25)
    assert ((got.double() - want).abs() <= tol).all()


# stages of 64 codes: eight to a turn of the loop, up to seven after it
@pytest.mark.parametrize("stages", [1, 2, 3, 4, 5, 6, 7, 8, 9, 12, 14, 15, 23, 31])
@pytest.mark.parametrize("M,N,dtype,kernel", [
    (30000, 1152, F16, "256 x 128"), (40000, 90, BF16, "256 x 96"), (2000, 2000, F16, "128 x 128")])
def test_every_rest_of_the_k_loop(clq, M, N, dtype, kernel, stages):
    c, rows = _units(), _div(M, 256)
    assert _div(M, 64) * _div(N, 64) > 2 * c                       # not split over the k loop
    if _div(M, 128) * _div(N, 128) <= c:
        picked = "128 x 128"
    else:
        picked = "256 x 96" if rows * _div(N, 96) <= _div(rows * _div(N, 128), c) * c else "256 x 128"
    assert picked == kernel
    K = 64 * stages
    x, w, b = _rand(stages, M, K, dtype=dtype), _rand(N, N, K, scale=K ** -0.5, dtype=dtype), _rand(3, N, dtype=dtype)
    q, qw = clq.clq_mx4_quantize(x), clq.clq_mx4_quantize_weights(w)
    xv, wv = _values(clq, q), _values(clq, qw)
    want = xv.double() @ wv.double().t().contiguous() + b.double()
    mass = xv.abs() @ wv.abs().t().contiguous() + b.abs().float()
    first = None
    for _ in range(5):
        got = clq.clq_mx4_linear(q, qw, b, dtype=dtype)
        _within(got, want, mass, K, dtype)
        first = got if first is None else first
        assert torch.equal(got, first)
