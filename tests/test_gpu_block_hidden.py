"""The hidden values of an MLP whose caller names no type: they reach the next quantizer in 32 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_block import BF16, F16, F32, U, act64, gen, operands, randn, rotated64

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


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("M,K,N,bits", [(1, 64, 64, 8), (45, 192, 320, 4), (777, 128, 1152, 8)])
def test_hidden_values_are_quantized_unrounded(clq, M, K, N, bits, act):
    """Codes of the activated product against its definition: h is off by S (the product's 3 roundings, behind a
    slope under 1.13, the activation's 2^-20 of its value or 2^-22), which a block's sum passes on; the rotation's 6
    stages add a rounding of the block's sum each; then half a step, 2 roundings of the scale and what moves the
    code's argument.  Values rounded to 16 bits ahead of the rotation are off by 2^-11 of a block's sum."""
    g = gen(M + N)
    q, xs, qw, p = operands(clq, g, M, K, N, bits)
    bias = randn(g, N, dtype=F16)
    h = clq.clq_a8_linear_act(q, xs, qw, bias, act=act)
    q2, xs2 = clq.clq_rotate_quant_act8(h, 64)
    y = act64(p + bias.double(), act)
    S = 1.13 * 3 * U * (p.abs() + bias.double().abs()) + 2.0 ** -20 * y.abs() + 2.0 ** -22
    v, total = rotated64(y, None, 64)
    E = S.view(M, -1, 64).sum(2).amax(1, keepdim=True) + 6 * U * total
    top, scale = v.abs().amax(1, keepdim=True), xs2.double().unsqueeze(1)
    assert ((scale - top / 127).abs() <= E / 127 + 3 * U * top / 127).all()
    off = (clq.clq_unswizzle_act8(q2, M, N).double() * scale - v).abs()
    assert (off <= scale / 2 + 2 * E + 4 * U * top).all(), f"{float((off - scale / 2).max() / top.max()):.3g}"
    assert h.dtype is F32 and torch.equal(h, clq.clq_a8_linear_act(q, xs, qw, bias, act=act, dtype=F32))


def test_types_of_results(clq):
    """A type that is named, or given with `out` or a residual, stays; without an activation it is fp16, and behind one
    too where a row is longer than the quantizer of fp32 takes."""
    g = gen(3)
    q, xs, qw, _ = operands(clq, g, 5, 64, 64, 8)
    call = clq.clq_a8_linear_act
    assert call(q, xs, qw).dtype is F16
    for act in ("gelu", "silu"):
        assert call(q, xs, qw, act=act, dtype=F16).dtype is F16
        assert call(q, xs, qw, act=act, residual=randn(g, 5, 64, dtype=BF16)).dtype is BF16
        assert call(q, xs, qw, act=act, out=torch.empty(5, 64, dtype=F16, device="cuda")).dtype is F16
    for N, want in ((16384, F32), (16448, F16)):
        _, _, wide, _ = operands(clq, g, 1, 64, N, 8)
        h = call(q, xs, wide, act="silu")
        assert h.dtype is want
        codes, scale = clq.clq_rotate_quant_act8(h, 64)
        assert scale.isfinite().all() and codes.numel() == clq.clq_act8_bytes(5, N)


@pytest.mark.parametrize("t", [F16, BF16, F32])
def test_the_quantizer_takes_them(clq, t):
    """clq_rotate_quant_act8 of bf16 and fp32 is clq_quantize_act8: columns gathered, buffers and a stream of the
    caller's."""
    g = gen(4)
    x = randn(g, 70, 640, dtype=t, scale=3)
    perm = torch.randperm(640, device="cuda", generator=g).to(torch.int32)
    want, scales = clq.clq_quantize_act8(x, 128, perm)
    out, scale_out = torch.full_like(want, 9), torch.full_like(scales, math.nan)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q, xs = clq.clq_rotate_quant_act8(x, 128, perm, out=out, scale_out=scale_out, stream=s)
    s.synchronize()
    assert q.data_ptr() == out.data_ptr() and xs.data_ptr() == scale_out.data_ptr()
    assert torch.equal(q, want) and torch.equal(xs, scales)
