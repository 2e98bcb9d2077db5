"""GPU parity of the MX4 quantizer and products against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import mx4 as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
UNIT = {F16: 2.0 ** -11, BF16: 2.0 ** -8}   # half a unit in the last place


@pytest.fixture(scope="module")
def clq():
    import paper_2509_24416_amd as m
    return m


def _rand(seed, *shape, dtype=F16, scale=1.0):
    """Gaussian rows with a few channels 50 times as large."""
    g = np.random.default_rng(seed)
    x = g.standard_normal(shape) * scale
    x[..., :: max(1, shape[-1] // 3)] *= 50.0
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def _np(t):
    return t.detach().float().cpu().double().numpy()


def _perm(seed, K):
    return np.random.default_rng(seed).permutation(K).astype(np.int32)


def _same(got, want):
    assert got.shape == want.shape
    assert np.array_equal(got, want, equal_nan=True), f"{(~((got == want) | (np.isnan(got) & np.isnan(want)))).sum()} values differ"


# ---- quantizer -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block", [0, 32, 64, 128])
@pytest.mark.parametrize("M,K", [(1, 128), (31, 256), (33, 384), (70, 1152), (5, 4608), (257, 640)])
def test_quantize_matches_oracle(clq, M, K, block, dtype):
    if block and K % block:
        pytest.skip("block does not divide K")
    x = _rand(M * K + block, M, K, dtype=dtype)
    q = clq.clq_mx4_quantize(x.cuda(), block=block)
    _same(_np(clq.clq_mx4_dequantize(q, torch.float32)), ref.quantize(_np(x), block))


@pytest.mark.parametrize("M,K,block", [(3, 64, 0), (3, 64, 32), (40, 192, 64), (2, 32768, 128), (9, 320, 32)])
def test_quantize_odd_widths(clq, M, K, block):
    x = _rand(K, M, K)
    q = clq.clq_mx4_quantize(x.cuda(), block=block)
    _same(_np(clq.clq_mx4_dequantize(q, torch.float32)), ref.quantize(_np(x), block))


@pytest.mark.parametrize("block", [0, 32, 64, 128])
def test_quantize_gathers_and_strides(clq, block):
    M, K, ld = 45, 1152, 1304
    wide = _rand(7, M, ld).cuda()
    perm = _perm(3, K)
    x = wide[:, 8:8 + K]   # 16-byte aligned view with a row stride of its own
    q = clq.clq_mx4_quantize(x, block=block, perm=torch.from_numpy(perm).cuda())
    _same(_np(clq.clq_mx4_dequantize(q, torch.float32)), ref.quantize(_np(x), block, perm))
    q = clq.clq_mx4_quantize(x, block=block)
    _same(_np(clq.clq_mx4_dequantize(q, torch.float32)), ref.quantize(_np(x), block))


@pytest.mark.parametrize("K", [64, 12288, 20480, 32768])
@pytest.mark.parametrize("shift", [0, 1])
def test_quantize_gathers_of_every_length(clq, K, shift):
    """Rows that fit LDS by four, rows that do not, and indices off 16-byte boundaries."""
    x, perm = _rand(K, 6, K, dtype=BF16), _perm(K, K)
    buf = torch.zeros(K + shift, dtype=torch.int32, device="cuda")
    buf[shift:] = torch.from_numpy(perm)
    q = clq.clq_mx4_quantize(x.cuda(), block=64, perm=buf[shift:])
    _same(_np(clq.clq_mx4_dequantize(q, torch.float32)), ref.quantize(_np(x), 64, perm))


def test_offsets_past_32_bits(clq):
    """Inputs and outputs of more than 2^32 bytes: the last rows are those of the last rows alone."""
    M, K = 70000, 32768
    x = torch.empty(M, K, dtype=F16, device="cuda")
    x[-40:] = torch.randn(40, K, device="cuda", dtype=F16)
    x[:-40] = 0
    v = clq.clq_mx4_dequantize(clq.clq_mx4_quantize(x, 64), BF16)
    assert torch.equal(v[-40:], clq.clq_mx4_dequantize(clq.clq_mx4_quantize(x[-40:], 64), BF16))
    assert (v[-140:-40] == 0).all()
    del x, v
    M, N = 300000, 8192
    x, w = torch.zeros(M, 64, dtype=F16, device="cuda"), torch.randn(N, 64, device="cuda", dtype=F16)
    x[-33:] = torch.randn(33, 64, device="cuda", dtype=F16)
    qw = clq.clq_mx4_quantize_weights(w)
    y = clq.clq_mx4_linear(clq.clq_mx4_quantize(x), qw)
    xv, wv = clq.clq_mx4_dequantize(clq.clq_mx4_quantize(x[-33:]), torch.float32), clq.clq_mx4_dequantize(qw, torch.float32)
    want, mass = xv.double() @ wv.double().t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    assert ((y[-33:].double() - want).abs() <= UNIT[F16] * want.abs() + 2.0 ** -18 * mass + 2.0 ** -25).all()
    assert (y[:-33:997] == 0).all() and (y[-34] == 0).all()


def test_quantize_every_rounding(clq):
    """Every fp16 magnitude up to 8 next to a 4 (scale 1): ties, saturation, both signs."""
    h = torch.arange(0, 0x4800 + 1, dtype=torch.int32).to(torch.int16).view(F16)
    h = torch.cat([h, -h])
    h = torch.cat([h, torch.zeros(-len(h) % 31, dtype=F16)]).view(-1, 31)
    x = torch.cat([torch.full((len(h), 1), 4.0, dtype=F16), h], 1)
    x = torch.cat([x, torch.zeros(-len(x) % 2, 32, dtype=F16)]).view(-1, 64)
    q = clq.clq_mx4_quantize(x.contiguous().cuda())
    _same(_np(clq.clq_mx4_dequantize(q, torch.float32)), ref.quantize(_np(x)))


def test_quantize_scales_over_the_range(clq):
    """A group of every binary magnitude bf16 has, from subnormals to the largest, and zeros."""
    g = np.random.default_rng(0)
    rows = []
    for e in range(-133, 128):
        rows.append(np.ldexp(g.uniform(-1.99, 1.99, 64), e))
    x = torch.from_numpy(np.array(rows + [np.zeros(64)]).astype(np.float32)).to(BF16)
    q = clq.clq_mx4_quantize(x.cuda())
    # (a product with a scale of 2^-126 may leave fp32's normal numbers, which are kept)
    _same(_np(clq.clq_mx4_dequantize(q, torch.float32)), ref.quantize(x.double().numpy()))


@pytest.mark.parametrize("block", [0, 64])
def test_quantize_marks_groups_that_are_not_finite(clq, block):
    x = _rand(1, 6, 256, dtype=BF16)
    x[0, 3], x[1, 70], x[2, 255], x[4, 100] = float("nan"), float("inf"), float("-inf"), 3e38
    x[4, 101] = 3e38
    got = _np(clq.clq_mx4_dequantize(clq.clq_mx4_quantize(x.cuda(), block=block), BF16))
    want = ref.quantize(x.double().numpy(), block)
    assert np.isnan(want[0]).sum() == (block or 32)
    _same(got, want)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("E,N,K,block", [(None, 100, 256, 64), (None, 192, 128, 0), (3, 128, 192, 32), (2, 64, 1152, 128)])
def test_weights(clq, E, N, K, block, gated):
    if gated and N % 64:
        pytest.skip("gated weights have a multiple of 64 rows")
    perm = _perm(5, K)
    w = _rand(N, *((E,) if E else ()), N, K, scale=K ** -0.5)
    qw = clq.clq_mx4_quantize_weights(w.cuda(), block=block, perm=torch.from_numpy(perm).cuda(), gated=gated)
    want = ref.quantize(_np(w), block, perm, divide=max(1, block))
    _same(_np(clq.clq_mx4_dequantize(qw, torch.float32)), want)
    # the same matrix from row-major codes and scale bytes
    e = ref.exponents(want)
    mag = np.abs(want) / np.ldexp(1.0, np.repeat(e, 32, -1))
    code = np.searchsorted(ref.GRID, mag).astype(np.uint8) | (np.signbit(want).astype(np.uint8) << 3)
    packed = torch.from_numpy(code[..., 0::2] | code[..., 1::2] << 4).cuda()
    # (a group may have rounded to a smaller exponent's range: any exact code serves)
    qp = clq.clq_mx4_pack_weights(packed, torch.from_numpy((e + 127).astype(np.uint8)).cuda(), block=block, gated=gated)
    _same(_np(clq.clq_mx4_dequantize(qp, torch.float32)), want)


def test_dequantize_types(clq):
    x = _rand(2, 9, 128)
    q = clq.clq_mx4_quantize(x.cuda())
    want = ref.quantize(_np(x))
    for t in (F16, BF16, torch.float32):
        _same(_np(clq.clq_mx4_dequantize(q, t)), want)


# ---- products ---------------------------------------------------------------------------

def _check_product(got, want, mass, K, dtype):
    """One rounding to dtype, and at most K roundings of a 24-bit sum of `mass` = sum |terms|."""
    err = np.abs(got - want)
    tol = UNIT[dtype] * np.abs(want) + K * 2.0 ** -24 * mass + 2.0 ** -25
    assert (err <= tol).all(), f"error {(err / tol).max():.3g} times the tolerance"


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,N,K,block,bias", [
    (1, 16, 64, 0, False), (1, 3456, 1152, 64, True), (2, 100, 128, 32, True), (31, 1, 192, 0, True),
    (33, 129, 320, 64, False), (64, 128, 256, 128, True), (100, 1000, 1216, 32, True), (257, 130, 448, 64, True),
    (300, 384, 4608, 128, False), (513, 72, 128, 64, True), (16, 4608, 768, 64, True), (5, 40, 32768, 64, True)])
def test_linear(clq, M, N, K, block, bias, dtype):
    if block and K % block:
        pytest.skip("block does not divide K")
    x, w = _rand(M + N, M, K, dtype=dtype), _rand(K, N, K, scale=K ** -0.5, dtype=dtype)
    b = _rand(9, N, dtype=dtype) if bias else None
    q = clq.clq_mx4_quantize(x.cuda(), block=block)
    qw = clq.clq_mx4_quantize_weights(w.cuda(), block=block)
    got = _np(clq.clq_mx4_linear(q, qw, None if b is None else b.cuda(), dtype=dtype))
    xv, wv = ref.quantize(_np(x), block), ref.quantize(_np(w), block, divide=max(1, block))
    want = xv @ wv.T + (0.0 if b is None else _np(b))
    _check_product(got, want, np.abs(xv) @ np.abs(wv).T + (0.0 if b is None else np.abs(_np(b))), K, dtype)


@pytest.mark.parametrize("M,N,K", [(1, 40, 128), (100, 131, 192), (70, 1152, 4608), (3000, 1000, 256)])
def test_linear_fp32_result(clq, M, N, K):
    """The sums as they are, on every kernel, ragged or not."""
    x, w, b = _rand(M, M, K), _rand(N, N, K, scale=K ** -0.5), _rand(5, N)
    q, qw = clq.clq_mx4_quantize(x.cuda(), 64), clq.clq_mx4_quantize_weights(w.cuda(), 64)
    y = clq.clq_mx4_linear(q, qw, b.cuda(), dtype=torch.float32)
    assert y.dtype == torch.float32 and y.shape == (M, N)
    xv, wv = ref.quantize(_np(x), 64), ref.quantize(_np(w), 64, divide=64)
    err = np.abs(_np(y) - (xv @ wv.T + _np(b)))
    assert (err <= K * 2.0 ** -24 * (np.abs(xv) @ np.abs(wv).T + np.abs(_np(b)))).all()


@pytest.mark.parametrize("M,N,K", [(64, 256, 256), (700, 3456, 1152), (2050, 1152, 4608), (4096, 4608, 320)])
def test_linear_large(clq, M, N, K):
    x, w = _rand(M, M, K), _rand(N, N, K, scale=K ** -0.5)
    q, qw = clq.clq_mx4_quantize(x.cuda(), block=64), clq.clq_mx4_quantize_weights(w.cuda(), block=64)
    got = _np(clq.clq_mx4_linear(q, qw))
    xv = torch.from_numpy(ref.quantize(_np(x), 64))
    wv = torch.from_numpy(ref.quantize(_np(w), 64, divide=64))
    _check_product(got, (xv @ wv.T).numpy(), (xv.abs() @ wv.abs().T).numpy(), K, F16)


@pytest.mark.parametrize("dtype", [F16, BF16, torch.float32])
@pytest.mark.parametrize("M,N,K", [(4100, 1152, 4608), (8195, 1147, 192), (20001, 288, 64), (40000, 90, 320), (40000, 57, 128)])
def test_linear_narrow_tiles(clq, M, N, K, dtype):
    """Tiles of 96 channels: whole and ragged, every length of the last eight stages' rest."""
    bd = BF16 if dtype is BF16 else F16
    x, w, b = _rand(M, M, K, dtype=bd), _rand(N, N, K, scale=K ** -0.5, dtype=bd), _rand(7, N, dtype=bd)
    q, qw = clq.clq_mx4_quantize(x.cuda(), 64), clq.clq_mx4_quantize_weights(w.cuda(), 64)
    buf = torch.full((M + 1, (N + 7) // 8 * 8 + 8), 7.0, dtype=dtype, device="cuda")
    got = clq.clq_mx4_linear(q, qw, b.cuda(), dtype=dtype, out=buf[:M, :N])
    xv, wv = clq.clq_mx4_dequantize(q, torch.float32).cpu(), clq.clq_mx4_dequantize(qw, torch.float32).cpu()
    want = (xv.double() @ wv.double().T + b.double()).numpy()
    mass = (xv.abs() @ wv.abs().T + b.abs().float()).numpy()
    if dtype is torch.float32:
        assert (np.abs(_np(got) - want) <= K * 2.0 ** -24 * mass).all()
    else:
        _check_product(_np(got), want, mass, K, dtype)
    assert (buf[:, N:] == 7).all() and (buf[M] == 7).all()


@pytest.mark.parametrize("M,N,K", [(43200, 4608, 1152), (20000, 1152, 4608), (30000, 3456, 192)])
def test_linear_many_tiles(clq, M, N, K):
    """Many rounds of workgroups under full memory load, several times over: a transfer that was
    not waited for shows here and not in a launch of a few tiles.  Against fp64 on the GPU."""
    x, w = torch.randn(M, K, device="cuda", dtype=F16), torch.randn(N, K, device="cuda", dtype=F16) * K ** -0.5
    q, qw = clq.clq_mx4_quantize(x, 64), clq.clq_mx4_quantize_weights(w, 64)
    xv, wv = clq.clq_mx4_dequantize(q, torch.float32), clq.clq_mx4_dequantize(qw, torch.float32)
    want = xv.double() @ wv.double().t().contiguous()
    mass = xv.abs() @ wv.abs().t().contiguous()
    tol = UNIT[F16] * want.abs() + K * 2.0 ** -24 * mass + 2.0 ** -25
    for i in range(5):
        got = clq.clq_mx4_linear(q, qw).double()
        assert ((got - want).abs() <= tol).all(), i


def test_linear_of_rotated_is_the_linear(clq):
    """The rotation is absorbed: the product approximates x . w^T."""
    x, w = _rand(1, 64, 1152), _rand(2, 256, 1152, scale=1152 ** -0.5)
    perm = torch.from_numpy(_perm(4, 1152)).cuda()
    got = _np(clq.clq_mx4_linear(clq.clq_mx4_quantize(x.cuda(), 64, perm),
                                 clq.clq_mx4_quantize_weights(w.cuda(), 64, perm)))
    want = _np(x) @ _np(w).T
    # 4-bit grids on both sides: about 12 % of a value each
    assert np.linalg.norm(got - want) < 0.25 * np.linalg.norm(want)


def test_linear_strided_output_and_reused_buffers(clq):
    x, w = _rand(1, 40, 256), _rand(2, 96, 256)
    q = clq.clq_mx4_quantize(_rand(3, 64, 256).cuda(), 32)
    clq.clq_mx4_quantize(x.cuda(), 32, out=q)
    qw = clq.clq_mx4_quantize_weights(w.cuda(), 32)
    want = clq.clq_mx4_linear(q, qw)
    buf = torch.full((42, 128), 7.0, dtype=F16, device="cuda")
    clq.clq_mx4_linear(q, qw, out=buf[:40, 16:112])
    assert torch.equal(buf[:40, 16:112], want)
    assert (buf[:, :16] == 7).all() and (buf[:, 112:] == 7).all() and (buf[40:] == 7).all()


def test_nan_groups_reach_only_their_rows(clq):
    x, w = _rand(1, 70, 512), _rand(2, 200, 512)
    x[33, 100], x[69, 511] = float("nan"), float("inf")
    qw = clq.clq_mx4_quantize_weights(w.cuda())
    got = _np(clq.clq_mx4_linear(clq.clq_mx4_quantize(x.cuda()), qw))
    bad = np.zeros(70, bool)
    bad[[33, 69]] = True
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    w[17, 3] = float("nan")
    got = _np(clq.clq_mx4_linear(clq.clq_mx4_quantize(_rand(1, 70, 512).cuda()),
                                 clq.clq_mx4_quantize_weights(w.cuda())))
    col = np.zeros(200, bool)
    col[17] = True
    assert np.isnan(got[:, col]).all() and np.isfinite(got[:, ~col]).all()


def test_linear_overflow_and_infinite_bias(clq):
    x, w = torch.full((3, 64), 6000.0, dtype=F16), torch.full((16, 64), 100.0, dtype=F16)
    b = torch.zeros(16, dtype=F16)
    b[5] = float("-inf")
    y = clq.clq_mx4_linear(clq.clq_mx4_quantize(x.cuda()), clq.clq_mx4_quantize_weights(w.cuda()), b.cuda()).cpu()
    assert torch.isposinf(y[:, :5]).all() and torch.isneginf(y[:, 5]).all()


# ---- products with an MX4 result -----------------------------------------------------------

def _check_requantized(got, h, block, slack):
    """got: the values of the MX4 result for h (fp64, activated, not yet rotated), whose error is
    at most slack.  A value within the slack of a boundary may take either side, and so may a
    group's scale."""
    v = ref.rotate(h, block).astype(np.float64)
    d = slack * max(1, block) ** 0.5 * 4 + np.abs(v) * 2.0 ** -20
    top, spread = np.abs(v).reshape(*v.shape[:-1], -1, 32).max(-1), d.reshape(*v.shape[:-1], -1, 32).max(-1)

    def ex(t):
        return np.where(t <= 0, -126, np.maximum(np.frexp(t)[1] - 3, -126))

    ok = np.zeros(v.shape, bool)
    for e in (ex(top - spread), ex(top + spread)):
        lo, hi = ref.on_grid(v - d, e), ref.on_grid(v + d, e)
        ok_e = ((got >= lo) & (got <= hi)).reshape(*v.shape[:-1], -1, 32).all(-1)
        ok |= np.repeat(ok_e, 32, -1)
    assert ok.all(), f"{(~ok).sum()} of {ok.size} values"
    # and hardly any of them needs the slack
    assert (got != ref.on_grid(v, ref.exponents(v))).mean() < 2e-3


@pytest.mark.parametrize("act", [None, "gelu", "swiglu"])
@pytest.mark.parametrize("block", [0, 32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(1, 128, 64), (37, 256, 192), (300, 640, 1152), (70, 4608, 256)])
def test_linear_mx4(clq, M, N, K, block, act):
    columns = N // 2 if act == "swiglu" else N
    if act == "swiglu" and block == 128 or block and columns % block:
        pytest.skip("not a block of this activation or width")
    x, w, b = _rand(M, M, K, scale=0.2), _rand(N, N, K, scale=K ** -0.5), _rand(3, N, dtype=BF16, scale=0.1)
    q, qw = clq.clq_mx4_quantize(x.cuda()), clq.clq_mx4_quantize_weights(w.cuda(), gated=act == "swiglu")
    o = clq.clq_mx4_linear_mx4(q, qw, b.cuda(), act=act, block=block)
    assert (o.rows, o.K, o.block) == (M, columns, block)
    xv, wv = ref.quantize(_np(x)), ref.quantize(_np(w))
    h = xv @ wv.T + _np(b)
    # the sum's error (K roundings at most, each of 2^-24 of the mass, rarely in one direction),
    # through an activation whose slope (swiglu: times the other half) is at most 1.13
    mass = np.abs(xv) @ np.abs(wv).T + np.abs(_np(b))
    err = np.sqrt(K) * 2.0 ** -23 * mass
    if act == "swiglu":
        f = N // 2
        err = 1.13 * (err[:, :f] * np.abs(h[:, f:]) + err[:, f:] * np.abs(h[:, :f]))
    _check_requantized(_np(clq.clq_mx4_dequantize(o, torch.float32)), ref.activate(h, act), block,
                       1.13 * err.max())


def test_mlp_through_both_products(clq):
    x, w1, w2 = _rand(1, 130, 256), _rand(2, 512, 256, scale=0.01), _rand(3, 192, 512, scale=0.05)
    b1, b2 = _rand(4, 512, scale=0.1), _rand(5, 192)
    h = clq.clq_mx4_linear_mx4(clq.clq_mx4_quantize(x.cuda(), 64), clq.clq_mx4_quantize_weights(w1.cuda(), 64),
                               b1.cuda(), act="gelu", block=32)
    y = _np(clq.clq_mx4_linear(h, clq.clq_mx4_quantize_weights(w2.cuda(), 32), b2.cuda()))
    hv = ref.gelu(ref.quantize(_np(x), 64) @ ref.quantize(_np(w1), 64, divide=64).T + _np(b1))
    want = ref.quantize(hv, 32) @ ref.quantize(_np(w2), 32, divide=32).T + _np(b2)
    # an fp16 rounding, and codes that fell on the other side of a boundary
    assert np.linalg.norm(y - want) < 3e-3 * np.linalg.norm(want)


# ---- streams and graphs ------------------------------------------------------------------------

def test_refused_calls_leave_their_output_alone(clq):
    x, w = _rand(1, 300, 1152).cuda(), _rand(2, 640, 1152).cuda()
    q, qw = clq.clq_mx4_quantize(x, 64), clq.clq_mx4_quantize_weights(w, 64)
    o = clq.clq_mx4_quantize(x[:70, :256], 32)
    want = clq.clq_mx4_dequantize(o)
    o.data.resize_(1 << 20)
    for call in (lambda: clq.clq_mx4_quantize(x[:, 1:65], 64, out=o), lambda: clq.clq_mx4_quantize(x, 48, out=o),
                 lambda: clq.clq_mx4_linear_mx4(q, qw, block=48, out=o)):
        with pytest.raises(clq.ClqError):
            call()
        assert (o.rows, o.K, o.block) == (70, 256, 32)
    assert torch.equal(clq.clq_mx4_dequantize(o), want)


def test_buffers_of_the_wrong_size_are_refused(clq):
    def u8(n):
        return torch.zeros(n, dtype=torch.uint8, device="cuda")

    clq.MX4(u8(2 * 512 * 2 + 512), 33, 64)
    clq.MX4Weight(u8(2 * 64 * 160), u8(2 * 2 * 512), 64, 320, experts=2)
    for make in (lambda: clq.MX4(u8(2 * 512 * 2 + 511), 33, 64), lambda: clq.MX4(u8(4096).half(), 33, 64),
                 lambda: clq.MX4(u8(8192)[::2], 33, 64),
                 lambda: clq.MX4Weight(u8(2 * 64 * 160 - 1), u8(2 * 2 * 512), 64, 320, experts=2),
                 lambda: clq.MX4Weight(u8(2 * 64 * 160), u8(2 * 2 * 512 - 1), 64, 320, experts=2),
                 lambda: clq.MX4Weight(u8(2 * 64 * 160), u8(2 * 2 * 512).cpu(), 64, 320, experts=2)):
        with pytest.raises(ValueError):
            make()


def test_side_stream(clq):
    x, w = _rand(1, 300, 1152).cuda(), _rand(2, 640, 1152).cuda()
    want = clq.clq_mx4_linear(clq.clq_mx4_quantize(x, 64), clq.clq_mx4_quantize_weights(w, 64))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    q = clq.clq_mx4_quantize(x, 64, stream=s)
    qw = clq.clq_mx4_quantize_weights(w, 64, stream=s)
    y = clq.clq_mx4_linear(q, qw, stream=s)
    s.synchronize()
    assert torch.equal(y, want)


def test_graph_replays(clq):
    w1, w2 = _rand(2, 512, 256, scale=0.05).cuda(), _rand(3, 256, 512, scale=0.05).cuda()
    q1, q2 = clq.clq_mx4_quantize_weights(w1, 64), clq.clq_mx4_quantize_weights(w2, 64)
    x = _rand(1, 90, 256).cuda()

    def step():
        h = clq.clq_mx4_linear_mx4(clq.clq_mx4_quantize(x, 64), q1, act="gelu", block=64)
        return clq.clq_mx4_linear(h, q2)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = step()
    for i in range(4):
        x.copy_(_rand(10 + i, 90, 256))
        g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, step()), i
