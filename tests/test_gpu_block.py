"""RMS norm, rotary positions and the 8-bit linear's epilogue against their definitions in 64 bits.

Tolerances are sums of roundings: half a step of the output's type, plus what the fp32 arithmetic of each
formula can lose (U = 2^-24, one fp32 rounding; each test says how many it counts)."""
import dataclasses
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
EPS = 1e-6


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


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32, scale=1.0):
    return (scale * torch.randn(*shape, device="cuda", generator=g)).to(dtype)


def strided(t, pad=8):
    """The same values in rows with `pad` further columns of NaN."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + pad), math.nan, device=t.device, dtype=t.dtype)
    wide[..., :t.shape[-1]] = t
    return wide[..., :t.shape[-1]]


def half_step(t):
    """Half a step of a type relative to a value, and of its smallest numbers."""
    return torch.finfo(t).eps / 2, torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def close(got, want, slack, what=""):
    """got = want rounded to its type, from a value that is off by up to `slack` (of want's shape)."""
    rel, least = half_step(got.dtype)
    off = (got.double() - want).abs()
    allowed = (want.abs() + slack) * rel + slack + least
    bad = ~(off <= allowed)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / allowed).nan_to_num().max()):.3g} times"


def by_sample(w, M):
    w = w.double()
    return w.expand(M, -1) if w.dim() == 1 else w.repeat_interleave(M // w.shape[0], 0)


def norm64(x, r, w, eps=EPS):
    s = x.double() if r is None else x.double() + r.double()
    n = s / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    return s, n if w is None else n * by_sample(w, x.shape[0])


# The factor of a row: a sum of squares over K values of s (each off by U where a residual is added, counted
# twice in the square) in a chain of 16 per lane, at most 16 partials and 6 exchanges, so 40 roundings and the
# 2; halved by the root; the mean, eps, root and reciprocal add 4.  Then s, weight and factor: 3.
NORM = 28 * U


@pytest.mark.parametrize("M,K,xt,rt,wt,samples", [
    (1, 64, F16, None, None, 1), (1, 1152, F16, F16, F16, 1), (2, 8, BF16, None, F32, 2), (3, 72, F16, F32, F16, 3),
    (31, 1160, BF16, BF16, BF16, 1), (33, 520, F16, BF16, F32, 3), (100, 4096, BF16, None, F16, 2), (6, 8192, F16, F32, BF16, 2),
    (5, 8200, BF16, F16, F16, 1), (9, 1152, F32, F32, F32, 3), (64, 200, F32, F16, None, 1), (12, 9216, F32, None, BF16, 2), (3, 16384, F16, BF16, None, 1), (70, 16376, BF16, F32, F32, 7), (1030, 136, F16, F16, F16, 2)])
def test_norm(clq, M, K, xt, rt, wt, samples):
    g = gen(M * K)
    x = strided(randn(g, M, K, dtype=xt, scale=3))
    r = None if rt is None else strided(randn(g, M, K, dtype=rt, scale=5), 16)
    w = None if wt is None else 1 + randn(g, samples, K, dtype=wt, scale=0.3)
    w = w[0] if w is not None and samples == 1 else w
    s, n = norm64(x, r, w)
    for yt in (None, F32, F16):
        y = clq.clq_rms_norm(x, w, r, EPS, dtype=yt)
        if r is not None:
            y, total = y
            assert total.dtype is rt
            close(total, s, s.abs() * U, "sum")
        assert y.dtype is (yt or xt) and y.shape == (M, K)
        close(y, n, n.abs() * NORM, f"norm as {y.dtype}")


def test_norm_in_place_and_given_buffers(clq):
    g = gen(1)
    x, r, w = randn(g, 77, 1152, dtype=F16), randn(g, 77, 1152, dtype=F32), 1 + randn(g, 1152, dtype=F16, scale=0.1)
    y, s = clq.clq_rms_norm(x, w, r)
    x2, r2 = x.clone(), r.clone()
    y2, s2 = clq.clq_rms_norm(x2, w, r2, out=x2, sum_out=r2)
    assert y2 is x2 and s2 is r2 and torch.equal(y2, y) and torch.equal(s2, s)
    out, total = strided(torch.empty_like(x)), strided(torch.empty_like(r), 24)
    y3, s3 = clq.clq_rms_norm(x, w, r, out=out, sum_out=total)
    assert torch.equal(y3, y) and torch.equal(s3, s)
    for t, pad in ((out, 8), (total, 24)):   # the columns behind a row stay what they were
        wide = t.as_strided((77, 1152 + pad), (1152 + pad, 1))
        assert wide[:, 1152:].isnan().all()
    r4 = r.clone()
    q, xs, s4 = clq.clq_rms_norm_act8(x, 64, w, r4, sum_out=r4)
    assert s4 is r4 and torch.equal(s4, s)


def hadamard(b):
    i = torch.arange(b)
    bits = i.unsqueeze(0) & i.unsqueeze(1)
    odd = sum((bits >> j) & 1 for j in range(8)) % 2
    return (1.0 - 2.0 * odd.double()).cuda()


def rotated64(n, perm, block):
    n = n if perm is None else n[:, perm.long()]
    blocks = n.reshape(n.shape[0], -1, block)
    return (blocks @ hadamard(block)).flatten(1), blocks.abs().sum(2).amax(1, keepdim=True)


def check_codes(clq, q, xs, n, perm, block, K, what=""):
    """A value v of the rotated row and the row's maximum are off by E at most: each stage of a block adds a
    rounding of sums no larger than the block's sum of magnitudes.  The scale is then off by E / 127 and 2
    roundings, a code by half a step and what moves its argument, and |code| <= 127."""
    M = n.shape[0]
    v, total = rotated64(n, perm, block)
    E = (math.log2(block) + 28) * U * total
    top = v.abs().amax(1, keepdim=True)
    scale = xs.double().unsqueeze(1)
    assert ((scale - top / 127).abs() <= E / 127 + 3 * U * top / 127).all(), what
    codes = clq.clq_unswizzle_act8(q, M, K).double()
    assert codes.abs().max() <= 127
    off = (codes * scale - v).abs()
    allowed = scale / 2 + 2 * E + 4 * U * top
    assert (off <= allowed).all(), f"{what}: {float((off / allowed).max()):.4g}"


@pytest.mark.parametrize("M,K,block,xt,rt,wt,samples,perm", [
    (1, 64, 64, F16, None, None, 1, False), (1, 1152, 64, F16, F16, F16, 1, False), (2, 1152, 128, BF16, F32, F32, 2, True),
    (45, 1216, 32, BF16, F32, BF16, 1, True), (33, 64, 32, F16, BF16, F16, 3, True), (600, 4096, 128, BF16, None, F16, 2, False),
    (9, 8192, 64, F16, F32, F16, 1, True), (66, 1152, 64, F32, F32, F32, 6, True), (40, 320, 32, F32, F16, F16, 10, False),
    (33, 8320, 128, F32, None, F32, 3, False), (5, 8256, 64, F16, F16, F16, 5, True), (40, 12288, 128, BF16, BF16, None, 1, False),
    (3, 16384, 32, F16, F32, F32, 1, True), (2049, 320, 64, F16, F16, F16, 1, True), (1030, 2048, 32, BF16, None, None, 1, False)])
def test_norm_act8(clq, M, K, block, xt, rt, wt, samples, perm):
    g = gen(M + K)
    x = strided(randn(g, M, K, dtype=xt, scale=2))
    x[:, K // 3] *= 50   # an outlier channel
    r = None if rt is None else strided(randn(g, M, K, dtype=rt, scale=4))
    w = None if wt is None else 1 + randn(g, samples, K, dtype=wt, scale=0.3)
    w = w[0] if w is not None and samples == 1 else w
    p = torch.randperm(K, device="cuda", generator=g).to(torch.int32) if perm else None
    s, n = norm64(x, r, w)
    q, xs, *total = clq.clq_rms_norm_act8(x, block, w, r, EPS, perm=p)
    assert q.numel() == clq.clq_act8_bytes(M, K) and xs.shape == (M,)
    check_codes(clq, q, xs, n, p, block, K)
    if r is not None:
        close(total[0], s, s.abs() * U, "sum")
    # rows that pad the last unit hold zero codes, as the quantizer's do
    rows = (M + 31) // 32 * 32
    assert (clq.clq_unswizzle_act8(q, rows, K)[M:] == 0).all()
    codes = clq.clq_unswizzle_act8(q, M, K).double()
    for t in (F16, BF16, F32):
        d = clq.clq_dequantize_act8(q, xs, K, dtype=t)
        close(d, codes * xs.double().unsqueeze(1), codes.abs() * xs.double().unsqueeze(1) * U, f"dequantized to {t}")
    q2, xs2 = clq.clq_rms_norm_act8(x, block, w, r, EPS, perm=p, out=torch.full_like(q, 77), scale_out=torch.empty_like(xs))[:2]
    assert torch.equal(q2, q) and torch.equal(xs2, xs)


@pytest.mark.parametrize("perm", [False, True])
@pytest.mark.parametrize("M,K,block", [(1, 64, 64), (1, 4608, 64), (45, 1216, 32), (600, 1152, 128), (70, 8192, 32), (40, 12288, 64)])
def test_quantizer(clq, M, K, block, perm):
    """fp16: bit for bit clq_rotate_quant_act8.  bf16 and fp32: the values' exact rotation within the roundings of
    its stages."""
    g = gen(M + K)
    p = torch.randperm(K, device="cuda", generator=g).to(torch.int32) if perm else None
    x = strided(randn(g, M, K, dtype=F16, scale=3))
    q, xs = clq.clq_quantize_act8(x, block, p)
    want, scales = clq.clq_rotate_quant_act8(x.contiguous(), block, p)
    assert torch.equal(q, want) and torch.equal(xs, scales)
    for t in (BF16, F32):
        x = strided(randn(g, M, K, dtype=t, scale=3))
        x[0] = 0
        q, xs = clq.clq_quantize_act8(x, block, p)
        assert xs[0] == 0 and (clq.clq_unswizzle_act8(q, M, K)[0] == 0).all()
        check_codes(clq, q, xs, x.double(), p, block, K, str(t))
        rows = (M + 31) // 32 * 32
        assert (clq.clq_unswizzle_act8(q, rows, K)[M:] == 0).all()
        q2, xs2 = clq.clq_quantize_act8(x, block, p, out=torch.full_like(q, 5), scale_out=torch.empty_like(xs))
        assert torch.equal(q2, q) and torch.equal(xs2, xs)
    x = randn(g, M, K)
    x[M - 1, 3] = math.nan
    assert clq.clq_quantize_act8(x, block)[1][M - 1].isnan()


def test_norm_of_zeros_infinities_and_nans(clq):
    g = gen(3)
    x = randn(g, 12, 256, dtype=F16)
    x[1] = 0
    x[3, 7] = math.inf
    x[4, 8] = math.nan
    x[6, 3], x[6, 4] = math.inf, -math.inf
    x[7, :4] = torch.tensor([math.inf, math.inf, math.inf, -math.inf])
    x[8] = 6e-8    # the smallest fp16 number, far under eps
    x[9, :] = 65504
    y = clq.clq_rms_norm(x, dtype=F32)
    want = norm64(x, None, None)[1]
    want[3], want[6], want[7] = 0, 0, 0
    want[3, 7], want[4], want[6, 3:5], want[7, :4] = math.nan, math.nan, math.nan, math.nan
    assert torch.equal(y.isnan(), want.isnan())
    close(y.nan_to_num(7.0), want.nan_to_num(7.0), want.nan_to_num(7.0).abs() * NORM)
    for block in (32, 64, 128):
        q, xs = clq.clq_rms_norm_act8(x, block)
        d = clq.clq_dequantize_act8(q, xs, 256)
        for row in (3, 4, 6, 7):
            assert xs[row].isnan() and d[row].isnan().all()
        rest = [0, 1, 2, 5, 8, 9, 10, 11]
        assert xs[1] == 0 and (d[1] == 0).all() and not d[rest].isnan().any() and (xs[rest] >= 0).all()
        v = rotated64(norm64(x[rest], None, None)[1], None, block)[0]
        assert ((clq.clq_dequantize_act8(q, xs, 256, dtype=F32)[rest].double() - v).abs() <= 0.51 * xs[rest].double().unsqueeze(1)).all()


@pytest.mark.parametrize("t", [BF16, F32])
def test_rows_of_tiny_values(clq, t):
    """8-bit rows down to a maximum of 2^-119; smaller ones are zeros."""
    g = gen(17)
    x = randn(g, 6, 256)
    for row, power in enumerate((-60, -99, -105, -112, -128, -140)):
        x[row] = x[row].clamp(-4, 4) * 2.0 ** power
    x = x.to(t)
    for q, xs, n in ((*clq.clq_quantize_act8(x, 64), x.double()),
                     (*clq.clq_rms_norm_act8(x, 64, eps=2.0 ** -126), norm64(x, None, None, 2.0 ** -126)[1])):
        codes = clq.clq_unswizzle_act8(q, 6, 256)
        assert (xs[4:] == 0).all() and (codes[4:] == 0).all()
        assert (xs[:4] > 0).all() and (codes[:4].abs().amax(1) == 127).all()
        check_codes(clq, q, xs[:4], n[:4], None, 64, 256, str(t))


def rope64(x, pos, freqs, axes, interleaved, inverse, w, eps=EPS):
    v, n = x.double(), freqs.numel()
    if w is not None:
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * w.double()
    axis = torch.repeat_interleave(torch.arange(len(axes)), torch.tensor([d // 2 for d in axes])).cuda()
    angle = (pos.double()[:, axis] * freqs).repeat(x.shape[0] // pos.shape[0], 1).unsqueeze(1)
    c, s = torch.cos(angle), torch.sin(angle) * (-1 if inverse else 1)
    a, b = (v[..., 0:2 * n:2], v[..., 1:2 * n:2]) if interleaved else (v[..., :n], v[..., n:2 * n])
    p, q = a * c - b * s, b * c + a * s
    size = (a.abs() + b.abs())
    join = (lambda u, z: torch.stack((u, z), -1).flatten(-2)) if interleaved else (lambda u, z: torch.cat((u, z), -1))
    return torch.cat((join(p, q), v[..., 2 * n:]), -1), torch.cat((join(size, size), v[..., 2 * n:].abs()), -1)


# A turned value: the fp32 argument in half turns (U of pi, 4 U), sine and cosine (4 units), two products and
# a sum: 12 U of |a| + |b|.  A head's norm: 8 squares in a chain (16 of a pair of chunks), 6 exchanges, halved,
# and 7 more.
ROPE, HEAD_NORM = 12 * U, 19 * U


@pytest.mark.parametrize("M,tokens,H,D,axes,t,inter,inverse,norm,pt", [
    (1, 1, 1, 8, (8,), F16, True, False, None, torch.int32), (2, 1, 32, 72, (24, 24, 24), F16, True, False, None, torch.int32),
    (54, 27, 32, 72, (24, 24, 24), BF16, False, False, "head", torch.int32), (33, 33, 3, 128, (16, 56, 56), F16, True, True, "one", F32),
    (33, 11, 5, 128, (16, 56, 56), BF16, False, False, "one", torch.int32), (10, 5, 7, 96, (32, 32), F16, False, True, "head", F32),
    (300, 300, 1, 64, (16, 24, 24), F16, True, False, None, torch.int32), (4, 4, 2, 256, (64, 64, 64, 64), F16, False, False, "head", F32),
    (7, 7, 64, 160, (44, 42, 42), BF16, True, False, "head", torch.int32), (7, 7, 9, 160, (44, 42, 42), F16, False, False, None, torch.int32),
    (5, 1, 4, 256, (2, 4, 2), F16, False, False, "one", torch.int32), (2100, 1050, 2, 40, (8,), BF16, True, False, "head", torch.int32),
    (9, 3, 8, 24, (10, 14), F16, False, False, None, F32)])
def test_rope(clq, M, tokens, H, D, axes, t, inter, inverse, norm, pt):
    g = gen(M + D)
    x = randn(g, M, H * D + 64, dtype=t, scale=2)[:, 24:24 + H * D].view(M, H, D)
    if pt is F32:
        pos = 100 * randn(g, tokens, len(axes))
    else:
        pos = torch.randint(-5000, 100000, (tokens, len(axes)), device="cuda", generator=g).to(torch.int32)
        pos[0] = torch.tensor([2 ** 31 - 1, -2 ** 31, 0, 1][:len(axes)])
    freqs = clq.clq_rope_freqs(axes)
    w = None if norm is None else 1 + randn(g, *((D,) if norm == "one" else (H, D)), dtype=F32 if D == 160 else t, scale=0.3)
    want, size = rope64(x, pos, freqs, axes, inter, inverse, w)
    slack = (ROPE if norm is None else ROPE + HEAD_NORM) * size
    y = clq.clq_rope_axes(x, pos, freqs, axes, interleaved=inter, inverse=inverse, weight=w)
    assert y.dtype is t and y.is_contiguous()
    close(y, want, slack)
    if norm is None:   # columns that no axis turns are copied
        assert torch.equal(y[..., sum(axes):], x[..., sum(axes):])
    # in place, on rows that hold other columns: those stay
    wide = randn(g, M, H * D + 16, dtype=t)
    before = wide.clone()
    inside = wide[:, 8:8 + H * D].view(M, H, D)
    inside.copy_(x)
    assert clq.clq_rope_axes(inside, pos, freqs, axes, interleaved=inter, inverse=inverse, weight=w, out=inside) is inside
    assert torch.equal(inside, y) and torch.equal(wide[:, :8], before[:, :8]) and torch.equal(wide[:, -8:], before[:, -8:])
    # heads first
    heads = torch.empty(H, M, D, dtype=t, device="cuda").transpose(0, 1)
    clq.clq_rope_axes(x.transpose(0, 1).contiguous().transpose(0, 1), pos, freqs, axes, interleaved=inter, inverse=inverse,
                      weight=w, out=heads)
    assert torch.equal(heads, y)


def test_rope_undone_by_its_inverse(clq):
    """The inverse is the transpose: it takes a turn back, and is its gradient (checked by differences
    along a direction, in the inner product that defines it)."""
    g = gen(5)
    axes, pos = (16, 24, 24), torch.randint(0, 50, (40, 3), device="cuda", generator=g).to(torch.int32)
    x, d = randn(g, 40, 4, 64, dtype=F16), randn(g, 40, 4, 64, dtype=F16)
    freqs = clq.clq_rope_freqs(axes)
    for inter in (True, False):
        y = clq.clq_rope_axes(x, pos, freqs, axes, interleaved=inter)
        back = clq.clq_rope_axes(y, pos, freqs, axes, interleaved=inter, inverse=True)
        size = x.double().abs() + 4   # |a| + |b| of a pair, of values under 4.5
        assert ((back.double() - x.double()).abs() <= (2 * 2.0 ** -11) * 2 * size).all()
        # <R x, d> = <x, R^T d>: roundings of 2^-11 of each product's values
        z = clq.clq_rope_axes(d, pos, freqs, axes, interleaved=inter, inverse=True)
        left, right = (y.double() * d.double()).sum(), (x.double() * z.double()).sum()
        assert (left - right).abs() <= 2.0 ** -11 * ((y.double() * d.double()).abs().sum() + (x.double() * z.double()).abs().sum())


def test_rope_rows_past_the_last_position_repeat(clq):
    g = gen(6)
    axes = (24, 24, 24)
    x = randn(g, 3 * 50, 5, 72, dtype=F16)
    pos = torch.randint(0, 50, (50, 3), device="cuda", generator=g).to(torch.int32)
    f = clq.clq_rope_freqs(axes)
    y = clq.clq_rope_axes(x, pos, f, axes)
    assert torch.equal(y, clq.clq_rope_axes(x, pos.repeat(3, 1), f, axes))


def operands(clq, g, M, K, N, bits, block=64):
    x, W = randn(g, M, K, dtype=F16, scale=2), randn(g, N, K, dtype=F16, scale=K ** -0.5)
    q, xs = clq.clq_rotate_quant_act8(x, block)
    qw = (clq.clq_quantize_weights8 if bits == 8 else clq.clq_quantize_weights)(W, block)
    a = clq.clq_unswizzle_act8(q, M, K).double()
    if bits == 8:
        b = clq.clq_unswizzle_weights8(qw).double()
    else:
        c = clq.clq_unswizzle_weights(qw).to(torch.int16)
        c = torch.stack((c & 15, c >> 4), -1).flatten(1)
        b = torch.where(c > 7, c - 16, c).double()
    return q, xs, qw, (a @ b.t()) * xs.double().unsqueeze(1) * qw.w_scale.double()


def act64(h, act):
    if act == "gelu":
        return h * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (h + 0.044715 * h ** 3))
    return h * torch.sigmoid(h) if act == "silu" else h


def check_linear(clq, q, xs, qw, p, bias, act, gate, res, dtype, **kw):
    """Ahead of the activation 3 roundings of the product and the bias (its slope is under 1.13); the
    activation 2^-20 of its value or 2^-22; gate and residual a rounding each."""
    M = p.shape[0]
    h = p if bias is None else p + bias.double()
    slack = 3 * U * (p.abs() + (0 if bias is None else bias.double().abs()))
    y = act64(h, act)
    if act:
        slack = 1.13 * slack + 2.0 ** -20 * y.abs() + 2.0 ** -22
    if gate is not None:
        gate = by_sample(gate, M)
        y, slack = y * gate, slack * gate.abs() + U * (y * gate).abs()
    if res is not None:
        y = y + res.double()
        slack = slack + U * y.abs()
    got = clq.clq_a8_linear_act(q, xs, qw, bias, act=act, gate=gate_arg(kw), residual=res, dtype=dtype, out=kw.get("out"))
    close(got, y, slack)
    return got


def gate_arg(kw):
    return kw.get("gate_tensor")


@pytest.mark.parametrize("M,K,N,bits,bt,act,gt,samples,res,dtype", [
    (1, 64, 16, 8, None, None, None, 1, False, F16), (1, 1152, 4608, 8, F16, "gelu", None, 1, False, F16),
    (2, 4608, 1152, 4, BF16, "silu", F32, 2, True, F32), (777, 1216, 1000, 4, F16, "silu", BF16, 1, True, BF16),
    (96, 192, 1, 8, F16, "gelu", F16, 3, True, F16), (130, 128, 129, 8, BF16, None, F32, 2, True, BF16),
    (300, 64, 515, 8, None, "gelu", None, 1, True, F32), (64, 32768, 72, 8, F16, None, None, 1, True, F16),
    (1300, 640, 1304, 8, F16, "gelu", F16, 13, True, F16), (2048, 1152, 1152, 4, F16, None, F16, 2, True, F16),
    (5000, 320, 1160, 8, F16, "silu", F32, 2, True, BF16), (8192, 256, 4608, 4, BF16, "gelu", None, 1, False, BF16),
    (6000, 64, 2000, 8, F16, "gelu", BF16, 6, True, F32), (2304, 1152, 3456, 8, F16, None, None, 1, False, F16),
    (4100, 128, 1152, 4, F16, None, F32, 4, True, F32), (3000, 192, 3456, 4, F16, "gelu", F16, 3, True, F16),
    (4200, 320, 1100, 4, BF16, "silu", F16, 7, True, BF16), (4200, 448, 1101, 8, F16, "gelu", BF16, 4200, True, F32),
    (32, 2048, 512, 8, F16, None, F32, 32, True, BF16), (31, 64, 33, 4, None, "silu", F16, 31, True, F32)])
def test_linear_act(clq, M, K, N, bits, bt, act, gt, samples, res, dtype):
    g = gen(M + N)
    q, xs, qw, p = operands(clq, g, M, K, N, bits)
    bias = None if bt is None else randn(g, N, dtype=bt)
    gate = None if gt is None else randn(g, samples, N, dtype=gt)
    gate = gate[0].contiguous() if gate is not None and samples == 1 else gate
    r = randn(g, M, N, dtype=dtype, scale=3) if res else None
    y = check_linear(clq, q, xs, qw, p, bias, act, gate, r, dtype, gate_tensor=gate)
    assert y.shape == (M, N) and y.dtype is dtype
    if res:
        # in place, and from rows at another distance
        pad = (N + 7) // 8 * 8 + 8
        wide = torch.full((M, pad), math.nan, dtype=dtype, device="cuda")
        inside = wide[:, :N]
        inside.copy_(r)
        assert clq.clq_a8_linear_act(q, xs, qw, bias, act=act, gate=gate, residual=inside, out=inside) is inside
        assert torch.equal(inside, y) and wide[:, N:].isnan().all()
        odd = torch.empty(M, N + 3, dtype=dtype, device="cuda")[:, 1:N + 1]
        odd.copy_(r)
        assert torch.equal(clq.clq_a8_linear_act(q, xs, qw, bias, act=act, gate=gate, residual=odd), y)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,K,N", [(40, 64, 64), (40, 1152, 200), (900, 1152, 1152), (1536, 192, 4608), (3000, 128, 3456),
                                   (9000, 128, 3456)])
def test_without_activation_it_is_the_linear(clq, M, K, N, bits):
    """The same fma of the same sums, whichever kernel a shape gets: clq_a8_linear rounds it to fp16 at once,
    this one to fp32 first.  The two roundings part only where the fp32 one (U of the value, behind those of
    sum, scale and fma: 4 U) lands on the other side of the middle between two neighbouring fp16 values."""
    g = gen(M)
    q, xs, qw, p = operands(clq, g, M, K, N, bits)
    bias = randn(g, N, dtype=F16)
    a, b = clq.clq_a8_linear_act(q, xs, qw, bias), clq.clq_a8_linear(q, xs, qw, bias)
    differ = a != b
    middle, h = (a.double() + b.double()) / 2, p + bias.double()
    assert ((middle - h).abs()[differ] <= 4 * U * (p.abs() + bias.double().abs())[differ]).all()
    # (a value in 2^13 lies so near a middle where sum and bias are its size)
    assert differ.double().mean() < 2.0 ** -10


@pytest.mark.parametrize("t", [F16, BF16, F32])
@pytest.mark.parametrize("M,K,N", [(5, 128, 13), (700, 512, 333), (700, 64, 2900), (6000, 128, 1001), (3000, 192, 3457)])
def test_residuals_of_any_alignment(clq, M, K, N, t):
    """Rows without padding, from an odd element on, and padded ones: the same result, bit for bit."""
    g = gen(M + N)
    q, xs, qw, _ = operands(clq, g, M, K, N, 8)
    padded = torch.full((M, (N + 7) // 8 * 8), math.nan, device="cuda", dtype=t)[:, :N]
    padded[:] = randn(g, M, N, dtype=t)
    gate = randn(g, N, dtype=F16)
    want = clq.clq_a8_linear_act(q, xs, qw, act="silu", gate=gate, residual=padded)
    assert want.isfinite().all()
    tight = padded.contiguous()
    odd = torch.full((M * N + 1,), math.nan, device="cuda", dtype=t)[1:].view(M, N)
    odd[:] = padded
    for res in (tight, odd):
        assert torch.equal(clq.clq_a8_linear_act(q, xs, qw, act="silu", gate=gate, residual=res), want)


def test_linear_act_far_from_zero(clq):
    """Activations at large arguments: no overflow in between."""
    g = gen(9)
    q, xs, qw, p = operands(clq, g, 64, 64, 64, 8)
    for size in (30.0, 3e3, 6e4):
        bias = torch.linspace(-size, size, 64, device="cuda").to(F16)
        for act in ("gelu", "silu"):
            y = clq.clq_a8_linear_act(q, xs, qw, bias, act=act, dtype=F32)
            assert y.isfinite().all()
            check_linear(clq, q, xs, qw, p, bias, act, None, None, F32)


def mlp(clq, x, r, n, w1, b1, w2, b2, gate):
    q, xs, s = clq.clq_rms_norm_act8(x, 64, n, r)
    h = clq.clq_a8_linear_act(q, xs, w1, b1, act="gelu", dtype=F32)
    q, xs = clq.clq_quantize_act8(h, 64)
    return clq.clq_a8_linear_act(q, xs, w2, b2, gate=gate, residual=s), s


def attention_inputs(clq, s, w, b, pos, freqs, axes, heads, hw):
    """Queries, keys and values of a block: norm, projection, head norms and positions in place."""
    q, xs = clq.clq_rms_norm_act8(s, 64)
    qkv = clq.clq_a8_linear_act(q, xs, w, b)
    hidden = qkv.shape[1] // 3
    qk = qkv[:, :2 * hidden].view(len(s), 2 * heads, hidden // heads)
    clq.clq_rope_axes(qk, pos, freqs, axes, weight=hw, out=qk)
    return qkv


def block_inputs(clq, seed, M=270, K=576, F=1152, heads=8):
    g = gen(seed)
    x, r = randn(g, M, K, dtype=F16, scale=2), randn(g, M, K, dtype=F16, scale=3)
    n, gate = 1 + randn(g, 2, K, dtype=F16, scale=0.2), randn(g, 2, K, dtype=F16)
    quant = lambda N, C: clq.clq_quantize_weights8(randn(g, N, C, dtype=F16, scale=C ** -0.5), 64)  # noqa: E731
    pos = torch.stack(torch.meshgrid(torch.arange(3), torch.arange(5), torch.arange(9), indexing="ij"), -1).view(-1, 3)
    return (x, r, n, quant(F, K), randn(g, F, dtype=F16), quant(K, F), randn(g, K, dtype=F16), gate), (
        quant(3 * K, K), randn(g, 3 * K, dtype=F16), pos.to(torch.int32).cuda(), clq.clq_rope_freqs((24, 24, 24)), (24, 24, 24),
        heads, 1 + randn(g, 2 * heads, K // heads, dtype=F16, scale=0.2))


def test_a_block_step_by_step(clq):
    """The MLP half and the attention's inputs as one run; every step against its definition on what the
    step before it gave."""
    (x, r, n, w1, b1, w2, b2, gate), (w, b, pos, freqs, axes, heads, hw) = block_inputs(clq, 11)
    M, K = x.shape
    y, s = mlp(clq, x, r, n, w1, b1, w2, b2, gate)
    s64, n64 = norm64(x, r, n)
    close(s, s64, s64.abs() * U)
    q, xs, _ = clq.clq_rms_norm_act8(x, 64, n, r)
    check_codes(clq, q, xs, n64, None, 64, K)

    def product(q, xs, qw):
        return (clq.clq_unswizzle_act8(q, M, qw.K).double() @ clq.clq_unswizzle_weights8(qw).double().t()) * \
            xs.double().unsqueeze(1) * qw.w_scale.double()

    h = check_linear(clq, q, xs, w1, product(q, xs, w1), b1, "gelu", None, None, F32)
    q, xs = clq.clq_quantize_act8(h, 64)
    check_codes(clq, q, xs, h.double(), None, 64, h.shape[1])
    last = check_linear(clq, q, xs, w2, product(q, xs, w2), b2, None, gate, s, F16, gate_tensor=gate)
    assert torch.equal(last, y)
    qkv = attention_inputs(clq, y, w, b, pos, freqs, axes, heads, hw)
    q, xs = clq.clq_rms_norm_act8(y, 64)
    plain = clq.clq_a8_linear_act(q, xs, w, b)   # (the projection of that run, bit for bit)
    want, size = rope64(plain[:, :2 * K].view(M, 2 * heads, -1), pos, freqs, axes, True, False, hw)
    close(qkv[:, :2 * K].view(M, 2 * heads, -1), want, (ROPE + HEAD_NORM) * size)
    assert torch.equal(qkv[:, 2 * K:], plain[:, 2 * K:])


def test_captured_runs_replay(clq):
    """Two graphs of a block's halves with other work between their replays: every replay equals the
    eager run."""
    first, second = block_inputs(clq, 12)
    x, r = first[0], first[1]
    mlp(clq, *first)
    attention_inputs(clq, x, *second)
    torch.cuda.synchronize()
    graphs = []
    for f in (lambda: mlp(clq, *first), lambda: attention_inputs(clq, r, *second)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = f()
        graphs.append((graph, out))
    for seed in range(4):
        g = gen(20 + seed)
        x.copy_(randn(g, *x.shape, dtype=F16))
        r.copy_(randn(g, *r.shape, dtype=F16))
        want = (*mlp(clq, *first), attention_inputs(clq, r, *second))
        torch.cuda.synchronize()
        graphs[0][0].replay()
        graphs[1][0].replay()
        graphs[0][0].replay()
        torch.cuda.synchronize()
        got = (*graphs[0][1], graphs[1][1])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_streams(clq):
    """Calls given a stream run there, and two at once do not meet."""
    first, _ = block_inputs(clq, 13)
    other, _ = block_inputs(clq, 14)
    want, want2 = mlp(clq, *first)[0], mlp(clq, *other)[0]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    a.wait_stream(torch.cuda.current_stream())
    b.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(5):
        for st, args in ((a, first), (b, other)):
            with torch.cuda.stream(st):
                got.append(mlp(clq, *args)[0])
    x, r, n = first[:3]
    y, s = clq.clq_rms_norm(x, n, r, stream=a)
    z = clq.clq_rope_axes(x.view(len(x), 8, 72), torch.zeros(1, 1, dtype=torch.int32, device="cuda"),
                          clq.clq_rope_freqs((72,)), (72,), stream=b)
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, [want, want2] * 5))
    assert torch.equal(y, clq.clq_rms_norm(x, n, r)[0]) and torch.equal(z.view_as(x), x)


def test_offsets_past_32_bits(clq):
    """Rows whose elements lie past 2^31 of their matrix's start (and past 2^32 bytes)."""
    g = gen(16)
    M, ld = 70000, 32768
    big = torch.empty(M, ld, dtype=F16, device="cuda")
    x, r, y = big[:, :64], big[:, 1024:1088], big[:, 2048:2112]
    x.copy_(randn(g, M, 64, dtype=F16))
    r.copy_(randn(g, M, 64, dtype=F16))
    want64 = norm64(x, r, None)[1]
    want, total = clq.clq_rms_norm(x.contiguous(), None, r.contiguous())
    got, s = clq.clq_rms_norm(x, None, r, out=y, sum_out=big[:, 4096:4160])
    assert torch.equal(got, want) and torch.equal(s, total)
    q, xs, _ = clq.clq_rms_norm_act8(x, 64, None, r, sum_out=r)
    d = clq.clq_dequantize_act8(q, xs, 64, out=big[:, 8192:8256])
    assert torch.equal(d, clq.clq_dequantize_act8(q, xs, 64)) and torch.equal(r, total)
    check_codes(clq, q, xs, want64, None, 64, 64)
    pos, f = torch.arange(M, dtype=torch.int32, device="cuda").unsqueeze(1), clq.clq_rope_freqs((64,))
    turned = clq.clq_rope_axes(x.unsqueeze(1), pos, f, (64,), out=big[:, 16384:16448].unsqueeze(1))
    assert torch.equal(turned, clq.clq_rope_axes(x.contiguous().unsqueeze(1), pos, f, (64,)))
    W = clq.clq_quantize_weights8(randn(g, 64, 64, dtype=F16), 64)
    lin = clq.clq_a8_linear_act(q, xs, W, residual=r, out=big[:, 30000:30064])
    assert torch.equal(lin, clq.clq_a8_linear_act(q, xs, W, residual=total))


def test_captured_with_gathered_rows(clq):
    """Gathered rows need more LDS than a launch has by itself: set up in a capture as well."""
    g = gen(17)
    x, p = randn(g, 40, 8192, dtype=F16), torch.randperm(8192, device="cuda", generator=g).to(torch.int32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, xs = clq.clq_rms_norm_act8(x, 128, perm=p)
    for seed in range(3):
        x.copy_(randn(gen(seed), 40, 8192, dtype=F16))
        want = clq.clq_rms_norm_act8(x, 128, perm=p)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, want[0]) and torch.equal(xs, want[1])


def test_binding_refusals(clq):
    g = gen(15)
    x = randn(g, 8, 128, dtype=F16)
    wide = randn(g, 16, 128, dtype=F16)
    r = randn(g, 8, 128)
    flat = torch.empty(4096, dtype=F16, device="cuda")
    with pytest.raises(TypeError, match="X"):
        clq.clq_rms_norm(r.double())
    with pytest.raises(TypeError, match="X"):
        clq.clq_rms_norm([1.0])
    for bad in (x.t(), x[0], x.unsqueeze(0)):
        with pytest.raises(ValueError, match="2-D"):
            clq.clq_rms_norm(bad)
    for f in (lambda **k: clq.clq_rms_norm(x, **k), lambda **k: clq.clq_dequantize_act8(*clq.clq_quantize_act8(x, 64), 128, **k)):
        with pytest.raises(TypeError, match="dtype"):
            f(dtype=torch.float64)
    for bad, kw in (("weight", dict(weight=wide[0, :64])), ("weight", dict(weight=wide[0, 0])), ("samples", dict(weight=wide[:3])), ("residual", dict(residual=r[:4])),
                    ("without a residual", dict(sum_out=r)), ("sum_out", dict(residual=r, sum_out=r[:4])),
                    ("overlaps", dict(out=wide[4:12], residual=wide[8:])), ("overlaps", dict(residual=wide[:8], sum_out=wide[4:12])),
                    ("overlaps", dict(out=flat[:1024].view(8, 128), residual=flat.as_strided((8, 128), (256, 1), 512))),
                    ("overlaps", dict(weight=flat[512:640], out=flat[:1024].view(8, 128)))):
        with pytest.raises(ValueError, match=bad):
            clq.clq_rms_norm(x, **kw)
    with pytest.raises(ValueError, match="overlaps"):
        clq.clq_rms_norm(wide[:8], out=wide[1:9])
    with pytest.raises(ValueError, match="overlaps"):   # both results in one place
        clq.clq_rms_norm(x, residual=x.clone(), out=wide[:8], sum_out=wide[:8])
    with pytest.raises(clq.ClqError):
        clq.clq_rms_norm(x, eps=0.0)
    with pytest.raises(clq.ClqError):
        clq.clq_rms_norm_act8(x, 48)
    with pytest.raises(ValueError, match="perm"):
        clq.clq_rms_norm_act8(x, 64, perm=torch.arange(64, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="too small"):
        clq.clq_rms_norm_act8(x, 64, out=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="scale_out"):
        clq.clq_rms_norm_act8(x, 64, scale_out=torch.empty(4, device="cuda"))
    assert clq.clq_rms_norm_act8(x, 64, scale_out=torch.empty(20, device="cuda"))[1].shape == (8,)
    with pytest.raises(ValueError, match="overlaps"):
        clq.clq_rms_norm_act8(flat[:1024].view(8, 128), 64, out=flat.view(torch.uint8))
    total = torch.zeros(8, 128, device="cuda")   # (zeros: a gather of column 0)
    with pytest.raises(ValueError, match="overlaps"):
        clq.clq_rms_norm_act8(x, 64, residual=r, sum_out=total, perm=total[7].view(torch.int32))
    for theta in (0.0, -2.0, math.inf, math.nan):
        with pytest.raises(ValueError, match="theta"):
            clq.clq_rope_freqs((64,), theta)
    h, f = x.view(8, 2, 64), clq.clq_rope_freqs((64,))
    pos = torch.zeros(8, 1, dtype=torch.int32, device="cuda")
    for bad, args in (("positions", (pos.repeat(1, 2), f, (64,))), ("repeat", (pos[:3], f, (64,))), ("freqs", (pos, f[:16], (64,))),
                      ("axes", (pos, f, (63,))), ("a head has", (pos, clq.clq_rope_freqs((128,)), (128,)))):
        with pytest.raises(ValueError, match=bad):
            clq.clq_rope_axes(h, *args)
    with pytest.raises(ValueError, match="weight"):
        clq.clq_rope_axes(h, pos, f, (64,), weight=wide[0])
    with pytest.raises(ValueError, match="overlaps"):
        clq.clq_rope_axes(wide[:8].view(8, 2, 64), pos, f, (64,), out=wide[4:12].view(8, 2, 64))
    with pytest.raises(clq.ClqError):   # all rows in one place
        clq.clq_rope_axes(h, pos, f, (64,), out=flat.as_strided((8, 2, 64), (64, 64, 1)))
    q, xs, qw, _ = operands(clq, g, 8, 128, 64, 8)
    res = randn(g, 8, 64, dtype=F16)
    for bad, kw in (("act", dict(act="swiglu")), ("bias", dict(bias=x[0])), ("gate", dict(gate=x[:2])),
                    ("samples", dict(gate=randn(g, 3, 64, dtype=F16))), ("residual", dict(residual=res[:4])),
                    ("overlaps", dict(out=flat[:512].view(8, 64), residual=flat[64:576].view(8, 64)))):
        with pytest.raises(ValueError, match=bad):
            clq.clq_a8_linear_act(q, xs, qw, **kw)
    with pytest.raises(clq.ClqError):
        clq.clq_a8_linear_act(q, xs, clq.clq_qweight_f6(clq.clq_quantize_weights(randn(g, 64, 128, dtype=F16), 64)))
    for bits in (4, 8):   # buffers without the rows that pad them to 64, of another type
        _, _, odd, _ = operands(clq, g, 8, 128, 40, bits)
        assert clq.clq_a8_linear_act(q, xs, odd).shape == (8, 40)
        for change in (dict(wq=odd.wq[:40 * 128 * bits // 8]), dict(wq=odd.wq.view(torch.int32)), dict(w_scale=odd.w_scale[:39]),
                       dict(w_scale=odd.w_scale.half())):
            with pytest.raises(ValueError, match="weights"):
                clq.clq_a8_linear_act(q, xs, dataclasses.replace(odd, **change))
    with pytest.raises(TypeError, match="residual"):
        clq.clq_a8_linear_act(q, xs, qw, residual=res, dtype=F32)
    with pytest.raises(ValueError, match="Xq8"):
        clq.clq_a8_linear_act(q[:64], xs, qw)
