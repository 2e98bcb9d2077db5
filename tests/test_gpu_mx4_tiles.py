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


# ---- dense products with an MX4 result -------------------------------------------------------

def _slack(xv, wv, b, h, K, act, gate_of):
    """The error of act(h), as for the smaller sizes: the sum's (K roundings at most, each of 2^-24
    of the mass, rarely in one direction) through an activation whose slope (swiglu: times the other
    half) is at most 1.13."""
    err = K ** 0.5 * 2.0 ** -23 * (xv.abs() @ wv.abs().t().contiguous() + b.abs().float()).double()
    if act == "swiglu":
        f = gate_of
        err = 1.13 * (err[:, :f] * h[:, f:].abs() + err[:, f:] * h[:, :f].abs())
    return 1.13 * err.max().item()


def _activated(h, act):
    if act == "swiglu":
        f = h.shape[1] // 2
        return h[:, :f] / (1.0 + torch.exp(-h[:, :f])) * h[:, f:]
    if act == "gelu":
        return h / (1.0 + torch.exp(-2.0 * 0.7978845608028654 * (h + 0.044715 * h ** 3)))
    return h


def _check_codes(got, h, block, slack):
    from test_gpu_mx4 import _check_requantized
    _check_requantized(got.double().cpu().numpy(), h.cpu().numpy(), block, slack)


def _some(n):
    """The first and last rows of n and every ninth (the oracle's rotation is slow)."""
    i = torch.arange(n, device="cuda")
    return i[(i < 40) | (i >= n - 40) | (i % 9 == 0)]


@pytest.mark.parametrize("act", [None, "gelu", "swiglu"])
@pytest.mark.parametrize("block", [0, 32, 64, 128])
@pytest.mark.parametrize("M,N,K,kernel", [(1001, 2048, 448, "128 x 128"), (2117, 2432, 1152, "256 x 128"),
                                          (8200, 1152, 64, "256 x 128")])
def test_requantized_tiles(clq, M, N, K, kernel, block, act):
    """Whole and ragged row tiles of every activation and rotation block; channels that end inside
    a tile where the activation leaves them to."""
    if act == "swiglu" and block == 128:
        pytest.skip("not a block of this activation")
    N += 64 if N == 2432 and act != "swiglu" and block != 128 else 0
    c, n = _units(), _div(N, 128)
    assert _div(M, 32) * n > 7 * c // 4 and (kernel == "128 x 128") == (_div(M, 128) * n <= c)
    x, w, b = _rand(M, M, K, scale=0.2), _rand(N, N, K, scale=K ** -0.5), _rand(3, N, dtype=BF16, scale=0.1)
    q, qw = clq.clq_mx4_quantize(x), clq.clq_mx4_quantize_weights(w, gated=act == "swiglu")
    o = clq.clq_mx4_linear_mx4(q, qw, b, act=act, block=block)
    xv, wv = _values(clq, q), _values(clq, qw)
    h = xv.double() @ wv.double().t().contiguous() + b.double()
    got = _values(clq, o)
    i = _some(M)
    _check_codes(got[i], _activated(h[i], act), block, _slack(xv, wv, b, h, K, act, N // 2))
    again = clq.clq_mx4_linear_mx4(q, qw, b, act=act, block=block)
    assert torch.equal(_values(clq, again), got)


# ---- grouped products ---------------------------------------------------------------------------

def _ids(seed, T, k, E, kind):
    g = torch.Generator().manual_seed(seed)
    if kind == "skew":   # a few experts with most of the tokens, some with none
        p = torch.exp(-torch.arange(E) / (E / 6.0))
        p[E // 2] = 0
        ids = torch.multinomial(p.expand(T, E), k, generator=g)
    else:
        ids = torch.rand(T, E, generator=g).argsort(1)[:, :k]
    ids = ids.to(torch.int32)
    if kind == "skew":
        ids[torch.rand(T, k, generator=g) < 0.05] = -1
    return ids


def _per_expert(clq, plan, q, qw, b):
    """(rows, fp64 result, sum of magnitudes) of every expert that has rows, padding left out."""
    xv, wv = _values(clq, q), _values(clq, qw)
    counts, first = plan.counts.tolist(), plan.offsets().tolist()
    for e, n in enumerate(counts):
        if n:
            v = xv[first[e]:first[e] + n]
            yield (slice(first[e], first[e] + n), v, wv[e], b[e],
                   v.double() @ wv[e].double().t().contiguous() + b[e].double(),
                   v.abs() @ wv[e].abs().t().contiguous() + b[e].abs().float())


# (tokens, experts of each, experts, rows of a tile)
PLANS = [(1500, 2, 40, 128, "even"), (1200, 3, 130, 128, "skew"), (3001, 2, 3, 256, "even"), (4500, 2, 7, 256, "skew"),
         (33500, 2, 130, 256, "skew")]


def _picked(T, k, E, N, split):
    """Rows of the tile that a grouped product of N channels takes (0: split over the k loop);
    split: whether it would be, by its own rule."""
    n, tiles = T * k, _div(N, 128)
    if split:
        return 0
    return 128 if n < 512 * E or (n // 128 + min(E, n)) * tiles <= _units() else 256


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("N,K", [(1280, 128), (1275, 448), (1280, 576)])
@pytest.mark.parametrize("T,k,E,rows,kind", PLANS)
def test_grouped_tiles(clq, T, k, E, rows, kind, N, K, dtype):
    units = T * k // 32 + E
    assert _picked(T, k, E, N, units * _div(N, 32) <= 3 * _units()) == rows
    bd = BF16 if dtype is BF16 else F16
    plan = clq.clq_expert_plan(_ids(T, T, k, E, kind).cuda(), E)
    x, w, b = _rand(T, T, K, dtype=bd), _rand(N, E, N, K, scale=K ** -0.5, dtype=bd), _rand(5, E, N, dtype=bd)
    q, qw = clq.clq_mx4_dispatch(x, plan), clq.clq_mx4_quantize_weights(w)
    del x, w
    buf = torch.full((plan.plan_rows + 1, _div(N, 8) * 8 + 8), 7.0, dtype=dtype, device="cuda")
    got = clq.clq_mx4_experts(q, plan, qw, b, dtype=dtype, out=buf[:-1, :N])
    for r, _, _, _, want, mass in _per_expert(clq, plan, q, qw, b):
        _within(got[r], want, mass, K, dtype)
    end = int(plan.offsets()[-1])
    assert (buf[:, N:] == 7).all() and (buf[end:] == 7).all()
    pad = torch.ones(plan.plan_rows, dtype=torch.bool, device="cuda")
    pad[plan.rows.flatten()[plan.rows.flatten() >= 0].long()] = False
    e_of = torch.searchsorted(plan.offsets().long(), torch.arange(end, device="cuda"), right=True) - 1
    assert torch.equal(got[:end][pad[:end]], b[e_of[pad[:end]]].to(dtype))   # (inputs of zeros)
    again = clq.clq_mx4_experts(q, plan, qw, b, dtype=dtype)
    assert torch.equal(again[:end], got[:end])


@pytest.mark.parametrize("act,block", [(None, 0), (None, 32), (None, 64), (None, 128), ("gelu", 0), ("gelu", 32),
                                       ("gelu", 64), ("gelu", 128), ("swiglu", 0), ("swiglu", 32), ("swiglu", 64)])
@pytest.mark.parametrize("N,K", [(1280, 448), (1280, 64)])
@pytest.mark.parametrize("T,k,E,rows,kind", PLANS[:4])
def test_grouped_requantized_tiles(clq, T, k, E, rows, kind, N, K, act, block):
    units, c = T * k // 32 + E, _units()
    N -= 64 if act != "swiglu" and block != 128 else 0   # channels that end inside a tile
    assert _picked(T, k, E, N, units * _div(N, 128) <= (c if act == "swiglu" else 7 * c // 4)) == rows
    plan = clq.clq_expert_plan(_ids(T, T, k, E, kind).cuda(), E)
    x, w, b = _rand(T, T, K, scale=0.2), _rand(N, E, N, K, scale=K ** -0.5), _rand(5, E, N, dtype=BF16, scale=0.1)
    q, qw = clq.clq_mx4_dispatch(x, plan), clq.clq_mx4_quantize_weights(w, gated=act == "swiglu")
    o = clq.clq_mx4_experts_mx4(q, plan, qw, b, act=act, block=block)
    got = _values(clq, o)
    parts, slack = [], 0.0
    for r, v, wv, be, h, _ in _per_expert(clq, plan, q, qw, b):
        i = _some(len(h))
        parts.append((got[r][i], _activated(h[i], act)))
        slack = max(slack, _slack(v, wv, be, h, K, act, N // 2))
    _check_codes(torch.cat([v for v, _ in parts]), torch.cat([h for _, h in parts]), block, slack)
    again = _values(clq, clq.clq_mx4_experts_mx4(q, plan, qw, b, act=act, block=block))
    end = int(plan.offsets()[-1])
    assert torch.equal(again[:end], got[:end])
