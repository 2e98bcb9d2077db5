"""GPU parity of the expert layer: routing, plan, grouped products, combination."""
import numpy as np
import pytest
import torch

from oracle import mx4 as ref

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def clq():
    import paper_2509_24416_amd as m
    return m


def _np(t):
    return t.detach().float().cpu().double().numpy()


def _check_route(clq, x, k, exact_ties=False, **kw):
    dev = {n: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for n, v in kw.items()}
    ids, w = clq.clq_expert_route(x.cuda(), k, **dev)
    ids, w = ids.cpu().numpy(), _np(w)
    want_ids, want_w, rank = ref.route(_np(x), k, **kw)
    assert ids.shape == want_ids.shape and ids.min() >= 0 and ids.max() < x.shape[1]
    assert all(len(set(r)) == k for r in ids)
    if exact_ties:
        assert np.array_equal(ids, want_ids)
    # a choice may differ only between ranks that fp32 does not tell apart: a few roundings
    got_r, want_r = np.take_along_axis(rank, ids, -1), np.take_along_axis(rank, want_ids, -1)
    same = ids == want_ids
    assert (same | (np.abs(got_r - want_r) <= 8 * 2.0 ** -24 * (1 + np.abs(want_r)))).all()
    close = same.all(-1)
    assert close.mean() > 0.99
    # scores: exp and a division, a sum of up to 512, then the sum of k
    assert np.allclose(w[close], want_w[close], rtol=16 * 2.0 ** -23, atol=2.0 ** -126)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 6), (5, 3, 3), (130, 65, 8), (77, 256, 8), (9, 512, 32), (33, 100, 1)])
def test_route(clq, T, E, k, score, dtype):
    g = np.random.default_rng(T * E + k)
    x = torch.from_numpy((2 * g.standard_normal((T, E))).astype(np.float32)).to(dtype)
    # (16-bit logits tie often: the lower index has to win)
    _check_route(clq, x, k, exact_ties=True, score=score)
    _check_route(clq, x, k, score=score, renormalize=False, scale=2.5)
    _check_route(clq, x, k, score=score, bias=(0.1 * g.standard_normal(E)).astype(np.float32))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups,top,k", [(256, 8, 4, 8), (64, 64, 5, 5), (12, 4, 2, 6), (60, 3, 1, 4), (512, 2, 1, 8), (8, 8, 8, 2)])
def test_route_groups(clq, E, groups, top, k, score):
    g = np.random.default_rng(E + groups)
    x = torch.from_numpy(g.standard_normal((200, E)).astype(np.float32))
    _check_route(clq, x, k, score=score, groups=groups, top_groups=top)
    _check_route(clq, x, k, score=score, groups=groups, top_groups=top, bias=g.standard_normal(E).astype(np.float32))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_ties_masks_and_empty_rows(clq, score):
    x = torch.zeros(6, 70)
    x[1, 40:] = 1.0
    x[2] = float("-inf")                       # nothing left
    x[3] = float("-inf")
    x[3, 69] = 0.5                             # fewer experts than top_k
    x[4] = torch.finfo(F32).min                # masked by the lowest value
    x[4, 5] = 2.0
    x[5] = torch.arange(70.0) * 20             # scores that round to 0 or 1
    ids, w = clq.clq_expert_route(x.cuda(), 4, score=score)
    ids, w = ids.cpu().numpy(), _np(w)
    want_ids, want_w, _ = ref.route(x.double().numpy(), 4, score=score)
    assert np.array_equal(ids, want_ids)
    assert np.allclose(w, want_w, rtol=2e-6)
    assert (w[2] == 0).all() and w[3, 0] == 1 and (w[3, 1:] == 0).all()


def test_route_nan_and_infinite_logits(clq):
    x = torch.randn(4, 20)
    x[1, 3] = float("nan")
    x[2] = float("nan")
    x[3, 7] = float("inf")
    ids, w = clq.clq_expert_route(x.cuda(), 3)
    assert ids.min() >= 0 and ids.max() < 20
    assert torch.isfinite(w[0]).all() and torch.isnan(w[1]).all() and torch.isnan(w[2]).all()
    assert ids[3, 0] == 7 and torch.isnan(w[3]).any()
    ids, w = clq.clq_expert_route(x.cuda(), 3, score="sigmoid")
    assert ids[3, 0] == 7 and torch.isfinite(w[3]).all() and torch.isnan(w[1]).all()


def test_route_strided_logits(clq):
    x = torch.randn(50, 90)
    a = clq.clq_expert_route(x[:, 7:40].cuda().contiguous(), 4)
    b = clq.clq_expert_route(x.cuda()[:, 7:40], 4)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k,groups,top,biased", [
    (4097, 1, 1, 1, 1, False), (4099, 33, 5, 1, 1, False), (5000, 64, 6, 1, 1, True), (4103, 100, 32, 1, 1, True),
    (4096, 128, 8, 32, 9, True), (24577, 256, 8, 8, 4, True), (24579, 130, 3, 1, 1, False), (30001, 192, 8, 32, 3, False)])
def test_route_of_many_tokens_is_that_of_few(clq, T, E, k, groups, top, biased, score):
    """With equal ranks, masked experts, masked rows and NaN among the tokens."""
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, E, generator=g)
    x[::5] = x[::5].round()
    x[::7, : E // 2] = -float("inf")
    x[3::1001] = -float("inf")
    x[5::997, E // 3] = float("nan")
    x[6::991, E // 4] = float("inf")
    x = x.cuda()
    b = torch.randn(E, generator=g).cuda() if biased else None
    f = lambda x: clq.clq_expert_route(x, k, score=score, bias=b, groups=groups, top_groups=top)  # noqa: E731
    ids, w = f(x)
    parts = [f(x[i:i + 3000]) for i in range(0, T, 3000)]
    assert torch.equal(ids, torch.cat([p[0] for p in parts]))
    assert torch.equal(w.view(torch.int32), torch.cat([p[1] for p in parts]).view(torch.int32))


def test_route_refuses_rows_that_overlap(clq):
    x = torch.randn(4, 64, device="cuda")
    for bad in (x[:1].expand(50, 64), x[:, :1].as_strided((50, 1), (0, 1)), x.as_strided((50, 64), (3, 1))):
        with pytest.raises(clq.ClqError):
            clq.clq_expert_route(bad, 1)
    one = clq.clq_expert_route(x[:1].expand(1, 64), 6)
    assert torch.equal(one[0], clq.clq_expert_route(x, 6)[0][:1])


# ---- plan ----------------------------------------------------------------------------------

@pytest.mark.parametrize("T,k,E,kind", [
    (1, 1, 1, "even"), (1, 8, 64, "even"), (3, 2, 5, "even"), (500, 6, 64, "even"), (700, 2, 3, "one"),
    (4096, 1, 7, "even"), (4097, 1, 512, "even"), (3000, 8, 100, "skew"), (20000, 3, 33, "drop"), (64, 4, 8, "none")])
def test_plan(clq, T, k, E, kind):
    g = np.random.default_rng(T + E)
    ids = g.integers(0, E, (T, k))
    if kind == "one":
        ids[:] = 1
    if kind == "skew":
        ids = np.minimum(g.geometric(0.05, (T, k)) - 1, E - 1)
    if kind == "drop":
        ids = g.integers(-2, E + 2, (T, k))   # entries outside belong to nobody here
    if kind == "none":
        ids[:] = -1
    ids = ids.astype(np.int32)
    p = clq.clq_expert_plan(torch.from_numpy(ids).cuda(), E)
    counts, rows, source = ref.plan(ids, E)
    assert np.array_equal(p.counts.cpu().numpy(), counts)
    assert np.array_equal(p.rows.cpu().numpy(), rows)
    assert len(source) <= p.plan_rows == p.source.numel()
    assert np.array_equal(p.source.cpu().numpy()[:len(source)], source)
    off = p.offsets().cpu().numpy()
    assert off[-1] == len(source) and (np.diff(off) == (counts + 31) // 32 * 32).all()


@pytest.mark.parametrize("T,k,E", [(1025, 1, 7), (600, 3, 512), (2500, 4, 512), (20000, 8, 256), (100000, 8, 64), (70000, 2, 512)])
def test_plan_runs_of_every_length(clq, T, k, E):
    ids = torch.from_numpy(np.random.default_rng(T).integers(-1, E, (T, k)).astype(np.int32))
    p = clq.clq_expert_plan(ids.cuda(), E)
    flat = ids.flatten().long()
    order = torch.sort(torch.where(flat < 0, E, flat), stable=True)[1]
    order = order[:int((flat >= 0).sum())]
    counts = torch.bincount(flat[flat >= 0], minlength=E)
    first = torch.cumsum((counts + 31) // 32 * 32, 0) - (counts + 31) // 32 * 32
    row = torch.full((T * k,), -1, dtype=torch.int64)
    row[order] = torch.arange(len(order)) - (torch.cumsum(counts, 0) - counts)[flat[order]] + first[flat[order]]
    assert torch.equal(p.counts.cpu().long(), counts) and torch.equal(p.rows.flatten().cpu().long(), row)
    source = torch.full((int(p.offsets()[-1]),), -1, dtype=torch.int64)
    source[row[order]] = order // k
    assert torch.equal(p.source[:len(source)].cpu().long(), source)


# ---- grouped products --------------------------------------------------------------------------

def _layer(seed, T, K, F, E, k, act, dtype):
    g = np.random.default_rng(seed)
    up = 2 * F if act == "swiglu" else F
    f = lambda *s, scale=1.0: torch.from_numpy((scale * g.standard_normal(s)).astype(np.float32)).to(dtype)  # noqa: E731
    x = f(T, K)
    return (x, f(E, up, K, scale=K ** -0.5), f(E, up, scale=0.1), f(E, K, F, scale=F ** -0.5), f(E, K, scale=0.1),
            torch.from_numpy(g.random((T, k)).astype(np.float32)))


@pytest.mark.parametrize("act,block,dtype", [("gelu", 64, F16), ("swiglu", 32, BF16), (None, 0, F16), ("gelu", 128, BF16)])
@pytest.mark.parametrize("T,K,F,E,k,kind", [
    (1, 128, 128, 4, 2, "even"), (2, 1152, 256, 16, 2, "even"), (50, 128, 384, 3, 1, "one"),
    (300, 256, 256, 5, 3, "drop"), (900, 256, 128, 4, 2, "even"), (200, 128, 128, 70, 6, "even"), (7, 128, 128, 2, 2, "none")])
def test_expert_mlp(clq, T, K, F, E, k, kind, act, block, dtype):
    x, w1, b1, w2, b2, gates = _layer(T + E, T, K, F, E, k, act, dtype)
    g = np.random.default_rng(E)
    ids = np.array([g.permutation(E)[:k] if k <= E else g.integers(0, E, k) for _ in range(T)], np.int32)
    if kind == "one":
        ids[:] = E - 1
    if kind == "drop":
        ids[g.random(ids.shape) < 0.3] = -1
    if kind == "none":
        ids[:] = E
    plan = clq.clq_expert_plan(torch.from_numpy(ids).cuda(), E)
    q = clq.clq_mx4_dispatch(x.cuda(), plan, block=block)
    q1 = clq.clq_mx4_quantize_weights(w1.cuda(), block=block, gated=act == "swiglu")
    q2 = clq.clq_mx4_quantize_weights(w2.cuda(), block=block)
    h = clq.clq_mx4_experts_mx4(q, plan, q1, b1.cuda(), act=act, block=block)
    y = clq.clq_mx4_experts(h, plan, q2, b2.cuda())
    out = _np(clq.clq_expert_combine(y, plan, gates.cuda()))
    xv = ref.quantize(_np(x), block)
    want = np.zeros((T, K))
    for e in range(E):
        t, j = np.nonzero(ids == e)
        if len(t):
            v1, v2 = (ref.quantize(_np(w[e]), block, divide=max(1, block)) for w in (w1, w2))
            hv = ref.quantize(ref.activate(xv[t] @ v1.T + _np(b1[e]), act), block)
            np.add.at(want, t, (hv @ v2.T + _np(b2[e])) * _np(gates)[t, j][:, None])
    assert out.shape == want.shape
    if kind == "none":
        assert (out == 0).all()
        return
    # two roundings to the type (the expert's output and the sum; a sum may cancel), and codes on
    # the other side of a boundary
    tol = (3e-3 if dtype == F16 else 8e-3)
    assert np.linalg.norm(out - want) < tol * np.linalg.norm(want)
    assert (out[(ids < 0).all(1)] == 0).all()


def test_dispatch_is_the_quantizer_in_the_plans_rows(clq):
    T, K, E, k = 90, 320, 6, 3
    x = torch.randn(T, K, dtype=F16)
    ids = torch.randint(0, E, (T, k), dtype=torch.int32)
    perm = torch.randperm(K).to(torch.int32)
    plan = clq.clq_expert_plan(ids.cuda(), E)
    got = clq.clq_mx4_dequantize(clq.clq_mx4_dispatch(x.cuda(), plan, 64, perm.cuda()), F32).cpu()
    want = clq.clq_mx4_dequantize(clq.clq_mx4_quantize(x.cuda(), 64, perm.cuda()), F32).cpu()
    src = plan.source.cpu()[:int(plan.offsets()[-1])].long()
    assert torch.equal(got[:len(src)][src >= 0], want[src[src >= 0]])
    assert (got[:len(src)][src < 0] == 0).all()


@pytest.mark.parametrize("N", [40, 129])
def test_combine(clq, N):
    T, k, E = 37, 4, 5
    ids = torch.randint(-1, E, (T, k), dtype=torch.int32)
    plan = clq.clq_expert_plan(ids.cuda(), E)
    y = torch.randn(plan.plan_rows, (N + 7) // 8 * 8, dtype=BF16).cuda()[:, :N]   # (rows on 16-byte boundaries)
    w = torch.rand(T, k)
    got = _np(clq.clq_expert_combine(y, plan, w.cuda()))
    rows = plan.rows.cpu().numpy()
    want = np.zeros((T, N))
    for j in range(k):
        use = rows[:, j] >= 0
        want[use] += _np(w)[use, j:j + 1] * _np(y)[rows[use, j]]
    # the sum's roundings in fp32 and one to bf16
    mass = k * np.abs(_np(y)).max()
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + k * 2.0 ** -23 * mass).all()


@pytest.mark.parametrize("ydt", [F16, BF16, F32])
@pytest.mark.parametrize("odt", [F16, BF16, F32])
def test_combine_types(clq, ydt, odt):
    T, k, E, N = 20, 3, 4, 24
    plan = clq.clq_expert_plan(torch.randint(0, E, (T, k), dtype=torch.int32).cuda(), E)
    y, w = torch.randn(plan.plan_rows, N).to(ydt).cuda(), torch.rand(T, k).cuda()
    got = clq.clq_expert_combine(y, plan, w, dtype=odt)
    assert got.dtype == odt
    rows = plan.rows.cpu().numpy()
    want = (_np(w)[:, :, None] * _np(y)[rows]).sum(1)
    unit = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}[odt]
    mass = (np.abs(_np(w))[:, :, None] * np.abs(_np(y)[rows])).sum(1)
    assert (np.abs(_np(got) - want) <= unit * np.abs(want) + k * 2.0 ** -24 * mass + 2.0 ** -25).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_results_that_are_summed_keep_fp32_while_they_are_small(clq, dtype):
    """One rounding: half a unit of the layer's output, beside the fp32 sums'."""
    T, K, F, E, k = 33, 128, 128, 4, 3
    x, w1, b1, w2, b2, gates = _layer(2, T, K, F, E, k, None, dtype)
    ids = torch.randint(0, E, (T, k), dtype=torch.int32)
    plan = clq.clq_expert_plan(ids.cuda(), E)
    q1, q2 = clq.clq_mx4_quantize_weights(w1.cuda()), clq.clq_mx4_quantize_weights(w2.cuda())
    h = clq.clq_mx4_experts_mx4(clq.clq_mx4_dispatch(x.cuda(), plan), plan, q1, b1.cuda())
    y = clq.clq_mx4_experts(h, plan, q2, b2.cuda())
    out = clq.clq_expert_combine(y, plan, gates.cuda())
    assert y.dtype == F32 and out.dtype == dtype
    hv, rows = _np(clq.clq_mx4_dequantize(h, F32)), plan.rows.cpu().numpy()
    wv = _np(clq.clq_mx4_dequantize(q2, F32))
    want, mass = np.zeros((T, K)), np.zeros((T, K))
    for j in range(k):
        e = ids[:, j].numpy()
        v = hv[rows[:, j]]
        g = _np(gates)[:, j:j + 1]
        want += g * (np.einsum("tf,tnf->tn", v, wv[e]) + _np(b2)[e])
        mass += g * (np.einsum("tf,tnf->tn", np.abs(v), np.abs(wv[e])) + np.abs(_np(b2)[e]))
    unit = {F16: 2.0 ** -11, BF16: 2.0 ** -8}[dtype]
    assert (np.abs(_np(out) - want) <= unit * np.abs(want) + (F + k) * 2.0 ** -24 * mass + 2.0 ** -25).all()
    assert clq.clq_mx4_experts(h, plan, q2, b2.cuda(), dtype=F16).dtype == F16


def test_layer_graph_replays(clq):
    T, K, F, E, k = 40, 128, 256, 8, 2
    x, w1, b1, w2, b2, _ = (t.cuda() for t in _layer(3, T, K, F, E, k, "gelu", F16))
    q1, q2 = clq.clq_mx4_quantize_weights(w1, 64), clq.clq_mx4_quantize_weights(w2, 64)
    logits = torch.randn(T, E, device="cuda")

    def step():
        ids, gates = clq.clq_expert_route(logits, k)
        plan = clq.clq_expert_plan(ids, E)
        h = clq.clq_mx4_experts_mx4(clq.clq_mx4_dispatch(x, plan, 64), plan, q1, b1, act="gelu", block=64)
        return clq.clq_expert_combine(clq.clq_mx4_experts(h, plan, q2, b2), plan, gates)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    for i in range(4):
        logits.copy_(torch.randn(T, E) * (1 + i))   # other experts, other tile counts
        x.copy_(torch.randn(T, K))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, step()), i


@pytest.mark.parametrize("act,dtype", [("gelu", F16), ("swiglu", BF16)])
def test_expert_mlp_class(clq, act, dtype):
    """The layer as a program uses it, eager and as a graph, against fp64 on its own routing."""
    from paper_2509_24416_amd.experts import ExpertMLP
    T, K, F, E, k = 75, 256, 192, 8, 2
    x, w1, b1, w2, b2, _ = _layer(11, T, K, F, E, k, act, dtype)
    router = torch.randn(E, K) * K ** -0.5
    layer = ExpertMLP(router.cuda(), w1.cuda(), b1.cuda(), w2.cuda(), b2.cuda(), k, act=act, block=32)
    out = layer.forward(x.cuda())
    assert out.dtype == dtype
    ids, gates, _ = ref.route(_np(x) @ _np(router).T, k)
    xv, want = ref.quantize(_np(x), 32), np.zeros((T, K))
    for e in range(E):
        t, j = np.nonzero(ids == e)
        v1, v2 = (ref.quantize(_np(w[e]), 32, divide=32) for w in (w1, w2))
        hv = ref.quantize(ref.activate(xv[t] @ v1.T + _np(b1[e]), act), 32)
        np.add.at(want, t, (hv @ v2.T + _np(b2[e])) * gates[t, j][:, None])
    assert np.linalg.norm(_np(out) - want) < (3e-3 if dtype == F16 else 8e-3) * np.linalg.norm(want)
    layer.capture(T, dtype)
    for i in range(3):
        xi = (torch.randn(T, K) * (i + 1)).to(dtype).cuda()
        y = layer.replay(xi).clone()
        torch.cuda.synchronize()
        assert torch.equal(y, layer.forward(xi))
