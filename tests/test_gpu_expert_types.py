"""Result types of the expert layer: the library's own choices round once."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
UNIT = {F16: 2.0 ** -11, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def clq():
    import paper_2509_24416_amd as m
    return m


def _gates(T, k):
    g = torch.rand(T, k, device="cuda")
    return g / g.sum(1, keepdim=True)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T", [1, 3000])
def test_results_that_are_summed_keep_fp32_whatever_their_number(clq, T, dtype):
    k, E, K, N = 4, 8, 128, 1152
    x, w, b = torch.randn(T, K).to(dtype).cuda(), torch.randn(E, N, K).to(dtype).cuda(), torch.randn(E, N).to(dtype).cuda()
    ids = torch.rand(T, E).argsort(1)[:, :k].to(torch.int32).contiguous().cuda()
    plan, gates = clq.clq_expert_plan(ids, E), _gates(T, k)
    q, qw = clq.clq_mx4_dispatch(x, plan), clq.clq_mx4_quantize_weights(w)
    y = clq.clq_mx4_experts(q, plan, qw, b)
    out = clq.clq_expert_combine(y, plan, gates)
    assert y.dtype == F32 and out.dtype == dtype
    xv, wv = clq.clq_mx4_dequantize(q, F32), clq.clq_mx4_dequantize(qw, F32)
    want, mass = torch.zeros(T, N, dtype=torch.float64, device="cuda"), torch.zeros(T, N, device="cuda")
    for j in range(k):
        for e in range(E):
            t = (ids[:, j] == e).nonzero()[:, 0]
            v = xv[plan.rows[t, j].long()]
            g = gates[t, j, None]
            want[t] += g.double() * (v.double() @ wv[e].double().t().contiguous() + b[e].double())
            mass[t] += g * (v.abs() @ wv[e].abs().t().contiguous() + b[e].abs().float())
    assert ((out.double() - want).abs() <= UNIT[dtype] * want.abs() + (K + k) * 2.0 ** -24 * mass + 2.0 ** -25).all()
    # a type that the caller names is that type at every size
    assert clq.clq_mx4_experts(q, plan, qw, b, dtype=dtype).dtype == dtype
    assert clq.clq_mx4_experts(q, plan, qw, b, out=torch.empty(plan.plan_rows, N, dtype=dtype, device="cuda")).dtype == dtype


def test_layer_keeps_fp32_results_unless_asked(clq):
    from paper_2509_24416_amd.experts import ExpertMLP
    T, K, F, E, k = 2500, 1152, 128, 8, 2
    f = lambda *s: (torch.randn(*s) * s[-1] ** -0.5).half().cuda()  # noqa: E731
    router, w1, w2, x = f(E, K), f(E, F, K), f(E, K, F), torch.randn(T, K).half().cuda()
    b1, b2 = f(E, F), f(E, K)
    layer = ExpertMLP(router, w1, b1, w2, b2, k)
    half = ExpertMLP(router, w1, b1, w2, b2, k, results=F16)
    ids, gates = clq.clq_expert_route(x.float() @ router.float().t(), k)
    plan = clq.clq_expert_plan(ids, E)
    h = clq.clq_mx4_experts_mx4(clq.clq_mx4_dispatch(x, plan, 64), plan, layer.w1, b1, act="gelu", block=64)
    for m, t in ((layer, F32), (half, F16)):
        y = clq.clq_mx4_experts(h, plan, layer.w2, b2, dtype=t)
        assert torch.equal(m.forward(x), clq.clq_expert_combine(y, plan, gates, dtype=F16))


def test_tokens_of_two_types_with_one_plan(clq):
    """Neither chain takes the other's type, in whatever order their calls come."""
    T, k, E, K, N = 40, 2, 4, 128, 64
    ids, gates = torch.randint(0, E, (T, k), dtype=torch.int32).cuda(), _gates(T, k)
    w = clq.clq_mx4_quantize_weights(torch.randn(E, N, K).half().cuda())
    xs = {t: torch.randn(T, K).to(t).cuda() for t in (F16, BF16)}
    want = {}
    for t, x in xs.items():   # each with a plan of its own
        p = clq.clq_expert_plan(ids, E)
        want[t] = clq.clq_expert_combine(clq.clq_mx4_experts(clq.clq_mx4_dispatch(x, p), p, w), p, gates)
        assert want[t].dtype == p.dtype == t
    plan = clq.clq_expert_plan(ids, E)
    y = {F16: clq.clq_mx4_experts(clq.clq_mx4_dispatch(xs[F16], plan), plan, w)}
    y[BF16] = clq.clq_mx4_experts(clq.clq_mx4_dispatch(xs[BF16], plan), plan, w)
    for t in (F16, BF16):
        with pytest.raises(ValueError, match="two types"):
            clq.clq_expert_combine(y[t], plan, gates)
        assert torch.equal(clq.clq_expert_combine(y[t], plan, gates, dtype=t), want[t])
        out = torch.empty(T, N, dtype=t, device="cuda")
        assert torch.equal(clq.clq_expert_combine(y[t], plan, gates, out=out), want[t])
    # a plan that is used again with the same type keeps it
    again = clq.clq_expert_plan(ids, E)
    for _ in range(2):
        q = clq.clq_mx4_dispatch(xs[BF16], again)
    assert torch.equal(clq.clq_expert_combine(clq.clq_mx4_experts(q, again, w), again, gates), want[BF16])
