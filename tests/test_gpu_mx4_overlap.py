"""Outputs in the memory of what a call reads are refused, others beside it are written."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F16 = torch.float16


@pytest.fixture(scope="module")
def clq():
    import paper_2509_24416_amd as m
    return m


def test_every_output_is_kept_apart_from_its_inputs(clq):
    M, K, N, E, k = 64, 128, 128, 2, 1
    mx = 64 * 64 + 2 * 256                     # bytes of an MX4 of M x K
    buf = torch.zeros(1 << 18, dtype=torch.uint8, device="cuda")
    half = buf.view(F16)
    x = half[:M * K].view(M, K)                # bytes 0 .. 16383
    x.copy_(torch.randn(M, K))
    q = clq.MX4(buf[32768:32768 + mx], M, K)
    qw, qe = (clq.clq_mx4_quantize_weights(torch.randn(*s, N, K, device="cuda").half()) for s in ((), (E,)))
    plan = clq.clq_expert_plan(torch.zeros(M, k, dtype=torch.int32, device="cuda"), E)
    gates = torch.ones(M, k, device="cuda")
    clq.clq_mx4_quantize(x, out=q)
    want = clq.clq_mx4_quantize(x.clone())
    assert torch.equal(clq.clq_mx4_dequantize(q), clq.clq_mx4_dequantize(want))
    y = clq.clq_mx4_linear(q, qw)
    d, n = clq.clq_mx4_dispatch(x, plan), plan.plan_rows
    arena = torch.empty(n * 64 + n // 32 * 256 + 2 * n * N, dtype=torch.uint8, device="cuda")
    dn = clq.MX4(arena[:n * 64 + n // 32 * 256], n, K)
    e = clq.clq_mx4_experts(d, plan, qe, dtype=F16)
    before = buf.clone()
    in_x, in_q = clq.MX4(buf[16368:16368 + n * 64 + n // 32 * 256], M, K), half[(32768 + mx - 16) // 2:][:M * N].view(M, N)
    dq = clq.clq_mx4_dispatch(x, plan, out=dn)
    for call in (lambda: clq.clq_mx4_quantize(x, out=in_x), lambda: clq.clq_mx4_dispatch(x, plan, out=in_x),
                 lambda: clq.clq_mx4_linear(q, qw, out=in_q), lambda: clq.clq_mx4_dequantize(q, out=in_q),
                 lambda: clq.clq_mx4_linear_mx4(q, qw, out=clq.MX4(buf[32768 + 16:32768 + 16 + mx], M, N)),
                 lambda: clq.clq_mx4_experts(dq, plan, qe, out=arena[1024:1024 + 2 * n * N].view(F16).view(n, N)),
                 lambda: clq.clq_expert_combine(e, plan, gates, out=e[1:1 + M])):
        with pytest.raises(ValueError, match="overlaps"):
            call()
    assert torch.equal(buf, before)
    # beside it: the rest of the rows, and the other columns of one matrix
    out = half[M * K:][:M * N].view(M, N)
    assert torch.equal(clq.clq_mx4_linear(q, qw, out=out), y)
    wide = torch.zeros(n, 2 * N, dtype=F16, device="cuda")
    left = clq.clq_mx4_experts(d, plan, qe, out=wide[:, :N])
    sums = clq.clq_expert_combine(left, plan, gates, out=wide[:M, N:])
    assert torch.equal(sums, clq.clq_expert_combine(e, plan, gates, dtype=F16))
    with pytest.raises(ValueError, match="overlaps"):
        clq.clq_expert_combine(left, plan, gates, out=wide[:M, N - 8:-8])
