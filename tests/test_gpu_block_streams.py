"""The block operators' `stream=`: a call given a stream runs behind what that stream holds, with every argument
that it was given."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_block import BF16, F16, F32, gen, randn

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


def cases(clq, g):
    """Each entry point: what changes while the stream is busy, the call on it (every optional argument given, none of
    them its default), and the results' buffers."""
    M, K, N, H, D = 70, 256, 192, 4, 64
    x, r, y = randn(g, M, K, dtype=F16, scale=2), randn(g, M, K, dtype=BF16, scale=3), torch.empty(M, K, device="cuda")
    w, perm = 1 + randn(g, 2, K, dtype=F16, scale=0.3), torch.randperm(K, device="cuda", generator=g).to(torch.int32)
    total = torch.empty_like(r)
    codes, scale = torch.empty(clq.clq_act8_bytes(M, K), dtype=torch.uint8, device="cuda"), torch.empty(M, device="cuda")
    q, xs = clq.clq_rotate_quant_act8(x, 64)
    q2, xs2 = clq.clq_rotate_quant_act8(randn(g, M, K, dtype=F16, scale=3), 64)   # (so many codes, of other rows)
    heads, turned = randn(g, M, H, D, dtype=BF16), torch.empty(M, H, D, dtype=BF16, device="cuda")
    pos, freqs = torch.randint(0, 90, (M // 2, 2), device="cuda", generator=g).to(torch.int32), clq.clq_rope_freqs((24, 32))
    hw = 1 + randn(g, H, D, dtype=F16, scale=0.3)
    qw, bias = clq.clq_quantize_weights8(randn(g, N, K, dtype=F16, scale=K ** -0.5), 64), randn(g, N, dtype=BF16)
    gate, res, out = randn(g, 2, N, dtype=F16), randn(g, M, N), torch.empty(M, N, device="cuda")
    other = lambda t: randn(g, *t.shape, scale=2).to(t.dtype)  # noqa: E731
    return {
        "norm": (((x, other(x)), (r, other(r))),
                 lambda o, **k: clq.clq_rms_norm(x, w, r, 0.3, dtype=F32, **(dict(out=y, sum_out=total) if o else {}), **k)),
        "norm8": (((x, other(x)), (r, other(r))),
                  lambda o, **k: clq.clq_rms_norm_act8(x, 128, w, r, 0.3, perm,
                                                       **(dict(out=codes, scale_out=scale, sum_out=total) if o else {}), **k)),
        "quantize": (((x, other(x)),),
                     lambda o, **k: clq.clq_quantize_act8(x, 32, perm, **(dict(out=codes, scale_out=scale) if o else {}), **k)),
        "dequantize": (((q, q2), (xs, xs2)),
                       lambda o, **k: (clq.clq_dequantize_act8(q, xs, K, dtype=F32, **(dict(out=y) if o else {}), **k),)),
        "rope": (((heads, other(heads)),),
                 lambda o, **k: (clq.clq_rope_axes(heads, pos, freqs, (24, 32), interleaved=False, inverse=True, weight=hw,
                                                   eps=0.3, **(dict(out=turned) if o else {}), **k),)),
        "linear": (((q, q2), (xs, xs2), (res, other(res))),
                   lambda o, **k: (clq.clq_a8_linear_act(q, xs, qw, bias, act="silu", gate=gate, residual=res, dtype=F32,
                                                         **(dict(out=out) if o else {}), **k),)),
        # (no residual and no buffer: the type is what was named)
        "linear, typed": (((q, q2), (xs, xs2)),
                          lambda o, **k: (clq.clq_a8_linear_act(q, xs, qw, bias, act="gelu", gate=gate, dtype=BF16, **k),)),
        "norm, typed by its buffer": (((x, other(x)),), lambda o, **k: (clq.clq_rms_norm(x, w, eps=0.3, out=y, **k),)),
    }


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("name", ["norm", "norm8", "quantize", "dequantize", "rope", "linear", "linear, typed",
                                  "norm, typed by its buffer"])
def test_a_call_runs_on_its_stream(clq, name, given):
    """The inputs get their values on the stream, behind some milliseconds of other work: a call on the current
    stream would read what they held before.  (Streams share a few hardware queues, and one that shares the current
    stream's would wait all the same: neighbours do not both.)"""
    changes, call = cases(clq, gen(21))[name]
    first = [t.clone() for t in call(given)]
    kept = [(t, t.clone()) for t, _ in changes]
    for t, new in changes:
        t.copy_(new)
    want = [t.clone() for t in call(given)]
    assert any(not torch.equal(a, b) for a, b in zip(first, want))
    busy = torch.zeros(4096, 4096, dtype=F16, device="cuda")
    product = torch.empty_like(busy)
    for other in (torch.cuda.Stream(), torch.cuda.Stream()):
        for t, old in kept:
            t.copy_(old)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            for _ in range(60):
                torch.mm(busy, busy, out=product)
            for t, new in changes:
                t.copy_(new)
        got = call(given, stream=other)
        other.synchronize()
        torch.cuda.synchronize()
        assert len(got) == len(want)
        for a, b in zip(got, want):
            assert a.dtype is b.dtype and torch.equal(a, b)


def test_two_streams_at_once(clq):
    """Queries turned on one stream while another norms, positions and frequencies made ahead of both."""
    g = gen(22)
    x, r = randn(g, 2000, 576, dtype=F16), randn(g, 2000, 576, dtype=F16)
    pos, f = torch.randint(0, 300, (2000, 3), device="cuda", generator=g).to(torch.int32), clq.clq_rope_freqs((24, 24, 24))
    want, turned = clq.clq_rms_norm(x, None, r), clq.clq_rope_axes(x.view(2000, 8, 72), pos, f, (24, 24, 24))
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [(clq.clq_rms_norm(x, None, r, stream=a), clq.clq_rope_axes(x.view(2000, 8, 72), pos, f, (24, 24, 24), stream=b))
           for _ in range(5)]
    torch.cuda.synchronize()
    for (y, s), z in got:
        assert torch.equal(y, want[0]) and torch.equal(s, want[1]) and torch.equal(z, turned)
