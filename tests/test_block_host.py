"""Host-side checks of the norm, rotary position and 8-bit epilogue entry points (no GPU needed, no kernel
is launched): exports, and every refusal before anything is enqueued."""
import ctypes
import math
import os
import re

import pytest
import torch

import paper_2509_24416_amd as clq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, BLOCK, ALIGN, ARG, HIP, WORKSPACE = range(8)
A, MIS = 0x10000, 0x10002   # fake device addresses, never read
L = clq.lib()


def test_exports_and_binding_names():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "clq_block.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(clq_[a-z0-9_]+)\s*\(", text)))
    assert sorted(clq.BLOCK_EXPORTS) == names
    for n in names:
        assert hasattr(L, n) and callable(getattr(clq, n)), n


def test_header_compiles_as_c(tmp_path):
    import subprocess
    src = tmp_path / "t.c"
    src.write_text('#define __HIP_PLATFORM_AMD__\n#include "clq_block.h"\nint main(void) { return CLQ_ACT_SILU; }\n')
    subprocess.run(["gcc", "-std=c11", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    str(src)], check=True, capture_output=True)


def norm(X=A, xt=0, ldx=1152, R=None, rt=0, ldr=1152, W=None, wt=0, samples=1, eps=1e-6, M=4, K=1152, Y=A, yt=0, ldy=1152,
         S=None, lds=1152):
    return L.clq_rms_norm(X, xt, ldx, R, rt, ldr, W, wt, samples, eps, M, K, Y, yt, ldy, S, lds, None)


def norm8(X=A, xt=0, ldx=1152, R=None, rt=0, ldr=1152, W=None, wt=0, samples=1, eps=1e-6, perm=None, M=4, K=1152, block=64,
          q=A, xs=A, S=None, lds=1152):
    return L.clq_rms_norm_act8(X, xt, ldx, R, rt, ldr, W, wt, samples, eps, perm, M, K, block, q, xs, S, lds, None)


COMMON = [(dict(X=None), NULL), (dict(R=A), NULL), (dict(S=A), NULL), (dict(xt=3), ARG), (dict(xt=-1), ARG),
          (dict(R=A, S=A, rt=3), ARG), (dict(W=A, wt=5), ARG), (dict(eps=0.0), ARG), (dict(eps=1e-39), ARG), (dict(eps=-1.0), ARG),
          (dict(eps=math.inf), ARG), (dict(eps=math.nan), ARG), (dict(M=0), SHAPE), (dict(M=2 ** 31), SHAPE),
          (dict(samples=2), SHAPE), (dict(W=A, samples=3), SHAPE), (dict(W=A, samples=8), SHAPE), (dict(W=A, samples=0), SHAPE),
          (dict(K=0), SHAPE), (dict(K=16448, ldx=16448), SHAPE), (dict(ldx=1144), SHAPE), (dict(ldx=1156), SHAPE),
          (dict(R=A, S=A, ldr=1148), SHAPE), (dict(R=A, S=A, lds=1144), SHAPE), (dict(X=MIS), ALIGN), (dict(W=MIS), ALIGN),
          (dict(R=MIS, S=A), ALIGN), (dict(R=A, S=0x10008), ALIGN)]


@pytest.mark.parametrize("kw,want", [*COMMON, (dict(Y=None), NULL), (dict(yt=3), ARG), (dict(K=100, ldx=104), SHAPE),
                                     (dict(ldy=1144), SHAPE), (dict(Y=MIS), ALIGN)])
def test_norm_refusals(kw, want):
    assert norm(**kw) == want


@pytest.mark.parametrize("kw,want", [*COMMON, (dict(q=None), NULL), (dict(xs=None), NULL), (dict(K=72, ldx=72), SHAPE),
                                     (dict(block=0), BLOCK), (dict(block=16), BLOCK), (dict(K=192, ldx=192, block=128), BLOCK),
                                     (dict(q=MIS), ALIGN), (dict(xs=MIS), ALIGN), (dict(perm=MIS), ALIGN)])
def test_norm_act8_refusals(kw, want):
    assert norm8(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(X=None), NULL), (dict(q=None), NULL), (dict(xs=None), NULL), (dict(t=3), ARG), (dict(M=0), SHAPE), (dict(K=72, ldx=72), SHAPE),
    (dict(K=16448, ldx=16448), SHAPE), (dict(ldx=1148), SHAPE), (dict(block=0), BLOCK), (dict(K=192, ldx=192, block=128), BLOCK),
    (dict(X=MIS), ALIGN), (dict(q=MIS), ALIGN), (dict(xs=MIS), ALIGN), (dict(perm=MIS), ALIGN)])
def test_quantize_act8_refusals(kw, want):
    def call(X=A, t=0, ldx=1152, perm=None, M=4, K=1152, block=64, q=A, xs=A):
        return L.clq_quantize_act8(X, t, ldx, perm, M, K, block, q, xs, None)

    assert call(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(t=3), ARG), (dict(M=0), SHAPE), (dict(K=96), SHAPE), (dict(ldo=60), SHAPE),
    (dict(ldo=56), SHAPE), (dict(q=MIS), ALIGN), (dict(xs=MIS), ALIGN), (dict(out=MIS), ALIGN)])
def test_dequantize_refusals(kw, want):
    def call(q=A, xs=A, M=4, K=64, t=0, out=A, ldo=64):
        return L.clq_dequantize_act8(q, xs, M, K, t, out, ldo, None)

    assert call(**kw) == want


def rope(X=A, t=0, ldx=1152, lhx=72, pos=A, pt=0, tokens=4, f=A, ends=(12, 24, 36), axes=None, inter=1, inv=0, W=None, wt=0,
         wh=1, eps=1e-6, M=4, H=16, D=72, Y=A, ldy=1152, lhy=72):
    e = (ctypes.c_int32 * 8)(*ends) if ends is not None else None
    return L.clq_rope_axes(X, t, ldx, lhx, pos, pt, tokens, f, e, len(ends) if axes is None else axes, inter, inv, W, wt, wh,
                           eps, M, H, D, Y, ldy, lhy, None)


@pytest.mark.parametrize("kw,want", [
    (dict(X=None), NULL), (dict(Y=None), NULL), (dict(pos=None), NULL), (dict(f=None), NULL), (dict(ends=None, axes=1), NULL),
    (dict(t=2), ARG), (dict(pt=2), ARG), (dict(axes=0), ARG), (dict(axes=5), ARG), (dict(inter=2), ARG), (dict(inv=-1), ARG),
    (dict(W=A, wt=3), ARG), (dict(W=A, eps=0.0), ARG), (dict(M=0), SHAPE), (dict(H=0), SHAPE), (dict(H=2 ** 20 + 1), SHAPE), (dict(tokens=3), SHAPE),
    (dict(tokens=0), SHAPE), (dict(tokens=8), SHAPE), (dict(D=0), SHAPE), (dict(D=70), SHAPE), (dict(D=264, ldx=4224), SHAPE),
    (dict(W=A, wh=2), SHAPE), (dict(ends=(12, 12, 36)), SHAPE), (dict(ends=(0, 12, 36)), SHAPE), (dict(ends=(12, 24, 40)), SHAPE),
    (dict(ends=(12, 24, 34)), SHAPE), (dict(ldx=64), SHAPE), (dict(lhx=64), SHAPE), (dict(lhx=76), SHAPE), (dict(ldy=1148), SHAPE),
    (dict(lhy=64), SHAPE), (dict(ldy=576), SHAPE), (dict(ldy=72), SHAPE), (dict(X=MIS), ALIGN), (dict(Y=MIS), ALIGN),
    (dict(pos=MIS), ALIGN), (dict(f=0x10004), ALIGN), (dict(W=MIS), ALIGN)])
def test_rope_refusals(kw, want):
    assert rope(**kw) == want


def lin(Xq=A, xs=A, Wq=A, ws=A, bits=8, b=None, bt=0, act=0, g=None, gt=0, samples=1, R=None, ldr=64, M=4, N=64, K=256, t=0, Y=A,
        ldy=64):
    return L.clq_a8_linear_act(Xq, xs, Wq, ws, bits, b, bt, act, g, gt, samples, R, ldr, M, N, K, t, Y, ldy, None)


@pytest.mark.parametrize("kw,want", [
    (dict(Xq=None), NULL), (dict(xs=None), NULL), (dict(Wq=None), NULL), (dict(ws=None), NULL), (dict(Y=None), NULL),
    (dict(bits=6), ARG), (dict(act=2), ARG), (dict(act=4), ARG), (dict(t=3), ARG), (dict(b=A, bt=2), ARG), (dict(g=A, gt=3), ARG),
    (dict(M=0), SHAPE), (dict(N=0), SHAPE), (dict(K=32), SHAPE), (dict(K=96), SHAPE), (dict(K=65536), SHAPE), (dict(samples=2), SHAPE),
    (dict(g=A, samples=3), SHAPE), (dict(g=A, samples=0), SHAPE), (dict(ldy=56), SHAPE), (dict(ldy=68), SHAPE),
    (dict(R=A, ldr=63), SHAPE), (dict(M=2 ** 31 - 1, N=2 ** 16, ldy=2 ** 16), SHAPE), (dict(Xq=MIS), ALIGN), (dict(xs=MIS), ALIGN), (dict(Wq=MIS), ALIGN), (dict(ws=MIS), ALIGN),
    (dict(Y=MIS), ALIGN), (dict(b=0x10001), ALIGN), (dict(g=MIS), ALIGN), (dict(R=0x10001), ALIGN), (dict(R=MIS, t=2), ALIGN)])
def test_linear_act_refusals(kw, want):
    assert lin(**kw) == want


def test_rows_that_overlap():
    """Outputs of other spacing than an input are compared by the spans of both."""
    from paper_2509_24416_amd.block import _apart
    a = (1000, 5, 100, 40)                       # five pieces of 40 bytes, 100 apart
    for other, bad in (((1040, 5, 100, 60), False), ((1040, 5, 100, 61), True), ((900, 5, 100, 100), True), ((900, 1, 1, 100), False),
                       ((1050, 3, 200, 10), True), ((1440, 3, 200, 10), False), ((500, 5, 100, 40), False), ((500, 6, 100, 40), True), ((0, 11, 104, 40), True),
                       ((1440, 1, 1, 5), False), ((1439, 1, 1, 5), True)):
        if bad:
            with pytest.raises(ValueError, match="overlaps"):
                _apart(a, (0, 1, 1, 8), other)
        else:
            _apart(a, (0, 1, 1, 8), other)


def test_freqs():
    f = clq.clq_rope_freqs((4, 8), theta=100.0, device="cpu")
    want = [1.0, 0.1, 1.0, 100 ** -0.25, 0.1, 100 ** -0.75]
    assert f.dtype is torch.float64 and all(abs(a - b) < 1e-15 for a, b in zip(f.tolist(), want))
    for bad in ((), (2, 2, 2, 2, 2), (3,), (0, 4), (-2,)):
        with pytest.raises(ValueError, match="axes"):
            clq.clq_rope_freqs(bad, device="cpu")


def test_host_tensors_are_refused():
    x = torch.zeros(4, 64, dtype=torch.float16)
    with pytest.raises(TypeError, match="CUDA"):
        clq.clq_rms_norm(x)
    with pytest.raises(TypeError, match="CUDA"):
        clq.clq_rms_norm_act8(x, 64)
    with pytest.raises(TypeError, match="CUDA"):
        clq.clq_rope_axes(x.view(4, 1, 64), torch.zeros(4, 1, dtype=torch.int32), torch.zeros(32, dtype=torch.float64), (64,))
