"""Host-side checks of the MX4 and expert entry points (no GPU needed, no kernel is
launched): exports, sizes, and every refusal before anything is enqueued."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2509_24416_amd as clq
from oracle import mx4 as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, BLOCK, ALIGN, ARG, HIP, WORKSPACE = range(8)
A, MIS = 0x10000, 0x10002   # fake device addresses, never read
L = clq.lib()


def test_plan_workspace_grows_with_the_assignments():
    """One that is large enough for some number of tokens is so for fewer."""
    for E in (1, 7, 64, 256, 512):
        sizes = [clq.clq_expert_plan_workspace_bytes(T, 8, E) for T in range(1, 200000, 97)]
        assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[-1] >= 4 * E * (8 * 199000 // 4096)


def test_exports_and_binding_names():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "clq_mx4.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(clq_[a-z0-9_]+)\s*\(", text)))
    assert sorted(clq.MX4_EXPORTS) == names
    for n in names:
        assert hasattr(L, n) and callable(getattr(clq, n)), n


def test_header_compiles_as_c(tmp_path):
    import subprocess
    src = tmp_path / "t.c"
    src.write_text('#define __HIP_PLATFORM_AMD__\n#include "clq_mx4.h"\nint main(void) { return CLQ_ACT_NONE; }\n')
    subprocess.run(["gcc", "-std=c11", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    str(src)], check=True, capture_output=True)


def test_sizes():
    assert clq.clq_mx4_code_bytes(64, 256) == 64 * 128
    assert clq.clq_mx4_code_bytes(33, 64) == 64 * 32          # rows padded to 32
    assert clq.clq_mx4_code_bytes(33, 64, True) == 64 * 32
    assert clq.clq_mx4_code_bytes(65, 64, True) == 128 * 32   # weights: to 64
    assert clq.clq_mx4_scale_bytes(64, 256) == 64 * 8
    assert clq.clq_mx4_scale_bytes(1, 64) == 256              # whole rows of four k units
    assert clq.clq_mx4_code_bytes(0, 64) == clq.clq_mx4_code_bytes(8, 96) == clq.clq_mx4_scale_bytes(8, 65536) == 0
    assert clq.clq_expert_plan_rows(1, 2, 16) == 64
    assert clq.clq_expert_plan_rows(100, 2, 3) == 32 * (200 // 32 + 3)
    assert clq.clq_expert_plan_rows(0, 1, 1) == clq.clq_expert_plan_rows(1, 33, 64) == 0
    assert clq.clq_expert_plan_rows(1, 1, 513) == clq.clq_expert_plan_rows(2 ** 31, 1, 1) == 0
    assert clq.clq_expert_plan_ints(0) == clq.clq_expert_plan_ints(513) == 0
    assert clq.clq_expert_plan_workspace_bytes(10, 2, 8) == 0
    assert clq.clq_expert_plan_workspace_bytes(43200, 8, 256) > 0


def q(X=A, t=0, ldx=1152, perm=None, M=4, K=1152, block=64, codes=A, scales=A):
    return L.clq_mx4_quantize(X, t, ldx, perm, M, K, block, codes, scales, None)


@pytest.mark.parametrize("kw,want", [
    (dict(X=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(t=2), ARG), (dict(t=7), ARG),
    (dict(M=0), SHAPE), (dict(M=2 ** 31), SHAPE), (dict(K=32, ldx=32), SHAPE), (dict(K=96, ldx=96), SHAPE),
    (dict(K=65536, ldx=65536), SHAPE), (dict(ldx=1144), SHAPE), (dict(ldx=1156), SHAPE), (dict(block=16), BLOCK),
    (dict(block=-1), BLOCK), (dict(K=192, ldx=192, block=128), BLOCK), (dict(X=MIS), ALIGN), (dict(codes=MIS), ALIGN),
    (dict(scales=0x10008), ALIGN), (dict(perm=0x10001), ALIGN)])
def test_quantize_refusals(kw, want):
    assert q(**kw) == want


def qw(W=A, t=0, perm=None, E=1, N=128, K=256, block=64, gated=0, codes=A, scales=A):
    return L.clq_mx4_quantize_weights(W, t, perm, E, N, K, block, gated, codes, scales, None)


@pytest.mark.parametrize("kw,want", [
    (dict(W=None), NULL), (dict(t=2), ARG), (dict(gated=2), ARG), (dict(E=0), SHAPE), (dict(E=513), SHAPE),
    (dict(N=0), SHAPE), (dict(E=512, N=2 ** 23), SHAPE), (dict(N=96, gated=1), SHAPE), (dict(K=100), SHAPE),
    (dict(block=48), BLOCK), (dict(W=MIS), ALIGN), (dict(scales=MIS), ALIGN)])
def test_quantize_weights_refusals(kw, want):
    assert qw(**kw) == want


def test_pack_and_dequantize_refusals():
    def pack(c=A, s=A, E=1, N=64, K=64, gated=0, co=A, so=A):
        return L.clq_mx4_pack_weights(c, s, E, N, K, gated, co, so, None)

    def deq(c=A, s=A, w=0, gated=0, mats=1, rows=4, K=64, t=0, out=A, ldo=64):
        return L.clq_mx4_dequantize(c, s, w, gated, mats, rows, K, t, out, ldo, None)

    assert pack(c=None) == pack(so=None) == NULL and pack(gated=3) == ARG and pack(N=32, gated=1) == SHAPE
    assert pack(K=80) == SHAPE and pack(c=MIS) == ALIGN
    assert deq(out=None) == NULL and deq(t=3) == ARG and deq(gated=1) == ARG and deq(mats=2) == ARG and deq(w=2) == ARG
    assert deq(ldo=56) == SHAPE and deq(ldo=68) == SHAPE and deq(rows=0) == SHAPE and deq(out=MIS) == ALIGN


def lin(Xq=A, Xs=A, Wq=A, Ws=A, b=None, bt=0, M=4, N=64, K=256, t=0, Y=A, ldy=64):
    return L.clq_mx4_linear(Xq, Xs, Wq, Ws, b, bt, M, N, K, t, Y, ldy, None)


@pytest.mark.parametrize("kw,want", [
    (dict(Xq=None), NULL), (dict(Ws=None), NULL), (dict(Y=None), NULL), (dict(M=0), SHAPE), (dict(N=0), SHAPE),
    (dict(K=32), SHAPE), (dict(t=3), ARG), (dict(b=A, bt=2), ARG), (dict(ldy=56), SHAPE), (dict(ldy=68), SHAPE),
    (dict(Xs=MIS), ALIGN), (dict(Y=MIS), ALIGN), (dict(b=0x10001), ALIGN), (dict(M=2 ** 31 - 1, N=2 ** 16, ldy=2 ** 16), SHAPE)])
def test_linear_refusals(kw, want):
    assert lin(**kw) == want


def lin4(Xq=A, Xs=A, Wq=A, Ws=A, b=None, bt=0, M=4, N=128, K=256, act=1, block=64, co=A, so=A):
    return L.clq_mx4_linear_mx4(Xq, Xs, Wq, Ws, b, bt, M, N, K, act, block, co, so, None)


@pytest.mark.parametrize("kw,want", [
    (dict(co=None), NULL), (dict(act=3), ARG), (dict(N=100), SHAPE), (dict(N=64, act=2), SHAPE), (dict(block=8), BLOCK),
    (dict(N=64, block=128), BLOCK), (dict(N=256, act=2, block=128), BLOCK), (dict(N=65536), SHAPE), (dict(so=MIS), ALIGN)])
def test_linear_mx4_refusals(kw, want):
    assert lin4(**kw) == want


def route(x=A, t=2, ld=64, T=4, E=64, k=2, score=0, b=None, groups=1, top=1, norm=1, scale=1.0, ids=A, w=A):
    return L.clq_expert_route(x, t, ld, T, E, k, score, b, groups, top, norm, scale, ids, w, None)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(ids=None), NULL), (dict(t=3), ARG), (dict(score=2), ARG), (dict(norm=2), ARG),
    (dict(scale=float("inf")), ARG), (dict(scale=float("nan")), ARG), (dict(T=0), SHAPE), (dict(E=513, ld=513), SHAPE),
    (dict(k=0), SHAPE), (dict(k=33), SHAPE), (dict(ld=63), SHAPE), (dict(groups=0), ARG), (dict(groups=5), ARG),
    (dict(groups=4, top=5), ARG), (dict(groups=32, top=1, k=3), ARG), (dict(E=2, ld=2, k=3), ARG),
    (dict(E=128, ld=128, groups=128), ARG), (dict(x=0x10001), ALIGN), (dict(b=MIS), ALIGN), (dict(w=MIS), ALIGN)])
def test_route_refusals(kw, want):
    assert route(**kw) == want


def test_plan_and_layer_refusals():
    def plan(ids=A, T=8, k=2, E=4, tables=A, rows=A, source=A, ws=None, wb=0):
        return L.clq_expert_plan(ids, T, k, E, tables, rows, source, ws, wb, None)

    def disp(X=A, t=0, ldx=64, T=8, k=2, E=4, K=64, block=0, tables=A, source=A, co=A, so=A):
        return L.clq_mx4_dispatch(X, t, ldx, None, T, k, E, K, block, tables, source, co, so, None)

    def exp(tables=A, T=8, k=2, E=4, N=64, Y=A, ldy=64, t=0):
        return L.clq_mx4_experts(A, A, tables, T, k, E, A, A, None, 0, N, 64, t, Y, ldy, None)

    def exp4(tables=A, T=8, k=2, E=4, N=64, act=0, block=0, co=A):
        return L.clq_mx4_experts_mx4(A, A, tables, T, k, E, A, A, None, 0, N, 64, act, block, co, A, None)

    def comb(Y=A, t=0, ldy=64, rows=A, w=A, T=8, k=2, E=4, N=64, out=A, to=0, ldo=64):
        return L.clq_expert_combine(Y, t, ldy, rows, w, T, k, E, N, out, to, ldo, None)

    assert plan(ids=None) == plan(source=None) == NULL and plan(E=0) == plan(k=33) == SHAPE
    assert plan(T=43200, k=8) == NULL and plan(T=43200, k=8, ws=A, wb=16) == WORKSPACE and plan(rows=MIS) == ALIGN
    assert disp(tables=None) == NULL and disp(t=2) == ARG and disp(E=513) == SHAPE and disp(source=MIS) == ALIGN
    assert disp(ldx=60) == SHAPE and disp(block=128) == BLOCK
    assert exp(tables=None) == exp(Y=None) == NULL and exp(T=0) == SHAPE and exp(ldy=60) == SHAPE and exp(t=3) == ARG
    assert exp(tables=MIS) == ALIGN
    assert exp4(co=None) == NULL and exp4(act=2) == SHAPE and exp4(block=128) == BLOCK and exp4(E=600) == SHAPE
    assert comb(w=None) == NULL and comb(t=3) == ARG and comb(to=3) == ARG and comb(N=0) == SHAPE and comb(ldo=60) == SHAPE
    assert comb(out=MIS) == ALIGN and comb(k=40) == SHAPE


def test_binding_refuses_host_tensors_and_wrong_kinds():
    x = torch.zeros(4, 64, dtype=torch.float16)
    for call in (lambda: clq.clq_mx4_quantize(x), lambda: clq.clq_mx4_quantize_weights(x),
                 lambda: clq.clq_expert_route(x.float(), 2), lambda: clq.clq_expert_plan(x.int(), 4),
                 lambda: clq.clq_mx4_linear(x, x), lambda: clq.clq_mx4_dequantize(None, torch.int8)):
        with pytest.raises(TypeError):
            call()
    a, w = clq.MX4(x, 4, 64, 64), clq.MX4Weight(x, x, 64, 64, 32)
    with pytest.raises(ValueError, match="rotated"):
        clq.clq_mx4_linear(a, w)
    w.block, w.K = 64, 128
    with pytest.raises(ValueError, match="columns"):
        clq.clq_mx4_linear(a, w)
    w.K, w.experts = 64, 3
    with pytest.raises(ValueError, match="experts"):
        clq.clq_mx4_linear(a, w)
    w.experts, w.gated = None, True
    with pytest.raises(ValueError, match="gated"):
        clq.clq_mx4_linear(a, w)
    with pytest.raises(ValueError, match="act"):
        clq.clq_mx4_linear_mx4(a, w, act="relu")


def test_binding_refuses_to_write_over_its_input():
    q = clq.MX4(torch.zeros(32 * 32 + 256, dtype=torch.uint8), 4, 64)
    w = clq.MX4Weight(torch.zeros(64 * 32, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 64, 64)
    plan = clq.ExpertPlan(torch.zeros(4, dtype=torch.int32), 1, 1, None, 4, 0)
    for out in (q, clq.MX4(q.data, 4, 64), clq.MX4(q.data.view(-1), 4, 64)):
        with pytest.raises(ValueError, match="output"):
            clq.clq_mx4_linear_mx4(q, w, out=out)
        with pytest.raises(ValueError, match="output"):
            clq.clq_mx4_experts_mx4(q, plan, w, out=out)


# ---- pins of the oracle itself -----------------------------------------------------------

def test_oracle_grid_by_hand():
    x = np.zeros(32)
    x[:16] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, 0.26, -0.25, -0.74, -5.01, -7.9, 0.2499, 6]
    want = [4, 0, 1, 1, 2, 2, 4, 4, 6, 0.5, 0, -0.5, -6, -6, 0, 6]
    assert ref.quantize(x)[:16].tolist() == want
    assert ref.exponents(np.full(32, 8.0)) == 1 and ref.exponents(np.full(32, 7.99)) == 0
    assert ref.exponents(np.zeros(32)) == -126 and ref.exponents(np.full(32, 2.0 ** -126)) == -126
    assert np.isnan(ref.quantize(np.r_[np.inf, np.zeros(31)])).all()


def test_oracle_rotation_is_the_hadamard_matrix():
    h = np.array([[1.0]])
    for _ in range(6):
        h = np.block([[h, h], [h, -h]])
    x = np.arange(128.0).reshape(2, 64) % 17 - 8
    assert np.array_equal(ref.rotate(x, 64), x @ h)


def test_oracle_route_and_plan_by_hand():
    ids, w, _ = ref.route([[1.0, 3.0, 3.0, 0.0]], 2)
    assert ids.tolist() == [[1, 2]] and np.allclose(w, 0.5)
    ids, _, _ = ref.route([[5.0, 0.0, 1.0, 4.9, -9.0, 3.0]], 2, score="sigmoid", groups=3, top_groups=1)
    assert ids.tolist() == [[3, 2]]   # (1, 4.9) beats (5, 0) and (-9, 3)
    counts, rows, source = ref.plan(np.array([[1, 0], [1, 5]]), 3)
    assert counts.tolist() == [1, 2, 0] and rows.tolist() == [[32, 0], [33, -1]]
    assert source[[0, 32, 33]].tolist() == [0, 0, 1] and len(source) == 64
