"""The kernels whose waves share the k loop need a stage for every wave: their launchers refuse shorter loops (no
GPU; the launches themselves are replaced by a count)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SOURCE = r"""
#include <hip/hip_runtime.h>
#include <stdio.h>
static int launches = 0;
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(...) ((void)++launches)
#include "a8_act.h"

using namespace clq;
template <class F>
static void show(const char *what, int K, F &&launch) {
    tg::Args a{};
    a.M = 64, a.N = 128, a.K = K;
    launches = 0;
    const hipError_t e = launch(a);
    printf("%s %d %d %d\n", what, K, launches, (int)(e == hipErrorInvalidValue));
}
int main() {
    for (int K = 64; K <= 320; K += 64) {
        show("act4", K, [](const tg::Args &a) {
            return launch_act_split<tg::SplitCfg<tg::Fmt::W8A8, 4>, ActEpi<Act8::Gelu, MxType::F16>>(a, nullptr);
        });
        show("plain4", K, [](const tg::Args &a) { return tg::launch_split<tg::SplitCfg<tg::Fmt::W4A8, 4>>(a, false, false, nullptr); });
        show("plain2", K, [](const tg::Args &a) { return tg::launch_split<tg::SplitCfg<tg::Fmt::W8A8, 2>>(a, true, true, nullptr); });
    }
    return 0;
}
"""


def test_a_stage_for_every_wave(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    src, exe = tmp_path / "t.hip", tmp_path / "t"
    src.write_text(SOURCE)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-ffp-contract=off", "-Xclang", "-target-feature",
                    "-Xclang", "-packed-fp32-ops", "-Wno-unused-function", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2509_24416_amd", "csrc"), str(src), "-o", str(exe)],
                   check=True, capture_output=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    seen = {(w, int(k)): (int(n), int(bad)) for w, k, n, bad in (line.split() for line in out if line)}
    assert len(seen) == 15
    for (what, K), got in seen.items():
        waves = int(what[-1])
        assert got == ((0, 1) if K // 64 < waves else (1, 0)), (what, K, got)
