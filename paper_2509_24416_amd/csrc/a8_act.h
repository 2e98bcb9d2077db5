// Launches of the 8-bit linear with activation, gate and residual, for one output type (each type is a source
// file of its own, so that they compile side by side).  The kernels are tile_gemm.h's behind
// act_epilogue.h's epilogue; the rule that picks one is the same.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdlib.h>

#include "a8_tile.h"
#include "act_epilogue.h"
#include "block.h"
#include "clq_internal.h"
#include "tile_gemm.h"

namespace clq {
namespace {

template <class C, class E>
hipError_t launch_act_tile(tg::Args a, hipStream_t stream) {
    a.tiles_m = (int)tg::tile_count(a.M, C::BM);
    a.tiles_n = (int)tg::tile_count(a.N, C::BN);
    hipLaunchKernelGGL((tg::tile_gemm_kernel<C, false, false, true, false, E>), dim3((unsigned)(a.tiles_m * a.tiles_n)),
                       dim3(C::NT), 0, stream, a);
    return hipGetLastError();
}
template <class C, class E>
hipError_t launch_act_split(tg::Args a, hipStream_t stream) {
    a.tiles_m = (int)tg::tile_count(a.M, C::BM);
    a.tiles_n = (int)tg::tile_count(a.N, C::BN);
    hipLaunchKernelGGL((tg::split_gemm_kernel<C, false, false, true, E>), dim3((unsigned)(a.tiles_m * a.tiles_n)),
                       dim3(C::NT), 0, stream, a);
    return hipGetLastError();
}

template <tg::Fmt F, int NW, int FN, class E>
hipError_t launch_act_direct(tg::Args a, hipStream_t stream) {
    a.tiles_m = (int)tg::tile_count(a.M, 64 * NW);
    a.tiles_n = (int)tg::tile_count(a.N, 32 * FN);
    hipLaunchKernelGGL((a8::a8_tile_kernel<F, NW, FN, E>), dim3((unsigned)(a.tiles_m * a.tiles_n)), dim3(NW * 64), 0, stream, a);
    return hipGetLastError();
}

template <tg::Fmt F, class E>
hipError_t launch_act_shape(const tg::Args &a, hipStream_t stream) {
    if (const char *v = getenv("CLQ_V")) switch (atoi(v)) {
        case 1: return launch_act_direct<F, 4, 4, E>(a, stream);
        case 2: return launch_act_direct<F, 2, 4, E>(a, stream);
        case 3: return launch_act_direct<F, 4, 3, E>(a, stream);
        case 4: return launch_act_direct<F, 2, 3, E>(a, stream);
        case 5: return launch_act_split<tg::SplitCfg<F, 4>, E>(a, stream);
        case 6: return launch_act_split<tg::SplitCfg<F, 2>, E>(a, stream);
    }
    switch (tg::pick_variant<F>(a.M, a.N, a.K, compute_units())) {
        case tg::kTile256: return launch_act_direct<F, 4, 4, E>(a, stream);
        case tg::kTile128: return launch_act_direct<F, 2, 4, E>(a, stream);
        case tg::kSplit4: return launch_act_split<tg::SplitCfg<F, 4>, E>(a, stream);
        case tg::kSplit2: return launch_act_split<tg::SplitCfg<F, 2>, E>(a, stream);
        case tg::kVariants: break;
    }
    return hipErrorInvalidValue;
}

template <Act8 A, MxType T>
hipError_t launch_act_format(const tg::Args &a, int wbits, hipStream_t stream) {
    return wbits == 4 ? launch_act_shape<tg::Fmt::W4A8, ActEpi<A, T>>(a, stream)
                      : launch_act_shape<tg::Fmt::W8A8, ActEpi<A, T>>(a, stream);
}

template <MxType T>
hipError_t launch_act_type(const Act8Args &g, hipStream_t stream) {
    tg::Args t{};
    t.Xq = g.Xq;
    t.xs = g.xs;
    t.Wq = g.Wq;
    t.ws = g.ws;
    t.bias = static_cast<const uint16_t *>(g.bias);
    t.bias_type = g.bias_type;
    t.gate = g.gate;
    t.gate_type = g.gate_type;
    t.sample_rows = (int)g.sample_rows;
    t.res = g.R;
    t.ldr = g.ldr;
    t.res_vec = g.ldr % 8 == 0 && reinterpret_cast<uintptr_t>(g.R) % 16 == 0;
    t.Y = g.Y;
    t.ldy = g.ldy;
    t.M = g.M;
    t.N = g.N;
    t.K = g.K;
    t.group_m = tg::kGroupPanels;
    switch (g.act) {
        case Act8::None: return launch_act_format<Act8::None, T>(t, g.wbits, stream);
        case Act8::Gelu: return launch_act_format<Act8::Gelu, T>(t, g.wbits, stream);
        case Act8::Silu: return launch_act_format<Act8::Silu, T>(t, g.wbits, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace
}  // namespace clq
