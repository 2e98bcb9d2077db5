// Launches of the 8-bit linear with activation, gate and residual, for one output type (each type is a source
// file of its own, so that they compile side by side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "a8_rows.h"
#include "a8_tile.h"
#include "act_epilogue.h"
#include "block.h"
#include "clq_internal.h"
#include "tile_gemm.h"

namespace clq {
namespace {

template <class C, class E>
hipError_t launch_act_split(tg::Args a, hipStream_t stream) {
    if (!tg::stage_each<C>(a)) return hipErrorInvalidValue;
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

template <tg::Fmt F, Act8 A, MxType T>
hipError_t launch_act_rows(tg::Args a, hipStream_t stream) {
    a.tiles_m = (int)tg::tile_count(a.M, 32);
    a.tiles_n = (int)tg::tile_count(a.N, 32);
    hipLaunchKernelGGL((a8::a8_rows_kernel<F, A, T>), dim3((unsigned)(a.tiles_m * a.tiles_n)), dim3(a8::kRowWaves * 64), 0,
                       stream, a);
    return hipGetLastError();
}

// The kernel of a shape, c compute units (us: 8-bit weights, GELU, replayed from a graph):
//   few tiles of 32 x 32     the rows kernel up to 2 c of them (one token x 4608 -> 1152 5.7, on 64 x 128 tiles with
//                            the k loop over four waves 10.8; 300 x 1152 -> 1152, 1.4 c, 6.3 / 7.8; 128 x 1152 -> 4608,
//                            2.25 c, 8.2 / 7.8);
//   t = M / 64 x N / 128     k over four waves up to t = 2 c, where they have a stage each (2560 x 4608 -> 1152,
//   (rounded up)             1.4 c, 26.0, 96-channel tiles 27.8; 4096 x 4608 -> 1152, 2.25 c, 37.7 / 31.5);
//   otherwise                256-token tiles, of 96 channels where these are no more to a compute unit than those
//                            of 128 (8192 x 4608 -> 1152: 384 and 288 of them, two a unit, 51.8 / 57.8; 4096 x 1152 ->
//                            4608: 768 and 576, three a unit, 36.0 / 37.4; 12000 x 4608 -> 1152: 564 and 423, 77.5 /
//                            65.8; 6144: 288 and 216, 48.0 / 38.4; 8192 x 1152 -> 4608: 1536 and 1152, 63.6 / 61.7).
// Tiles of 128 tokens and the k loop over two waves won nowhere by more than 3%.  4-bit weights, residuals and fp32
// results go by the same lines, which were not measured with them; with the k loop over four waves the epilogue spills 64
// registers, 124 to 144 for fp32 results.
template <tg::Fmt F, Act8 A, MxType T>
hipError_t launch_act_shape(const tg::Args &a, hipStream_t stream) {
    using E = ActEpi<A, T>;
    const int64_t c = compute_units(), M = a.M, N = a.N;
    if (tg::tile_count(M, 32) * tg::tile_count(N, 32) <= 2 * c) return launch_act_rows<F, A, T>(a, stream);
    if (tg::tile_count(M, 64) * tg::tile_count(N, 128) <= 2 * c && tg::stage_each<tg::SplitCfg<F, 4>>(a))
        return launch_act_split<tg::SplitCfg<F, 4>, E>(a, stream);
    const int64_t t128 = tg::tile_count(M, 256) * tg::tile_count(N, 128), t96 = tg::tile_count(M, 256) * tg::tile_count(N, 96);
    if ((t96 + c - 1) / c <= (t128 + c - 1) / c) return launch_act_direct<F, 4, 3, E>(a, stream);
    return launch_act_direct<F, 4, 4, E>(a, stream);
}

template <Act8 A, MxType T>
hipError_t launch_act_format(const tg::Args &a, int wbits, hipStream_t stream) {
    return wbits == 4 ? launch_act_shape<tg::Fmt::W4A8, A, T>(a, stream) : launch_act_shape<tg::Fmt::W8A8, A, T>(a, stream);
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
