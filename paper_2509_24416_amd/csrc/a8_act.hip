// W4A8 and W8A8 linear with activation, gate and residual in its epilogue:
//   Y = R + gate[sample] * act(sum * x_scale * w_scale + bias),
// all of it in fp32 on the exact integer sums, rounded once.
//
// The kernels are tile_gemm.h's with another epilogue; the rule that picks one is the same.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.h"
#include "clq_internal.h"
#include "tile_gemm.h"

namespace clq {
namespace {

template <class C, tg::Epi E>
hipError_t launch_tile(tg::Args a, hipStream_t stream) {
    a.tiles_m = (int)tg::tile_count(a.M, C::BM);
    a.tiles_n = (int)tg::tile_count(a.N, C::BN);
    hipLaunchKernelGGL((tg::tile_gemm_kernel<C, false, false, true, false, E>), dim3((unsigned)(a.tiles_m * a.tiles_n)),
                       dim3(C::NT), 0, stream, a);
    return hipGetLastError();
}
template <class C, tg::Epi E>
hipError_t launch_split(tg::Args a, hipStream_t stream) {
    a.tiles_m = (int)tg::tile_count(a.M, C::BM);
    a.tiles_n = (int)tg::tile_count(a.N, C::BN);
    hipLaunchKernelGGL((tg::split_gemm_kernel<C, false, false, true, E>), dim3((unsigned)(a.tiles_m * a.tiles_n)),
                       dim3(C::NT), 0, stream, a);
    return hipGetLastError();
}

template <tg::Fmt F, tg::Epi E>
hipError_t launch_shape(const tg::Args &a, hipStream_t stream) {
    switch (tg::pick_variant<F>(a.M, a.N, a.K, compute_units())) {
        case tg::kTile256: return launch_tile<tg::Cfg<F, 4, tg::kRing256<F>>, E>(a, stream);
        case tg::kTile128: return launch_tile<tg::Cfg<F, 2, tg::kRing128<F>>, E>(a, stream);
        case tg::kSplit4: return launch_split<tg::SplitCfg<F, 4>, E>(a, stream);
        case tg::kSplit2: return launch_split<tg::SplitCfg<F, 2>, E>(a, stream);
        case tg::kVariants: break;
    }
    return hipErrorInvalidValue;
}

template <tg::Fmt F>
hipError_t launch_type(const tg::Args &a, MxType type, hipStream_t stream) {
    switch (type) {
        case MxType::F16: return launch_shape<F, tg::Epi::F16>(a, stream);
        case MxType::BF16: return launch_shape<F, tg::Epi::BF16>(a, stream);
        case MxType::F32: return launch_shape<F, tg::Epi::F32>(a, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_a8_act(const Act8Args &g, hipStream_t stream) {
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
    t.act = (int)g.act;
    t.res = g.R;
    t.ldr = g.ldr;
    t.res_vec = g.ldr % 8 == 0 && reinterpret_cast<uintptr_t>(g.R) % 16 == 0;
    t.Y = g.Y;
    t.ldy = g.ldy;
    t.M = g.M;
    t.N = g.N;
    t.K = g.K;
    t.group_m = tg::kGroupPanels;
    return g.wbits == 4 ? launch_type<tg::Fmt::W4A8>(t, g.type, stream) : launch_type<tg::Fmt::W8A8>(t, g.type, stream);
}

}  // namespace clq
