// The 8-bit linears with an epilogue on few rows: with few tiles of a8_tile.h's kernel most compute units are
// idle and a launch takes the length of one wave's k loop.  Here a workgroup computes 32 tokens x 32 channels,
// its eight waves an eighth of the k loop each, with operands straight from memory (nothing is shared between
// them), kAhead stages of 64 codes ahead.  The partial sums, exact integers, meet in LDS; each thread then
// finishes two channels of a token.  What bounds it is latency: one token x 1152 -> 4608 4.4 us, x 4608 -> 1152 5.7 (weights of
// 5.3 MB, 0.9 TB/s), 300 tokens x 1152 -> 1152 6.3.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "act_epilogue.h"
#include "block.h"
#include "clq_internal.h"
#include "tile_gemm.h"

namespace clq {
namespace {
namespace a8 {

constexpr int kRowWaves = 8, kAhead = 4;

template <tg::Fmt F, Act8 A, MxType T>
__global__ void __launch_bounds__(kRowWaves * 64) a8_rows_kernel(tg::Args a)
{
    using tg::v4i;
    using tg::v4u;
    constexpr int kPitch = 36;   // ints between the rows of a partial tile, for the banks
    constexpr int HW = F == tg::Fmt::W8A8 ? 2 : 1;
    __shared__ __align__(16) int part[kRowWaves][32 * kPitch];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nks = a.K >> 6;
    const int tm = blockIdx.x / a.tiles_n, tn = blockIdx.x - tm * a.tiles_n;
    const int kb = wave * nks / kRowWaves, ke = (wave + 1) * nks / kRowWaves;
    const uint8_t *w = a.Wq + (int64_t)tn * nks * (1024 * HW) + lane * 16;   // (rows are padded to 64)
    const uint8_t *x = a.Xq + (int64_t)tm * nks * 2048 + lane * 16;
    v4u ws[kAhead][HW], xs[kAhead][2];
    auto load = [&](auto dc, int k) __attribute__((always_inline)) {
        constexpr int D = decltype(dc)::value;
#pragma unroll
        for (int h = 0; h < HW; ++h) ws[D][h] = *reinterpret_cast<const v4u *>(w + (int64_t)k * (1024 * HW) + h * 1024);
#pragma unroll
        for (int h = 0; h < 2; ++h) xs[D][h] = *reinterpret_cast<const v4u *>(x + (int64_t)k * 2048 + h * 1024);
    };

    // this thread's two channels of a token: their operands are on their way through the k loop
    const int r = tid >> 4, m = tm * 32 + r, n = tn * 32 + 2 * (tid & 15);
    const int mc = min(m, a.M - 1), n0 = min(n, a.N - 1), n1 = min(n + 1, a.N - 1);
    const float sx = a.xs[mc], sw[2] = {a.ws[n0], a.ws[n1]};
    auto value = [](const void *p, int64_t at, MxType t) {
        return t == MxType::F32 ? static_cast<const float *>(p)[at]
                                : clq::widen16(static_cast<const uint16_t *>(p)[at], t == MxType::BF16);
    };
    float b[2] = {0.0f, 0.0f}, g[2] = {1.0f, 1.0f}, res[2] = {0.0f, 0.0f};
    if (a.bias != nullptr) b[0] = value(a.bias, n0, a.bias_type), b[1] = value(a.bias, n1, a.bias_type);
    if (a.gate != nullptr) {
        const int64_t at = (int64_t)((uint32_t)mc / (uint32_t)a.sample_rows) * a.N;
        g[0] = value(a.gate, at + n0, a.gate_type), g[1] = value(a.gate, at + n1, a.gate_type);
    }
    if (a.res != nullptr) res[0] = value(a.res, (int64_t)mc * a.ldr + n0, T), res[1] = value(a.res, (int64_t)mc * a.ldr + n1, T);

    tg::v16i acc = {};
    if (kb < ke) {   // (loads past the end repeat the last stage)
        tg::static_for<0, kAhead>([&](auto d) { load(d, min(kb + decltype(d)::value, ke - 1)); });
        for (int k = kb; k < ke; k += kAhead)
            tg::static_for<0, kAhead>([&](auto dc) {
                constexpr int D = decltype(dc)::value;
                if (k + D < ke) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        v4i wi;
                        if constexpr (HW == 2) wi = __builtin_bit_cast(v4i, ws[D][h]);
                        else wi = tg::widen16(ws[D][0][2 * h], ws[D][0][2 * h + 1]);
                        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(wi, __builtin_bit_cast(v4i, xs[D][h]), acc, 0, 0, 0);
                    }
                    load(dc, min(k + D + kAhead, ke - 1));
                }
            });
    }
    // lane: token lane % 32, channels 16 (lane / 32) + 0 .. 15
    int *mine = part[wave] + (lane & 31) * kPitch + (lane >> 5) * 16;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        reinterpret_cast<v4i *>(mine)[q] = v4i{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    int s[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kRowWaves; ++i) {
        const int2 p = *reinterpret_cast<const int2 *>(part[i] + r * kPitch + 2 * (tid & 15));
        s[0] += p.x;
        s[1] += p.y;
    }
    if (m >= a.M) return;
    float y[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
        y[e] = res[e] + g[e] * activated<A>(__builtin_fmaf((float)s[e] * (sx * (1.0f / (float)(1 << tg::FmtInfo<F>::LOG))), sw[e], b[e]));
    const int64_t at = (int64_t)m * a.ldy + n;
    if constexpr (T == MxType::F32) {
        float *p = static_cast<float *>(a.Y) + at;
        if (n + 1 < a.N) *reinterpret_cast<float2 *>(p) = make_float2(y[0], y[1]);
        else if (n < a.N) p[0] = y[0];
    } else {
        uint16_t *p = static_cast<uint16_t *>(a.Y) + at;
        const uint32_t v = narrow2(y[0], y[1], T == MxType::BF16);
        if (n + 1 < a.N) *reinterpret_cast<uint32_t *>(p) = v;
        else if (n < a.N) p[0] = (uint16_t)v;
    }
}

}  // namespace a8
}  // namespace
}  // namespace clq
