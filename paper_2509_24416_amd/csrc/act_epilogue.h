// Epilogue of the 8-bit linear with activation, gate and residual (a policy of
// tile_gemm.h's kernels):
//   y = r + gate[sample] * act(sum * x_scale * w_scale + bias), fp32, rounded once.
//
// A lane's sums are 16 channels of one token, 32 tokens side by side: as they lie, a load or store of 16
// bytes a lane is 64 places, and each lane needs other channels' scales, biases and gates in every fragment.
// So a wave turns 32 tokens at a time in its own part of LDS (the sums themselves, before any arithmetic);
// each lane then owns the same eight channels of all its tokens, holds their scale, bias and gate in
// registers, and rows are read and stored in whole 256-byte pieces.  The residual is on its way before the
// turn: its loads are the longest wait of the epilogue.  (fp32 rows: the eight channels are four and four, half a
// tile apart, so that a store's lanes lie next to each other: 8192 x 1152 -> 4608 76 -> 65 us.)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.h"
#include "tile_gemm.h"

namespace clq {
namespace {

// The tanh form of GELU and SiLU with the hardware's exp2 and reciprocal (1 ulp each): h / (1 + 2^t).
// Relative errors under 6e-7 for h > -2; below, exp2 scales up its argument's rounding with the argument
// (1e-5 at -10, where GELU is -1e-37 and SiLU's error 1e-6); absolute errors for negative h under 1e-7.
template <Act8 A>
__device__ __forceinline__ float activated(float h) {
    if constexpr (A == Act8::None) return h;
    const float t = A == Act8::Gelu ? h * __builtin_fmaf(-0.10294324f, h * h, -2.3022082f) : h * -1.4426950408889634f;
    return h * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
}

template <Act8 A, MxType T>
struct ActEpi {
    static constexpr bool kActs = true;
    static constexpr int kPitch = 528;   // bytes between the turned rows of 128 sums, for the banks
    static constexpr int kTurnBytes = 32 * kPitch;
    template <int BN, int BM> static constexpr int kOperands = 3 * BN + BM;

    // Scale, bias and gate (the tile's first sample's) of a channel a thread and scale of a token a thread, on
    // their way through the k loop; as floats in LDS after it.
    template <int BN, int BM>
    struct Operands {
        float w, x, g32;
        uint16_t b, g16;
        __device__ __forceinline__ void load(const tg::Args &a, int tm, int tn, int tid) {
            const int n = min(tn * BN + min(tid, BN - 1), a.N - 1);
            w = a.ws[n];
            x = a.xs[min(tm * BM + min(tid, BM - 1), a.M - 1)];
            if (a.bias != nullptr) b = a.bias[n];
            if (a.gate != nullptr) {
                const int64_t at = (int64_t)((uint32_t)(tm * BM) / (uint32_t)a.sample_rows) * a.N + n;
                if (a.gate_type == MxType::F32) g32 = static_cast<const float *>(a.gate)[at];
                else g16 = static_cast<const uint16_t *>(a.gate)[at];
            }
        }
        __device__ __forceinline__ void store(const tg::Args &a, float *ep, int tid) const {
            if (tid < BN) {
                ep[tid] = w;
                ep[BN + tid] = a.bias != nullptr ? clq::widen16(b, a.bias_type == MxType::BF16) : 0.0f;
                ep[2 * BN + tid] = a.gate == nullptr             ? 1.0f
                                   : a.gate_type == MxType::F32 ? g32
                                                                : clq::widen16(g16, a.gate_type == MxType::BF16);
            }
            if (tid < BM) ep[3 * BN + tid] = x;
        }
    };

    // Channel e of lane c's eight, of 32 NF.
    template <int NF>
    __device__ static __forceinline__ int channel(int c, int e) {
        if constexpr (T == MxType::F32) return 4 * c + (e & 3) + (e < 4 ? 0 : 16 * NF);
        return 8 * c + e;
    }

    // The residual of 32 tokens x 32 NF channels, as the turned lanes take it: 16 bytes a load whatever the rows'
    // alignment (29881 x 768 -> 2900 in rows of 2900, value by value 244 us).
    template <int NF>
    struct Residual {
        static constexpr int LPR = NF == 3 ? 16 : 4 * NF, RPP = 64 / LPR,   // lanes a row (NF = 3: 4 of 16 idle), rows a pass
                              PASSES = 32 / RPP, W = T == MxType::F32 ? 2 : 1;
        uint4 v[PASSES][W];
        __device__ __forceinline__ void load(const tg::Args &a, int m0, int n0, int lane) {
            typedef uint32_t Piece __attribute__((ext_vector_type(4), aligned(2)));
            if (a.res == nullptr || a.N < 8) return;
            constexpr int E = 8 / W;   // values of a load
            const int c = min(lane & (LPR - 1), 4 * NF - 1);
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int64_t row = (int64_t)min(m0 + p * RPP + lane / LPR, a.M - 1) * a.ldr;
#pragma unroll
                for (int h = 0; h < W; ++h) {
                    const int64_t at = row + min(n0 + channel<NF>(c, E * h), a.N - E);
                    const Piece q = *reinterpret_cast<const Piece *>(T == MxType::F32
                                                                         ? static_cast<const void *>(static_cast<const float *>(a.res) + at)
                                                                         : static_cast<const uint16_t *>(a.res) + at);
                    v[p][h] = make_uint4(q.x, q.y, q.z, q.w);
                }
            }
        }
        __device__ __forceinline__ void widen(int p, float (&r)[8]) const {
            if constexpr (T == MxType::F32) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 q = v[p][h];
                    r[4 * h] = __uint_as_float(q.x), r[4 * h + 1] = __uint_as_float(q.y);
                    r[4 * h + 2] = __uint_as_float(q.z), r[4 * h + 3] = __uint_as_float(q.w);
                }
            } else {
                widen8(v[p][0], T == MxType::BF16, r);
            }
        }
    };

    __device__ static __forceinline__ float element(const void *p, int64_t at) {
        return T == MxType::F32 ? static_cast<const float *>(p)[at]
                                : clq::widen16(static_cast<const uint16_t *>(p)[at], T == MxType::BF16);
    }

    // Tokens m0 .. m0 + 31 (tile tokens r0 on), fragments fn0 .. fn0 + NF - 1 of column fm of acc.
    template <tg::Fmt F, int FN, int FN0, int NF, int FM>
    __device__ static __forceinline__ void finish(const tg::Args &a, const tg::Acc<F> (&acc)[FN][2], const Residual<NF> &res,
                                                  uint8_t *turn, const float *ep, int BM, int m0, int r0, int tn, int lane) {
        constexpr int BN = 32 * FN, LPR = Residual<NF>::LPR, RPP = Residual<NF>::RPP;
        const int c = lane & (LPR - 1), rs = lane / LPR, n0 = tn * BN + FN0 * 32;
        const bool some = c < 4 * NF && n0 + channel<NF>(c, 0) < a.N;
        float w[8], b[8], g[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int ch = FN0 * 32 + channel<NF>(min(c, 4 * NF - 1), e);
            w[e] = ep[ch], b[e] = ep[BN + ch], g[e] = ep[2 * BN + ch];
        }
        const bool whole = n0 + channel<NF>(c, 7) < a.N;
        // (tiles whose tokens are of several samples: a lane looks its gates up where its sample changes; row by row
        // 43200 x 1152 -> 1152 with residual took 81 instead of 72 us for two samples, 128 instead of 104 for 5400)
        uint32_t held = a.gate == nullptr ? 0 : (uint32_t)(m0 - r0) / (uint32_t)a.sample_rows;
        const bool one = a.gate == nullptr || held == (uint32_t)min(m0 - r0 + BM - 1, a.M - 1) / (uint32_t)a.sample_rows;
        const bool gated = a.gate != nullptr, vec = a.res != nullptr && whole;
        constexpr float kDown = 1.0f / (float)(1 << tg::FmtInfo<F>::LOG);
        uint8_t *mine = turn + (lane & 31) * kPitch + (lane >> 5) * 64;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (a wave's LDS accesses stay in order)
        tg::static_for<0, NF>([&](auto fc) {
            const tg::Acc<F> &x = acc[FN0 + decltype(fc)::value][FM];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                reinterpret_cast<tg::v4i *>(mine + decltype(fc)::value * 128)[q] =
                    tg::v4i{(int)x[4 * q], (int)x[4 * q + 1], (int)x[4 * q + 2], (int)x[4 * q + 3]};
        });
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (!some) return;
#pragma unroll
        for (int p = 0; p < Residual<NF>::PASSES; ++p) {
            const int r = p * RPP + rs, m = m0 + r;
            const uint8_t *row = turn + r * kPitch;
            const int4 lo = *reinterpret_cast<const int4 *>(row + channel<NF>(c, 0) * 4);
            const int4 hi = *reinterpret_cast<const int4 *>(row + channel<NF>(c, 4) * 4);
            const int s[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            const float xs = ep[3 * BN + r0 + r] * kDown;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = activated<A>(__builtin_fmaf((float)s[e] * xs, w[e], b[e]));
            if (m >= a.M) continue;
            if (gated) {
                if (!one) {
                    const uint32_t sample = (uint32_t)m / (uint32_t)a.sample_rows;
                    if (sample != held) {
                        held = sample;
                        const int64_t at = (int64_t)sample * a.N;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int64_t i = at + min(n0 + channel<NF>(c, e), a.N - 1);
                            g[e] = a.gate_type == MxType::F32
                                       ? static_cast<const float *>(a.gate)[i]
                                       : clq::widen16(static_cast<const uint16_t *>(a.gate)[i], a.gate_type == MxType::BF16);
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= g[e];
            }
            if (vec) {
                float t[8];
                res.widen(p, t);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] += t[e];
            } else if (a.res != nullptr) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int n = n0 + channel<NF>(c, e);
                    if (n < a.N) y[e] += element(a.res, (int64_t)m * a.ldr + n);
                }
            }
            const int64_t at = (int64_t)m * a.ldy + n0;
            if (whole) {
                if constexpr (T == MxType::F32) {
                    float *dst = static_cast<float *>(a.Y) + at;
                    *reinterpret_cast<float4 *>(dst + channel<NF>(c, 0)) = make_float4(y[0], y[1], y[2], y[3]);
                    *reinterpret_cast<float4 *>(dst + channel<NF>(c, 4)) = make_float4(y[4], y[5], y[6], y[7]);
                } else {
                    store8(a.Y, at + channel<NF>(c, 0), T, y);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int n = channel<NF>(c, e);
                    if (n0 + n < a.N) {
                        if constexpr (T == MxType::F32) static_cast<float *>(a.Y)[at + n] = y[e];
                        else static_cast<uint16_t *>(a.Y)[at + n] = (uint16_t)narrow2(y[e], y[e], T == MxType::BF16);
                    }
                }
            }
        }
    }

    // a wave's FN x 2 fragments (behind the operands' barrier)
    template <tg::Fmt F, int FN>
    __device__ static __forceinline__ void finish_tile(const tg::Args &a, const tg::Acc<F> (&acc)[FN][2], uint8_t *turn,
                                                       const float *ep, int BM, int tm, int tn, int wave, int lane) {
        const int r0 = wave * 64, m0 = tm * BM + r0;
        if (m0 >= a.M) return;
        Residual<FN> first, second;
        first.load(a, m0, tn * 32 * FN, lane);
        if constexpr (T != MxType::F32) second.load(a, m0 + 32, tn * 32 * FN, lane);
        __builtin_amdgcn_sched_barrier(0);
        finish<F, FN, 0, FN, 0>(a, acc, first, turn, ep, BM, m0, r0, tn, lane);
        if (m0 + 32 >= a.M) return;
        if constexpr (T == MxType::F32) second.load(a, m0 + 32, tn * 32 * FN, lane);
        __builtin_amdgcn_sched_barrier(0);
        finish<F, FN, 0, FN, 1>(a, acc, second, turn, ep, BM, m0 + 32, r0 + 32, tn, lane);
    }
    // a wave's NF fragments of one token unit, after the k loop's parts have met
    template <tg::Fmt F, int FN0, int NF, int FM>
    __device__ static __forceinline__ void finish_unit(const tg::Args &a, const tg::Acc<F> (&acc)[4][2], uint8_t *turn,
                                                       const float *ep, int BM, int tm, int tn, int r0, int lane) {
        const int m0 = tm * BM + r0;
        if (m0 >= a.M) return;
        Residual<NF> res;
        res.load(a, m0, tn * 128 + FN0 * 32, lane);
        __builtin_amdgcn_sched_barrier(0);
        finish<F, 4, FN0, NF, FM>(a, acc, res, turn, ep, BM, m0, r0, tn, lane);
    }
};

}  // namespace
}  // namespace clq
