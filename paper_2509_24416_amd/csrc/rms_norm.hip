// RMS norm with the residual's addition, its result plain (fp16, bf16, fp32) or rotated
// (CLQ, arXiv 2509.24416, Sec. 3.3) and quantized to 8 bits a token (Sec. 3.1, Eq. (1) with
// n = 8) for the 8-bit linears.
//
//   s = x + r,  n = s w / sqrt(mean(s^2) + eps),  x~ = FWHT_b(gather(n, perm))
//
// The rotation is linear, so a row's factor 1 / sqrt(..) is left out of it: with v = FWHT_b(gather(s w))
// and m = max|v|, the codes are rne(v * 127 / m), which do not hold the factor at all, and the scale is
// m / 127 times the factor.  One pass over a row then yields its squares' sum and its maximum together,
// between one pair of barriers, and no value is kept anywhere but in registers.
//
// What bounds it is memory, so the split is the rotate+quantize kernels': a lane owns one 16-byte
// chunk (8 columns) of four rows.  Sums and maxima meet over 8 lanes by lane permutes, then through LDS
// in a fixed order (each lane of an octet adds every eighth octet's partials, then the octet adds up),
// so that results do not depend on the order in which waves arrive.
//
// Measured (a copy reaches 5.2 to 5.7 TB/s): 43200 x 1152 with a 16-bit residual to 8 bits 67 to 75 us (4.6 to 5.2
// TB/s), with an fp32 one 105 (5.2), without one 40 (3.7: vector instructions); plain with residual 77 (5.2); 8192 x 4608
// plain with residual 53 (5.7); 3000 x 12288 57 (5.2), to 8 bits 65 (3.9: two chunks a lane), gathered 76; fp32 rows of 43200 x
// 1152 quantized 45 (5.6).  Samples whose rows are no multiple of four: 43204 x 1152 in two plain with residual
// 111 us (two samples of 21600 rows 76), to 8 bits 114 (67), without a residual 67 (38): weights are read for each row, and
// registers spill.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "block.h"
#include "rq_device.h"

namespace clq {
namespace {

constexpr int kMaxGroups = 8;    // four-row groups per workgroup
constexpr int kMaxLanes = 1024;
constexpr int kLdsLimit = 160 * 1024 - 8192;   // gathered rows of a workgroup, beside the partials

struct NormArgs : RmsNormArgs {
    int groups, stride;   // four-row groups per workgroup, lanes of each
    float inv_k;
    int unit0, units;     // first 32-row unit of this launch, units
};

// the larger of two magnitudes, a NaN if either is one
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// over the eight lanes of an octet, in each of them
constexpr int kHalfMirror = 0x141;   // DPP control: lane ^ 7
template <class Op>
__device__ __forceinline__ float octet(float v, Op &&op) {
    v = op(v, lane_xchg<kLaneXor1>(v));
    v = op(v, lane_xchg<kLaneXor2>(v));
    return op(v, lane_xchg<kHalfMirror>(v));
}

template <int CTRL>
__device__ __forceinline__ void pair_exchange(uint32_t &lo, uint32_t &hi, bool b) {
    const uint32_t plo = lane_xchg<CTRL>(lo), phi = lane_xchg<CTRL>(hi);
    lo = b ? phi : lo;
    hi = b ? hi : plo;
}

// The codes of one chunk column of a quad's four rows (rows rho0 .. rho0 + 3 of unit u) from rotated
// values and the rows' signed reciprocals: a 16-byte operand piece is the even codes of 16, then the
// odd, of a lane pair; lane b0 of the pair stores rows b0 and 2 + b0.
__device__ __forceinline__ void store_codes8(const float (&x)[4][8], const float (&rs)[4], int64_t u, int rho0, int chunk,
                                             int K, uint8_t *__restrict__ out, bool active) {
    constexpr float M = Grid<8>::magic;
    const int lam = chunk & 3;
    const bool b0 = lam & 1;
    uint32_t ev[4], od[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(__builtin_fmaf(x[r][e], rs[r], M));
        ev[r] = low_bytes4(w[0], w[2], w[4], w[6]) ^ 0x80808080u;
        od[r] = low_bytes4(w[1], w[3], w[5], w[7]) ^ 0x80808080u;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        pair_exchange<kLaneXor1>(ev[2 * s], ev[2 * s + 1], b0);
        pair_exchange<kLaneXor1>(od[2 * s], od[2 * s + 1], b0);
        if (active)
            *reinterpret_cast<uint4 *>(out + q8_piece_offset(u, rho0 + 2 * s + (lam & 1), chunk >> 2, lam >> 1, K)) =
                make_uint4(ev[2 * s], ev[2 * s + 1], od[2 * s], od[2 * s + 1]);
    }
}

enum class Res { None, F16, BF16, F32 };

// Waves a SIMD that the registers are held to: what the forms of one sample with a chunk a lane need by themselves or a few
// less (4 of 57 spill, one register mostly, 10 at most).  It does not look at MIXED, whose forms spill up to 29 registers
// with one chunk a lane and 32 to 101 with two; of one sample and two chunks those to 8 bits spill 8 to 22.
template <int B, MxType XT, Res RT, bool NORM, int NCH>
constexpr int waves_per_simd() {
    if (NCH == 2) return 4;   // (a workgroup of 16 waves)
    return NORM ? 7 - (B != 0) - (XT == MxType::F32 || RT == Res::F32) : 7;
}

// B: Hadamard block (0: plain result).  XT, RT: types of X and the residual (as branches at run time they cost
// 8192 x 4608 with a residual 58.7 instead of 52.8 us, to 8 bits 59.4 instead of 55.0).  NORM: without it the rows
// are only rotated and quantized.  MIXED: four rows may be of several samples (a branch for it at run time costs
// every launch 20 registers).  NCH: chunks per lane (1: rows of up to 8192 columns, 2: up to 16384).
template <int B, MxType XT, Res RT, bool NORM, bool MIXED, int NCH>
__global__ void __launch_bounds__(kMaxLanes) __attribute__((amdgpu_waves_per_eu(waves_per_simd<B, XT, RT, NORM, NCH>())))
rms_norm_kernel(NormArgs a)
{
    constexpr bool XW = XT == MxType::F32;
    constexpr MxType kSum = RT == Res::F32 ? MxType::F32 : RT == Res::BF16 ? MxType::BF16 : MxType::F16;
    static_assert(NORM || (B != 0 && RT == Res::None), "a quantizer");
    extern __shared__ __align__(16) float gat[];   // gathered inputs: a column's rows side by side
    __shared__ float4 psum[NORM ? kMaxLanes / 8 : 1], pmax[B ? kMaxLanes / 8 : 1];
    const int t = threadIdx.x;
    const int groups = NCH == 2 ? 1 : a.groups, wpu = 8 / groups;   // workgroups per unit
    const int idx = blockIdx.x >> 3;
    const int ul = (int)(blockIdx.x & 7) + 8 * (idx / wpu);
    if (ul >= a.units) return;
    const int u = a.unit0 + ul;
    const int K = a.K, cpr = K >> 3;
    // (a workgroup of wide rows has one group: its rows' addresses are scalars)
    const int gl = NCH == 2 ? 0 : t / a.stride, t0 = t - gl * a.stride;
    const bool glive = NCH == 2 || gl < a.groups;
    const int s = (idx % wpu) * groups + (glive ? gl : 0);
    const uint32_t row0 = (uint32_t)u * 32 + 4 * s;
    const int lane_c = logical_lane(t0);   // its chunk among the octet's eight
    if (B == 0 && (uint32_t)u * 32 + 4 * ((idx % wpu) * groups) >= (uint32_t)a.M) return;   // (codes are written to the unit's end)
    // rows of the four that exist; the others read the last of all
    const int rows = glive && row0 < (uint32_t)a.M ? (int)min(4u, (uint32_t)a.M - row0) : 0;
    auto row_of = [&](int r) { return (int64_t)min(row0 + r, (uint32_t)a.M - 1); };

    // s w of each chunk, and the rows' sums of squares
    float x[NCH][4][8], sq[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    {
        auto as_floats = [](const uint4 &q, float *f) {
            f[0] = __uint_as_float(q.x), f[1] = __uint_as_float(q.y), f[2] = __uint_as_float(q.z), f[3] = __uint_as_float(q.w);
        };
        const uint32_t sr = (uint32_t)a.sample_rows;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int chunk = lane_c + i * a.stride, at = min(chunk, cpr - 1) * 8;
            const bool live = chunk < cpr;
            uint4 v[4][XW ? 2 : 1], res[4][RT == Res::F32 ? 2 : 1];
            // (unconditional, so that all of a chunk are in flight)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (XW) {
                    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const float *>(a.X) + row_of(r) * a.ldx + at);
                    v[r][0] = p[0];
                    v[r][1] = p[1];
                } else {
                    v[r][0] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.X) + row_of(r) * a.ldx + at);
                }
            }
            if constexpr (RT == Res::F16 || RT == Res::BF16) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    res[r][0] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.R) + row_of(r) * a.ldr + at);
            } else if constexpr (RT == Res::F32) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const float *>(a.R) + row_of(r) * a.ldr + at);
                    res[r][0] = p[0];
                    res[r][1] = p[1];
                }
            }
            float w[8];
            if constexpr (NORM) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = 1.0f;
                if (!MIXED && a.W != nullptr) load8(a.W, (int64_t)((uint32_t)row_of(0) / sr) * K + at, a.w_type, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = live ? w[e] : 0.0f;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float(&y)[8] = x[i][r];
                if constexpr (XW) as_floats(v[r][0], y), as_floats(v[r][1], y + 4);
                else widen8(v[r][0], XT == MxType::BF16, y);
                if constexpr (RT != Res::None) {
                    float q[8];
                    if constexpr (RT == Res::F32) as_floats(res[r][0], q), as_floats(res[r][1], q + 4);
                    else widen8(res[r][0], RT == Res::BF16, q);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] += q[e];
                    if (r < rows && live) store8(a.sum, row_of(r) * a.ld_sum + at, kSum, y);
                }
                if (r >= rows || !live) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = 0.0f;
                }
                if constexpr (NORM) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) sq[r] = __builtin_fmaf(y[e], y[e], sq[r]);
                    if (MIXED && live) load8(a.W, (int64_t)((uint32_t)row_of(r) / sr) * K + at, a.w_type, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] *= w[e];
                }
            }
            if (i + 1 < NCH) __builtin_amdgcn_sched_barrier(0);   // (both chunks' loads in flight: registers spill)
        }
    }

    const CrossSigns cs = cross_signs<B ? B : 32>(lane_c);
    if constexpr (B != 0) {
        if (a.perm != nullptr) {
            // P rows of the group at a time, a column's side by side: one LDS read serves them
            constexpr int P = NCH == 1 ? 4 : 2;
            float *mine = gat + (int64_t)(glive ? gl : 0) * K * P;
#pragma unroll
            for (int p0 = 0; p0 < 4; p0 += P) {
                if (p0 > 0) __syncthreads();
#pragma unroll
                for (int i = 0; i < NCH; ++i) {
                    const int chunk = lane_c + i * a.stride;
                    if (glive && chunk < cpr) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
#pragma unroll
                            for (int p = 0; p < P; ++p) mine[(chunk * 8 + e) * P + p] = x[i][p0 + p][e];
                    }
                }
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NCH; ++i) {
                    const int32_t *q = a.perm + min(lane_c + i * a.stride, cpr - 1) * 8;
                    float g[P][8];   // (read by all lanes: a condition around the reads costs 10 of 82 us)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float *c = mine + (int64_t)q[e] * P;
#pragma unroll
                        for (int p = 0; p < P; ++p) g[p][e] = c[p];
                    }
                    const bool live = lane_c + i * a.stride < cpr;
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[i][p0 + p][e] = live ? g[p][e] : 0.0f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float p = x[i][r][e], q = x[i][r][e + 1];
                    x[i][r][e] = p + q;
                    x[i][r][e + 1] = p - q;
                }
                fwht8_rest(x[i][r]);
            }
            cross_stages<B, 4>(x[i], cs);
        }
    }

    // the rows' sums and maxima: octet, LDS, octet
    float m[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [](float p, float q) { return p + q; };
    auto larger = [](float p, float q) { return max_nan(p, q); };
    if constexpr (B != 0) {
#pragma unroll
        for (int i = 0; i < NCH; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < 8; ++e) m[r] = max_nan(m[r], fabsf(x[i][r][e]));
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if constexpr (NORM) sq[r] = octet(sq[r], add);
        if constexpr (B != 0) m[r] = octet(m[r], larger);
    }
    if ((t & 7) == 0) {
        if constexpr (NORM) psum[t >> 3] = make_float4(sq[0], sq[1], sq[2], sq[3]);
        if constexpr (B != 0) pmax[t >> 3] = make_float4(m[0], m[1], m[2], m[3]);
    }
    __syncthreads();
    const int first = (glive ? gl : 0) * (a.stride >> 3);
#pragma unroll
    for (int r = 0; r < 4; ++r) sq[r] = m[r] = 0.0f;
    for (int j = t & 7; j < a.stride >> 3; j += 8) {
        if constexpr (NORM) {
            const float4 p = psum[first + j];
            sq[0] += p.x, sq[1] += p.y, sq[2] += p.z, sq[3] += p.w;
        }
        if constexpr (B != 0) {
            const float4 q = pmax[first + j];
            m[0] = max_nan(m[0], q.x), m[1] = max_nan(m[1], q.y), m[2] = max_nan(m[2], q.z), m[3] = max_nan(m[3], q.w);
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if constexpr (NORM) sq[r] = octet(sq[r], add);
        if constexpr (B != 0) m[r] = octet(m[r], larger);
    }
    // each lane of a quad works out one of its four rows, the quad shares the results
    const int mine = t & 3;
    auto of_mine = [&](const float (&v)[4]) { return mine == 0 ? v[0] : mine == 1 ? v[1] : mine == 2 ? v[2] : v[3]; };
    // (1 ulp; eps is a normal number)
    const float inv = NORM ? __builtin_amdgcn_rsqf(__builtin_fmaf(of_mine(sq), a.inv_k, a.eps)) : 1.0f;
    auto quad = [](float v, float (&all)[4]) {
        all[0] = lane_xchg<kQuadLane0>(v), all[1] = lane_xchg<kQuadLane1>(v);
        all[2] = lane_xchg<kQuadLane2>(v), all[3] = lane_xchg<kQuadLane3>(v);
    };

    if constexpr (B == 0) {
        float factor[4];
        quad(inv, factor);
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int chunk = lane_c + i * a.stride;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][r][e] *= factor[r];
                if (r < rows && chunk < cpr) store8(a.Y, row_of(r) * a.ldy + chunk * 8, a.y_type, x[i][r]);
            }
        }
    } else {
        // (maxima whose 127 / m would overflow count as zeros: eps keeps the factor finite)
        float top = of_mine(m);
        top = top < 0x1p-119f ? 0.0f : top;
        if (t0 < 4 && mine < rows) a.x_scale[row_of(mine)] = (top / 127.0f) * inv;
        float rs[4];
        quad(top == 0.0f ? 0.0f : 127.0f / top, rs);
#pragma unroll
        for (int r = 0; r < 4; ++r) rs[r] *= cs.sign;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int chunk = lane_c + i * a.stride;
            store_codes8(x[i], rs, u, 4 * s, chunk, K, a.Xq8, glive && chunk < cpr);
        }
    }
}

// Four-row groups per workgroup: the most live lanes on a compute unit (lane utilisation of whole waves times
// the share of its wave slots that whole workgroups fill), on a tie the fewest, since the other workgroups of a
// unit work while one waits at its barrier (43200 x 1152 with residual to 8 bits, 8 workgroups of 3 waves 73 us, 2
// of 9 82; 43200 x 576 36 / 45), but no more than leaves two workgroups per compute unit to the launch.
int pick_groups(int stride, int64_t total_groups, int cus, int most_waves) {
    int best = 1;
    double best_u = 0.0;
    for (int g = 1; g <= kMaxGroups && g * stride <= kMaxLanes; g <<= 1) {
        if (g > 1 && g * stride > 64 && total_groups / g < 2 * cus) break;
        const int waves = (g * stride + 63) / 64;
        if (g > 1 && waves > most_waves / 2) break;
        const double u = (double)(g * stride) * (most_waves / waves);
        if (u > best_u) {
            best_u = u;
            best = g;
        }
    }
    return best;
}

template <int B, MxType XT, Res RT, bool NORM, bool MIXED, int NCH>
hipError_t launch_norm(const RmsNormArgs &args, hipStream_t stream) {
    NormArgs a;
    static_cast<RmsNormArgs &>(a) = args;
    a.inv_k = 1.0f / (float)a.K;
    const int cpr = a.K >> 3;
    const int64_t units = padded_act_rows(a.M) / 32;
    constexpr int P = NCH == 1 ? 4 : 2;
    if constexpr (NCH == 1) {
        a.stride = (cpr + 7) / 8 * 8;
        a.groups = pick_groups(a.stride, units * 8, compute_units(), 4 * waves_per_simd<B, XT, RT, NORM, NCH>());
        while (B != 0 && a.perm != nullptr && a.groups > 1 && (size_t)a.groups * a.K * P * 4 > kLdsLimit) a.groups >>= 1;
    } else {
        a.groups = 1;
        a.stride = ((cpr + 1) / 2 + 63) / 64 * 64;
    }
    const int T = (a.groups * a.stride + 63) / 64 * 64;
    const size_t lds = B != 0 && a.perm != nullptr ? (size_t)a.groups * a.K * P * 4 : 0;
    if (T > kMaxLanes || lds > kLdsLimit) return hipErrorInvalidConfiguration;
    if (lds > 65536 - 8192) {
        hipError_t e = hipFuncSetAttribute((const void *)rms_norm_kernel<B, XT, RT, NORM, MIXED, NCH>,
                                           hipFuncAttributeMaxDynamicSharedMemorySize, kLdsLimit);
        if (e != hipSuccess) return e;
    }
    // launches of at most 2^31 lanes
    const int64_t per_unit = (int64_t)(8 / a.groups) * T;
    const int64_t most = std::max<int64_t>(8, (((int64_t)1 << 31) / per_unit) / 8 * 8);
    for (int64_t u0 = 0; u0 < units; u0 += most) {
        a.unit0 = (int)u0;
        a.units = (int)std::min<int64_t>(most, units - u0);
        const int64_t grid = ((int64_t)a.units + 7) / 8 * 8 * (8 / a.groups);
        hipLaunchKernelGGL((rms_norm_kernel<B, XT, RT, NORM, MIXED, NCH>), dim3((unsigned)grid), dim3(T), lds, stream, a);
    }
    return hipGetLastError();
}

template <int B, MxType XT, Res RT, bool NORM>
hipError_t launch_width(const RmsNormArgs &a, hipStream_t stream) {
    if constexpr (NORM)
        if (a.W != nullptr && a.sample_rows < a.M && a.sample_rows % 4 != 0)
            return a.K <= 8 * kMaxLanes ? launch_norm<B, XT, RT, NORM, true, 1>(a, stream)
                                        : launch_norm<B, XT, RT, NORM, true, 2>(a, stream);
    return a.K <= 8 * kMaxLanes ? launch_norm<B, XT, RT, NORM, false, 1>(a, stream)
                                : launch_norm<B, XT, RT, NORM, false, 2>(a, stream);
}
template <int B, MxType XT>
hipError_t launch_residual(const RmsNormArgs &a, hipStream_t stream) {
    if constexpr (B != 0)
        if (!a.norm) return launch_width<B, XT, Res::None, false>(a, stream);
    if (a.R == nullptr) return launch_width<B, XT, Res::None, true>(a, stream);
    switch (a.r_type) {
        case MxType::F16: return launch_width<B, XT, Res::F16, true>(a, stream);
        case MxType::BF16: return launch_width<B, XT, Res::BF16, true>(a, stream);
        default: return launch_width<B, XT, Res::F32, true>(a, stream);
    }
}
template <int B>
hipError_t launch_type(const RmsNormArgs &a, hipStream_t stream) {
    switch (a.x_type) {
        case MxType::F16: return launch_residual<B, MxType::F16>(a, stream);
        case MxType::BF16: return launch_residual<B, MxType::BF16>(a, stream);
        default: return launch_residual<B, MxType::F32>(a, stream);
    }
}

// One 16-byte operand piece (16 codes of a row) per thread: four threads write a row's 64 codes, sixteen
// rows a wave read whole 256-byte pieces.  Memory-bound: 43200 x 1152 to fp16 23 to 25 us (6 TB/s, partly from cache).
__global__ void dequantize_act8_kernel(const uint8_t *__restrict__ q8, const float *__restrict__ scale, int64_t M, int K,
                                       MxType type, void *__restrict__ out, int64_t ldo) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int piece = (int)(i & 3), rho = (int)(i >> 2) & 31;
    const int64_t unit = i >> 7, kus = K >> 6, u = unit / kus, ku = unit - u * kus;
    const int64_t row = u * 32 + rho;
    if (row >= M) return;
    const int h = piece >> 1, q = piece & 1;
    const uint4 v = *reinterpret_cast<const uint4 *>(q8 + q8_piece_offset(u, rho, 2 * ku + h, q, K));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const float sc = scale[row];
    const int64_t at = row * ldo + ku * 64 + h * 32 + q * 16;
#pragma unroll
    for (int half = 0; half < 2; ++half) {   // (bytes 0 .. 7: even codes, 8 .. 15: odd ones)
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = (float)(int8_t)(w[2 * (e & 1) + half] >> (8 * (e >> 1))) * sc;
        store8(out, at + 8 * half, type, x);
    }
}

}  // namespace

hipError_t launch_rms_norm(const RmsNormArgs &a, hipStream_t stream) {
    if (a.Y != nullptr) return launch_type<0>(a, stream);
    switch (a.block) {
        case 32: return launch_type<32>(a, stream);
        case 64: return launch_type<64>(a, stream);
        case 128: return launch_type<128>(a, stream);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_dequantize_act8(const uint8_t *Xq8, const float *x_scale, int64_t M, int K, MxType type, void *out,
                                  int64_t ldo, hipStream_t stream) {
    // units of 32 rows x 64 codes, 128 threads each; launches of at most 2^31 lanes
    const int64_t units = (padded_act_rows(M) >> 5) * (K >> 6), kus = K >> 6;
    const int64_t most = (((int64_t)1 << 24) / kus) * kus;   // whole row units
    for (int64_t u0 = 0; u0 < units; u0 += most) {
        const int64_t n = std::min(most, units - u0), rows0 = u0 / kus * 32;
        hipLaunchKernelGGL(dequantize_act8_kernel, dim3((unsigned)((n + 1) / 2)), dim3(256), 0, stream,
                           Xq8 + u0 * 2048, x_scale + rows0, M - rows0, K, type,
                           static_cast<uint8_t *>(out) + rows0 * ldo * (type == MxType::F32 ? 4 : 2), ldo);
    }
    return hipGetLastError();
}

}  // namespace clq
