// Rotary positions with several axes (time, height, width), on heads that may be normed first:
// pair i of a head, (a, b) -> (a cos - b sin, b cos + a sin) at the angle
// position[row, axis(i)] * freq[i].
//
// Angles are formed as revolutions, position * freq / 2 pi, each of the two products as the sum of two fp64 numbers
// (rounded once to fp64, 2^31 positions on, an angle is off by 2e-7, as much as 4 fp32 roundings of its sine), and
// reduced there (less their nearest whole number), so that far positions are as exact as near ones; sine and cosine
// then take an fp32 argument of half a revolution at most.
//
// What bounds it is memory (every value read and written once), and on few heads the sines, which a row's heads
// share.  So a lane owns the same piece of every head that it works on, an item: eight columns (interleaved
// pairs), or V columns and their partners (halves paired; V = 8, or 4 where half of the turned columns is no
// multiple of 8), and a wave takes as many heads side by side as its 64 lanes hold, several rows where a row's
// heads do not fill it.  Its lanes work out the angles of its rows together and take their items' from LDS.
//
// Measured: 43200 rows of 32 heads of 72 columns, pairs 70 to 78 us (5.1 to 5.7 TB/s), halves (8 bytes a lane) 96, heads
// normed 90 (one set of weights) and 96; 4608 rows of 48 heads of 128, halves, normed 24 to 27 (from the cache in part); 20000 rows of
// 8 heads of 64 13 to 14.  With the angles worked out by each lane for itself 84, 100, 98 and 104; 29; 17 to 18.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "block.h"

namespace clq {
namespace {

struct RopeLaunch : RopeArgs {
    int items, turned;   // items of a head, those that turn
    int side;            // heads side by side in a wave
    int rows;            // rows of a wave
    int slices;          // waves that share a row's heads
    int64_t m0, m1;      // rows of this launch
    float inv_d;
};

// V 16-bit values as they lie, and widened
template <int V> struct Raw;
template <> struct Raw<8> { uint4 v; };
template <> struct Raw<4> { uint2 v; };
template <int V>
__device__ __forceinline__ Raw<V> load_raw(const uint16_t *p) {
    return {*reinterpret_cast<const decltype(Raw<V>::v) *>(p)};
}
template <int V>
__device__ __forceinline__ void widen(const Raw<V> &r, bool bf16, float (&x)[V]) {
    if constexpr (V == 8) {
        widen8(r.v, bf16, x);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = widen16((uint16_t)((e < 2 ? r.v.x : r.v.y) >> (16 * (e & 1))), bf16);
    }
}
template <int V>
__device__ __forceinline__ void store_v(uint16_t *p, bool bf16, const float (&x)[V]) {
    if constexpr (V == 8) *reinterpret_cast<uint4 *>(p) = narrow8(x, bf16);
    else *reinterpret_cast<uint2 *>(p) = make_uint2(narrow2(x[0], x[1], bf16), narrow2(x[2], x[3], bf16));
}
// V weights from element `at` on
template <int V>
__device__ __forceinline__ void load_weights(const void *W, MxType type, int64_t at, float (&w)[V]) {
    if (type == MxType::F32) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const float4 f = reinterpret_cast<const float4 *>(static_cast<const float *>(W) + at)[q];
            w[4 * q] = f.x, w[4 * q + 1] = f.y, w[4 * q + 2] = f.z, w[4 * q + 3] = f.w;
        }
    } else {
        widen<V>(load_raw<V>(static_cast<const uint16_t *>(W) + at), type == MxType::BF16, w);
    }
}

// PAIRS: interleaved pairs (V = 8 columns an item), otherwise an item's V columns pair with V others.
constexpr int kMaxTurns = 512;   // pairs of a wave's rows: 64 lanes of at most 8
template <bool PAIRS, int V, bool NORM>
__global__ void __launch_bounds__(256) rope_kernel(RopeLaunch a)
{
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t rowgroup = wave / a.slices;
    const int slice = (int)(wave - rowgroup * a.slices);
    const int hd = lane / a.items, c = lane - hd * a.items;   // head of the wave's, item
    const int sub = hd / a.side, g = hd - sub * a.side;        // row of the wave's, head of the row's
    const int64_t m = a.m0 + rowgroup * a.rows + sub;
    const bool live = sub < a.rows && m < a.m1;
    const int half = a.ends[3];                               // pairs
    const bool turns = c < a.turned;
    // the item's columns: c0 onwards, and (halves paired) half + c0 onwards
    const int c0 = PAIRS ? 8 * c : turns ? V * c : 2 * half + V * (c - a.turned);

    // Sine and cosine of the wave's rows' pairs, one of each a lane at a time, meet in LDS.
    constexpr int NP = PAIRS ? V / 2 : V;   // pairs of an item
    __shared__ __align__(16) float2 turns_of[4][kMaxTurns];
    float2 *table = turns_of[threadIdx.x >> 6];
    for (int q = lane; q < a.rows * half; q += 64) {
        const int r = q / half, i = q - r * half;
        const uint32_t row = (uint32_t)min(m - sub + r, a.m1 - 1);
        const int axis = (i >= a.ends[0]) + (i >= a.ends[1]) + (i >= a.ends[2]);
        const int64_t at = (int64_t)(row % (uint32_t)a.tokens) * a.axes + axis;
        const double p = a.float_positions ? (double)static_cast<const float *>(a.positions)[at]
                                           : (double)static_cast<const int32_t *>(a.positions)[at];
        // 1 / 2 pi = 0x1.45f306dc9c883p-3 + kLow, |kLow| under half a step of it
        constexpr double kTurns = 0x1.45f306dc9c883p-3, kLow = -0x1.6b01ec5417056p-57;
        const double f = a.freqs[i], angle = p * f, rest = __builtin_fma(p, f, -angle);
        const double high = angle * kTurns;
        double rev = high - rint(high) + __builtin_fma(angle, kLow, __builtin_fma(rest, kTurns, __builtin_fma(angle, kTurns, -high)));
        rev -= rint(rev);
        float2 t;
        sincospif(2.0f * (float)rev, &t.y, &t.x);
        table[q] = make_float2(t.x, a.inverse ? -t.y : t.y);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (a wave's LDS accesses stay in order)
    float cs[NP], sn[NP];
    {
        const float4 *p = reinterpret_cast<const float4 *>(table + (live && turns ? sub * half + NP * c : 0));
#pragma unroll
        for (int j = 0; j < NP; j += 2) {
            const float4 t = p[j / 2];
            cs[j] = t.x, sn[j] = t.y, cs[j + 1] = t.z, sn[j + 1] = t.w;
        }
    }

    const uint16_t *xr = a.X + (live ? m : 0) * a.ldx + c0;
    uint16_t *yr = a.Y + (live ? m : 0) * a.ldy + c0;
    // (one set of weights for all heads stays in registers)
    float wx[NORM ? V : 1], wy[NORM && !PAIRS ? V : 1];
    auto weights = [&](int64_t at) {
        if constexpr (NORM) load_weights<V>(a.W, a.w_type, at + c0, wx);
        if constexpr (NORM && !PAIRS) load_weights<V>(a.W, a.w_type, at + c0 + (turns ? half : 0), wy);
    };
    if (NORM && a.w_stride == 0 && live) weights(0);
    // A head's values are on their way while the one before it is turned.  (The trip count is the wave's own, so
    // that its lanes meet at the norm's exchanges; loads past the last head repeat it.)
    const int step = a.slices * a.side;
    Raw<V> nx, ny;
    auto fetch = [&](int h) {
        const uint16_t *p = xr + (int64_t)min(h, a.heads - 1) * a.lhx;
        nx = load_raw<V>(p);
        if constexpr (!PAIRS) ny = load_raw<V>(p + (turns ? half : 0));
    };
    if (live) fetch(slice * a.side + g);
    for (int h0 = slice * a.side; h0 < a.heads; h0 += step) {
        const int h = h0 + g;
        const bool on = live && h < a.heads;
        float x[V], y[V];
        if (live) {
            widen<V>(nx, a.bf16, x);
            if constexpr (!PAIRS) widen<V>(ny, a.bf16, y);
            if (h0 + step < a.heads) fetch(h + step);
        }
        if constexpr (NORM) {
            float s = 0.0f;
            if (on) {
                if (a.w_stride != 0) weights(h * a.w_stride);
#pragma unroll
                for (int e = 0; e < V; ++e) s = __builtin_fmaf(x[e], x[e], s);
                if (!PAIRS && turns) {
#pragma unroll
                    for (int e = 0; e < V; ++e) s = __builtin_fmaf(y[e], y[e], s);
                }
            }
            // the head's items are neighbours: each adds what lies 1, 2, 4, .. items behind it, in a
            // fixed order, until the first holds the sum
            for (int off = 1; off < a.items; off <<= 1) {
                const float o = __shfl(s, lane + off);
                if (c + off < a.items) s += o;
            }
            s = __shfl(s, lane - c);
            const float inv = __builtin_amdgcn_rsqf(__builtin_fmaf(s, a.inv_d, a.eps));   // (1 ulp; eps is a normal number)
            if (on) {
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = x[e] * inv * wx[e];
                if constexpr (!PAIRS) {
#pragma unroll
                    for (int e = 0; e < V; ++e) y[e] = y[e] * inv * wy[e];
                }
            }
        }
        if (!on) continue;
        uint16_t *yp = yr + (int64_t)h * a.lhy;
        if (!turns) {
            store_v<V>(yp, a.bf16, x);
        } else if constexpr (PAIRS) {
            float z[V];
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                z[2 * j] = __builtin_fmaf(x[2 * j], cs[j], -(x[2 * j + 1] * sn[j]));
                z[2 * j + 1] = __builtin_fmaf(x[2 * j + 1], cs[j], x[2 * j] * sn[j]);
            }
            store_v<V>(yp, a.bf16, z);
        } else {
            float z[V];
#pragma unroll
            for (int j = 0; j < V; ++j) z[j] = __builtin_fmaf(x[j], cs[j], -(y[j] * sn[j]));
            store_v<V>(yp, a.bf16, z);
#pragma unroll
            for (int j = 0; j < V; ++j) z[j] = __builtin_fmaf(y[j], cs[j], x[j] * sn[j]);
            store_v<V>(yp + half, a.bf16, z);
        }
    }
}

template <bool PAIRS, int V>
hipError_t launch(RopeLaunch a, hipStream_t stream) {
    a.turned = PAIRS ? 2 * a.ends[3] / 8 : a.ends[3] / V;
    a.items = a.turned + (a.D - 2 * a.ends[3]) / V;
    if (a.items < 1 || a.items > 64) return hipErrorInvalidValue;
    const int fit = 64 / a.items;
    a.inv_d = 1.0f / (float)a.D;
    a.side = std::min(fit, a.heads);
    a.rows = fit / a.side;
    const int steps = (a.heads + a.side - 1) / a.side;
    const int64_t groups = (a.M + a.rows - 1) / a.rows;
    // few rows: their heads to several waves, up to eight waves a compute unit (64: 4608 x 48 x 128 24 -> 27 us)
    a.slices = (int)std::max<int64_t>(1, std::min<int64_t>(steps, 8 * (int64_t)compute_units() / groups));
    // launches of at most 2^31 lanes
    const int64_t most = (((int64_t)1 << 25) / a.slices) * a.rows;
    for (a.m0 = 0; a.m0 < a.M; a.m0 += most) {
        a.m1 = std::min(a.M, a.m0 + most);
        const int64_t waves = (a.m1 - a.m0 + a.rows - 1) / a.rows * a.slices;
        const dim3 grid((unsigned)((waves + 3) / 4));
        if (a.W != nullptr) hipLaunchKernelGGL((rope_kernel<PAIRS, V, true>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((rope_kernel<PAIRS, V, false>), grid, dim3(256), 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeArgs &args, hipStream_t stream) {
    RopeLaunch a;
    static_cast<RopeArgs &>(a) = args;
    if (a.interleaved) return launch<true, 8>(a, stream);
    return a.ends[3] % 8 == 0 && (a.D - 2 * a.ends[3]) % 8 == 0 ? launch<false, 8>(a, stream) : launch<false, 4>(a, stream);
}

}  // namespace clq
