// Block-Hadamard rotation (CLQ, arXiv 2509.24416, Sec. 3.3) followed by the MX4
// quantizer, the inverse of the quantizer, and the layout of checkpoint weights.
//
// x~ = FWHT_b(gather(x, perm)) in fp32 with the stage order h = 1, 2, ..., b / 2,
// then for each 32 values the scale 2^e, e = floor(log2 max|x~|) - 2, and the codes
// rne(x~ / 2^e) on the e2m1 grid.  A group needs no other column of its row (a
// per-token scale needs the whole row), so a workgroup takes a 32-row x 256-column
// tile and nothing passes through LDS.
//
// What bounds it is memory: 2 bytes in and 17/32 out per element.  A lane owns one
// 16-byte chunk (8 columns) of four rows, so that a wave's loads are whole 256-byte
// pieces, four in flight per lane; stages h = 1, 2, 4 run inside the lane, 8 .. 64
// across lanes; the group's maximum is over a quad of lanes; the quad transposes
// 4 rows x 4 chunks of codes, each lane then storing the 32 codes of one row, the
// quad 64 contiguous bytes.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "clq_internal.h"
#include "mx4.h"
#include "rq_device.h"

namespace clq {
namespace {

constexpr int kTileCols = 256, kChunkLanes = kTileCols / 8, kRowGroups = 8;
constexpr int kThreads = kChunkLanes * kRowGroups;   // 32 rows x 256 columns

// the larger of two magnitudes, a NaN if either is one
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Exchange between the two lanes of a pair (CTRL: xor 1 or 2; b: the lane's side).
template <int CTRL>
__device__ __forceinline__ void pair_exchange(uint32_t &lo, uint32_t &hi, bool b) {
    const uint32_t plo = lane_xchg<CTRL>(lo), phi = lane_xchg<CTRL>(hi);
    lo = b ? phi : lo;
    hi = b ? hi : plo;
}
// transposes a quad's 4 x 4 dwords: lane k (logical bits b0, b1) ends with d[j] =
// lane j's d[k]
__device__ __forceinline__ void quad_transpose(uint32_t (&d)[4], bool b0, bool b1) {
    pair_exchange<kLaneXor1>(d[0], d[1], b0);
    pair_exchange<kLaneXor1>(d[2], d[3], b0);
    pair_exchange<kLaneXor2>(d[0], d[2], b1);
    pair_exchange<kLaneXor2>(d[1], d[3], b1);
}

__device__ __forceinline__ float widen(uint16_t h, bool bf16) {
    return bf16 ? __uint_as_float((uint32_t)h << 16) : __half2float(__ushort_as_half(h));
}

// row of W that output row n holds
__device__ __forceinline__ int64_t gated_row(int64_t n, int64_t rows) {
    const int64_t j = n >> 6, t = n & 63;
    return t < 32 ? 32 * j + t : rows / 2 + 32 * j + (t - 32);
}

struct QuantParams {
    const uint16_t *X;
    int64_t ldx, rows, units, mat_units;   // mat_units: units of each matrix
    const int32_t *perm;
    int K, log_div, tiles;                 // tiles: 256-column tiles of a unit
    bool weights, gated;
    const int32_t *source, *total_units;
    uint8_t *codes, *scales;
};

template <int B, bool BF16, bool PERM>
__global__ void __launch_bounds__(kThreads) mx_quant_kernel(QuantParams p)
{
    const int t = threadIdx.x;
    const int lc = t & (kChunkLanes - 1), rg = t / kChunkLanes;
    // chunk order over lanes: see rq_device.h
    const int chunk = (lc & ~7) | logical_lane(lc & 7);
    const bool b0 = chunk & 1, b1 = chunk & 2;
    const CrossSigns cs = cross_signs<B ? B : 32>(chunk);
    const uint32_t flip = B && cs.sign < 0.0f ? 0x88888888u : 0u;
    int64_t units = p.units;
    if (p.total_units) units = min((int64_t)*p.total_units, units);
    const int64_t work = units * p.tiles;
    for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const int64_t u = w / p.tiles;
        const int ct = (int)(w - u * p.tiles);
        const int col = ct * kTileCols + 8 * chunk;
        const int64_t mat = u / p.mat_units, um = u - mat * p.mat_units;
        // four consecutive rows; in the weights' fragment order four rows aligned to
        // four stay together
        const int64_t r0 = um * 32 + rg * 4;
        const int rho0 = p.weights ? wq_rho(rg * 4) : rg * 4;
        const bool in = col < p.K;   // (whole octets and, for B = 128, whole 16 lanes)
        float x[4][8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t n = r0 + r;
            int64_t src = n < p.rows ? (p.gated ? gated_row(n, p.rows) : n) + mat * p.rows : -1;
            if (p.source) {
                src = p.source[u * 32 + rg * 4 + r];
                if (src >= p.rows) src = -1;
            }
            uint32_t d[4] = {0u, 0u, 0u, 0u};
            if (in && src >= 0) {
                const uint16_t *row = p.X + src * p.ldx;
                if constexpr (PERM) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        d[e] = (uint32_t)row[p.perm[col + 2 * e]] | (uint32_t)row[p.perm[col + 2 * e + 1]] << 16;
                } else {
                    const uint4 v = *reinterpret_cast<const uint4 *>(row + col);
                    d[0] = v.x; d[1] = v.y; d[2] = v.z; d[3] = v.w;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float lo = widen((uint16_t)d[e], BF16), hi = widen((uint16_t)(d[e] >> 16), BF16);
                x[r][2 * e] = B ? lo + hi : lo;
                x[r][2 * e + 1] = B ? lo - hi : hi;
            }
            if constexpr (B != 0) fwht8_rest(x[r]);
        }
        if constexpr (B != 0) cross_stages<B, 4>(x, cs);
        uint32_t codes[4];
        int byte[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float m = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max_nan(m, fabsf(x[r][e]));
            m = max_nan(m, lane_xchg<kLaneXor1>(m));
            m = max_nan(m, lane_xchg<kLaneXor2>(m));
            byte[r] = mx_scale_byte(__float_as_uint(m) & 0x7fffffffu, p.log_div);
            codes[r] = mx_pack8(x[r], mx_scale_value(byte[r], p.log_div)) ^ flip;
        }
        quad_transpose(codes, b0, b1);
        const int k4 = chunk & 3;   // the row of the four that this lane stores
        if (in) {
            const int c32 = col >> 5;
            *reinterpret_cast<uint4 *>(p.codes + mx_code_offset(u, rho0 + k4, c32, p.K)) =
                make_uint4(codes[0], codes[1], codes[2], codes[3]);
            const int sb = k4 == 0 ? byte[0] : k4 == 1 ? byte[1] : k4 == 2 ? byte[2] : byte[3];
            p.scales[mx_scale_offset(u, rho0 + k4, c32, p.K)] = (uint8_t)sb;
        }
    }
}

// 8 codes of a row per thread, 16 neighbouring threads on 128 columns
template <class T>
__global__ void __launch_bounds__(256) mx_dequant_kernel(const uint8_t *codes, const uint8_t *scales, int64_t rows,
                                                         int K, bool weights, bool gated, int64_t mats, T *out,
                                                         int64_t ldo)
{
    const int tiles = (K + 127) / 128;
    const int64_t mat_units = weights ? padded_rows(rows) >> 5 : padded_act_rows(rows) >> 5;
    const int64_t total = mats * mat_units * 32 * tiles * 16;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t ur = i / (512 * tiles);   // unit
        const int in_unit = (int)(i - ur * 512 * tiles);
        const int tile = in_unit / 512, q = in_unit & 511;
        const int row = q >> 4, col = tile * 128 + (q & 15) * 8;
        const int64_t mat = ur / mat_units, n = (ur - mat * mat_units) * 32 + row;
        if (n >= rows || col >= K) continue;
        const int rho = weights ? wq_rho(row) : row;
        const uint32_t d = *reinterpret_cast<const uint32_t *>(codes + mx_code_offset(ur, rho, col >> 5, K) +
                                                               (col & 31) / 2);
        const int byte = scales[mx_scale_offset(ur, rho, col >> 5, K)];
        const float s = __uint_as_float(byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : (uint32_t)byte << 23);
        const int64_t dst = mat * rows + (gated ? gated_row(n, rows) : n);
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = (int)(d >> (4 * e)) & 15, ex = (c >> 1) & 3, m = c & 1;
            const float a = ex ? __uint_as_float((uint32_t)(126 + ex) << 23 | (uint32_t)m << 22) : 0.5f * (float)m;
            const float f = (c & 8 ? -a : a) * s;
            if constexpr (sizeof(T) == 4) v[e] = f;
            else v[e] = (T)f;
        }
        T *o = out + dst * ldo + col;
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4 *>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4 *>(o) = *reinterpret_cast<uint4 *>(v);
        }
    }
}

// one 16-byte chunk (32 codes) per thread
__global__ void __launch_bounds__(256) mx_pack_kernel(const uint8_t *codes, const uint8_t *scales, int64_t rows, int K,
                                                      bool gated, int64_t mats, uint8_t *co, uint8_t *so)
{
    const int cpr = K >> 5;
    const int64_t prow = padded_rows(rows), total = mats * prow * cpr;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        // rows fastest: 32 neighbouring threads fill a unit's half
        const int64_t u = i / (32 * cpr);
        const int q = (int)(i - u * 32 * cpr), c = q >> 5, row = q & 31;
        const int64_t mat = u / (prow >> 5), n = (u - mat * (prow >> 5)) * 32 + row;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        uint8_t s = 1;
        if (n < rows) {
            const int64_t src = mat * rows + (gated ? gated_row(n, rows) : n);
            v = *reinterpret_cast<const uint4 *>(codes + src * (K >> 1) + c * 16);
            s = scales[src * cpr + c];
        }
        const int rho = wq_rho(row);
        *reinterpret_cast<uint4 *>(co + mx_code_offset(u, rho, c, K)) = v;
        so[mx_scale_offset(u, rho, c, K)] = s;
    }
}

template <int B, bool BF16>
void launch_quant(const QuantParams &p, unsigned grid, hipStream_t stream) {
    if (p.perm) hipLaunchKernelGGL((mx_quant_kernel<B, BF16, true>), dim3(grid), dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((mx_quant_kernel<B, BF16, false>), dim3(grid), dim3(kThreads), 0, stream, p);
}
template <int B>
void launch_quant(const QuantParams &p, bool bf16, unsigned grid, hipStream_t stream) {
    if (bf16) launch_quant<B, true>(p, grid, stream);
    else launch_quant<B, false>(p, grid, stream);
}

}  // namespace

constexpr int64_t kMaxGrid = 1 << 20;   // workgroups of a launch; the rest by a loop

hipError_t launch_mx_quantize(const MxQuantArgs &a, hipStream_t stream) {
    QuantParams p;
    p.X = static_cast<const uint16_t *>(a.X);
    p.ldx = a.ldx;
    p.rows = a.rows;
    p.mat_units = a.units;
    p.units = a.units * a.mats;
    p.perm = a.perm;
    p.K = a.K;
    p.log_div = a.log_div;
    p.tiles = (a.K + kTileCols - 1) / kTileCols;
    p.weights = a.weights;
    p.gated = a.gated;
    p.source = a.source;
    p.total_units = a.total_units;
    p.codes = a.codes;
    p.scales = a.scales;
    const int64_t work = p.units * p.tiles;
    const unsigned grid = (unsigned)(work < kMaxGrid ? work : kMaxGrid);
    const bool bf16 = a.type == MxType::BF16;
    switch (a.block) {
        case 0: launch_quant<0>(p, bf16, grid, stream); break;
        case 32: launch_quant<32>(p, bf16, grid, stream); break;
        case 64: launch_quant<64>(p, bf16, grid, stream); break;
        default: launch_quant<128>(p, bf16, grid, stream); break;
    }
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int K, bool weights,
                                bool gated, int mats, MxType type, void *out, int64_t ldo, hipStream_t stream) {
    const int64_t units = (weights ? padded_rows(rows) : padded_act_rows(rows)) / 32 * mats;
    const int64_t want = units * ((K + 127) / 128) * 2;
    const dim3 grid((unsigned)(want < kMaxGrid ? want : kMaxGrid)), block(256);
    switch (type) {
        case MxType::F16:
            hipLaunchKernelGGL((mx_dequant_kernel<_Float16>), grid, block, 0, stream, codes, scales, rows, K, weights,
                               gated, (int64_t)mats, static_cast<_Float16 *>(out), ldo);
            break;
        case MxType::BF16:
            hipLaunchKernelGGL((mx_dequant_kernel<__bf16>), grid, block, 0, stream, codes, scales, rows, K, weights,
                               gated, (int64_t)mats, static_cast<__bf16 *>(out), ldo);
            break;
        case MxType::F32:
            hipLaunchKernelGGL((mx_dequant_kernel<float>), grid, block, 0, stream, codes, scales, rows, K, weights,
                               gated, (int64_t)mats, static_cast<float *>(out), ldo);
            break;
    }
    return hipGetLastError();
}

hipError_t launch_mx_pack(const uint8_t *codes, const uint8_t *scales, int64_t rows, int K, bool gated, int mats,
                          uint8_t *codes_out, uint8_t *scales_out, hipStream_t stream) {
    const int64_t want = (padded_rows(rows) * mats * (K >> 5) + 255) / 256;
    const dim3 grid((unsigned)(want < kMaxGrid ? want : kMaxGrid)), block(256);
    hipLaunchKernelGGL(mx_pack_kernel, grid, block, 0, stream, codes, scales, rows, K, gated, (int64_t)mats, codes_out,
                       scales_out);
    return hipGetLastError();
}

}  // namespace clq
