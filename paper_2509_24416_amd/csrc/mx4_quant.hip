// Block-Hadamard rotation (CLQ, arXiv 2509.24416, Sec. 3.3) followed by the MX4
// quantizer, the inverse of the quantizer, and the layout of checkpoint weights.
//
// x~ = FWHT_b(gather(x, perm)) in fp32 with the stage order h = 1, 2, ..., b / 2,
// then for each 32 values the scale 2^e, e = floor(log2 max|x~|) - 2, and the codes
// rne(x~ / 2^e) on the e2m1 grid.  A group needs no other column of its row (a
// per-token scale needs the whole row), so a workgroup takes a 32-row x 256-column
// tile and nothing passes through LDS.
//
// What bounds it is memory: 2 bytes in and 17/32 out per element (43200 x 4608, b = 64: 97
// to 118 us, 4.3 to 5.2 TB/s; 8192 x 1152 7 us).  A lane owns one
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
constexpr int kGatherThreads = 256;
constexpr int kGatherLds = 160 * 1024;               // four rows of up to 20480 columns

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

// A launch covers row units first .. first + units - 1 (fewer than 2^31 tiles, so that the
// index arithmetic is 32-bit).
struct QuantParams {
    const uint16_t *X;
    int64_t ldx, rows;
    int first, units, mat_units;   // mat_units: units of each matrix
    const int32_t *perm;
    int K, log_div, tiles;         // tiles: 256-column tiles of a unit
    bool weights, gated;
    const int32_t *source, *total_units;
    uint8_t *codes, *scales;
};

// Source rows of W or X of output rows r .. r + 3 of unit u; negative: zeros.
__device__ __forceinline__ void source_rows(const QuantParams &p, int u, int r, int64_t (&src)[4]) {
    if (p.source) {
        int v[4];
        __builtin_memcpy(v, p.source + (int64_t)u * 32 + r, sizeof v);   // (4-byte aligned)
#pragma unroll
        for (int i = 0; i < 4; ++i) src[i] = v[i] < p.rows ? v[i] : -1;
        return;
    }
    const int mat = u < p.mat_units ? 0 : u / p.mat_units;
    const int64_t n = (int64_t)(u - mat * p.mat_units) * 32 + r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        src[i] = n + i < p.rows ? (p.gated ? gated_row(n + i, p.rows) : n + i) + mat * p.rows : -1;
}
// the launch's share of the row units in use
__device__ __forceinline__ int used_units(const QuantParams &p) {
    return p.total_units ? max(min(*p.total_units - p.first, p.units), 0) : p.units;
}

// Stage h = 1 of a lane's pair of columns (the values themselves without a rotation).
template <int B>
__device__ __forceinline__ void pair_in(float lo, float hi, float &a, float &b) {
    a = B ? lo + hi : lo;
    b = B ? lo - hi : hi;
}

// The rest of the rotation, the codes and the stores of four rows' chunk of 8 columns,
// x[row][column] after stage h = 1; rho0: the first row's fragment row.
template <int B>
__device__ __forceinline__ void quantize_chunk(const QuantParams &p, float (&x)[4][8], int chunk, const CrossSigns &cs,
                                               int u, int rho0) {
    if constexpr (B != 0) {
#pragma unroll
        for (int r = 0; r < 4; ++r) fwht8_rest(x[r]);
        cross_stages<B, 4>(x, cs);
    }
    const uint32_t flip = B && cs.sign < 0.0f ? 0x88888888u : 0u;
    uint32_t codes[4];
    int byte[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float m0 = 0.0f, m1 = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            m0 = max_nan(max_nan(m0, fabsf(x[r][e])), fabsf(x[r][e + 1]));
            m1 = max_nan(max_nan(m1, fabsf(x[r][e + 2])), fabsf(x[r][e + 3]));
        }
        float m = max_nan(m0, m1);
        m = max_nan(m, lane_xchg<kLaneXor1>(m));
        m = max_nan(m, lane_xchg<kLaneXor2>(m));
        byte[r] = mx_scale_byte(__float_as_uint(m) & 0x7fffffffu, p.log_div);
        codes[r] = mx_pack8(x[r], mx_scale_value(byte[r], p.log_div)) ^ flip;
    }
    quad_transpose(codes, chunk & 1, chunk & 2);
    const int k4 = chunk & 3, c32 = chunk >> 2;   // the row of the four that this lane stores
    if (8 * chunk < p.K) {
        *reinterpret_cast<uint4 *>(p.codes + mx_code_offset(u, rho0 + k4, c32, p.K)) =
            make_uint4(codes[0], codes[1], codes[2], codes[3]);
        const int sb = k4 == 0 ? byte[0] : k4 == 1 ? byte[1] : k4 == 2 ? byte[2] : byte[3];
        p.scales[mx_scale_offset(u, rho0 + k4, c32, p.K)] = (uint8_t)sb;
    }
}

// A workgroup takes 32 rows x 256 columns.  Gathered inputs (PERM): from memory.
template <int B, bool BF16, bool PERM>
__global__ void __launch_bounds__(kThreads) mx_quant_kernel(QuantParams p)
{
    const int t = threadIdx.x;
    const int lc = t & (kChunkLanes - 1), rg = t / kChunkLanes;
    // chunk order over lanes: see rq_device.h
    const int lane_chunk = (lc & ~7) | logical_lane(lc & 7);
    const CrossSigns cs = cross_signs<B ? B : 32>(lane_chunk);
    const int w = (int)(blockIdx.x / (unsigned)p.tiles);
    if (w >= used_units(p)) return;
    const int u = p.first + w, chunk = ((int)blockIdx.x - w * p.tiles) * kChunkLanes + lane_chunk, col = 8 * chunk;
    const bool in = col < p.K;   // (whole octets and, for B = 128, whole 16 lanes)
    int64_t src[4];
    source_rows(p, u, rg * 4, src);
    uint32_t d[4][4] = {};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (!in || src[r] < 0) continue;
        const uint16_t *row = p.X + src[r] * p.ldx;
        if constexpr (PERM) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                d[r][e] = (uint32_t)row[p.perm[col + 2 * e]] | (uint32_t)row[p.perm[col + 2 * e + 1]] << 16;
        } else {
            const uint4 v = *reinterpret_cast<const uint4 *>(row + col);
            d[r][0] = v.x; d[r][1] = v.y; d[r][2] = v.z; d[r][3] = v.w;
        }
    }
    float x[4][8];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            pair_in<B>(widen((uint16_t)d[r][e], BF16), widen((uint16_t)(d[r][e] >> 16), BF16), x[r][2 * e], x[r][2 * e + 1]);
    // (in the weights' fragment order four rows aligned to four stay together)
    quantize_chunk<B>(p, x, chunk, cs, u, p.weights ? wq_rho(rg * 4) : rg * 4);
}

// Gathered inputs whose four rows fit LDS: a workgroup takes four rows, staged with the
// rows' values of a column side by side, so that one 8-byte read gathers a column of all
// four: 2777 x 4608 14 us, from memory column by column 45.
template <int B, bool BF16>
__global__ void __launch_bounds__(kGatherThreads) mx_gather_kernel(QuantParams p)
{
    extern __shared__ __align__(16) uint8_t staged[];
    const int t = threadIdx.x, chunks = p.K >> 3, padded = (chunks + 15) & ~15;
    const int u = p.first + (int)(blockIdx.x >> 3), rg = blockIdx.x & 7;
    if (u - p.first >= used_units(p)) return;
    int64_t src[4];
    source_rows(p, u, rg * 4, src);
    {
        const uint16_t *row[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) row[r] = src[r] < 0 ? nullptr : p.X + src[r] * p.ldx;
        for (int c = t; c < chunks; c += kGatherThreads) {
            uint4 v[4];
#pragma unroll
            for (int r = 0; r < 4; ++r)
                v[r] = row[r] ? reinterpret_cast<const uint4 *>(row[r])[c] : make_uint4(0u, 0u, 0u, 0u);
            uint32_t q[16];
            interleave_rows(v, q);
            uint4 *dst = reinterpret_cast<uint4 *>(staged) + c * 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[i] = make_uint4(q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]);
        }
        __syncthreads();
        for (int c0 = t; c0 < padded; c0 += kGatherThreads) {   // (whole 16-lane rows)
            const int chunk = (c0 & ~7) | logical_lane(c0 & 7);
            const CrossSigns cs = cross_signs<B ? B : 32>(chunk);
            float x[4][8];
            const bool in = chunk < chunks;
            int s[8] = {};
            if (in) {
                const int4 s0 = reinterpret_cast<const int4 *>(p.perm)[2 * chunk];
                const int4 s1 = reinterpret_cast<const int4 *>(p.perm)[2 * chunk + 1];
                s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w;
                s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint2 lo = reinterpret_cast<const uint2 *>(staged)[s[e]];
                const uint2 hi = reinterpret_cast<const uint2 *>(staged)[s[e + 1]];
                const uint32_t l[2] = {lo.x, lo.y}, h[2] = {hi.x, hi.y};
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    pair_in<B>(widen((uint16_t)(l[r >> 1] >> (16 * (r & 1))), BF16),
                               widen((uint16_t)(h[r >> 1] >> (16 * (r & 1))), BF16), x[r][e], x[r][e + 1]);
            }
            quantize_chunk<B>(p, x, chunk, cs, u, p.weights ? wq_rho(rg * 4) : rg * 4);
        }
    }
}

// The inverse, bound by memory (43200 x 4608 to bf16: 90 to 99 us, 5.1 to 5.6 TB/s).  A
// workgroup takes 32 rows x 128 columns, a thread 8 codes of one row twice
// over: 16 neighbouring threads store 256 bytes of a row (16-bit types), and the 4-byte
// pieces of codes that they read are all of the tile's two units between them.
template <class T>
__global__ void __launch_bounds__(256) mx_dequant_kernel(const uint8_t *codes, const uint8_t *scales, int64_t rows,
                                                         int K, bool weights, bool gated, int64_t mats, T *out,
                                                         int64_t ldo)
{
    const int tiles = (K + 127) / 128, t = threadIdx.x;
    const int64_t mat_units = (weights ? padded_rows(rows) : padded_act_rows(rows)) >> 5;
    const int64_t work = mats * mat_units * tiles;
    for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const int64_t u = w / tiles, mat = u / mat_units;
        const int col = (int)(w - u * tiles) * 128 + (t & 15) * 8, c = col >> 5;
        if (col >= K) continue;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = half * 16 + (t >> 4), rho = weights ? wq_rho(row) : row;
            const int64_t n = (u - mat * mat_units) * 32 + row;
            if (n >= rows) continue;
            const uint32_t d = *reinterpret_cast<const uint32_t *>(codes + mx_code_offset(u, rho, c, K) + (col & 31) / 2);
            const int byte = scales[mx_scale_offset(u, rho, c, K)];
            // (byte 255: NaN; byte 0, 2^-127, is fp32's subnormal)
            const float s = __uint_as_float(byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : (uint32_t)byte << 23);
            typedef float f2 __attribute__((ext_vector_type(2)));
            const f2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d, 1.0f, 0),
                             __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d, 1.0f, 1),
                             __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d, 1.0f, 2),
                             __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d, 1.0f, 3)};
            T v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (T)(p[e >> 1][e & 1] * s);
            T *o = out + (mat * rows + (gated ? gated_row(n, rows) : n)) * ldo + col;
            if constexpr (sizeof(T) == 4) {
                reinterpret_cast<float4 *>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4 *>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                *reinterpret_cast<uint4 *>(o) = *reinterpret_cast<uint4 *>(v);
            }
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

constexpr int64_t kMaxGrid = 1 << 23;   // workgroups of a launch

template <int B, bool BF16>
hipError_t launch_quant(QuantParams p, hipStream_t stream) {
    const size_t lds = (size_t)p.K * 8;
    // (the vector loads of the indices need 16 bytes of alignment)
    const bool staged = p.perm && lds <= (size_t)kGatherLds && (reinterpret_cast<uintptr_t>(p.perm) & 15) == 0;
    if (staged && lds > 64 * 1024) {
        const hipError_t set = hipFuncSetAttribute(reinterpret_cast<const void *>(&mx_gather_kernel<B, BF16>),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, kGatherLds);
        if (set != hipSuccess) return set;
    }
    const int per = staged ? 8 : p.tiles, all = p.units;
    for (int left = all, first = 0; left > 0;) {
        p.first = first;
        p.units = left < kMaxGrid / per ? left : (int)(kMaxGrid / per);
        const dim3 grid((unsigned)(p.units * per));
        if (staged) hipLaunchKernelGGL((mx_gather_kernel<B, BF16>), grid, dim3(kGatherThreads), lds, stream, p);
        else if (p.perm) hipLaunchKernelGGL((mx_quant_kernel<B, BF16, true>), grid, dim3(kThreads), 0, stream, p);
        else hipLaunchKernelGGL((mx_quant_kernel<B, BF16, false>), grid, dim3(kThreads), 0, stream, p);
        first += p.units;
        left -= p.units;
    }
    return hipGetLastError();
}
template <int B>
hipError_t launch_quant(const QuantParams &p, bool bf16, hipStream_t stream) {
    return bf16 ? launch_quant<B, true>(p, stream) : launch_quant<B, false>(p, stream);
}

}  // namespace

hipError_t launch_mx_quantize(const MxQuantArgs &a, hipStream_t stream) {
    QuantParams p;
    p.X = static_cast<const uint16_t *>(a.X);
    p.ldx = a.ldx;
    p.rows = a.rows;
    p.mat_units = (int)a.units;
    p.units = (int)(a.units * a.mats);   // (under 2^26)
    p.first = 0;
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
    const bool bf16 = a.type == MxType::BF16;
    switch (a.block) {
        case 0: return launch_quant<0>(p, bf16, stream);
        case 32: return launch_quant<32>(p, bf16, stream);
        case 64: return launch_quant<64>(p, bf16, stream);
        default: return launch_quant<128>(p, bf16, stream);
    }
}

hipError_t launch_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int K, bool weights,
                                bool gated, int mats, MxType type, void *out, int64_t ldo, hipStream_t stream) {
    const int64_t units = (weights ? padded_rows(rows) : padded_act_rows(rows)) / 32 * mats;
    const int64_t want = units * ((K + 127) / 128);
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
