// MX4 products: Y = dequant(Xq) . dequant(Wq)^T + bias on the fp4 matrix cores of
// gfx950, dense and grouped by expert, with the result either stored (fp16, bf16, fp32)
// or activated, rotated (CLQ, arXiv 2509.24416, Sec. 3.3) and requantized to MX4 for
// the next product without leaving the registers.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 multiplies 32 fp4 codes a lane and applies each
// operand's scale byte itself: the sum over a 32-value group times both scales is
// added to an fp32 accumulator, so there is no dequantization anywhere.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "clq_internal.h"
#include "mx4.h"
#include "tile_gemm.h"

namespace clq {
namespace {
namespace mx {

using tg::IC;
using tg::lds_addr;
using tg::read16;
using tg::static_for;
using tg::v16f;
using tg::v4f;
using tg::v4u;
using tg::v8i;
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

struct Args {
    const uint8_t *Xq, *Xs, *Wq, *Ws;
    const uint16_t *bias;
    int64_t w_stride, ws_stride;   // bytes of one expert's codes and scales
    int M, N, K, tiles_m, tiles_n, group_m;
    int xunits, wunits;
    const int32_t *info;
    int experts, log_units;   // of a tile
    void *Y;
    int64_t ldy;
    bool bias_bf16;
    MxType out_type;
    uint8_t *Oq, *Os;
    int oK;   // channels of the MX4 output
};

// Buffer transfers into LDS of 16 and 4 bytes a lane from byte `lane_off` + `off` of a
// buffer: the compiler counts them among the loads in flight, where behind a transfer
// by a global address it waits for all of them ahead of every loaded register's use.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const uint8_t *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p), 0, (int)bytes, 0x00027000);
}
__device__ __forceinline__ void dma16(Buffer b, uint32_t lane_off, uint32_t off, uint32_t dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (CLQ_LDS void *)(size_t)dst, 16, (int)lane_off, (int)off, 0, 0);
}
__device__ __forceinline__ void dma4(Buffer b, uint32_t lane_off, uint32_t off, uint32_t dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (CLQ_LDS void *)(size_t)dst, 4, (int)lane_off, (int)off, 0, 0);
}
template <int OFF>
__device__ __forceinline__ uint32_t read4(uint32_t addr) {
    uint32_t v;
    asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}

// D = A . B + D on fp4 operands, scale bytes P of sa and sb
template <int P>
__device__ __forceinline__ v16f mfma_mx4(v4u a, v4u b, v16f c, uint32_t sa, uint32_t sb) {
    const v8i a8 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const v8i b8 = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a8, b8, c, 4, 4, P, (int)sa, P, (int)sb);
}

__device__ __forceinline__ float widen(uint16_t h, bool bf16) {
    return bf16 ? __uint_as_float((uint32_t)h << 16) : __half2float(__ushort_as_half(h));
}
// two 16-bit outputs, rounded to nearest even
template <MxType T>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    if constexpr (T == MxType::BF16) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        const b2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// The tanh form of GELU: 0.5 h (1 + tanh u) = h / (1 + exp(-2u)), the exponent's constants
// times log2 e.  With the hardware's exp2 and reciprocal (1 ulp each) the relative error is under
// 6e-7 for h > -2; below, exp2 scales up its argument's rounding with the argument (2e-6 at -5,
// 1e-5 at -10, where the results are -2e-7 and -1e-37).  The absolute error is under 1e-7 for
// negative h: that of the sum it is applied to, or less.  SiLU, whose argument is h itself: 1e-6 at
// -16.
__device__ __forceinline__ float gelu(float h) {
    const float t = h * __builtin_fmaf(-0.10294324f, h * h, -2.3022082f);   // -2u log2 e
    return h * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
}
__device__ __forceinline__ float silu(float g) {
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g));
}

// the row tile a workgroup works on
struct RowTile {
    int unit0, unit_end;   // its first row unit; the end of the rows it may touch
    int expert;
};

// Expert and first unit of grouped tile t: the number of experts whose tiles all
// come before it, 64 table entries at a time.
__device__ __forceinline__ RowTile find_tile(const Args &a, int t, int lane) {
    const int32_t *table = a.info + plan_table_offset(a.experts, a.log_units);
    const int32_t *first = a.info + plan_table_offset(a.experts, 0);
    int e = 0;
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
        const int i = e0 + lane;
        const bool before = i < a.experts && table[i + 1] <= t;
        const int n = __popcll(__ballot(before));
        e += n;
        if (n < 64) break;
    }
    e = __builtin_amdgcn_readfirstlane(e);
    RowTile r;
    r.expert = e;
    r.unit0 = first[e] + ((t - table[e]) << a.log_units);
    r.unit_end = first[e + 1];
    return r;
}

// ---- the tile kernel ---------------------------------------------------------------
// A workgroup of NW waves computes 32 FN channels x 64 NW tokens, each wave all of the channels
// x 64 tokens (FN x 2 fragments of 32 x 32; FN = 4, or 3 where that fills the chip better).  A
// k-stage is 64 codes, one matrix instruction per fragment.  The channel units are shared by
// the waves: they go global -> LDS without registers through a ring of NS stages, and a wave
// reads a stage's units back one stage ahead of its use.  The token units belong to one wave
// each and go straight to registers, kDepth stages ahead (through LDS the reads and writes of
// both operands came to 144 of its 128 bytes a clock at full rate).  The scale dwords of four
// stages (a quad) take the same two ways, the channels' through a ring of two, read at the end
// of the quad before.
//
// Ring protocol: iteration s waits until stage s + 1 has landed (transfers and loads
// complete in issue order: at most the later stages' may be outstanding) and its own LDS
// reads of stage s are in, then the workgroup barrier: every wave holds stage s in
// registers, so its slot is refilled with stage s + NS.  Quad q's scale slot is likewise
// free after the barrier of the quad's first iteration and refilled there with quad q + 2,
// needed at the end of quad q + 1.  Within the loop transfers past the end repeat the last
// stage or quad, so that its wait counts are constant; the stages after it have their own.
//
// What bounds it: on long k loops the matrix instructions (8 per wave and stage of 32 cycles) at
// the clock that the power limit leaves (8192^3 228 to 244 us, 4.5 to 4.8 PFLOP/s, matrix cores
// 68% busy; 43200 x 4608 -> 1152 104 to 116 us, 4.0 to 4.4 PFLOP/s); with GELU and requantization
// on many rows the epilogue's vector instructions (62% of issue beside 30% of matrix cycles).
// Otherwise no unit by itself: a tile's prologue, its few stages and its stores follow one another,
// and the other workgroup of the compute unit covers a part of that.  43200 x 1152 -> 4608: 140
// to 186 us, matrix cores 36% busy, vector issue 16%, 2.0 of 2.4 GHz (76 us with one stage of k
// loop); 8192 x 1152 -> 4608 with GELU and requantization 41 us, 20% and 42% at full clock, its
// 1152 tiles being 2.25 rounds of the 512 workgroups that run at a time.
constexpr int kBN = 128;                        // channels (FN = 4)
constexpr int kStageBytes = 4 * kMxUnit;        // 4 / NW units from each wave (FN = 3: the last twice)
constexpr int kQuadBytes = 4 * kMxScaleRow;
constexpr int kDepth = 4;                       // stages of token units in registers
// Ring of channel units: one more than kDepth, so that the stages that the prologue leaves in
// flight are as many transfers and loads as the loop's wait counts take them for.
constexpr int kStages = kDepth + 1;

// What a stage at position p of eight fetches (negative: of the eight before, or of the
// prologue): channel units for NS stages on, token units for kDepth stages on, at the start of
// a quad the token scales of the next and the channel scales of the one after it.  The stages
// after the loop (`last`, positions 0 .. 6) are followed by no others.
constexpr bool fetches_w(int p, bool last) { return !last || p + kStages < 7; }
constexpr bool fetches_x(int p, bool last) { return !last || p + kDepth < 7; }
constexpr bool fetches_xs(int p, bool last) { return p % 4 == 0 && (!last || p == 0); }
constexpr bool fetches_ws(int p, bool last) { return p % 4 == 0 && !last; }
// its transfers and loads, per_wave transfers of each kind a wave
constexpr int fetched(int p, bool last, int per_wave) {
    if (p < 0) last = false;
    return per_wave * (fetches_w(p, last) + fetches_ws(p, last)) + 2 * (fetches_x(p, last) + fetches_xs(p, last));
}

template <int FN>
struct Operands {
    v4u w[FN];
    __device__ __forceinline__ void read(uint32_t wa) {
        static_for<0, FN>([&](auto f) { w[f] = read16<decltype(f)::value * kMxUnit>(wa); });
    }
};
template <int FN>
struct Scales {
    uint32_t s[FN];
};
// At most VM transfers outstanding, the LDS reads in, the workgroup barrier.  The
// destinations of those reads are named, so that nothing touches them before; a
// register set whose value is used once, in place, is never copied while a read of it
// is in flight (hence two sets of scales, too: a copy from one into the other was moved
// ahead of this wait).
#define CLQ_MX_WAIT "s_waitcnt vmcnt(%c[vm]) lgkmcnt(0)\n\ts_barrier"
template <int VM>
__device__ __forceinline__ void wait_stage(Operands<4> &o) {
    asm volatile(CLQ_MX_WAIT : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]), "+v"(o.w[3]) : [vm] "n"(VM) : "memory");
}
template <int VM>
__device__ __forceinline__ void wait_stage(Operands<4> &o, Scales<4> &s) {
    asm volatile(CLQ_MX_WAIT
                 : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]), "+v"(o.w[3]), "+v"(s.s[0]), "+v"(s.s[1]), "+v"(s.s[2]),
                   "+v"(s.s[3])
                 : [vm] "n"(VM)
                 : "memory");
}
template <int VM>
__device__ __forceinline__ void wait_stage(Operands<3> &o) {
    asm volatile(CLQ_MX_WAIT : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]) : [vm] "n"(VM) : "memory");
}
template <int VM>
__device__ __forceinline__ void wait_stage(Operands<3> &o, Scales<3> &s) {
    asm volatile(CLQ_MX_WAIT
                 : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]), "+v"(s.s[0]), "+v"(s.s[1]), "+v"(s.s[2])
                 : [vm] "n"(VM)
                 : "memory");
}
#undef CLQ_MX_WAIT

enum class Out { Plain, None, Gelu, Swiglu };   // None, Gelu, Swiglu: MX4 output

// 16 bias values of channels n0 .. n0 + 15 (a gated layer's biases are in the order of
// its two halves)
__device__ __forceinline__ int bias_index(int n, int N, bool gated) {
    if (!gated) return n;
    const int j = n >> 6, t = n & 63;
    return t < 32 ? 32 * j + t : N / 2 + 32 * j + (t - 32);
}

// Eight outputs of a row from channel n on, s in fp32.
template <bool RAGGED, MxType T>
__device__ __forceinline__ void store8(const Args &a, const float *s, int64_t m, int n) {
    const bool whole = !RAGGED || n <= a.N - 8;
    if constexpr (T == MxType::F32) {
        float *dst = static_cast<float *>(a.Y) + m * a.ldy + n;
        if (whole) {
            reinterpret_cast<v4f *>(dst)[0] = v4f{s[0], s[1], s[2], s[3]};
            reinterpret_cast<v4f *>(dst)[1] = v4f{s[4], s[5], s[6], s[7]};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (n + e < a.N) dst[e] = s[e];
        }
    } else {
        const v4u v = {narrow2<T>(s[0], s[1]), narrow2<T>(s[2], s[3]), narrow2<T>(s[4], s[5]), narrow2<T>(s[6], s[7])};
        uint16_t *dst = static_cast<uint16_t *>(a.Y) + m * a.ldy + n;
        if (whole) {
            *reinterpret_cast<v4u *>(dst) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (n + e < a.N) dst[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
        }
    }
}

// Stores the 16-bit outputs of one 32-row unit (row0 ..), 128 channels from n0.  A lane's
// 16 channels of a row are 32 bytes of 32 different rows to a store, and the L2 takes a
// request for each; so the wave turns the unit in its own part of LDS (rows kRowPitch bytes
// apart, for the banks) and stores four whole 256-byte row pieces at a time.  (fp32 outputs are
// stored as they lie, 16 bytes of 64 places at a time: 43200 x 1152 -> 4608 322 us, 2.5 TB/s of
// results.)
constexpr int kRowPitch = 272, kTurnBytes = 32 * kRowPitch;

template <int FN, bool RAGGED, MxType T>
__device__ __forceinline__ void store_plain(const Args &a, const v16f (&acc)[FN][2], int fm, uint8_t *turn, int64_t row0,
                                            int64_t row_end, int n0, int lane) {
    const int h16 = (lane >> 5) * 16;
    if constexpr (T == MxType::F32) {
        const int64_t m = row0 + (lane & 31);
        if (m >= row_end) return;
#pragma unroll
        for (int fn = 0; fn < FN; ++fn)
#pragma unroll
            for (int q = 0; q < 16; q += 8) {
                const int n = n0 + fn * 32 + h16 + q;
                float s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = acc[fn][fm][q + e];
                if (n < a.N) store8<RAGGED, T>(a, s, m, n);
            }
        return;
    }
    uint8_t *w = turn + (lane & 31) * kRowPitch + h16 * 2;
#pragma unroll
    for (int fn = 0; fn < FN; ++fn) {
        const v16f &x = acc[fn][fm];
        uint32_t h[8];
#pragma unroll
        for (int v = 0; v < 16; v += 2) h[v / 2] = narrow2<T>(x[v], x[v + 1]);
        reinterpret_cast<v4u *>(w + fn * 64)[0] = v4u{h[0], h[1], h[2], h[3]};
        reinterpret_cast<v4u *>(w + fn * 64)[1] = v4u{h[4], h[5], h[6], h[7]};
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (a wave's LDS accesses stay in order)
    const int c = lane & 15, n = n0 + 8 * c;
    if (c >= 4 * FN || n >= a.N) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i * 4 + (lane >> 4);
        const v4u v = *reinterpret_cast<const v4u *>(turn + r * kRowPitch + c * 16);
        if (row0 + r >= row_end) break;
        uint16_t *dst = static_cast<uint16_t *>(a.Y) + (row0 + r) * a.ldy + n;
        if (!RAGGED || n <= a.N - 8) {
            *reinterpret_cast<v4u *>(dst) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (n + e < a.N) dst[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
        }
    }
}

// Rotates and quantizes NF fragments of one 32-row unit: f[i][v] is channel
// 32 i + 16 (lane / 32) + v (of the output) of row lane % 32.  Writes the chunks
// c0 .. c0 + NF - 1 of unit u.
//
// Stages h = 1 .. 8 stay in the lane, 32 and 64 pair fragments.  Stage 16 pairs the lane
// halves: one exchange of two registers, v and v + 8, leaves the lower lanes with both
// halves' values of v and the upper ones with those of v + 8, so that a sum and a
// difference finish two channels on every lane.  The lane then holds channels 8 h' .. + 7 and
// 16 + 8 h' .. + 7 of each fragment (h' = lane / 32): two whole dwords of codes.
template <int B, int NF>
__device__ __forceinline__ void requantize(const Args &a, float (&f)[NF][16], int lane, int64_t u, int c0) {
    const int h = lane >> 5, row = lane & 31, oK = a.oK;
    if constexpr (B >= 32) {
#pragma unroll
        for (int i = 0; i < NF; ++i) {
#pragma unroll
            for (int st = 1; st < 16; st <<= 1)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if ((v & st) == 0) {
                        const float p = f[i][v], q = f[i][v + st];
                        f[i][v] = p + q;
                        f[i][v + st] = p - q;
                    }
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(f[i][v]), __float_as_uint(f[i][v + 8]),
                                                                false, false);
                const float p = __uint_as_float(r[0]), q = __uint_as_float(r[1]);
                f[i][v] = p + q;
                f[i][v + 8] = p - q;
            }
        }
        if constexpr (B >= 64) {
            static_assert(B < 64 || NF >= B / 32, "fragments of a rotation block");
#pragma unroll
            for (int st = 1; st < B / 32; st <<= 1)
#pragma unroll
                for (int i = 0; i < NF; ++i)
                    if ((i & st) == 0)
#pragma unroll
                        for (int v = 0; v < 16; ++v) {
                            const float p = f[i][v], q = f[i + st][v];
                            f[i][v] = p + q;
                            f[i + st][v] = p - q;
                        }
        }
    }
    int byte[NF];
    v2u codes[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        float m0 = 0.0f, m1 = 0.0f;
#pragma unroll
        for (int v = 0; v < 16; v += 4) {
            m0 = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m0, fabsf(f[i][v])), fabsf(f[i][v + 1]));
            m1 = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m1, fabsf(f[i][v + 2])), fabsf(f[i][v + 3]));
        }
        const uint32_t b = __float_as_uint(__builtin_elementwise_maximum(m0, m1));
        const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        const float m = __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
        byte[i] = mx_scale_byte(__float_as_uint(m) & 0x7fffffffu, 0);
        const float s = mx_scale_value(byte[i], 0);
        codes[i] = v2u{mx_pack8(f[i], s), mx_pack8(f[i] + 8, s)};
    }
    // a chunk's halves meet: lanes 0..31 take the even chunk of a pair, 32..63 the odd
    static_assert(NF % 2 == 0, "chunks in pairs");
#pragma unroll
    for (int i = 0; i < NF; i += 2) {
        const auto lo = __builtin_amdgcn_permlane32_swap(codes[i][0], codes[i + 1][0], false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(codes[i][1], codes[i + 1][1], false, false);
        const int c = c0 + i + h;
        if (32 * c < oK) {
            *reinterpret_cast<v4u *>(a.Oq + mx_code_offset(u, row, c, oK)) =
                B >= 32 ? v4u{lo[0], lo[1], hi[0], hi[1]} : v4u{lo[0], hi[0], lo[1], hi[1]};
            a.Os[mx_scale_offset(u, row, c, oK)] = (uint8_t)(h ? byte[i + 1] : byte[i]);
        }
    }
}

template <int NW, int FN, Out OUT, int B, bool GROUPED, bool RAGGED, MxType T>
__global__ void __launch_bounds__(NW * 64, 2) mx_tile_kernel(Args a)
{
    constexpr int NS = kStages, PPW = 4 / NW;   // transfers per wave and stage
    constexpr int BN = 32 * FN;   // channels
    constexpr bool GATED = OUT == Out::Swiglu;
    static_assert(FN == 4 || OUT == Out::Plain, "a requantized tile");
    constexpr int kRing = NS * kStageBytes + 2 * kQuadBytes, kTurn = OUT == Out::Plain && T != MxType::F32 ? NW * kTurnBytes : 0;
    __shared__ __align__(16) uint8_t pool[kRing > kTurn ? kRing : kTurn];
    __shared__ __align__(16) float ep[BN];   // biases
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nks = a.K >> 6, nq = (a.K + 255) >> 8;

    // ---- which tile ------------------------------------------------------------------
    int tn;
    RowTile rt;
    if constexpr (GROUPED) {
        // the launch covers the most tiles there can be; those in use are dealt evenly to
        // the XCDs, a contiguous run each, channels fastest
        const int total = a.info[plan_table_offset(a.experts, a.log_units) + a.experts] * a.tiles_n;
        const int x = blockIdx.x & 7, j = blockIdx.x >> 3, per = total >> 3, rem = total & 7;
        if (j >= per + (x < rem ? 1 : 0)) return;
        const int L = x * per + min(x, rem) + j;
        tn = L % a.tiles_n;
        rt = find_tile(a, L / a.tiles_n, lane);
    } else {
        int tm;
        tg::Args t;
        t.group_m = a.group_m; t.tiles_m = a.tiles_m; t.tiles_n = a.tiles_n;
        tg::tile_coords(t, tg::tile_of_block(), tm, tn);
        rt.unit0 = tm * (2 * NW);
        rt.unit_end = a.xunits;
        rt.expert = 0;
    }
    const uint8_t *Wq = a.Wq + rt.expert * a.w_stride, *Ws = a.Ws + rt.expert * a.ws_stride;

    // ---- sources: this wave's channel units, its two token units, their scales ----------
    const uint32_t l16 = (uint32_t)lane * 16, l4 = (uint32_t)lane * 4;
    Buffer wsrc[PPW], wssrc[PPW];
    static_for<0, PPW>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        const int64_t wu = min(tn * FN + min(wave * PPW + i, FN - 1), a.wunits - 1);
        wsrc[i] = buffer_of(Wq + wu * nks * kMxUnit, (uint32_t)(nks * kMxUnit));
        wssrc[i] = buffer_of(Ws + wu * nq * kMxScaleRow, (uint32_t)(nq * kMxScaleRow));
    });
    const uint8_t *xsrc[2], *xssrc[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        const int64_t xu = min(rt.unit0 + 2 * wave + f, rt.unit_end - 1);
        xsrc[f] = a.Xq + xu * nks * kMxUnit;
        xssrc[f] = a.Xs + xu * nq * kMxScaleRow;
    }
    const uint32_t pool0 = lds_addr(pool), spool = pool0 + NS * kStageBytes;
    auto produce = [&](uint32_t slot, int k) __attribute__((always_inline)) {
        const uint32_t off = (uint32_t)min(k, nks - 1) * kMxUnit;
        static_for<0, PPW>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            dma16(wsrc[i], l16, off, pool0 + slot + (uint32_t)(wave * PPW + i) * kMxUnit);
        });
    };
    auto produce_scales = [&](uint32_t slot, int q) __attribute__((always_inline)) {
        const uint32_t off = (uint32_t)min(q, nq - 1) * kMxScaleRow;
        static_for<0, PPW>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            dma4(wssrc[i], l4, off, spool + slot + (uint32_t)(wave * PPW + i) * kMxScaleRow);
        });
    };
    v4u x[kDepth][2];        // token units of stages k .. k + kDepth - 1
    uint32_t xs[2][2];       // token scales of even and odd quads
    auto load_x = [&](auto dc, int k) __attribute__((always_inline)) {
        const uint32_t off = l16 + (uint32_t)min(k, nks - 1) * kMxUnit;
#pragma unroll
        for (int f = 0; f < 2; ++f) x[decltype(dc)::value][f] = *reinterpret_cast<const v4u *>(xsrc[f] + off);
    };
    auto load_xs = [&](auto qc, int q) __attribute__((always_inline)) {
        const uint32_t off = l4 + (uint32_t)min(q, nq - 1) * kMxScaleRow;
#pragma unroll
        for (int f = 0; f < 2; ++f) xs[decltype(qc)::value][f] = *reinterpret_cast<const uint32_t *>(xssrc[f] + off);
    };

    // a channel's bias per thread: every sum starts from it
    static_assert(NW * 64 >= BN, "a thread per channel");
    uint16_t bv = 0;
    if (a.bias && tid < BN)
        bv = a.bias[(int64_t)rt.expert * a.N + bias_index(min(tn * BN + tid, a.N - 1), a.N, GATED)];
    __builtin_amdgcn_sched_barrier(0);

    // ---- k loop ------------------------------------------------------------------------
    Operands<FN> op[2];
    Scales<FN> sc[2];   // channel scales of even and odd quads
    const uint32_t wl = pool0 + l16, sl = spool + l4;
    auto read_scales = [&](auto qc) __attribute__((always_inline)) {
        constexpr int Q = decltype(qc)::value;
        static_for<0, FN>([&](auto f) { sc[Q].s[f] = read4<Q * kQuadBytes + decltype(f)::value * kMxScaleRow>(sl); });
    };
    // prologue: two quads of scales and NS stages in flight, stage 0 and quad 0 landed
    produce_scales(0, 0);
    produce_scales(kQuadBytes, 1);
    load_xs(IC<0>{}, 0);
    static_for<0, NS>([&](auto qc) {
        constexpr int Q = decltype(qc)::value;
        produce(Q * kStageBytes, Q);
        __builtin_amdgcn_sched_barrier(0);   // (the loop's first wait counts rely on this order)
        if constexpr (Q < kDepth) load_x(qc, Q);
        __builtin_amdgcn_sched_barrier(0);
    });
    if (tid < BN) ep[tid] = widen(bv, a.bias_bf16);
    // outstanding: what came after stage 0's transfers and loads
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NS - 1) * PPW + 2 * (kDepth - 1)) : "memory");
    v16f acc[FN][2];
    const int h16 = (lane >> 5) * 16;
    static_for<0, FN>([&](auto fc) {
        constexpr int fn = decltype(fc)::value;
        const v4f *b = reinterpret_cast<const v4f *>(ep + fn * 32 + h16);
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[fn][0][v] = acc[fn][1][v] = b[v >> 2][v & 3];
    });
    __builtin_amdgcn_sched_barrier(0);
    op[0].read(wl);
    read_scales(IC<0>{});
    uint32_t cur = 0;
    int k = 0, q = 1;
    // Position P8 of the eight stages of an even and an odd quad.  LAST: one of the stages after
    // the loop, at most seven, which start on a quad; they fetch only what such a stage can still
    // use, so that no load among those that the waits count is one without a use (the compiler
    // drops it).
    auto stage = [&](auto pc, auto lc) __attribute__((always_inline)) {
        constexpr bool LAST = decltype(lc)::value;
        constexpr int P8 = decltype(pc)::value, P = P8 & 3, Q = P8 >> 2, R = P & 1;
        // Outstanding: what the three stages before this one fetch, whatever the order within
        // each; the next stage's transfers are those of the stage before them.
        constexpr int VM = fetched(P8 - 1, LAST, PPW) + fetched(P8 - 2, LAST, PPW) + fetched(P8 - 3, LAST, PPW);
        static_assert(NS == 5, "three stages between a transfer and the wait for it");
        if constexpr (P == 0) wait_stage<VM>(op[R], sc[Q]);
        else wait_stage<VM>(op[R]);
        const uint32_t nxt = cur == (uint32_t)((NS - 1) * kStageBytes) ? 0u : cur + kStageBytes;
        op[1 - R].read(wl + nxt);
        if constexpr (P == 3) read_scales(IC<1 - Q>{});
        if constexpr (fetches_w(P8, LAST)) produce(cur, k + NS);
        if constexpr (fetches_xs(P8, LAST)) load_xs(IC<1 - Q>{}, q);
        if constexpr (fetches_ws(P8, LAST)) produce_scales(Q * kQuadBytes, ++q);
        static_for<0, FN>([&](auto fc) {
            static_for<0, 2>([&](auto mc) {
                constexpr int fn = decltype(fc)::value, fm = decltype(mc)::value;
                acc[fn][fm] = mfma_mx4<P>(op[R].w[fn], x[P][fm], acc[fn][fm], sc[Q].s[fn], xs[Q][fm]);
            });
        });
        if constexpr (fetches_x(P8, LAST)) load_x(IC<P>{}, k + kDepth);
        cur = nxt;
        ++k;
    };
    for (int pairs = nks >> 3; pairs > 0; --pairs) static_for<0, 8>([&](auto p) { stage(p, std::false_type{}); });
    const int rest = nks & 7;
    static_for<0, 7>([&](auto p) {
        if (rest > decltype(p)::value) stage(p, std::true_type{});
    });
    // drain: the last transfers, and the last reads, whose data is not used (all register
    // sets are named, so that no register of theirs serves another value meanwhile)
    wait_stage<0>(op[0], sc[0]);
    wait_stage<0>(op[1], sc[1]);

    // ---- epilogue: lane owns row m and 16 consecutive channels of each fragment ---------
    static_for<0, 2>([&](auto mc) {
        constexpr int fm = decltype(mc)::value;
        const int u = rt.unit0 + wave * 2 + fm;
        if (u >= rt.unit_end) return;
        if constexpr (OUT == Out::Plain) {
            const int64_t end = GROUPED ? (int64_t)rt.unit_end * 32 : a.M;
            store_plain<FN, RAGGED, T>(a, acc, fm, pool + wave * kTurnBytes, (int64_t)u * 32, end, tn * BN, lane);
        } else if constexpr (GATED) {
            float f[2][16];
            static_for<0, 2>([&](auto pc) {
                constexpr int i = decltype(pc)::value;
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    f[i][v] = silu(acc[2 * i][fm][v]) * acc[2 * i + 1][fm][v];
            });
            requantize<B, 2>(a, f, lane, u, tn * 2);
        } else {
            float f[4][16];
            static_for<0, 4>([&](auto pc) {
                constexpr int i = decltype(pc)::value;
#pragma unroll
                for (int v = 0; v < 16; ++v) f[i][v] = OUT == Out::Gelu ? gelu(acc[i][fm][v]) : acc[i][fm][v];
            });
            requantize<B, 4>(a, f, lane, u, tn * 4);
        }
    });
}

// ---- few rows ----------------------------------------------------------------------------
// With few tiles of the kernel above most compute units are idle and a launch takes the
// length of one wave's k loop.  Here a workgroup computes 32 FM rows x 32 FN channels, its KS
// waves each a part of the k loop with operands straight from memory (nothing is shared
// between them), kAhead stages ahead; the partial sums meet in LDS.  A plain result needs no
// channel but its own: 1 x 1 fragments make the most workgroups, 2 x 2 read half the operand
// bytes an instruction.  A requantized one needs the channels of a rotation block (FN = 4).
template <int FN_, int FM_, int KS_, int AHEAD>
struct Split {
    static constexpr int FN = FN_, FM = FM_, KS = KS_, kAhead = AHEAD, NT = KS * 64, BN = 32 * FN, BM = 32 * FM;
    static constexpr int kPitch = BN + 4;   // floats between rows of a partial tile, for the banks
};
using Split1 = Split<1, 1, 8, 6>;
using Split2 = Split<2, 2, 4, 4>;
using SplitMx = Split<4, 1, 4, 3>;

template <class C, Out OUT, int B, bool GROUPED, bool RAGGED, MxType T>
__global__ void __launch_bounds__(C::NT) mx_split_kernel(Args a)
{
    constexpr bool MX4 = OUT != Out::Plain, GATED = OUT == Out::Swiglu;
    constexpr int FN = C::FN, FM = C::FM, KS = C::KS, D = C::kAhead;
    static_assert(!MX4 || (FN == 4 && FM == 1), "a requantized tile");
    __shared__ __align__(16) float part[KS][C::BM * C::kPitch];
    __shared__ __align__(16) float ep[C::BN];   // biases
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nks = a.K >> 6, nq = (a.K + 255) >> 8;
    int tn;
    RowTile rt;
    if constexpr (GROUPED) {
        const int total = a.info[plan_table_offset(a.experts, a.log_units) + a.experts] * a.tiles_n;
        if ((int)blockIdx.x >= total) return;
        tn = blockIdx.x % a.tiles_n;
        rt = find_tile(a, blockIdx.x / a.tiles_n, lane);
    } else {
        tn = blockIdx.x % a.tiles_n;
        rt.unit0 = blockIdx.x / a.tiles_n * FM;
        rt.unit_end = a.xunits;
        rt.expert = 0;
    }
    const int u = rt.unit0;
    // this wave's stages; bytes of a scale row: lane's dword, then the stage's byte
    const int kb = wave * nks / KS, ke = (wave + 1) * nks / KS;
    const uint8_t *wsrc[FN], *wssrc[FN];
#pragma unroll
    for (int f = 0; f < FN; ++f) {
        const int64_t wu = min(tn * FN + f, a.wunits - 1);
        wsrc[f] = a.Wq + rt.expert * a.w_stride + wu * nks * kMxUnit + lane * 16;
        wssrc[f] = a.Ws + rt.expert * a.ws_stride + wu * nq * kMxScaleRow + lane * 4;
    }
    // a channel's bias per thread, on its way while the k loop runs
    static_assert(C::NT >= C::BN, "a thread per channel");
    uint16_t bv = 0;
    if (a.bias && tid < C::BN)
        bv = a.bias[(int64_t)rt.expert * a.N + bias_index(min(tn * C::BN + tid, a.N - 1), a.N, GATED)];
    const uint8_t *xsrc[FM], *xssrc[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) {
        const int64_t xu = min(u + f, rt.unit_end - 1);
        xsrc[f] = a.Xq + xu * nks * kMxUnit + lane * 16;
        xssrc[f] = a.Xs + xu * nq * kMxScaleRow + lane * 4;
    }
    v16f acc[FN][FM];
#pragma unroll
    for (int f = 0; f < FN; ++f)
#pragma unroll
        for (int g = 0; g < FM; ++g) acc[f][g] = v16f{};
    if (kb < ke) {
        v4u w[D][FN], x[D][FM];
        uint8_t ws[D][FN], xs[D][FM];
        auto load = [&](auto dc, int k) __attribute__((always_inline)) {
            constexpr int d = decltype(dc)::value;
            const uint32_t off = (uint32_t)k * kMxUnit, soff = (uint32_t)(k >> 2) * kMxScaleRow + (k & 3);
#pragma unroll
            for (int f = 0; f < FN; ++f) {
                w[d][f] = *reinterpret_cast<const v4u *>(wsrc[f] + off);
                ws[d][f] = wssrc[f][soff];
            }
#pragma unroll
            for (int f = 0; f < FM; ++f) {
                x[d][f] = *reinterpret_cast<const v4u *>(xsrc[f] + off);
                xs[d][f] = xssrc[f][soff];
            }
        };
        auto mma = [&](auto dc) __attribute__((always_inline)) {
            constexpr int d = decltype(dc)::value;
#pragma unroll
            for (int f = 0; f < FN; ++f)
#pragma unroll
                for (int g = 0; g < FM; ++g) acc[f][g] = mfma_mx4<0>(w[d][f], x[d][g], acc[f][g], ws[d][f], xs[d][g]);
        };
        const int last = ke - 1;   // loads past the end repeat the last stage
        static_for<0, D>([&](auto dc) {
            load(dc, min(kb + decltype(dc)::value, last));
            __builtin_amdgcn_sched_barrier(0);
        });
        // whole groups of D stages, then the rest one by one: one loop with one exit, so that
        // the compiler's waits count only the loads that matter
        const int groups = (ke - kb) / D, rest = (ke - kb) - groups * D;
        int k = kb + D;
        for (int g = 0; g < groups; ++g)
            static_for<0, D>([&](auto dc) {
                mma(dc);
                load(dc, min(k, last));
                __builtin_amdgcn_sched_barrier(0);
                ++k;
            });
        static_for<0, D - 1>([&](auto dc) {
            if (rest > decltype(dc)::value) mma(dc);
        });
    }
    if (tid < C::BN) ep[tid] = widen(bv, a.bias_bf16);
    // lane's 16 channels of its row
    const int row = lane & 31, h16 = (lane >> 5) * 16;
#pragma unroll
    for (int f = 0; f < FN; ++f)
#pragma unroll
        for (int g = 0; g < FM; ++g) {
            v4f *dst = reinterpret_cast<v4f *>(&part[wave][(g * 32 + row) * C::kPitch + f * 32 + h16]);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                dst[q] = v4f{acc[f][g][4 * q], acc[f][g][4 * q + 1], acc[f][g][4 * q + 2], acc[f][g][4 * q + 3]};
        }
    __syncthreads();
    if constexpr (!MX4) {
        // eight channels of a row at a time
        constexpr int kPieces = C::BN / 8;
        for (int p = tid; p < C::BM * kPieces; p += C::NT) {
            const int r = p / kPieces, c = (p % kPieces) * 8, n = tn * C::BN + c;
            const int64_t m = (int64_t)u * 32 + r;
            if (n >= a.N || m >= (GROUPED ? (int64_t)rt.unit_end * 32 : (int64_t)a.M)) continue;
            float s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = ep[c + e];
#pragma unroll
            for (int w = 0; w < KS; ++w) {
                const v4f *src = reinterpret_cast<const v4f *>(&part[w][r * C::kPitch + c]);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += src[e >> 2][e & 3];
            }
            store8<RAGGED, T>(a, s, m, n);
        }
    } else {
        // wave 0 .. NW - 1: the fragments of a rotation block each, summed in the products' layout
        constexpr int NW = GATED || B == 128 ? 1 : 2, NF = FN / NW;
        if (wave >= NW) return;
        float s[NF][16];
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            const int c = (wave * NF + i) * 32 + h16;
#pragma unroll
            for (int v = 0; v < 16; ++v) s[i][v] = ep[c + v];
#pragma unroll
            for (int w = 0; w < KS; ++w) {
                const v4f *src = reinterpret_cast<const v4f *>(&part[w][row * C::kPitch + c]);
#pragma unroll
                for (int v = 0; v < 16; ++v) s[i][v] += src[v >> 2][v & 3];
            }
        }
        if constexpr (GATED) {
            float f[2][16];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) f[i][v] = silu(s[2 * i][v]) * s[2 * i + 1][v];
            requantize<B, 2>(a, f, lane, u, tn * 2);
        } else {
            if constexpr (OUT == Out::Gelu) {
#pragma unroll
                for (int i = 0; i < NF; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) s[i][v] = gelu(s[i][v]);
            }
            requantize<B, NF>(a, s, lane, u, tn * 4 + wave * NF);
        }
    }
}

// The kernels: tiles of 32 and 64 rows split over the k loop, of 128 and of 256 rows, the latter
// also of 96 channels.  (A plan has tables for those of 1, 4 and 8 row units.)
enum Kernel { kSplit1, kSplit2, kTile128, kTile256, kTile256x96 };
constexpr int kLogUnits[] = {0, 1, 2, 3, 3};   // row units of a tile

template <Out OUT, int B, bool GROUPED, bool RAGGED, MxType T>
void launch_one(Args a, Kernel kernel, int64_t row_tiles, hipStream_t stream) {
    constexpr bool DENSE = OUT == Out::Plain && !GROUPED;   // what kSplit2 and kTile256x96 are for
    using S1 = std::conditional_t<OUT == Out::Plain, Split1, SplitMx>;
    const int bn = kernel == kSplit1 ? S1::BN : kernel == kSplit2 ? Split2::BN : kernel == kTile256x96 ? 96 : kBN;
    a.tiles_n = (a.N + bn - 1) / bn;
    const dim3 grid((unsigned)(row_tiles * a.tiles_n));
    switch (kernel) {
        case kSplit1:
            hipLaunchKernelGGL((mx_split_kernel<S1, OUT, B, GROUPED, RAGGED, T>), grid, dim3(S1::NT), 0, stream, a);
            break;
        case kSplit2:
            if constexpr (DENSE)
                hipLaunchKernelGGL((mx_split_kernel<Split2, OUT, B, GROUPED, RAGGED, T>), grid, dim3(Split2::NT), 0, stream,
                                   a);
            break;
        case kTile128:
            hipLaunchKernelGGL((mx_tile_kernel<2, 4, OUT, B, GROUPED, RAGGED, T>), grid, dim3(128), 0, stream, a);
            break;
        case kTile256:
            hipLaunchKernelGGL((mx_tile_kernel<4, 4, OUT, B, GROUPED, RAGGED, T>), grid, dim3(256), 0, stream, a);
            break;
        case kTile256x96:
            if constexpr (DENSE)
                hipLaunchKernelGGL((mx_tile_kernel<4, 3, OUT, B, GROUPED, RAGGED, T>), grid, dim3(256), 0, stream, a);
            break;
    }
}

template <Out OUT, int B, bool GROUPED>
void launch_kernel(const Args &a, Kernel kernel, int64_t row_tiles, hipStream_t stream) {
    if constexpr (OUT == Out::Plain) {
        auto by_type = [&](auto rc) {
            constexpr bool RAGGED = decltype(rc)::value;
            switch (a.out_type) {
                case MxType::F16: launch_one<OUT, B, GROUPED, RAGGED, MxType::F16>(a, kernel, row_tiles, stream); break;
                case MxType::BF16: launch_one<OUT, B, GROUPED, RAGGED, MxType::BF16>(a, kernel, row_tiles, stream); break;
                case MxType::F32: launch_one<OUT, B, GROUPED, RAGGED, MxType::F32>(a, kernel, row_tiles, stream); break;
            }
        };
        if (a.N % 8 != 0) by_type(std::true_type{});
        else by_type(std::false_type{});
    } else {
        launch_one<OUT, B, GROUPED, false, MxType::F16>(a, kernel, row_tiles, stream);
    }
}

template <bool GROUPED>
hipError_t launch_out(const Args &a, MxAct act, int block, Kernel kernel, int64_t row_tiles, hipStream_t stream) {
    if (a.Y) {
        launch_kernel<Out::Plain, 0, GROUPED>(a, kernel, row_tiles, stream);
    } else {
        auto by_block = [&](auto oc) {
            constexpr Out OUT = decltype(oc)::value;
            switch (block) {
                case 0: launch_kernel<OUT, 0, GROUPED>(a, kernel, row_tiles, stream); break;
                case 32: launch_kernel<OUT, 32, GROUPED>(a, kernel, row_tiles, stream); break;
                case 64: launch_kernel<OUT, 64, GROUPED>(a, kernel, row_tiles, stream); break;
                default:
                    if constexpr (OUT != Out::Swiglu) launch_kernel<OUT, 128, GROUPED>(a, kernel, row_tiles, stream);
                    break;
            }
        };
        switch (act) {
            case MxAct::None: by_block(std::integral_constant<Out, Out::None>{}); break;
            case MxAct::Gelu: by_block(std::integral_constant<Out, Out::Gelu>{}); break;
            case MxAct::Swiglu: by_block(std::integral_constant<Out, Out::Swiglu>{}); break;
        }
    }
    return hipGetLastError();
}

// The kernel of a product, by the workgroups it would be cut into (c compute units; of a
// plan the row units it can have at most, which a few tokens nearly reach).  us, measured
// on tiles of 32 / 64 (both split) / 128 / 256 rows:
//   32   one row unit, plain, up to 2 c workgroups (3 c on long k loops): 1 x 4608 -> 1152
//        6.2 / - / 12.9 / 14.3; experts, 2 tokens to 2 of 16, 4608 -> 1152, 144 workgroups:
//        7.5 / - / 13.5 / 14.7, 64 tokens, 720: 13.1 / - / 14.8 / 16.4, 256, 1152: 16.4 / - /
//        15.7 / 17.5.  Requantized, up to 1.75 c: 384 x 1152 -> 4608, 432: 8.8 / - / 10.7 /
//        12.8; 512, 576: 12.1 / - / 10.9 / 11.4; where one wave finishes a tile whose
//        channels gate each other, up to c: 8 tokens to 6 of 64 experts, 1152 -> 1536, 588:
//        14.9 / - / 10.3 / 11.2.
//   64   more units, plain, while every workgroup has a unit to itself: 777 x 4608 -> 1152,
//        234: 13.4 / 8.5 / 13.8 / 15.5; 512 x 1152 -> 1152, 144: 7.1 / 6.3 / 6.6 / 7.3; 512 x
//        1152 -> 2304, 288: 9.8 / 7.7 / 6.9 / 7.3; on long k loops up to 1.75 c: 1536 x 4608 ->
//        1152, 432: 22.1 / 13.8 / 14.4 / 15.8, 2048, 576: 27.5 / 18.7 / 14.8 / 16.1.
//   128  while those tiles are one to a unit (3072 x 4608 -> 1152, 216: 40.9 / 23.8 / 15.8 /
//        17.2; 4096, 288: 51.4 / 28.6 / 24.2 / 18.0), and for experts of under 512 rows on
//        average, whose last tiles are half empty (384 rows, 1152 -> 1536 gated: 38.5 of 128 /
//        41.8 of 256; 512 rows, 1152 -> 4608: 51.6 / 50.2; 5400: 405 / 399);
//   256  otherwise: the fewest operand bytes (43200 x 1152 -> 4608: 189 of 128 / 171 of 256);
//        96 channels instead of 128, plain, where they take no more rounds of one tile to a unit
//        (us of 128 / 96 channels, tiles: 4608 -> 1152 with 4096 rows, 144 / 192, 19.1 / 16.9; 8192,
//        288 / 384, 30.0 / 26.5; 16384, 576 / 768, 49.0 / 44.7; but 5400, 198 / 264, 20.8 / 25.7;
//        20000, 711 / 948, 52.9 / 58.1; 8192 x 1152 -> 1152, 288 / 384, 16.1 / 14.6; 8192^3, 2048 /
//        2752, 230 / 251).
inline Kernel pick_kernel(const MxGemmArgs &g, int64_t units, int64_t c) {
    const bool mx4 = g.Y == nullptr, longk = g.K >= 48 * 64;
    if (mx4) {
        const int64_t split = units * ((g.N + SplitMx::BN - 1) / SplitMx::BN);
        if (split <= (g.act == MxAct::Swiglu ? c : c * 7 / 4)) return kSplit1;
    } else if (g.info || units == 1) {
        const int64_t split = units * ((g.N + Split1::BN - 1) / Split1::BN);
        if (split <= (longk ? 3 * c : 2 * c)) return kSplit1;
    } else {
        const int64_t split = (units + 1) / 2 * ((g.N + Split2::BN - 1) / Split2::BN);
        if (split <= (longk ? c * 7 / 4 : c)) return kSplit2;
    }
    const int64_t tiles_n = (g.N + kBN - 1) / kBN;
    if (g.info) {
        const int64_t nonempty = g.experts < g.assignments ? g.experts : g.assignments;
        if (g.assignments < 512 * (int64_t)g.experts || (g.assignments / 128 + nonempty) * tiles_n <= c) return kTile128;
        return kTile256;
    }
    if ((units + 3) / 4 * tiles_n <= c) return kTile128;
    const int64_t rows = (units + 7) / 8, rounds = (rows * tiles_n + c - 1) / c;
    return !mx4 && rows * ((g.N + 95) / 96) <= rounds * c ? kTile256x96 : kTile256;
}

}  // namespace mx
}  // namespace

hipError_t launch_mx_gemm(const MxGemmArgs &g, hipStream_t stream) {
    mx::Args a = {};
    a.Xq = g.Xq; a.Xs = g.Xs; a.Wq = g.Wq; a.Ws = g.Ws;
    a.bias = static_cast<const uint16_t *>(g.bias);
    a.bias_bf16 = g.bias_type == MxType::BF16;
    a.out_type = g.out_type;
    a.M = (int)g.M;
    a.N = (int)g.N;
    a.K = g.K;
    a.wunits = (int)(padded_rows(g.N) >> 5);
    a.w_stride = (int64_t)a.wunits * (g.K >> 6) * kMxUnit;
    a.ws_stride = mx_scale_bytes(a.wunits, g.K);
    a.group_m = 4;
    a.info = g.info;
    a.experts = g.experts;
    a.Y = g.Y;
    a.ldy = g.ldy;
    a.Oq = g.Oq;
    a.Os = g.Os;
    a.oK = (int)(g.act == MxAct::Swiglu ? g.N / 2 : g.N);
    a.xunits = (int)(g.info ? g.units : padded_act_rows(g.M) >> 5);
    const mx::Kernel kernel = mx::pick_kernel(g, a.xunits, compute_units());
    a.log_units = mx::kLogUnits[kernel];
    const int64_t per = 1 << a.log_units;
    if (g.info) {
        // every expert's last tile may be a part of one
        const int64_t most = per == 1 ? g.units : g.units / per + (g.experts < g.units ? g.experts : g.units);
        return mx::launch_out<true>(a, g.act, g.block, kernel, most, stream);
    }
    a.tiles_m = (int)((a.xunits + per - 1) / per);
    return mx::launch_out<false>(a, g.act, g.block, kernel, a.tiles_m, stream);
}

}  // namespace clq
