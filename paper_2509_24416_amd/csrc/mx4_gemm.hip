// MX4 products: Y = dequant(Xq) . dequant(Wq)^T + bias on the fp4 matrix cores of
// gfx950, dense and grouped by expert, with the result either stored as fp16 / bf16
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
    uint16_t *Y;
    int64_t ldy;
    bool bias_bf16, out_bf16;
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
// two outputs, rounded to nearest even
template <bool BF16>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    if constexpr (BF16) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        const b2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// The tanh form of GELU: 0.5 h (1 + tanh u) = h / (1 + exp(-2u)).  The hardware's exp2
// and reciprocal (1 ulp each) keep the relative error near 3e-7, under that of the
// sum it is applied to.
__device__ __forceinline__ float gelu(float h) {
    const float u2 = h * (1.5957691216057308f + 0.07135481282553575f * h * h);   // 2u
    return h * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * u2));
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
// A workgroup of 4 waves computes 128 channels x 256 tokens, each wave 128 channels x 64
// tokens (4 x 2 fragments of 32 x 32).  A k-stage is 64 codes, one matrix instruction per
// fragment.  The channel units are shared by the waves: they go global -> LDS without
// registers through a ring of NS stages, and a wave reads a stage's units back one stage
// ahead of its use.  The token units belong to one wave each and go straight to registers,
// kDepth stages ahead (through LDS the reads and writes of both operands came to 144 of
// its 128 bytes a clock at full rate).  The scale dwords of four stages (a quad) take the
// same two ways, the channels' through a ring of two, read at the end of the quad before.
//
// Ring protocol: iteration s waits until stage s + 1 has landed (transfers and loads
// complete in issue order: at most the later stages' may be outstanding) and its own LDS
// reads of stage s are in, then the workgroup barrier: every wave holds stage s in
// registers, so its slot is refilled with stage s + NS.  Quad q's scale slot is likewise
// free after the barrier of the quad's first iteration and refilled there with quad q + 2,
// needed at the end of quad q + 1.  Transfers past the end repeat the last stage or quad,
// so the wait counts stay constant.
constexpr int kWaves = 4, kThreads = kWaves * 64, kBN = 128, kBM = 256;
constexpr int kStages = 5;                      // ring of channel units
constexpr int kStageBytes = 4 * kMxUnit;        // one unit transferred by each wave
constexpr int kQuadBytes = 4 * kMxScaleRow;
constexpr int kDepth = 4;                       // stages of token units in registers

struct Operands {
    v4u w[4];
    __device__ __forceinline__ void read(uint32_t wa) {
        static_for<0, 4>([&](auto f) { w[f] = read16<decltype(f)::value * kMxUnit>(wa); });
    }
};
struct Scales {
    uint32_t s[4];
};
// At most VM transfers outstanding, the LDS reads in, the workgroup barrier.  The
// destinations of those reads are named, so that nothing touches them before; a
// register set whose value is used once, in place, is never copied while a read of it
// is in flight (hence two sets of scales, too: a copy from one into the other was moved
// ahead of this wait).
#define CLQ_MX_WAIT "s_waitcnt vmcnt(%c[vm]) lgkmcnt(0)\n\ts_barrier"
template <int VM>
__device__ __forceinline__ void wait_stage(Operands &o) {
    asm volatile(CLQ_MX_WAIT : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]), "+v"(o.w[3]) : [vm] "n"(VM) : "memory");
}
template <int VM>
__device__ __forceinline__ void wait_stage(Operands &o, Scales &s) {
    asm volatile(CLQ_MX_WAIT
                 : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]), "+v"(o.w[3]), "+v"(s.s[0]), "+v"(s.s[1]), "+v"(s.s[2]),
                   "+v"(s.s[3])
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

// Stores the plain outputs of one 32-row unit (row0 ..), 128 channels from n0.  A lane's
// 16 channels of a row are 32 bytes of 32 different rows to a store, and the L2 takes a
// request for each; so the wave turns the unit in its own part of LDS (rows kRowPitch bytes
// apart, for the banks) and stores four whole 256-byte row pieces at a time.
constexpr int kRowPitch = 272, kTurnBytes = 32 * kRowPitch;

template <bool RAGGED, bool BF16>
__device__ __forceinline__ void store_plain(const Args &a, const v16f (&acc)[4][2], int fm, const float *bias,
                                            uint8_t *turn, int64_t row0, int64_t row_end, int n0, int lane) {
    const int h16 = (lane >> 5) * 16;
    uint8_t *w = turn + (lane & 31) * kRowPitch + h16 * 2;
#pragma unroll
    for (int fn = 0; fn < 4; ++fn) {
        const v16f &x = acc[fn][fm];
        const float *b = bias + fn * 32 + h16;
        uint32_t h[8];
#pragma unroll
        for (int v = 0; v < 16; v += 2) h[v / 2] = narrow2<BF16>(x[v] + b[v], x[v + 1] + b[v + 1]);
        reinterpret_cast<v4u *>(w + fn * 64)[0] = v4u{h[0], h[1], h[2], h[3]};
        reinterpret_cast<v4u *>(w + fn * 64)[1] = v4u{h[4], h[5], h[6], h[7]};
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (a wave's LDS accesses stay in order)
    const int c = lane & 15, n = n0 + 8 * c;
    if (n >= a.N) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i * 4 + (lane >> 4);
        const v4u v = *reinterpret_cast<const v4u *>(turn + r * kRowPitch + c * 16);
        if (row0 + r >= row_end) break;
        uint16_t *dst = a.Y + (row0 + r) * a.ldy + n;
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

template <Out OUT, int B, bool GROUPED, bool RAGGED, bool BF16>
__global__ void __launch_bounds__(kThreads, 2) mx_tile_kernel(Args a)
{
    constexpr int NS = kStages;
    constexpr bool GATED = OUT == Out::Swiglu;
    constexpr int kRing = NS * kStageBytes + 2 * kQuadBytes, kTurn = OUT == Out::Plain ? kWaves * kTurnBytes : 0;
    __shared__ __align__(16) uint8_t pool[kRing > kTurn ? kRing : kTurn];
    __shared__ __align__(16) float ep[kBN];   // biases
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
        rt.unit0 = tm * (kBM / 32);
        rt.unit_end = a.xunits;
        rt.expert = 0;
    }
    const uint8_t *Wq = a.Wq + rt.expert * a.w_stride, *Ws = a.Ws + rt.expert * a.ws_stride;

    // ---- sources: this wave's channel unit, its two token units, their scales -----------
    const uint32_t l16 = (uint32_t)lane * 16, l4 = (uint32_t)lane * 4;
    const int64_t wu = min(tn * 4 + wave, a.wunits - 1);
    const Buffer wsrc = buffer_of(Wq + wu * nks * kMxUnit, (uint32_t)(nks * kMxUnit));
    const Buffer wssrc = buffer_of(Ws + wu * nq * kMxScaleRow, (uint32_t)(nq * kMxScaleRow));
    const uint8_t *xsrc[2], *xssrc[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        const int64_t xu = min(rt.unit0 + 2 * wave + f, rt.unit_end - 1);
        xsrc[f] = a.Xq + xu * nks * kMxUnit;
        xssrc[f] = a.Xs + xu * nq * kMxScaleRow;
    }
    const uint32_t pool0 = lds_addr(pool), spool = pool0 + NS * kStageBytes;
    auto produce = [&](uint32_t slot, int k) __attribute__((always_inline)) {
        dma16(wsrc, l16, (uint32_t)min(k, nks - 1) * kMxUnit, pool0 + slot + (uint32_t)wave * kMxUnit);
    };
    auto produce_scales = [&](uint32_t slot, int q) __attribute__((always_inline)) {
        dma4(wssrc, l4, (uint32_t)min(q, nq - 1) * kMxScaleRow, spool + slot + (uint32_t)wave * kMxScaleRow);
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

    // the tile's biases, in registers until the ring is done with
    float bv = 0.0f;
    if (a.bias && tid < kBN) {
        const int n = min(tn * kBN + tid, a.N - 1);
        bv = widen(a.bias[(int64_t)rt.expert * a.N + bias_index(n, a.N, GATED)], a.bias_bf16);
    }
    __builtin_amdgcn_sched_barrier(0);

    // ---- k loop ------------------------------------------------------------------------
    Operands op[2];
    Scales sc[2];   // channel scales of even and odd quads
    const uint32_t wl = pool0 + l16, sl = spool + l4;
    auto read_scales = [&](auto qc) __attribute__((always_inline)) {
        constexpr int Q = decltype(qc)::value;
        static_for<0, 4>([&](auto f) { sc[Q].s[f] = read4<Q * kQuadBytes + decltype(f)::value * kMxScaleRow>(sl); });
    };
    v16f acc[4][2];
    static_for<0, 4>([&](auto i) { static_for<0, 2>([&](auto j) { acc[decltype(i)::value][decltype(j)::value] = v16f{}; }); });

    // prologue: two quads of scales and NS stages in flight, stage 0 and quad 0 landed
    produce_scales(0, 0);
    produce_scales(kQuadBytes, 1);
    load_xs(IC<0>{}, 0);
    static_for<0, NS>([&](auto qc) {
        constexpr int Q = decltype(qc)::value;
        produce(Q * kStageBytes, Q);
        if constexpr (Q < kDepth) load_x(qc, Q);
        __builtin_amdgcn_sched_barrier(0);
    });
    // after stage 0's transfer: at least that of every other stage
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(NS - 1 + 2 * (kDepth - 1)) : "memory");
    op[0].read(wl);
    read_scales(IC<0>{});
    uint32_t cur = 0;
    int k = 0, q = 1;
    // position P8 of the eight stages of an even and an odd quad
    auto stage = [&](auto pc) __attribute__((always_inline)) {
        constexpr int P8 = decltype(pc)::value, P = P8 & 3, Q = P8 >> 2, R = P & 1;
        // Outstanding: the last NS - 2 stages' transfer and two loads, and the three of the
        // scales if a quad began among them.
        constexpr int VM = (NS - 2) * 3 + (P >= 1 && P <= NS - 2 ? 3 : 0);
        if constexpr (P == 0) wait_stage<VM>(op[R], sc[Q]);
        else wait_stage<VM>(op[R]);
        const uint32_t nxt = cur == (uint32_t)((NS - 1) * kStageBytes) ? 0u : cur + kStageBytes;
        op[1 - R].read(wl + nxt);
        if constexpr (P == 3) read_scales(IC<1 - Q>{});
        produce(cur, k + NS);
        if constexpr (P == 0) {
            load_xs(IC<1 - Q>{}, q);
            produce_scales(Q * kQuadBytes, ++q);
        }
        static_for<0, 4>([&](auto fc) {
            static_for<0, 2>([&](auto mc) {
                constexpr int fn = decltype(fc)::value, fm = decltype(mc)::value;
                acc[fn][fm] = mfma_mx4<P>(op[R].w[fn], x[P][fm], acc[fn][fm], sc[Q].s[fn], xs[Q][fm]);
            });
        });
        load_x(IC<P>{}, k + kDepth);
        cur = nxt;
        ++k;
    };
    for (int pairs = nks >> 3; pairs > 0; --pairs) static_for<0, 8>([&](auto p) { stage(p); });
    const int rest = nks & 7;
    static_for<0, 7>([&](auto p) {
        if (rest > decltype(p)::value) stage(p);
    });
    // drain: the last transfers, and the last reads, whose data is not used (all register
    // sets are named, so that no register of theirs serves another value meanwhile)
    wait_stage<0>(op[0], sc[0]);
    wait_stage<0>(op[1], sc[1]);
    if (tid < kBN) ep[tid] = bv;
    __syncthreads();

    // ---- epilogue: lane owns row m and 16 consecutive channels of each fragment ---------
    const int h16 = (lane >> 5) * 16;
    static_for<0, 2>([&](auto mc) {
        constexpr int fm = decltype(mc)::value;
        const int u = rt.unit0 + wave * 2 + fm;
        if (u >= rt.unit_end) return;
        if constexpr (OUT == Out::Plain) {
            const int64_t end = GROUPED ? (int64_t)rt.unit_end * 32 : a.M;
            store_plain<RAGGED, BF16>(a, acc, fm, ep, pool + wave * kTurnBytes, (int64_t)u * 32, end, tn * kBN, lane);
        } else if constexpr (GATED) {
            float f[2][16];
            static_for<0, 2>([&](auto pc) {
                constexpr int i = decltype(pc)::value;
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    f[i][v] = silu(acc[2 * i][fm][v] + ep[64 * i + h16 + v]) * (acc[2 * i + 1][fm][v] + ep[64 * i + 32 + h16 + v]);
            });
            requantize<B, 2>(a, f, lane, u, tn * 2);
        } else {
            float f[4][16];
            static_for<0, 4>([&](auto pc) {
                constexpr int i = decltype(pc)::value;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float y = acc[i][fm][v] + ep[32 * i + h16 + v];
                    f[i][v] = OUT == Out::Gelu ? gelu(y) : y;
                }
            });
            requantize<B, 4>(a, f, lane, u, tn * 4);
        }
    });
}

template <Out OUT, int B, bool GROUPED>
void launch_kernel(const Args &a, unsigned grid, hipStream_t stream) {
    const dim3 g(grid), b(kThreads);
    if constexpr (OUT == Out::Plain) {
        const bool ragged = a.N % 8 != 0;
        if (ragged && a.out_bf16) hipLaunchKernelGGL((mx_tile_kernel<OUT, B, GROUPED, true, true>), g, b, 0, stream, a);
        else if (ragged) hipLaunchKernelGGL((mx_tile_kernel<OUT, B, GROUPED, true, false>), g, b, 0, stream, a);
        else if (a.out_bf16) hipLaunchKernelGGL((mx_tile_kernel<OUT, B, GROUPED, false, true>), g, b, 0, stream, a);
        else hipLaunchKernelGGL((mx_tile_kernel<OUT, B, GROUPED, false, false>), g, b, 0, stream, a);
    } else {
        hipLaunchKernelGGL((mx_tile_kernel<OUT, B, GROUPED, false, false>), g, b, 0, stream, a);
    }
}

template <bool GROUPED>
hipError_t launch_out(Args &a, MxAct act, int block, unsigned grid, hipStream_t stream) {
    if (a.Y) {
        launch_kernel<Out::Plain, 0, GROUPED>(a, grid, stream);
    } else {
        auto by_block = [&](auto oc) {
            constexpr Out OUT = decltype(oc)::value;
            switch (block) {
                case 0: launch_kernel<OUT, 0, GROUPED>(a, grid, stream); break;
                case 32: launch_kernel<OUT, 32, GROUPED>(a, grid, stream); break;
                case 64: launch_kernel<OUT, 64, GROUPED>(a, grid, stream); break;
                default:
                    if constexpr (OUT != Out::Swiglu) launch_kernel<OUT, 128, GROUPED>(a, grid, stream);
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

}  // namespace mx
}  // namespace

hipError_t launch_mx_gemm(const MxGemmArgs &g, hipStream_t stream) {
    mx::Args a = {};
    a.Xq = g.Xq; a.Xs = g.Xs; a.Wq = g.Wq; a.Ws = g.Ws;
    a.bias = static_cast<const uint16_t *>(g.bias);
    a.bias_bf16 = g.bias_type == MxType::BF16;
    a.out_bf16 = g.out_type == MxType::BF16;
    a.M = (int)g.M;
    a.N = (int)g.N;
    a.K = g.K;
    a.wunits = (int)(padded_rows(g.N) >> 5);
    a.w_stride = (int64_t)a.wunits * (g.K >> 6) * kMxUnit;
    a.ws_stride = mx_scale_bytes(a.wunits, g.K);
    a.tiles_n = (int)((g.N + mx::kBN - 1) / mx::kBN);
    a.group_m = 4;
    a.info = g.info;
    a.experts = g.experts;
    a.Y = static_cast<uint16_t *>(g.Y);
    a.ldy = g.ldy;
    a.Oq = g.Oq;
    a.Os = g.Os;
    a.oK = (int)(g.act == MxAct::Swiglu ? g.N / 2 : g.N);
    if (g.info) {
        a.log_units = 3;
        a.xunits = (int)g.units;
        const int64_t most = g.units / 8 + (g.experts < g.units ? g.experts : g.units);
        return mx::launch_out<true>(a, g.act, g.block, (unsigned)(most * a.tiles_n), stream);
    }
    a.xunits = (int)(padded_act_rows(g.M) >> 5);
    a.tiles_m = (int)((g.M + mx::kBM - 1) / mx::kBM);
    return mx::launch_out<false>(a, g.act, g.block, (unsigned)((int64_t)a.tiles_m * a.tiles_n), stream);
}

}  // namespace clq
