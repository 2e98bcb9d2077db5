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

using tg::dma16;
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
__device__ __forceinline__ uint32_t narrow2(float a, float b, bool bf16) {
    if (bf16) {
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
// A workgroup of WM waves computes 128 channels x 64 WM tokens, each wave 128 channels x
// 64 tokens (4 x 2 fragments of 32 x 32).  A k-stage is 64 codes, one matrix
// instruction per fragment.  Units go global -> LDS without registers through a ring of
// NS stages; a wave reads a stage's units back one stage ahead of its use.  The scale
// dwords of four stages (a quad) come the same way through a ring of two, read into
// registers at the end of the quad before.
//
// Ring protocol: iteration s waits until stage s + 1 has landed (transfers complete in
// issue order: at most the later stages' may be outstanding) and its own LDS reads of
// stage s are in, then the workgroup barrier: every wave holds stage s in registers, so
// its slot is refilled with stage s + NS.  Quad q's scale slot is likewise free after
// the barrier of the quad's first iteration and refilled there with quad q + 2, needed
// at the end of quad q + 1.  Transfers past the end repeat the last stage or quad, so
// the wait counts stay constant.
template <int WM_, int NS_>
struct Cfg {
    static constexpr int WM = WM_, NS = NS_, NT = WM * 64, BN = 128, BM = WM * 64;
    static constexpr int UNITS = 4 + 2 * WM, STAGE = UNITS * kMxUnit;
    static constexpr int PPW = UNITS / WM;                 // transfers per wave and stage
    static constexpr int SQ = UNITS * kMxScaleRow;         // scale bytes of a quad
    static constexpr int SPIECES = (UNITS + 3) / 4;        // transfers of four units' scales
    static_assert(UNITS % WM == 0 && UNITS % 4 == 0, "transfers split evenly");
};

struct Operands {
    v4u w[4], x[2];
    __device__ __forceinline__ void read(uint32_t wa, uint32_t xa, int lane) {
        const uint32_t wl = wa + lane * 16, xl = xa + lane * 16;
        static_for<0, 4>([&](auto f) { w[f] = read16<decltype(f)::value * kMxUnit>(wl); });
        static_for<0, 2>([&](auto f) { x[f] = read16<decltype(f)::value * kMxUnit>(xl); });
    }
};
struct Scales {
    uint32_t s[6];   // four channel units, two token units
};
// At most VM transfers outstanding, the LDS reads in, the workgroup barrier.  The
// destinations of those reads are named, so that nothing touches them before; a
// register set whose value is used once, in place, is never copied while a read of it
// is in flight (hence two sets of scales, too: a copy from one into the other was moved
// ahead of this wait).
#define CLQ_MX_WAIT "s_waitcnt vmcnt(%c[vm]) lgkmcnt(0)\n\ts_barrier"
template <int VM>
__device__ __forceinline__ void wait_stage(Operands &o) {
    asm volatile(CLQ_MX_WAIT
                 : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]), "+v"(o.w[3]), "+v"(o.x[0]), "+v"(o.x[1])
                 : [vm] "n"(VM)
                 : "memory");
}
template <int VM>
__device__ __forceinline__ void wait_stage(Operands &o, Scales &s) {
    asm volatile(CLQ_MX_WAIT
                 : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]), "+v"(o.w[3]), "+v"(o.x[0]), "+v"(o.x[1]), "+v"(s.s[0]),
                   "+v"(s.s[1]), "+v"(s.s[2]), "+v"(s.s[3]), "+v"(s.s[4]), "+v"(s.s[5])
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

// Stores the plain outputs of a fragment: the lane's 16 channels n0 .. of row m.
template <bool RAGGED>
__device__ __forceinline__ void store_plain(const Args &a, const v16f &x, const float *bias, int64_t m, int n0) {
    uint32_t h[8];
#pragma unroll
    for (int v = 0; v < 16; v += 2) h[v / 2] = narrow2(x[v] + bias[v], x[v + 1] + bias[v + 1], a.out_bf16);
    uint16_t *dst = a.Y + m * a.ldy + n0;
    if (!RAGGED || n0 <= a.N - 16) {
        reinterpret_cast<v4u *>(dst)[0] = v4u{h[0], h[1], h[2], h[3]};
        reinterpret_cast<v4u *>(dst)[1] = v4u{h[4], h[5], h[6], h[7]};
    } else {
#pragma unroll
        for (int v = 0; v < 16; ++v)
            if (n0 + v < a.N) dst[v] = (uint16_t)(h[v >> 1] >> (16 * (v & 1)));
    }
}

// Rotates and quantizes NF fragments of one 32-row unit: f[i][v] is channel
// 32 i + 16 (lane / 32) + v (of the output) of row lane % 32.  Stage h = 16 pairs
// the lane halves, 32 and 64 the fragments.  Writes the chunks c0 .. c0 + NF - 1 of unit u.
template <int B, int NF>
__device__ __forceinline__ void requantize(const Args &a, float (&f)[NF][16], int lane, int64_t u, int c0) {
    const int h = lane >> 5, row = lane & 31, oK = a.oK;
    if constexpr (B >= 32) {
        const float sg = h ? -1.0f : 1.0f;
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
            for (int v = 0; v < 16; ++v) {
                const uint32_t b = __float_as_uint(f[i][v]);
                const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
                // lower half's value + or - upper half's (the product with 1 is exact)
                f[i][v] = __builtin_fmaf(__uint_as_float(r[1]), sg, __uint_as_float(r[0]));
            }
        }
        if constexpr (B >= 64) {
            static_assert(B < 64 || NF >= 2, "fragments of a rotation block");
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
        float m = 0.0f;
#pragma unroll
        for (int v = 0; v < 16; ++v) m = __builtin_elementwise_maximum(m, fabsf(f[i][v]));
        const uint32_t b = __float_as_uint(m);
        const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        m = __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
        byte[i] = mx_scale_byte(__float_as_uint(m) & 0x7fffffffu, 0);
        const float s = mx_scale_value(byte[i], 0);
        codes[i] = v2u{mx_pack8(f[i], s), mx_pack8(f[i] + 8, s)};
    }
    // a chunk's two halves meet: lanes 0..31 take the even chunk of a pair, 32..63 the odd
#pragma unroll
    for (int i = 0; i < NF; i += 2) {
        if constexpr (NF >= 2) {
            const auto lo = __builtin_amdgcn_permlane32_swap(codes[i][0], codes[i + 1][0], false, false);
            const auto hi = __builtin_amdgcn_permlane32_swap(codes[i][1], codes[i + 1][1], false, false);
            // lower lanes: own and the upper lanes' chunk i; upper: the lower lanes' and own chunk i + 1
            const int c = c0 + i + h;
            if (32 * c < oK) {
                *reinterpret_cast<v4u *>(a.Oq + mx_code_offset(u, row, c, oK)) = v4u{lo[0], hi[0], lo[1], hi[1]};
                a.Os[mx_scale_offset(u, row, c, oK)] = (uint8_t)(h ? byte[i + 1] : byte[i]);
            }
        }
    }
}

template <class C, Out OUT, int B, bool GROUPED, bool RAGGED>
__global__ void __launch_bounds__(C::NT, 2) mx_tile_kernel(Args a)
{
    constexpr int NS = C::NS;
    constexpr bool GATED = OUT == Out::Swiglu;
    __shared__ __align__(16) uint8_t pool[NS * C::STAGE + 2 * C::SQ];
    __shared__ float ep[C::BN];   // biases
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
        rt.unit0 = tm * (C::BM / 32);
        rt.unit_end = a.xunits;
        rt.expert = 0;
    }
    const uint8_t *Wq = a.Wq + rt.expert * a.w_stride, *Ws = a.Ws + rt.expert * a.ws_stride;

    // ---- producer --------------------------------------------------------------------
    const uint32_t l16 = (uint32_t)lane * 16;
    const uint8_t *src[C::PPW];
    uint32_t dsto[C::PPW];
    static_for<0, C::PPW>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        const int p = wave * C::PPW + i;   // channel units first
        src[i] = p < 4 ? Wq + (int64_t)min(tn * 4 + p, a.wunits - 1) * nks * kMxUnit
                       : a.Xq + (int64_t)min(rt.unit0 + p - 4, rt.unit_end - 1) * nks * kMxUnit;
        dsto[i] = (uint32_t)(p * kMxUnit);
    });
    // scales: a transfer brings the 256 bytes of four units; waves past the last piece
    // repeat it
    const int sp = min(wave, C::SPIECES - 1), su = sp * 4 + (lane >> 4);
    const uint8_t *ssrc = (su < 4 ? Ws + (int64_t)min(tn * 4 + su, a.wunits - 1) * nq * kMxScaleRow
                                  : a.Xs + (int64_t)min(rt.unit0 + su - 4, rt.unit_end - 1) * nq * kMxScaleRow) +
                          (lane & 15) * 16;
    const uint32_t pool0 = lds_addr(pool), spool = pool0 + NS * C::STAGE;
    auto produce = [&](uint32_t slot, int k) __attribute__((always_inline)) {
        const uint32_t off = l16 + (uint32_t)min(k, nks - 1) * kMxUnit;
        static_for<0, C::PPW>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            const uint8_t *s = src[i] + off;
            dma16(s, pool0 + slot + dsto[i]);
        });
    };
    auto produce_scales = [&](uint32_t slot, int q) __attribute__((always_inline)) {
        const uint8_t *s = ssrc + (uint32_t)min(q, nq - 1) * kMxScaleRow;
        dma16(s, spool + slot + (uint32_t)sp * 1024);
    };

    // the tile's biases, in registers until the ring is done with
    float bv = 0.0f;
    if (a.bias && tid < C::BN) {
        const int n = min(tn * C::BN + tid, a.N - 1);
        bv = widen(a.bias[(int64_t)rt.expert * a.N + bias_index(n, a.N, GATED)], a.bias_bf16);
    }
    __builtin_amdgcn_sched_barrier(0);

    // ---- consumer --------------------------------------------------------------------
    Operands op[2];
    Scales sc[2];   // of even and odd quads
    const uint32_t xo = (uint32_t)((4 + 2 * wave) * kMxUnit);
    auto read_stage = [&](uint32_t slot, auto pc) __attribute__((always_inline)) {
        op[decltype(pc)::value].read(pool0 + slot, pool0 + slot + xo, lane);
    };
    const uint32_t sw = spool + (uint32_t)lane * 4, sx = sw + (uint32_t)(4 + 2 * wave) * kMxScaleRow;
    auto read_scales = [&](auto qc) __attribute__((always_inline)) {
        constexpr int Q = decltype(qc)::value;
        static_for<0, 4>([&](auto f) { sc[Q].s[f] = read4<Q * C::SQ + decltype(f)::value * kMxScaleRow>(sw); });
        static_for<0, 2>([&](auto f) {
            sc[Q].s[4 + decltype(f)::value] = read4<Q * C::SQ + decltype(f)::value * kMxScaleRow>(sx);
        });
    };
    v16f acc[4][2];
    static_for<0, 4>([&](auto i) { static_for<0, 2>([&](auto j) { acc[decltype(i)::value][decltype(j)::value] = v16f{}; }); });

    // prologue: two quads of scales and NS stages in flight, stage 0 and quad 0 landed
    produce_scales(0, 0);
    produce_scales(C::SQ, 1);
    static_for<0, NS>([&](auto qc) { produce(decltype(qc)::value * C::STAGE, decltype(qc)::value); });
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 1) * C::PPW) : "memory");
    read_stage(0, IC<0>{});
    read_scales(IC<0>{});
    uint32_t cur = 0;
    int k = 0, q = 2;
    // position P of the eight stages of an even and an odd quad
    auto stage = [&](auto pc) __attribute__((always_inline)) {
        constexpr int P8 = decltype(pc)::value, P = P8 & 3, Q = P8 >> 2, R = P & 1;
        // outstanding: the last NS - 2 stages, and the scale transfer if a quad began among them
        constexpr int VM = (NS - 2) * C::PPW + (P >= 1 && P <= NS - 2 ? 1 : 0);
        if constexpr (P == 0) wait_stage<VM>(op[R], sc[Q]);
        else wait_stage<VM>(op[R]);
        const uint32_t nxt = cur == (uint32_t)((NS - 1) * C::STAGE) ? 0u : cur + C::STAGE;
        read_stage(nxt, IC<1 - R>{});
        if constexpr (P == 3) read_scales(IC<1 - Q>{});
        produce(cur, k + NS);
        if constexpr (P == 0) produce_scales(Q * C::SQ, q++);
        static_for<0, 4>([&](auto fc) {
            static_for<0, 2>([&](auto mc) {
                constexpr int fn = decltype(fc)::value, fm = decltype(mc)::value;
                acc[fn][fm] = mfma_mx4<P>(op[R].w[fn], op[R].x[fm], acc[fn][fm], sc[Q].s[fn], sc[Q].s[4 + fm]);
            });
        });
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
    if (tid < C::BN) ep[tid] = bv;
    __syncthreads();

    // ---- epilogue: lane owns row m and 16 consecutive channels of each fragment ---------
    const int h16 = (lane >> 5) * 16;
    static_for<0, 2>([&](auto mc) {
        constexpr int fm = decltype(mc)::value;
        const int u = rt.unit0 + wave * 2 + fm;
        if (u >= rt.unit_end) return;
        if constexpr (OUT == Out::Plain) {
            const int64_t m = (int64_t)u * 32 + (lane & 31);
            static_for<0, 4>([&](auto fc) {
                constexpr int fn = decltype(fc)::value;
                const int c = fn * 32 + h16, n0 = tn * C::BN + c;
                if ((GROUPED || m < a.M) && n0 < a.N) store_plain<RAGGED>(a, acc[fn][fm], ep + c, m, n0);
            });
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

template <class C, Out OUT, int B, bool GROUPED>
void launch_kernel(const Args &a, unsigned grid, hipStream_t stream) {
    const dim3 g(grid), b(C::NT);
    if constexpr (OUT == Out::Plain) {
        if (a.N % 16 != 0) {
            hipLaunchKernelGGL((mx_tile_kernel<C, OUT, B, GROUPED, true>), g, b, 0, stream, a);
            return;
        }
    }
    hipLaunchKernelGGL((mx_tile_kernel<C, OUT, B, GROUPED, false>), g, b, 0, stream, a);
}

template <class C, bool GROUPED>
hipError_t launch_out(Args &a, MxAct act, int block, unsigned grid, hipStream_t stream) {
    if (a.Y) {
        launch_kernel<C, Out::Plain, 0, GROUPED>(a, grid, stream);
    } else {
        auto by_block = [&](auto oc) {
            constexpr Out OUT = decltype(oc)::value;
            switch (block) {
                case 0: launch_kernel<C, OUT, 0, GROUPED>(a, grid, stream); break;
                case 32: launch_kernel<C, OUT, 32, GROUPED>(a, grid, stream); break;
                case 64: launch_kernel<C, OUT, 64, GROUPED>(a, grid, stream); break;
                default:
                    if constexpr (OUT != Out::Swiglu) launch_kernel<C, OUT, 128, GROUPED>(a, grid, stream);
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
    using C = mx::Cfg<4, 5>;
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
    a.tiles_n = (int)((g.N + C::BN - 1) / C::BN);
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
        return mx::launch_out<C, true>(a, g.act, g.block, (unsigned)(most * a.tiles_n), stream);
    }
    a.xunits = (int)(padded_act_rows(g.M) >> 5);
    a.tiles_m = (int)((g.M + C::BM - 1) / C::BM);
    return mx::launch_out<C, false>(a, g.act, g.block, (unsigned)((int64_t)a.tiles_m * a.tiles_n), stream);
}

}  // namespace clq
