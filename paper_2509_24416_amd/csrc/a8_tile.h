// The tile kernel of the 8-bit linears with an epilogue policy (act_epilogue.h): int8 activations times
// int4 or int8 weights on v_mfma_i32_32x32x32_i8, layouts of clq_internal.h.
//
// A workgroup of NW waves computes 32 FN channels x 64 NW tokens, each wave all of the channels x 64 tokens
// (FN x 2 fragments of 32 x 32; FN = 4, or 3 where that fills the chip better).  A k-stage is one 1 KB channel unit a fragment:
// 32 codes of int8 weights (one matrix instruction a fragment) or 64 of int4 ones (two, the codes widened
// right before them).  The channel units are shared by the waves: global -> LDS without registers through a
// ring of NS stages, read back one stage ahead of their use.  The token units belong to one wave each and go
// straight to registers, kDepth stages ahead.  (With both operands through LDS, as in tile_gemm.h, int8
// weights take 576 of its cycles for every 512 of the matrix cores; so 320.)
//
// Ring protocol: stage s waits until stage s + 1 has landed (transfers and loads complete in the order of
// issue, so at most what the three stages before s fetched may be outstanding) and its own LDS reads of
// stage s are in, then the workgroup barrier: every wave holds stage s in registers, so its slot is refilled
// with stage s + NS.  The loop runs over whole groups of kDepth stages, each of which fetches the same
// (past the end the last stage again); the up to three stages behind it fetch nothing, and their waits count
// that.
//
// What bounds it: on long k loops the power limit (43200 x 4608 -> 1152 on int8 weights: 214 us, 2.15 POP/s at 1.7 of
// 2.4 GHz, matrix cores 63% busy at that clock; with gate and residual, 100 MB more, 235).  On short ones loop,
// epilogue and stores add up, at a clock that is held down as well (43200 x 1152 -> 4608 with GELU 279 us, 244 without
// the stores, 185 without the epilogue; 8192 rows 60 us at 2.16 GHz, 1152 tiles on 512 slots).  That the two workgroups
// of a compute unit are in step is not why: a later start of every other one changed nothing, and wave
// priorities (by wave slot or workgroup) made it 0 to 10% slower.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "clq_internal.h"
#include "tile_gemm.h"

namespace clq {
namespace {
namespace a8 {

using tg::Fmt;
using tg::IC;
using tg::static_for;
using tg::v4i;
using tg::v4u;

// (6 and 8 stages ahead took the same time on int8 weights: 43200 x 4608 -> 1152 214 to 216 us)
constexpr int kDepth = 4, kStages = kDepth + 1, kStageBytes = 4096;

// Buffer transfers into LDS, 16 bytes a lane from byte lane_off + off of a buffer: the compiler counts
// them among the loads in flight, where behind a transfer by a global address it waits for all of them
// ahead of every loaded register's use.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const uint8_t *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p), 0, (int)bytes, 0x00027000);
}
__device__ __forceinline__ void dma16(Buffer b, uint32_t lane_off, uint32_t off, uint32_t dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (CLQ_LDS void *)(size_t)dst, 16, (int)lane_off, (int)off, 0, 0);
}

template <int FN>
struct Units {
    v4u w[FN];
    __device__ __forceinline__ void read(uint32_t wa) {
        static_for<0, FN>([&](auto f) { w[f] = tg::read16<decltype(f)::value * 1024>(wa); });
    }
};
// At most VM transfers and loads outstanding, the LDS reads in, the workgroup barrier.
template <int VM>
__device__ __forceinline__ void wait_stage(Units<4> &o) {
    asm volatile("s_waitcnt vmcnt(%c[vm]) lgkmcnt(0)\n\ts_barrier"
                 : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2]), "+v"(o.w[3])
                 : [vm] "n"(VM)
                 : "memory");
}

template <int VM>
__device__ __forceinline__ void wait_stage(Units<3> &o) {
    asm volatile("s_waitcnt vmcnt(%c[vm]) lgkmcnt(0)\n\ts_barrier"
                 : "+v"(o.w[0]), "+v"(o.w[1]), "+v"(o.w[2])
                 : [vm] "n"(VM)
                 : "memory");
}

template <Fmt F, int NW, int FN, class E>
__global__ void __launch_bounds__(NW * 64, 2) a8_tile_kernel(tg::Args a)
{
    static_assert(F == Fmt::W4A8 || F == Fmt::W8A8, "8-bit activations");
    static_assert(NW == 4, "a piece of a stage each");
    constexpr int NS = kStages, PPW = 4 / NW, BN = 32 * FN, BM = 64 * NW;
    constexpr int H = F == Fmt::W4A8 ? 2 : 1;             // matrix instructions a fragment and stage
    constexpr int FETCH = PPW + 2 * H;                    // transfers and loads of a wave and stage
    constexpr int kRing = NS * kStageBytes, kTurn = NW * E::kTurnBytes;
    __shared__ __align__(16) uint8_t pool[kRing > kTurn ? kRing : kTurn];
    __shared__ __align__(16) float ep[E::template kOperands<BN, BM>];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nks = a.K >> (H == 2 ? 6 : 5);              // stages
    int tm, tn;
    tg::tile_coords(a, tg::tile_of_block(), tm, tn);
    const int wunits = (int)(padded_rows(a.N) >> 5), xunits = (int)(padded_act_rows(a.M) >> 5);

    // sources: this wave's channel units, its two token units
    const uint32_t l16 = (uint32_t)lane * 16;
    const uint32_t wbytes = (uint32_t)nks * 1024;         // of a channel unit's row
    Buffer wsrc[PPW];
    static_for<0, PPW>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        const int64_t wu = min(tn * FN + min(wave * PPW + i, FN - 1), wunits - 1);   // (FN = 3: the last twice)
        wsrc[i] = buffer_of(a.Wq + wu * wbytes, wbytes);
    });
    const uint8_t *xsrc[2];
#pragma unroll
    for (int f = 0; f < 2; ++f)
        xsrc[f] = a.Xq + (int64_t)min(tm * 2 * NW + 2 * wave + f, xunits - 1) * (a.K >> 6) * 2048;
    const uint32_t pool0 = tg::lds_addr(pool);
    auto produce = [&](uint32_t slot, int k) __attribute__((always_inline)) {
        const uint32_t off = (uint32_t)min(k, nks - 1) * 1024;
        static_for<0, PPW>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            dma16(wsrc[i], l16, off, pool0 + slot + (uint32_t)(wave * PPW + i) * 1024);
        });
    };
    v4u x[kDepth][2][H];   // token units of stages k .. k + kDepth - 1
    auto load_x = [&](auto dc, int k) __attribute__((always_inline)) {
        const uint32_t off = l16 + (uint32_t)min(k, nks - 1) * (1024 * H);
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int h = 0; h < H; ++h)
                x[decltype(dc)::value][f][h] = *reinterpret_cast<const v4u *>(xsrc[f] + off + h * 1024);
    };

    typename E::template Operands<BN, BM> eo;
    eo.load(a, tm, tn, tid);
    __builtin_amdgcn_sched_barrier(0);

    // prologue: NS stages in flight, stage 0 landed
    Units<FN> op[2];
    const uint32_t wl = pool0 + l16;
    static_for<0, NS>([&](auto qc) {
        constexpr int Q = decltype(qc)::value;
        produce(Q * kStageBytes, Q);
        __builtin_amdgcn_sched_barrier(0);   // (the first wait counts rely on this order)
        if constexpr (Q < kDepth) load_x(qc, Q);
        __builtin_amdgcn_sched_barrier(0);
    });
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NS - 1) * PPW + (kDepth - 1) * 2 * H) : "memory");
    tg::Acc<F> acc[FN][2];
    static_for<0, FN>([&](auto fn) {
        static_for<0, 2>([&](auto fm) { acc[decltype(fn)::value][decltype(fm)::value] = tg::Acc<F>{}; });
    });
    __builtin_amdgcn_sched_barrier(0);
    op[0].read(wl);
    uint32_t cur = 0;
    int k = 0;
    // stage at position P of a group; BEHIND: of those after the loop
    auto stage = [&](auto pc, auto bc) __attribute__((always_inline)) {
        constexpr int P = decltype(pc)::value, R = P & 1;
        constexpr bool BEHIND = decltype(bc)::value;
        wait_stage<BEHIND ? (kDepth - 1 - P) * FETCH : (kDepth - 1) * FETCH>(op[R]);
        const uint32_t nxt = cur == (uint32_t)((NS - 1) * kStageBytes) ? 0u : cur + kStageBytes;
        op[1 - R].read(wl + nxt);
        if constexpr (!BEHIND) produce(cur, k + NS);
        static_for<0, H>([&](auto hc) {
            constexpr int h = decltype(hc)::value;
            static_for<0, FN>([&](auto fc) {
                constexpr int fn = decltype(fc)::value;
                v4i w;
                if constexpr (H == 2) w = tg::widen16(op[R].w[fn][2 * h], op[R].w[fn][2 * h + 1]);
                else w = __builtin_bit_cast(v4i, op[R].w[fn]);
                static_for<0, 2>([&](auto mc) {
                    constexpr int fm = decltype(mc)::value;
                    acc[fn][fm] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, __builtin_bit_cast(v4i, x[P][fm][h]), acc[fn][fm],
                                                                         0, 0, 0);
                });
            });
        });
        if constexpr (!BEHIND) load_x(pc, k + kDepth);
        cur = nxt;
        ++k;
    };
#pragma clang loop unroll(disable)
    for (int groups = nks / kDepth; groups > 0; --groups) static_for<0, kDepth>([&](auto p) { stage(p, std::false_type{}); });
    const int rest = nks % kDepth;
    static_for<0, kDepth - 1>([&](auto p) {
        if (rest > decltype(p)::value) stage(p, std::true_type{});
    });
    // drain: the last transfers, and the last reads, whose data is not used (both register sets are named, so
    // that no register of theirs serves another value meanwhile)
    wait_stage<0>(op[0]);
    wait_stage<0>(op[1]);
    eo.store(a, ep, tid);
    __syncthreads();
    E::template finish_tile<F, FN>(a, acc, pool + wave * E::kTurnBytes, ep, BM, tm, tn, wave, lane);
}

}  // namespace a8
}  // namespace
}  // namespace clq
