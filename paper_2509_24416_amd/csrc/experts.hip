// Expert layer around the MX4 products: routing of tokens to experts, the plan that
// sorts them by expert, and the weighted sum of the experts' outputs.
//
// Routing.  score = softmax or sigmoid of the token's logits; the experts are ranked by
// score + bias (by the logits themselves where there is neither a bias nor groups:
// the scores keep their order, and far from 0 round to one value).  With G groups a
// group counts the sum of its two best ranks and only the experts of the best
// top_groups groups take part.  The k best experts, ties to the lower index, carry
// their scores (without the bias), divided by their sum if so asked, times a factor.
//
// Plan.  The assignments (token, slot) are sorted by expert, stable in their order;
// every expert's rows start on a multiple of 32, the row unit of the products, so that
// a grouped product is the dense one on a run of units.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "clq_internal.h"
#include "mx4.h"

namespace clq {
namespace {

// ---- routing ---------------------------------------------------------------------------
// LPT lanes per token, 64 or 32.  Lane l holds the VPL consecutive experts from l * VPL, so that
// among equal ranks the lowest lane's first one is the lowest index.  Ranks are compared as
// whole numbers in the floats' order, 0 for an expert that cannot be chosen.  A lane sorts
// its own experts once, in lists of up to four; each of the top_k rounds then is a maximum over the
// token's lanes of their heads (four to six lane permutes) and a pop.  What bounds it are these
// vector instructions, some 450 a token at 256 experts: 43200 tokens to 8 of them in 4 of 8 groups
// take 40 us, reading the logits 9 (one LDS read after another by a lane a group, and shuffles
// instead of permutes: 89).
constexpr int kRouteWaves = 4, kRouteMost = 32;   // waves of a workgroup, experts of a token

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false));
}
// largest value of the token's LPT lanes, in all of them
template <int LPT>
__device__ __forceinline__ uint32_t token_max(uint32_t v) {
    if constexpr (LPT == 64) {
        v = dpp_max<0x111>(v);        // row_shr 1, 2, 4, 8
        v = dpp_max<0x112>(v);
        v = dpp_max<0x114>(v);
        v = dpp_max<0x118>(v);
        v = dpp_max<0x142, 0xa>(v);   // row_bcast 15 into rows 1 and 3
        v = dpp_max<0x143, 0xc>(v);   // row_bcast 31 into rows 2 and 3
        return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
    } else {
        static_assert(LPT == 32);
        v = dpp_max<0xb1>(v);         // quad_perm 1 0 3 2, 2 3 0 1
        v = dpp_max<0x4e>(v);
        v = dpp_max<0x141>(v);        // row_half_mirror, row_mirror
        v = dpp_max<0x140>(v);
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);   // the other row of the pair
        return max((uint32_t)r[0], (uint32_t)r[1]);
    }
}
// the token's lanes of a wave mask, lowest bit first
template <int LPT>
__device__ __forceinline__ uint64_t token_mask(uint64_t m, bool upper) {
    if constexpr (LPT == 64) return m;
    else return upper ? (uint32_t)(m >> 32) : (uint32_t)m;
}
// whether this is the token's lowest lane of a wave mask
template <int LPT>
__device__ __forceinline__ bool first_lane(uint64_t m) {
    if constexpr (LPT == 64) return __builtin_amdgcn_inverse_ballot_w64(m & -m);
    const uint32_t lo = (uint32_t)m, hi = (uint32_t)(m >> 32);
    return __builtin_amdgcn_inverse_ballot_w64((uint64_t)(hi & -hi) << 32 | (lo & -lo));
}
// lane i of the token's lanes (i the same in all)
template <int LPT>
__device__ __forceinline__ uint32_t token_lane(uint32_t v, int i, bool upper) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)v, i);
    if constexpr (LPT == 64) return lo;
    else return upper ? (uint32_t)__builtin_amdgcn_readlane((int)v, 32 + i) : lo;
}
// floats (no NaN) as whole numbers of the same order, all above 0; equal zeros
__device__ __forceinline__ uint32_t order_of(float f) {
    const uint32_t b = __float_as_uint(f + 0.0f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float float_of(uint32_t o) {
    return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}

struct RouteArgs {
    const void *logits;
    MxType type;
    int64_t ld, T;
    int E, k, groups, top_groups;
    bool sigmoid, renormalize;
    const float *bias;
    float scale;
    int32_t *ids;
    float *weights;
};

template <int VPL>
__device__ __forceinline__ void load_logits(const RouteArgs &a, int64_t t, int lane, float (&x)[VPL]) {
    const int e0 = lane * VPL;
    if (a.type == MxType::F32) {
        const float *p = static_cast<const float *>(a.logits) + t * a.ld;
        if constexpr (VPL % 4 == 0) {
            if (a.E % 4 == 0 && a.ld % 4 == 0 && (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0) {
#pragma unroll
                for (int v = 0; v < VPL; v += 4) {
                    float4 q = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                    if (e0 + v < a.E) q = *reinterpret_cast<const float4 *>(p + e0 + v);
                    x[v] = q.x; x[v + 1] = q.y; x[v + 2] = q.z; x[v + 3] = q.w;
                }
                return;
            }
        }
#pragma unroll
        for (int v = 0; v < VPL; ++v) x[v] = e0 + v < a.E ? p[e0 + v] : -INFINITY;
    } else {
        const uint16_t *p = static_cast<const uint16_t *>(a.logits) + t * a.ld;
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const uint16_t h = e0 + v < a.E ? p[e0 + v] : 0;
            const float f = a.type == MxType::BF16 ? __uint_as_float((uint32_t)h << 16) : __half2float(__ushort_as_half(h));
            x[v] = e0 + v < a.E ? f : -INFINITY;
        }
    }
}

template <int VPL, int LPT>
__global__ void __launch_bounds__(64 * kRouteWaves) route_kernel(RouteArgs a)
{
    constexpr int TPW = 64 / LPT;   // tokens of a wave
    // lists of a lane's experts, each sorted
    constexpr int NL = VPL > 4 ? VPL / 4 : 1, LEN = VPL / NL;
    __shared__ __align__(16) float sh_score[kRouteWaves][TPW][VPL * LPT];
    __shared__ __align__(16) uint32_t sh_rank[kRouteWaves][TPW][VPL * LPT];
    __shared__ int sh_id[kRouteWaves][TPW][kRouteMost];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & (LPT - 1), token = (threadIdx.x & 63) / LPT;
    const bool upper = token != 0;
    constexpr float kNone = -INFINITY;
    float *scores = sh_score[wave][token];
    int *chosen = sh_id[wave][token];
    // lanes of a group: the largest power of two that gives every group as many
    int per_group = LPT;
    while (per_group * a.groups > LPT) per_group >>= 1;
    const bool by_logit = a.bias == nullptr && a.groups == 1;
    float balance[VPL];
#pragma unroll
    for (int v = 0; v < VPL; ++v) balance[v] = a.bias && lane * VPL + v < a.E ? a.bias[lane * VPL + v] : 0.0f;
    // (whole waves: the upper half of the last one may repeat the last token)
    const int64_t step = (int64_t)gridDim.x * kRouteWaves * TPW;
    int64_t t0 = ((int64_t)blockIdx.x * kRouteWaves + wave) * TPW;
    float next[VPL];
    if (t0 < a.T) load_logits<VPL>(a, min(t0 + token, a.T - 1), lane, next);
    for (; t0 < a.T; t0 += step) {
        const int64_t t = t0 + token;
        float x[VPL], score[VPL];
#pragma unroll
        for (int v = 0; v < VPL; ++v) x[v] = next[v];
        if (t0 + step < a.T) load_logits<VPL>(a, min(t + step, a.T - 1), lane, next);
        bool nan = false;
#pragma unroll
        for (int v = 0; v < VPL; ++v) nan |= x[v] != x[v];
        nan = token_mask<LPT>(__ballot(nan), upper) != 0;   // leaves the token's weights NaN; NaN ranks come last
        if (a.sigmoid) {
#pragma unroll
            for (int v = 0; v < VPL; ++v) score[v] = 1.0f / (1.0f + expf(-x[v]));
        } else {
            uint32_t mo = 0;
#pragma unroll
            for (int v = 0; v < VPL; ++v) mo = max(mo, x[v] == x[v] ? order_of(x[v]) : 0u);
            const float m = float_of(max(token_max<LPT>(mo), order_of(kNone)));
            // (the sum in 64 bits, so that the rounded sum does not depend on the order)
            double s = 0.0;
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
                score[v] = m == kNone ? 0.0f : expf(x[v] - m);
                s += (double)score[v];   // (0 past the last expert)
            }
#pragma unroll
            for (int o = LPT / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
            const float sum = m == kNone ? 1.0f : (float)s;
#pragma unroll
            for (int v = 0; v < VPL; ++v) score[v] = score[v] / sum;
        }
        uint32_t key[VPL];
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const int e = lane * VPL + v;
            const bool in = e < a.E;
            float r = by_logit ? x[v] : score[v];
            if (a.bias) r = score[v] + balance[v];
            key[v] = in ? order_of(r == r ? r : kNone) : 0u;
        }
#pragma unroll
        for (int v = 0; v < VPL; ++v) scores[lane * VPL + v] = score[v];
        if (a.groups > 1) {
            uint32_t *ranks = sh_rank[wave][token];
#pragma unroll
            for (int v = 0; v < VPL; ++v) ranks[lane * VPL + v] = key[v];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            // the two best of a group over its lanes
            const int gs = a.E / a.groups, g = lane / per_group, first = lane & (per_group - 1);
            uint32_t b0 = 0, b1 = 0;
            if (g < a.groups)
                for (int i = first; i < gs; i += per_group) {
                    const uint32_t r = ranks[g * gs + i];
                    b1 = max(b1, min(b0, r));
                    b0 = max(b0, r);
                }
            for (int o = 1; o < per_group; o <<= 1) {
                const uint32_t o0 = __shfl_xor(b0, o), o1 = __shfl_xor(b1, o);
                b1 = max(min(b0, o0), max(b1, o1));
                b0 = max(b0, o0);
            }
            float best = gs > 1 ? float_of(b0) + float_of(b1) : float_of(b0);
            if (best != best) best = kNone;   // (biases of both infinities)
            const uint32_t bo = g < a.groups ? order_of(best) : 0u;
            // a group is kept if fewer than top_groups groups come before it
            int before = 0;
            for (int o = 0; o < a.groups; ++o) {
                const uint32_t other = token_lane<LPT>(bo, o * per_group, upper);
                before += other > bo || (other == bo && o < g);
            }
            const uint64_t kept = token_mask<LPT>(__ballot(g < a.groups && before < a.top_groups), upper);
#pragma unroll
            for (int v = 0; v < VPL; ++v) {
                const int e = min(lane * VPL + v, a.E - 1);
                key[v] = (kept >> (e / gs * per_group)) & 1 ? key[v] : 0u;
            }
        }
        // each list best first (an equal one stays behind: its index is higher); the places of its
        // experts, four bits each, go along
        uint32_t order[NL];
#pragma unroll
        for (int n = 0; n < NL; ++n) {
            uint32_t *list = key + n * LEN, place[LEN];
#pragma unroll
            for (int v = 0; v < LEN; ++v) place[v] = (uint32_t)(n * LEN + v);
#pragma unroll
            for (int i = 1; i < LEN; ++i)
#pragma unroll
                for (int j = i; j > 0; --j) {
                    const bool swap = list[j] > list[j - 1];
                    const uint32_t hi = list[j - 1], lo = list[j], p = place[j - 1], q = place[j];
                    list[j - 1] = swap ? lo : hi;
                    list[j] = swap ? hi : lo;
                    place[j - 1] = swap ? q : p;
                    place[j] = swap ? p : q;
                }
            order[n] = 0;
#pragma unroll
            for (int v = 0; v < LEN; ++v) order[n] |= place[v] << (4 * v);
        }
        for (int j = 0; j < a.k; ++j) {
            uint32_t head = key[0], at = order[0];
            if constexpr (NL == 2) {
                at = key[LEN] > head ? order[1] : at;
                head = max(head, key[LEN]);
            }
            const uint32_t top = token_max<LPT>(head);
            const bool won = first_lane<LPT>(__ballot(head == top));
            if (won) chosen[j] = lane * VPL + (int)(at & 15);
            // the winner's list moves up (of two equal heads the first one's)
            const uint32_t in_first = key[0] == top ? ~0u : 0u, mask = won ? ~0u : 0u;
#pragma unroll
            for (int n = 0; n < NL; ++n) {
                uint32_t *list = key + n * LEN;
                const uint32_t pop = NL == 1 ? mask : n == 0 ? mask & in_first : mask & ~in_first;
#pragma unroll
                for (int v = 0; v + 1 < LEN; ++v) list[v] = (list[v + 1] & pop) | (list[v] & ~pop);
                list[LEN - 1] &= ~pop;
                order[n] = ((order[n] >> 4) & pop) | (order[n] & ~pop);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int my_id = lane < a.k ? chosen[lane] : 0;
        float w = lane < a.k ? scores[my_id] : 0.0f;
        if (a.renormalize) {
            float total = w;
            for (int o = 1; o < a.k; o <<= 1) total += __shfl_xor(total, o);   // (0 past the k-th lane)
            // (a total of 0, where every score is, leaves weights of 0)
            w = total > 0.0f ? w / total : total == 0.0f ? 0.0f : total;
        }
        w *= a.scale;
        if (nan) w = __uint_as_float(0x7fc00000u);
        if (lane < a.k && t < a.T) {
            a.ids[t * a.k + lane] = my_id;
            a.weights[t * a.k + lane] = w;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Two tokens share a wave where there are enough to fill the chip all the same: the rounds cost
// both of them what they cost one.  us of one / two tokens a wave: 64 experts, 6 of them, 1 token
// 2.9 / 3.2, 4096 4.4 / 4.1, 43200 19.2 / 14.8; 128 experts, 8, 4096 tokens 5.2 / 4.9, 8192 7.4 / 6.6;
// 256 experts, 8, in 4 of 8 groups, 4096 tokens 7.4 / 8.4, 20000 22.6 / 24.6, 24576 27.0 / 25.6, 43200
// 44.4 / 39.8, 100000 91 / 78.
inline bool route_shared(int64_t T, int E, int groups) {
    return groups <= 32 && E <= 256 && T >= (E <= 128 ? 4096 : 24576);
}

template <int VPL, int LPT>
void launch_route(const RouteArgs &a, hipStream_t stream) {
    // as many waves as the chip holds, each with every so-many-th token
    const int64_t tokens = kRouteWaves * (64 / LPT), want = (a.T + tokens - 1) / tokens, most = (int64_t)compute_units() * 8;
    hipLaunchKernelGGL((route_kernel<VPL, LPT>), dim3((unsigned)(want < most ? want : most)), dim3(64 * kRouteWaves), 0,
                       stream, a);
}

// ---- plan ---------------------------------------------------------------------------------
// A stable counting sort.  A block owns a run of 1024 PER assignments; the first kernel
// counts its experts, the second adds the counts of the runs before (every block for
// itself: they are a few hundred rows of E counts), and places its own.  One run is a single
// launch; past it two are quicker than every block counting all assignments (24576 to 64
// experts, 4 a thread: 4.8 + 6.9 us against 15.6).  Latency bounds it.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

template <int PER>
__global__ void __launch_bounds__(kPlanThreads) plan_count_kernel(const int32_t *ids, int64_t n, int E, int32_t *hist)
{
    extern __shared__ int32_t count[];
    for (int e = threadIdx.x; e < E; e += kPlanThreads) count[e] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * (kPlanThreads * PER);
    for (int j = 0; j < PER; ++j) {
        const int64_t i = i0 + j * kPlanThreads + threadIdx.x;
        if (i < n) {
            const int id = ids[i];
            if (id >= 0 && id < E) atomicAdd(&count[id], 1);   // (whole numbers: any order)
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kPlanThreads) hist[(int64_t)blockIdx.x * E + e] = count[e];
}

// hist: counts of every run (nullptr: there is one run, counted here)
template <int PER>
__global__ void __launch_bounds__(kPlanThreads) plan_place_kernel(const int32_t *ids, int64_t n, int k, int E, int runs,
                                                                  const int32_t *hist, int32_t *info, int32_t *rows,
                                                                  int32_t *source)
{
    extern __shared__ int32_t sm[];
    int32_t *wcount = sm;                    // [waves][E]: then the wave's next row of each expert
    int32_t *all = wcount + kPlanWaves * E;  // [E] counts over all runs
    int32_t *first = all + E;                // [E + 1] first row unit
    int32_t *prior = first + E + 1;          // [E] counts of the runs before
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool lead = blockIdx.x == 0;
    for (int i = tid; i < kPlanWaves * E; i += kPlanThreads) wcount[i] = 0;
    for (int i = tid; i < E; i += kPlanThreads) all[i] = prior[i] = 0;
    __syncthreads();
    // a wave owns 64 * PER consecutive assignments
    const int64_t i0 = (int64_t)blockIdx.x * (kPlanThreads * PER) + wave * 64 * PER;
    int id[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int64_t i = i0 + j * 64 + lane;
        id[j] = i < n ? ids[i] : -1;
        if (id[j] < 0 || id[j] >= E) id[j] = -1;
        if (id[j] >= 0) atomicAdd(&wcount[wave * E + id[j]], 1);
    }
    if (hist)
        // whole rows of counts at a time, summed in registers
        for (int e0 = 0; e0 < E; e0 += kPlanThreads) {
            const int width = min(E - e0, kPlanThreads), lines = kPlanThreads / width;
            const int line = tid / width, e = e0 + tid - line * width;
            if (line < lines) {
                int sum = 0, before = 0;
#pragma unroll 8
                for (int r = line; r < runs; r += lines) {
                    const int c = hist[(int64_t)r * E + e];
                    sum += c;
                    before += r < (int)blockIdx.x ? c : 0;
                }
                atomicAdd(&all[e], sum);
                atomicAdd(&prior[e], before);
            }
        }
    __syncthreads();
    // per expert: the waves' first ranks
    for (int e = tid; e < E; e += kPlanThreads) {
        int sum = prior[e];
        for (int w = 0; w < kPlanWaves; ++w) {
            const int c = wcount[w * E + e];
            wcount[w * E + e] = sum;
            sum += c;
        }
        if (!hist) all[e] = sum;
    }
    __syncthreads();
    // per expert: first row units and, for the products, first tiles of 4 and 8 units
    if (wave < kPlanTables) {
        const int log_units = plan_log_units(wave);
        int32_t *table = info + plan_table_offset(E, log_units);
        int run = 0;
        for (int e0 = 0; e0 < E; e0 += 64) {
            const int e = e0 + lane;
            const int units = e < E ? (all[e] + 31) >> 5 : 0;
            const int v = (units + (1 << log_units) - 1) >> log_units;
            int s = v;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int t = __shfl_up(s, o);
                if (lane >= o) s += t;
            }
            if (e < E) {
                if (lead) table[e] = run + s - v;
                if (wave == 0) first[e] = run + s - v;
            }
            run += __shfl(s, 63);
        }
        if (lane == 0) {
            if (lead) table[E] = run;
            if (wave == 0) first[E] = run;
        }
    }
    if (lead)
        for (int e = tid; e < E; e += kPlanThreads) info[e] = all[e];
    __syncthreads();
    // place: 64 assignments at a time, in order
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int64_t i = i0 + j * 64 + lane;
        // lanes with the same expert
        uint64_t same = __ballot(id[j] >= 0);
        for (int b = 0; (1 << b) < E; ++b) {
            const bool bit = id[j] >= 0 && (id[j] >> b & 1);
            const uint64_t m = __ballot(bit);
            same &= bit ? m : ~m;
        }
        int row = -1;
        if (id[j] >= 0) {
            const int rank = __popcll(same & ((1ull << lane) - 1));
            const int base = wcount[wave * E + id[j]];
            row = first[id[j]] * 32 + base + rank;
            source[row] = (int)(i / k);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        // the lowest lane of each expert moves its count on
        if (id[j] >= 0 && (same & ((1ull << lane) - 1)) == 0) wcount[wave * E + id[j]] += __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (i < n) rows[i] = row;
    }
    // rows that pad an expert's last unit have no source
    if (lead)
        for (int i = tid; i < E * 32; i += kPlanThreads) {
            const int e = i >> 5, r = first[e] * 32 + all[e] + (i & 31);
            if (r < first[e + 1] * 32) source[r] = -1;
        }
}

// Assignments of a thread.  Short runs fill more of the chip, until there is more than one a
// compute unit or the counts of all runs, which every block reads, take longer.  us with 1 / 2 / 4
// (both launches): 4096 x 6 to 64 experts 6.4 / 7.4 / 9.2; 8192 x 8 to 256, 64 / 32 / 16 runs,
// 9.6 / 10.0 / 12.5; 10800 x 8, 85 / 43 / 22, 11.5 / 10.7 / 12.9; 43200 x 8, 338 / 169 / 85, 22.6 /
// 14.2 / 14.7; 100000 x 8 to 64, 782 / 391 / 196, 25.8 / 14.5 / 13.0, to 512, 114 / 42.7 / 25.7.  One
// run, a single launch, where there can be one: 512 x 2 to 16 3.4 / 3.7 / 4.7.
inline int64_t plan_runs(int64_t n, int per) { return (n + kPlanThreads * per - 1) / (kPlanThreads * per); }
// the most runs that there are of `per` assignments a thread (no limit for 4)
inline int64_t plan_most(int per, int64_t E) {
    const int64_t counts = (per == 1 ? 16384 : 49152) / E;
    return counts < 256 ? counts : 256;
}
inline int plan_per(int64_t n, int64_t E) {
    const bool single = plan_runs(n, 4) == 1;
    for (int per = 1; per < 4; per *= 2)
        if (plan_runs(n, per) <= (single ? 1 : plan_most(per, E))) return per;
    return 4;
}

template <int PER>
hipError_t launch_plan(const int32_t *ids, int64_t n, int k, int E, int32_t *info, int32_t *rows, int32_t *source,
                       void *workspace, hipStream_t stream) {
    const int runs = (int)plan_runs(n, PER);
    int32_t *hist = runs > 1 ? static_cast<int32_t *>(workspace) : nullptr;
    if (hist) {
        hipLaunchKernelGGL((plan_count_kernel<PER>), dim3((unsigned)runs), dim3(kPlanThreads), E * sizeof(int32_t), stream,
                           ids, n, E, hist);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const size_t lds = ((size_t)(kPlanWaves + 3) * E + 1) * sizeof(int32_t);
    hipLaunchKernelGGL((plan_place_kernel<PER>), dim3((unsigned)runs), dim3(kPlanThreads), lds, stream, ids, n, k, E, runs,
                       hist, info, rows, source);
    return hipGetLastError();
}

// ---- combination ------------------------------------------------------------------------------
// out[t] = sum over the slots, in order and in fp32, of weight * Y[row]; a slot without
// a row adds nothing.  W columns per thread; the rows and weights of four slots are read
// ahead of their values, whose loads are then in flight together.  Bound by memory (43200 x 1152 of
// two slots, fp16: 51 us, 5.9 TB/s with the memory-side cache; fp32 values: 88 us, 5.6 TB/s).
struct CombineArgs {
    const void *Y;
    const int32_t *rows;
    const float *weights;
    void *out;
    int64_t ldy, ldo, plan_rows;
    int64_t first;         // token of the launch's first thread
    int tokens, k, per;    // per: pieces of W columns in a row
};
// (W consecutive values)
template <class T, int W>
struct __align__(W * sizeof(T) < 16 ? W * sizeof(T) : 16) Piece {
    T v[W];
};

template <class TI, class TO, int W>
__global__ void __launch_bounds__(256) combine_kernel(CombineArgs a)
{
    const unsigned i = blockIdx.x * 256 + threadIdx.x, tl = i / (unsigned)a.per;
    if (tl >= (unsigned)a.tokens) return;
    const int64_t t = a.first + tl;
    const int c = (int)(i - tl * a.per) * W;
    const TI *Y = static_cast<const TI *>(a.Y) + c;
    const int32_t *rows = a.rows + t * a.k;
    const float *weights = a.weights + t * a.k;
    float s[W] = {};
    for (int j = 0; j < a.k; j += 4) {
        int r[4];
        float w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            r[q] = j + q < a.k ? rows[j + q] : -1;
            w[q] = j + q < a.k ? weights[j + q] : 0.0f;
            if (r[q] >= a.plan_rows) r[q] = -1;
        }
        Piece<TI, W> v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (r[q] >= 0) v[q] = *reinterpret_cast<const Piece<TI, W> *>(Y + r[q] * a.ldy);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (r[q] < 0) continue;
#pragma unroll
            for (int e = 0; e < W; ++e) s[e] = __builtin_fmaf(w[q], (float)v[q].v[e], s[e]);
        }
    }
    Piece<TO, W> o;
#pragma unroll
    for (int e = 0; e < W; ++e) o.v[e] = (TO)s[e];
    *reinterpret_cast<Piece<TO, W> *>(static_cast<TO *>(a.out) + t * a.ldo + c) = o;
}

template <class TI, class TO, int W>
hipError_t launch_combine(CombineArgs a, int64_t tokens, hipStream_t stream) {
    // (a launch's threads stay within 2^30, or are one token's, fewer than 2^31)
    const int64_t fit = ((int64_t)1 << 30) / a.per, most = fit > 0 ? fit : 1;
    for (a.first = 0; a.first < tokens; a.first += a.tokens) {
        a.tokens = (int)(tokens - a.first < most ? tokens - a.first : most);
        const dim3 grid((unsigned)(((int64_t)a.tokens * a.per + 255) / 256));
        hipLaunchKernelGGL((combine_kernel<TI, TO, W>), grid, dim3(256), 0, stream, a);
    }
    return hipGetLastError();
}
template <class TI, class TO>
hipError_t launch_combine(CombineArgs a, int64_t tokens, int64_t N, hipStream_t stream) {
    const bool vec = N % 8 == 0;
    a.per = (int)(vec ? N / 8 : N);
    return vec ? launch_combine<TI, TO, 8>(a, tokens, stream) : launch_combine<TI, TO, 1>(a, tokens, stream);
}
template <class TI>
hipError_t launch_combine(const CombineArgs &a, MxType out, int64_t tokens, int64_t N, hipStream_t stream) {
    switch (out) {
        case MxType::F16: return launch_combine<TI, _Float16>(a, tokens, N, stream);
        case MxType::BF16: return launch_combine<TI, __bf16>(a, tokens, N, stream);
        case MxType::F32: return launch_combine<TI, float>(a, tokens, N, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_expert_route(const void *logits, MxType type, int64_t ld, int64_t T, int E, int k, bool sigmoid,
                               const float *bias, int groups, int top_groups, bool renormalize, float scale,
                               int32_t *ids, float *weights, hipStream_t stream) {
    const RouteArgs a = {logits, type, ld, T, E, k, groups, top_groups, sigmoid, renormalize, bias, scale, ids, weights};
    if (route_shared(T, E, groups)) {
        if (E <= 64) launch_route<2, 32>(a, stream);
        else if (E <= 128) launch_route<4, 32>(a, stream);
        else launch_route<8, 32>(a, stream);
    } else {
        if (E <= 64) launch_route<1, 64>(a, stream);
        else if (E <= 128) launch_route<2, 64>(a, stream);
        else if (E <= 256) launch_route<4, 64>(a, stream);
        else launch_route<8, 64>(a, stream);   // (512 at most)
    }
    return hipGetLastError();
}

size_t expert_plan_workspace_bytes(int64_t n, int64_t E) {
    int64_t runs = plan_runs(n, 4);
    if (runs == 1) return 0;
    // (no smaller n needs more)
    for (int per = 1; per < 4; per *= 2) {
        const int64_t most = plan_most(per, E), r = plan_runs(n, per) < most ? plan_runs(n, per) : most;
        runs = r > runs ? r : runs;
    }
    return (size_t)(runs * E) * sizeof(int32_t);
}

hipError_t launch_expert_plan(const int32_t *ids, int64_t n, int k, int E, int32_t *info, int32_t *rows,
                              int32_t *source, void *workspace, hipStream_t stream) {
    switch (plan_per(n, E)) {
        case 1: return launch_plan<1>(ids, n, k, E, info, rows, source, workspace, stream);
        case 2: return launch_plan<2>(ids, n, k, E, info, rows, source, workspace, stream);
        default: return launch_plan<4>(ids, n, k, E, info, rows, source, workspace, stream);
    }
}

hipError_t launch_expert_combine(const void *Y, MxType type, int64_t ldy, const int32_t *rows, const float *weights,
                                 int64_t T, int k, int64_t N, int64_t plan_rows, void *out, MxType out_type, int64_t ldo,
                                 hipStream_t stream) {
    const CombineArgs a = {Y, rows, weights, out, ldy, ldo, plan_rows, 0, 0, k, 0};
    switch (type) {
        case MxType::F16: return launch_combine<_Float16>(a, out_type, T, N, stream);
        case MxType::BF16: return launch_combine<__bf16>(a, out_type, T, N, stream);
        case MxType::F32: return launch_combine<float>(a, out_type, T, N, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace clq
