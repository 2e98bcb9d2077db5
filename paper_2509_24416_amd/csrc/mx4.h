// Microscaled 4-bit codes (MX4): layouts and the grid, shared by the quantizer
// and the products.
//
// Grid: e2m1 codes (sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3,
// 4, 6 and their negatives) with one scale 2^e for 32 consecutive values of a row,
// stored as the byte e + 127.  e = floor(log2(max|x|)) - 2 (6 = 1.5 * 2^2 is the
// largest code), at least -126; byte 255 marks a group that held an infinity or a
// NaN and stands for NaN.
//
// Layout (opaque to callers): the row units and lane order of the packed int4
// layouts in clq_internal.h.  A unit is 32 rows x 64 codes, 1 KB: lane
// l = 32h + rho holds the 16 bytes of codes 32h .. 32h+31 of fragment row rho, so
// that a lane's 16 bytes are its whole operand of a 32x32x64 matrix instruction and
// its h picks the scale group.  Weights keep their fragment-row order (an output
// lane then owns 16 consecutive channels).  Scales: [row unit][K / 256 rounded
// up][lane][4], byte j of lane l's dword belonging to lane l's 32 codes of k unit
// 4 q + j: one 256-byte row of dwords serves four matrix instructions, each taking
// its byte by an immediate selector.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "clq_internal.h"

namespace clq {

constexpr int kMxGroup = 32;      // values that share a scale
constexpr int kMxUnit = 1024;     // bytes of a 32 x 64 unit of codes
constexpr int kMxScaleRow = 256;  // scale bytes of 32 rows x 256 codes

__host__ __device__ inline int64_t mx_scale_quads(int64_t K) { return (K + 255) >> 8; }
// scale bytes of `units` row units
__host__ __device__ inline int64_t mx_scale_bytes(int64_t units, int64_t K) {
    return units * mx_scale_quads(K) * kMxScaleRow;
}
// byte offsets of row unit u, fragment row rho, chunk c (codes 32c .. 32c + 31)
__host__ __device__ inline int64_t mx_code_offset(int64_t u, int rho, int64_t c, int64_t K) {
    return ((u * (K >> 6) + (c >> 1)) * 64 + (c & 1) * 32 + rho) * 16;
}
__host__ __device__ inline int64_t mx_scale_offset(int64_t u, int rho, int64_t c, int64_t K) {
    return ((u * mx_scale_quads(K) + (c >> 3)) * 64 + (c & 1) * 32 + rho) * 4 + ((c >> 1) & 3);
}

enum class MxType { F16 = 0, BF16 = 1, F32 = 2 };
enum class MxAct { None = 0, Gelu = 1, Swiglu = 2 };

// Where the rows of an expert plan lie (experts.hip): per-expert tables of int32.
// counts [E], then for tiles of 1, 4 and 8 row units (those of the grouped products) the
// number of tiles before each expert, E + 1 entries (the last one the total).  The first of the
// three is the experts' first row units.
constexpr int kPlanTables = 3;
__host__ __device__ constexpr int plan_log_units(int table) { return table ? table + 1 : 0; }
__host__ __device__ inline int64_t plan_info_ints(int64_t E) { return E + kPlanTables * (E + 1); }
// log_units: 0, 2 or 3
__host__ __device__ inline int64_t plan_table_offset(int64_t E, int log_units) {
    return E + (log_units ? log_units - 1 : 0) * (E + 1);
}
// row units an expert plan of n assignments can need: every expert's last unit may
// hold a single row
__host__ __device__ inline int64_t plan_max_units(int64_t n, int64_t E) {
    return n / 32 + (E < n ? E : n);
}

#if defined(__HIP_DEVICE_COMPILE__) || defined(__HIPCC__)
// Scale byte of a group whose largest magnitude has the bits `top` (infinity or NaN
// if the group holds one); log_div: the values are to be divided by 2^log_div.
__device__ __forceinline__ int mx_scale_byte(uint32_t top, int log_div) {
    const int ex = (int)(top >> 23);
    return ex == 255 ? 255 : max(ex - 2 - log_div, 1);
}
// the float that the conversion instructions divide by (byte 255: any)
__device__ __forceinline__ float mx_scale_value(int byte, int log_div) {
    return __uint_as_float((uint32_t)min(byte + log_div, 254) << 23);
}
// eight values -> eight codes, element e at bits 4e .. 4e + 3, rounded to nearest,
// ties to even, saturated at 6
__device__ __forceinline__ uint32_t mx_pack8(const float *x, float scale) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
    return r;
}
#endif

// Quantizer of activations and weights.  source (activations): row r of the output
// is row source[r] of X (negative: zeros); info: the plan's tables, past whose last
// row unit nothing is written.  Weights: fragment-row order, values divided by
// 2^log_div, gated: row 64j + t is row 32j + t of the first half of W's rows for t < 32,
// of the second half for the others; `mats` matrices of `rows` rows each.
struct MxQuantArgs {
    const void *X;
    int64_t ldx;
    MxType type;
    const int32_t *perm;
    int64_t rows, units;   // valid rows; row units written (of each matrix)
    int K, block;
    bool weights, gated;
    int mats, log_div;
    const int32_t *source;
    const int32_t *total_units;   // device: row units in use (nullptr: all)
    uint8_t *codes, *scales;
};
hipError_t launch_mx_quantize(const MxQuantArgs &a, hipStream_t stream);

hipError_t launch_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int K, bool weights,
                                bool gated, int mats, MxType type, void *out, int64_t ldo, hipStream_t stream);

// canonical codes [rows][K / 2] and scale bytes [rows][K / 32] into the weight layout
hipError_t launch_mx_pack(const uint8_t *codes, const uint8_t *scales, int64_t rows, int K, bool gated, int mats,
                          uint8_t *codes_out, uint8_t *scales_out, hipStream_t stream);

// Products.  info != nullptr: the rows are an expert plan's (units row units at most)
// and W holds `experts` matrices; otherwise M rows.
struct MxGemmArgs {
    const uint8_t *Xq, *Xs, *Wq, *Ws;
    const void *bias;
    MxType bias_type;
    int64_t M, N;
    int K;
    const int32_t *info;
    int experts;
    int64_t units, assignments;   // plan: row units at most, assignments
    // plain output
    void *Y;
    int64_t ldy;
    MxType out_type;
    // MX4 output (Y == nullptr): activation and rotation ahead of the quantizer
    MxAct act;
    int block;
    uint8_t *Oq, *Os;
};
hipError_t launch_mx_gemm(const MxGemmArgs &a, hipStream_t stream);

// Routing.
hipError_t launch_expert_route(const void *logits, MxType type, int64_t ld, int64_t T, int E, int k, bool sigmoid,
                               const float *bias, int groups, int top_groups, bool renormalize, float scale,
                               int32_t *ids, float *weights, hipStream_t stream);
size_t expert_plan_workspace_bytes(int64_t n, int64_t E);
hipError_t launch_expert_plan(const int32_t *ids, int64_t n, int k, int E, int32_t *info, int32_t *rows,
                              int32_t *source, void *workspace, hipStream_t stream);
hipError_t launch_expert_combine(const void *Y, MxType type, int64_t ldy, const int32_t *rows, const float *weights,
                                 int64_t T, int k, int64_t N, int64_t plan_rows, void *out, MxType out_type, int64_t ldo,
                                 hipStream_t stream);

}  // namespace clq
