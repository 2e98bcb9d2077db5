// Operators around the 8-bit linears of a transformer block: launch arguments
// (host and device) and the conversions that their kernels share.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "clq_internal.h"
#include "mx4.h"

namespace clq {

struct RmsNormArgs {
    const void *X, *R, *W;   // R, W: may be null
    MxType x_type, r_type, w_type, y_type;
    int64_t ldx, ldr, ld_sum, ldy;
    int64_t M, sample_rows;  // rows of a sample
    int K;
    float eps;
    void *sum;               // R's type
    // plain result
    void *Y;
    // 8-bit codes (Y == nullptr); norm: false for a quantizer alone
    bool norm;
    const int32_t *perm;
    int block;
    uint8_t *Xq8;
    float *x_scale;
};
hipError_t launch_rms_norm(const RmsNormArgs &a, hipStream_t stream);

hipError_t launch_dequantize_act8(const uint8_t *Xq8, const float *x_scale, int64_t M, int K, MxType type, void *out,
                                  int64_t ldo, hipStream_t stream);

struct RopeArgs {
    const uint16_t *X;
    uint16_t *Y;
    int64_t ldx, lhx, ldy, lhy, M, tokens;
    const void *positions;
    bool bf16, float_positions, interleaved, inverse;
    const double *freqs;
    int ends[4];             // pairs of the axes so far (unused ones repeat the last)
    int axes, heads, D;
    const void *W;           // may be null
    MxType w_type;
    int64_t w_stride;        // elements between the heads' weights
    float eps;
};
hipError_t launch_rope(const RopeArgs &a, hipStream_t stream);

enum class Act8 { None = 0, Gelu = 1, Silu = 2 };
// What follows the sums of an 8-bit linear.
struct Act8Args {
    const uint8_t *Xq, *Wq;
    const float *xs, *ws;
    const void *bias, *gate, *R;   // may be null
    MxType bias_type, gate_type, type;   // type: R's and Y's
    Act8 act;
    int64_t sample_rows, ldr, ldy;
    void *Y;
    int M, N, K, wbits;
};
hipError_t launch_a8_act(const Act8Args &a, hipStream_t stream);
// by the output's type
hipError_t launch_a8_act_bf16(const Act8Args &a, hipStream_t stream);
hipError_t launch_a8_act_f32(const Act8Args &a, hipStream_t stream);

#if defined(__HIP_DEVICE_COMPILE__) || defined(__HIPCC__)
__device__ __forceinline__ float widen16(uint16_t h, bool bf16) {
    return bf16 ? __uint_as_float((uint32_t)h << 16) : __half2float(__ushort_as_half(h));
}
// eight 16-bit values
__device__ __forceinline__ void widen8(const uint4 &v, bool bf16, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if (bf16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __half2float(__ushort_as_half((uint16_t)w[e]));
            x[2 * e + 1] = __half2float(__ushort_as_half((uint16_t)(w[e] >> 16)));
        }
    }
}
// two values rounded to nearest even
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
__device__ __forceinline__ uint4 narrow8(const float (&x)[8], bool bf16) {
    return make_uint4(narrow2(x[0], x[1], bf16), narrow2(x[2], x[3], bf16), narrow2(x[4], x[5], bf16),
                      narrow2(x[6], x[7], bf16));
}
// eight values of a matrix of any of the three types
__device__ __forceinline__ void load8(const void *p, int64_t at, MxType type, float (&x)[8]) {
    if (type == MxType::F32) {
        const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at);
        const float4 a = q[0], b = q[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        widen8(*reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + at), type == MxType::BF16, x);
    }
}
__device__ __forceinline__ void store8(void *p, int64_t at, MxType type, const float (&x)[8]) {
    if (type == MxType::F32) {
        float4 *q = reinterpret_cast<float4 *>(static_cast<float *>(p) + at);
        q[0] = make_float4(x[0], x[1], x[2], x[3]);
        q[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {   // (one branch for the eight)
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + at) = type == MxType::BF16 ? narrow8(x, true) : narrow8(x, false);
    }
}
#endif

}  // namespace clq
