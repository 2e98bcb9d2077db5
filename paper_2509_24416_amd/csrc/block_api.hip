// C ABI of the operators around the 8-bit linears (clq_block.h): host-side checks and
// launches, as in clq_api.hip.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include "../../include/clq_block.h"
#include "api_checks.h"
#include "block.h"
#include "clq_internal.h"

using namespace clq::api;

namespace {

constexpr int64_t kMaxNormK = 16384, kMaxHead = 256, kMaxHeads = 1 << 20;

bool is_16bit(clq_type t) { return t == CLQ_F16 || t == CLQ_BF16; }
bool is_type(clq_type t) { return is_16bit(t) || t == CLQ_F32; }
clq::MxType mx_type(clq_type t) { return t == CLQ_F16 ? clq::MxType::F16 : t == CLQ_BF16 ? clq::MxType::BF16 : clq::MxType::F32; }
bool is_eps(float eps) { return isfinite(eps) && eps >= FLT_MIN; }

bool is_stride(int64_t ld, int64_t n) { return ld >= n && ld % 8 == 0; }
clq_status check_samples(int64_t M, int64_t samples) {
    return samples < 1 || samples > M || M % samples != 0 ? CLQ_ERR_SHAPE : CLQ_OK;
}

// the checks and arguments that both results of the norm share
clq_status norm(const void *X, clq_type x_type, int64_t ldx, const void *R, clq_type r_type, int64_t ldr, const void *W,
                clq_type w_type, int64_t samples, float eps, int64_t M, int64_t K, void *sum, int64_t ld_sum,
                clq::RmsNormArgs &a) {
    if ((R == nullptr) != (sum == nullptr)) return CLQ_ERR_NULL;
    if (!is_type(x_type) || (R && !is_type(r_type)) || (W && !is_type(w_type)) || !is_eps(eps)) return CLQ_ERR_ARG;
    clq_status s;
    if ((s = check_rows(M)) != CLQ_OK || (s = check_samples(M, samples)) != CLQ_OK) return s;
    if (K < 8 || K > kMaxNormK || K % 8 != 0 || (!W && samples != 1)) return CLQ_ERR_SHAPE;
    if (!is_stride(ldx, K) || (R && (!is_stride(ldr, K) || !is_stride(ld_sum, K)))) return CLQ_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(R, 16) || !aligned(sum, 16) || !aligned(W, 16)) return CLQ_ERR_ALIGN;
    a = {};
    a.X = X;
    a.x_type = mx_type(x_type);
    a.ldx = ldx;
    a.R = R;
    a.r_type = mx_type(r_type);
    a.ldr = ldr;
    a.W = W;
    a.w_type = mx_type(w_type);
    a.M = M;
    a.sample_rows = M / samples;
    a.K = (int)K;
    a.eps = eps;
    a.sum = sum;
    a.ld_sum = ld_sum;
    return CLQ_OK;
}

}  // namespace

extern "C" {

clq_status clq_rms_norm(const void *X, clq_type x_type, int64_t ldx, const void *R, clq_type r_type, int64_t ldr,
                        const void *W, clq_type w_type, int64_t samples, float eps, int64_t M, int64_t K, void *Y,
                        clq_type y_type, int64_t ldy, void *sum, int64_t ld_sum, hipStream_t stream) {
    if (!X || !Y) return CLQ_ERR_NULL;
    clq::RmsNormArgs a;
    clq_status s = norm(X, x_type, ldx, R, r_type, ldr, W, w_type, samples, eps, M, K, sum, ld_sum, a);
    if (s != CLQ_OK) return s;
    if (!is_type(y_type)) return CLQ_ERR_ARG;
    if (!is_stride(ldy, K)) return CLQ_ERR_SHAPE;
    if (!aligned(Y, 16)) return CLQ_ERR_ALIGN;
    a.Y = Y;
    a.y_type = mx_type(y_type);
    a.ldy = ldy;
    return done(stream, clq::launch_rms_norm(a, stream));
}

clq_status clq_rms_norm_act8(const void *X, clq_type x_type, int64_t ldx, const void *R, clq_type r_type, int64_t ldr,
                             const void *W, clq_type w_type, int64_t samples, float eps, const int32_t *perm,
                             int64_t M, int64_t K, int32_t block, void *Xq8, float *x_scale, void *sum, int64_t ld_sum,
                             hipStream_t stream) {
    if (!X || !Xq8 || !x_scale) return CLQ_ERR_NULL;
    clq::RmsNormArgs a;
    clq_status s = norm(X, x_type, ldx, R, r_type, ldr, W, w_type, samples, eps, M, K, sum, ld_sum, a);
    if (s != CLQ_OK || (s = check_k(K)) != CLQ_OK || (s = check_block(K, block)) != CLQ_OK) return s;
    if (!aligned(Xq8, 16) || !aligned(x_scale, 4) || !aligned(perm, 4)) return CLQ_ERR_ALIGN;
    a.norm = true;
    a.perm = perm;
    a.block = block;
    a.Xq8 = static_cast<uint8_t *>(Xq8);
    a.x_scale = x_scale;
    return done(stream, clq::launch_rms_norm(a, stream));
}

clq_status clq_quantize_act8(const void *X, clq_type x_type, int64_t ldx, const int32_t *perm, int64_t M, int64_t K,
                             int32_t block, void *Xq8, float *x_scale, hipStream_t stream) {
    if (!X || !Xq8 || !x_scale) return CLQ_ERR_NULL;
    if (!is_type(x_type)) return CLQ_ERR_ARG;
    clq_status s;
    if ((s = check_rows(M)) != CLQ_OK || (s = check_k(K)) != CLQ_OK || (s = check_block(K, block)) != CLQ_OK) return s;
    if (K > kMaxNormK || !is_stride(ldx, K)) return CLQ_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(Xq8, 16) || !aligned(x_scale, 4) || !aligned(perm, 4)) return CLQ_ERR_ALIGN;
    clq::RmsNormArgs a = {};
    a.X = X;
    a.x_type = mx_type(x_type);
    a.ldx = ldx;
    a.M = M;
    a.sample_rows = M;
    a.K = (int)K;
    a.perm = perm;
    a.block = block;
    a.Xq8 = static_cast<uint8_t *>(Xq8);
    a.x_scale = x_scale;
    return done(stream, clq::launch_rms_norm(a, stream));
}

clq_status clq_dequantize_act8(const void *Xq8, const float *x_scale, int64_t M, int64_t K, clq_type type, void *out,
                               int64_t ldo, hipStream_t stream) {
    if (!Xq8 || !x_scale || !out) return CLQ_ERR_NULL;
    if (!is_type(type)) return CLQ_ERR_ARG;
    clq_status s;
    if ((s = check_rows(M)) != CLQ_OK || (s = check_k(K)) != CLQ_OK) return s;
    if (!is_stride(ldo, K)) return CLQ_ERR_SHAPE;
    if (!aligned(Xq8, 16) || !aligned(x_scale, 4) || !aligned(out, 16)) return CLQ_ERR_ALIGN;
    return done(stream, clq::launch_dequantize_act8(static_cast<const uint8_t *>(Xq8), x_scale, M, (int)K, mx_type(type),
                                                    out, ldo, stream));
}

clq_status clq_rope_axes(const void *X, clq_type type, int64_t ldx, int64_t lhx, const void *positions,
                         int32_t position_type, int64_t tokens, const double *freqs, const int32_t *pair_ends,
                         int32_t axes, int32_t interleaved, int32_t inverse, const void *W, clq_type w_type,
                         int64_t weight_heads, float eps, int64_t M, int64_t heads, int64_t D, void *Y, int64_t ldy,
                         int64_t lhy, hipStream_t stream) {
    if (!X || !positions || !freqs || !pair_ends || !Y) return CLQ_ERR_NULL;
    if (!is_16bit(type) || position_type < 0 || position_type > 1 || axes < 1 || axes > 4 ||
        (interleaved != 0 && interleaved != 1) || (inverse != 0 && inverse != 1))
        return CLQ_ERR_ARG;
    if (W && (!is_type(w_type) || !is_eps(eps))) return CLQ_ERR_ARG;
    clq_status s;
    if ((s = check_rows(M)) != CLQ_OK || (s = check_rows(heads)) != CLQ_OK) return s;
    if (heads > kMaxHeads) return CLQ_ERR_SHAPE;
    if (tokens < 1 || tokens > M || M % tokens != 0) return CLQ_ERR_SHAPE;
    if (D < 8 || D > kMaxHead || D % 8 != 0) return CLQ_ERR_SHAPE;
    if (W && weight_heads != 1 && weight_heads != heads) return CLQ_ERR_SHAPE;
    int32_t last = 0;
    for (int i = 0; i < axes; ++i) {
        if (pair_ends[i] <= last || pair_ends[i] > D / 2) return CLQ_ERR_SHAPE;
        last = pair_ends[i];
    }
    if (last % 4 != 0) return CLQ_ERR_SHAPE;
    if (!is_stride(ldx, D) || !is_stride(lhx, D) || !is_stride(ldy, D) || !is_stride(lhy, D)) return CLQ_ERR_SHAPE;
    // the output's heads do not meet: rows of heads, or heads of rows
    if (ldy < (heads - 1) * lhy + D && lhy < (M - 1) * ldy + D) return CLQ_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(Y, 16) || !aligned(positions, 4) || !aligned(freqs, 8) ||
        !aligned(W, 16))
        return CLQ_ERR_ALIGN;
    clq::RopeArgs a = {};
    a.X = static_cast<const uint16_t *>(X);
    a.Y = static_cast<uint16_t *>(Y);
    a.ldx = ldx;
    a.lhx = lhx;
    a.ldy = ldy;
    a.lhy = lhy;
    a.M = M;
    a.tokens = tokens;
    a.positions = positions;
    a.bf16 = type == CLQ_BF16;
    a.float_positions = position_type == 1;
    a.interleaved = interleaved != 0;
    a.inverse = inverse != 0;
    a.freqs = freqs;
    for (int i = 0; i < 4; ++i) a.ends[i] = pair_ends[i < axes ? i : axes - 1];
    a.axes = axes;
    a.heads = (int)heads;
    a.D = (int)D;
    a.W = W;
    a.w_type = mx_type(w_type);
    a.w_stride = weight_heads == 1 ? 0 : D;
    a.eps = eps;
    return done(stream, clq::launch_rope(a, stream));
}

clq_status clq_a8_linear_act(const void *Xq8, const float *x_scale, const void *Wq, const float *w_scale,
                             int32_t wbits, const void *bias, clq_type bias_type, int32_t act, const void *gate,
                             clq_type gate_type, int64_t samples, const void *R, int64_t ldr, int64_t M, int64_t N,
                             int64_t K, clq_type type, void *Y, int64_t ldy, hipStream_t stream) {
    if (!Xq8 || !x_scale || !Wq || !w_scale || !Y) return CLQ_ERR_NULL;
    if (wbits != 4 && wbits != 8) return CLQ_ERR_ARG;
    if (act != CLQ_ACT_NONE && act != CLQ_ACT_GELU && act != CLQ_ACT_SILU) return CLQ_ERR_ARG;
    if (!is_type(type) || (bias && !is_16bit(bias_type)) || (gate && !is_type(gate_type))) return CLQ_ERR_ARG;
    clq_status s;
    if ((s = check_rows(M)) != CLQ_OK || (s = check_rows(N)) != CLQ_OK || (s = check_k(K)) != CLQ_OK ||
        (s = check_samples(M, samples)) != CLQ_OK)
        return s;
    // (a launch has fewer than 2^32 lanes)
    if (((M + 255) / 256) * ((N + 127) / 128) >= (int64_t)1 << 24) return CLQ_ERR_SHAPE;
    if ((!gate && samples != 1) || !is_stride(ldy, N) || (R && ldr < N)) return CLQ_ERR_SHAPE;
    if (!aligned(Xq8, 16) || !aligned(Wq, 16) || !aligned(Y, 16) || !aligned(R, type == CLQ_F32 ? 4 : 2) || !aligned(gate, 16) ||
        !aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 2))
        return CLQ_ERR_ALIGN;
    clq::Act8Args a = {};
    a.Xq = static_cast<const uint8_t *>(Xq8);
    a.xs = x_scale;
    a.Wq = static_cast<const uint8_t *>(Wq);
    a.ws = w_scale;
    a.wbits = wbits;
    a.bias = bias;
    a.bias_type = mx_type(bias_type);
    a.act = act == CLQ_ACT_GELU ? clq::Act8::Gelu : act == CLQ_ACT_SILU ? clq::Act8::Silu : clq::Act8::None;
    a.gate = gate;
    a.gate_type = mx_type(gate_type);
    a.sample_rows = M / samples;
    a.R = R;
    a.ldr = ldr;
    a.type = mx_type(type);
    a.Y = Y;
    a.ldy = ldy;
    a.M = (int)M;
    a.N = (int)N;
    a.K = (int)K;
    return done(stream, clq::launch_a8_act(a, stream));
}

}  // extern "C"
