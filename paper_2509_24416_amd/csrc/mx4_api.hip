// C ABI of the MX4 operators and of the expert layer (clq_mx4.h): host-side checks
// and launches, as in clq_api.hip.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/clq_mx4.h"
#include "api_checks.h"
#include "clq_internal.h"
#include "mx4.h"

using namespace clq::api;

namespace {

constexpr int64_t kMaxExperts = 512, kMaxTopK = 32, kMaxGroups = 64;

bool is_16bit(clq_type t) { return t == CLQ_F16 || t == CLQ_BF16; }
bool is_type(clq_type t) { return is_16bit(t) || t == CLQ_F32; }
clq::MxType mx_type(clq_type t) { return t == CLQ_F16 ? clq::MxType::F16 : t == CLQ_BF16 ? clq::MxType::BF16 : clq::MxType::F32; }

clq_status check_mx_block(int64_t K, int32_t block) { return block == 0 ? CLQ_OK : check_block(K, block); }
int log2_block(int32_t block) { return block == 32 ? 5 : block == 64 ? 6 : block == 128 ? 7 : 0; }
// row units of `rows` rows; rows of all matrices together stay below 2^31
int64_t row_units(int64_t rows, bool weights) { return (weights ? clq::padded_rows(rows) : clq::padded_act_rows(rows)) >> 5; }
clq_status check_matrices(int64_t mats, int64_t rows, int64_t K) {
    clq_status s;
    if (mats < 1 || mats > kMaxExperts) return CLQ_ERR_SHAPE;
    if ((s = check_rows(rows)) != CLQ_OK || (s = check_k(K)) != CLQ_OK) return s;
    if (mats * clq::padded_rows(rows) > kMaxRows) return CLQ_ERR_SHAPE;
    return CLQ_OK;
}
clq_status check_plan(int64_t T, int64_t top_k, int64_t experts) {
    if (T < 1 || T > kMaxRows || top_k < 1 || top_k > kMaxTopK || experts < 1 || experts > kMaxExperts)
        return CLQ_ERR_SHAPE;
    if (T * top_k + 32 * kMaxExperts > kMaxRows) return CLQ_ERR_SHAPE;
    return CLQ_OK;
}

clq_status quantize(const void *X, clq_type type, int64_t ldx, const int32_t *perm, int64_t rows, int64_t K,
                    int32_t block, const int32_t *source, const int32_t *total, int64_t units, void *codes,
                    void *scales, hipStream_t stream) {
    if (!is_16bit(type)) return CLQ_ERR_ARG;
    clq_status s;
    if ((s = check_rows(rows)) != CLQ_OK || (s = check_k(K)) != CLQ_OK || (s = check_mx_block(K, block)) != CLQ_OK)
        return s;
    if (ldx < K || ldx % 8 != 0) return CLQ_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(codes, 16) || !aligned(scales, 16) || (perm && !aligned(perm, 4)))
        return CLQ_ERR_ALIGN;
    clq::MxQuantArgs a = {};
    a.X = X;
    a.ldx = ldx;
    a.type = mx_type(type);
    a.perm = perm;
    a.rows = rows;
    a.units = units;
    a.K = (int)K;
    a.block = block;
    a.mats = 1;
    a.source = source;
    a.total_units = total;
    a.codes = static_cast<uint8_t *>(codes);
    a.scales = static_cast<uint8_t *>(scales);
    return done(stream, clq::launch_mx_quantize(a, stream));
}

// the checks and arguments that every product shares
clq_status product(const void *Xq, const void *Xs, const void *Wq, const void *Ws, const void *bias, clq_type bias_type,
                   int64_t experts, int64_t N, int64_t K, clq::MxGemmArgs &g) {
    clq_status s;
    if ((s = check_matrices(experts, N, K)) != CLQ_OK) return s;
    if (bias && !is_16bit(bias_type)) return CLQ_ERR_ARG;
    if (!aligned(Xq, 16) || !aligned(Xs, 16) || !aligned(Wq, 16) || !aligned(Ws, 16) || (bias && !aligned(bias, 2)))
        return CLQ_ERR_ALIGN;
    g = {};
    g.Xq = static_cast<const uint8_t *>(Xq);
    g.Xs = static_cast<const uint8_t *>(Xs);
    g.Wq = static_cast<const uint8_t *>(Wq);
    g.Ws = static_cast<const uint8_t *>(Ws);
    g.bias = bias;
    g.bias_type = mx_type(bias_type);
    g.N = N;
    g.K = (int)K;
    g.experts = (int)experts;
    return CLQ_OK;
}
// tiles of 256 x 128 outputs in one launch (under 2^32 lanes)
clq_status check_tiles(int64_t rows, int64_t N) {
    return ((rows + 255) / 256) * ((N + 127) / 128) < (int64_t)1 << 24 ? CLQ_OK : CLQ_ERR_SHAPE;
}
clq_status plain_output(clq::MxGemmArgs &g, clq_type type, void *Y, int64_t ldy) {
    if (!is_type(type)) return CLQ_ERR_ARG;
    if (ldy < g.N || ldy % 8 != 0) return CLQ_ERR_SHAPE;
    if (!aligned(Y, 16)) return CLQ_ERR_ALIGN;
    g.out_type = mx_type(type);
    g.Y = Y;
    g.ldy = ldy;
    return CLQ_OK;
}
clq_status mx4_output(clq::MxGemmArgs &g, clq_act act, int32_t block, void *codes, void *scales) {
    if (act != CLQ_ACT_NONE && act != CLQ_ACT_GELU && act != CLQ_ACT_SWIGLU) return CLQ_ERR_ARG;
    const bool gated = act == CLQ_ACT_SWIGLU;
    if (g.N % (gated ? 128 : 64) != 0) return CLQ_ERR_SHAPE;
    const int64_t columns = gated ? g.N / 2 : g.N;
    clq_status s;
    if ((s = check_k(columns)) != CLQ_OK || (s = check_mx_block(columns, block)) != CLQ_OK) return s;
    if (gated && block == 128) return CLQ_ERR_BLOCK;
    if (!aligned(codes, 16) || !aligned(scales, 16)) return CLQ_ERR_ALIGN;
    g.act = gated ? clq::MxAct::Swiglu : act == CLQ_ACT_GELU ? clq::MxAct::Gelu : clq::MxAct::None;
    g.block = block;
    g.Oq = static_cast<uint8_t *>(codes);
    g.Os = static_cast<uint8_t *>(scales);
    return CLQ_OK;
}
clq_status plan_rows(clq::MxGemmArgs &g, const int32_t *tables, int64_t T, int64_t top_k, int64_t experts) {
    clq_status s;
    if ((s = check_plan(T, top_k, experts)) != CLQ_OK) return s;
    if (!aligned(tables, 4)) return CLQ_ERR_ALIGN;
    g.info = tables;
    g.assignments = T * top_k;
    g.units = clq::plan_max_units(T * top_k, experts);
    return check_tiles(g.units * 32 + 256 * experts, g.N);
}

}  // namespace

extern "C" {

size_t clq_mx4_code_bytes(int64_t rows, int64_t K, int32_t weights) {
    if (check_rows(rows) != CLQ_OK || check_k(K) != CLQ_OK) return 0;
    return (size_t)row_units(rows, weights != 0) * (size_t)(K >> 6) * clq::kMxUnit;
}

size_t clq_mx4_scale_bytes(int64_t rows, int64_t K, int32_t weights) {
    if (check_rows(rows) != CLQ_OK || check_k(K) != CLQ_OK) return 0;
    return (size_t)clq::mx_scale_bytes(row_units(rows, weights != 0), K);
}

clq_status clq_mx4_quantize(const void *X, clq_type type, int64_t ldx, const int32_t *perm, int64_t M, int64_t K,
                            int32_t block, void *codes, void *scales, hipStream_t stream) {
    if (!X || !codes || !scales) return CLQ_ERR_NULL;
    return quantize(X, type, ldx, perm, M, K, block, nullptr, nullptr, row_units(M, false), codes, scales, stream);
}

clq_status clq_mx4_quantize_weights(const void *W, clq_type type, const int32_t *perm, int64_t experts, int64_t N,
                                    int64_t K, int32_t block, int32_t gated, void *codes, void *scales,
                                    hipStream_t stream) {
    if (!W || !codes || !scales) return CLQ_ERR_NULL;
    clq_status s;
    if (!is_16bit(type) || (gated != 0 && gated != 1)) return CLQ_ERR_ARG;
    if ((s = check_matrices(experts, N, K)) != CLQ_OK || (s = check_mx_block(K, block)) != CLQ_OK) return s;
    if (gated && N % 64 != 0) return CLQ_ERR_SHAPE;
    if (!aligned(W, 16) || !aligned(codes, 16) || !aligned(scales, 16) || (perm && !aligned(perm, 4)))
        return CLQ_ERR_ALIGN;
    clq::MxQuantArgs a = {};
    a.X = W;
    a.ldx = K;
    a.type = mx_type(type);
    a.perm = perm;
    a.rows = N;
    a.units = row_units(N, true);
    a.K = (int)K;
    a.block = block;
    a.weights = true;
    a.gated = gated != 0;
    a.mats = (int)experts;
    a.log_div = log2_block(block);
    a.codes = static_cast<uint8_t *>(codes);
    a.scales = static_cast<uint8_t *>(scales);
    return done(stream, clq::launch_mx_quantize(a, stream));
}

clq_status clq_mx4_pack_weights(const void *row_codes, const void *row_scales, int64_t experts, int64_t N, int64_t K,
                                int32_t gated, void *codes, void *scales, hipStream_t stream) {
    if (!row_codes || !row_scales || !codes || !scales) return CLQ_ERR_NULL;
    clq_status s;
    if (gated != 0 && gated != 1) return CLQ_ERR_ARG;
    if ((s = check_matrices(experts, N, K)) != CLQ_OK) return s;
    if (gated && N % 64 != 0) return CLQ_ERR_SHAPE;
    if (!aligned(row_codes, 16) || !aligned(codes, 16) || !aligned(scales, 16)) return CLQ_ERR_ALIGN;
    return done(stream, clq::launch_mx_pack(static_cast<const uint8_t *>(row_codes),
                                            static_cast<const uint8_t *>(row_scales), N, (int)K, gated != 0,
                                            (int)experts, static_cast<uint8_t *>(codes),
                                            static_cast<uint8_t *>(scales), stream));
}

clq_status clq_mx4_dequantize(const void *codes, const void *scales, int32_t weights, int32_t gated, int64_t matrices,
                              int64_t rows, int64_t K, clq_type type, void *out, int64_t ldo, hipStream_t stream) {
    if (!codes || !scales || !out) return CLQ_ERR_NULL;
    clq_status s;
    if ((weights != 0 && weights != 1) || (gated != 0 && gated != 1)) return CLQ_ERR_ARG;
    if (!is_type(type)) return CLQ_ERR_ARG;
    if (!weights && (gated || matrices != 1)) return CLQ_ERR_ARG;
    if (weights) s = check_matrices(matrices, rows, K);
    else s = check_rows(rows) != CLQ_OK ? CLQ_ERR_SHAPE : check_k(K);
    if (s != CLQ_OK) return s;
    if ((gated && rows % 64 != 0) || ldo < K || ldo % 8 != 0) return CLQ_ERR_SHAPE;
    if (!aligned(codes, 16) || !aligned(scales, 16) || !aligned(out, 16)) return CLQ_ERR_ALIGN;
    return done(stream, clq::launch_mx_dequantize(static_cast<const uint8_t *>(codes),
                                                  static_cast<const uint8_t *>(scales), rows, (int)K, weights != 0,
                                                  gated != 0, (int)matrices, mx_type(type), out, ldo, stream));
}

clq_status clq_mx4_linear(const void *Xq, const void *Xs, const void *Wq, const void *Ws, const void *bias,
                          clq_type bias_type, int64_t M, int64_t N, int64_t K, clq_type type, void *Y, int64_t ldy,
                          hipStream_t stream) {
    if (!Xq || !Xs || !Wq || !Ws || !Y) return CLQ_ERR_NULL;
    clq::MxGemmArgs g;
    clq_status s;
    if ((s = check_rows(M)) != CLQ_OK || (s = product(Xq, Xs, Wq, Ws, bias, bias_type, 1, N, K, g)) != CLQ_OK ||
        (s = plain_output(g, type, Y, ldy)) != CLQ_OK)
        return s;
    if ((s = check_tiles(M, N)) != CLQ_OK) return s;
    g.M = M;
    return done(stream, clq::launch_mx_gemm(g, stream));
}

clq_status clq_mx4_linear_mx4(const void *Xq, const void *Xs, const void *Wq, const void *Ws, const void *bias,
                              clq_type bias_type, int64_t M, int64_t N, int64_t K, clq_act act, int32_t block,
                              void *codes, void *scales, hipStream_t stream) {
    if (!Xq || !Xs || !Wq || !Ws || !codes || !scales) return CLQ_ERR_NULL;
    clq::MxGemmArgs g;
    clq_status s;
    if ((s = check_rows(M)) != CLQ_OK || (s = product(Xq, Xs, Wq, Ws, bias, bias_type, 1, N, K, g)) != CLQ_OK ||
        (s = mx4_output(g, act, block, codes, scales)) != CLQ_OK)
        return s;
    if ((s = check_tiles(M, N)) != CLQ_OK) return s;
    g.M = M;
    return done(stream, clq::launch_mx_gemm(g, stream));
}

clq_status clq_expert_route(const void *logits, clq_type type, int64_t ld, int64_t T, int64_t experts, int32_t top_k,
                            clq_score score, const float *bias, int32_t groups, int32_t top_groups,
                            int32_t renormalize, float scale, int32_t *ids, float *weights, hipStream_t stream) {
    if (!logits || !ids || !weights) return CLQ_ERR_NULL;
    clq_status s;
    if ((!is_type(type)) || (score != CLQ_SOFTMAX && score != CLQ_SIGMOID)) return CLQ_ERR_ARG;
    if ((renormalize != 0 && renormalize != 1) || !isfinite(scale)) return CLQ_ERR_ARG;
    if ((s = check_plan(T, top_k, experts)) != CLQ_OK) return s;
    if (ld < experts) return CLQ_ERR_SHAPE;
    if (groups < 1 || groups > kMaxGroups || experts % groups != 0 || top_groups < 1 || top_groups > groups)
        return CLQ_ERR_ARG;
    if (top_k > experts / groups * top_groups) return CLQ_ERR_ARG;
    if (!aligned(logits, type == CLQ_F32 ? 4 : 2) || (bias && !aligned(bias, 4)) || !aligned(ids, 4) ||
        !aligned(weights, 4))
        return CLQ_ERR_ALIGN;
    return done(stream, clq::launch_expert_route(logits, mx_type(type), ld, T, (int)experts, top_k,
                                                 score == CLQ_SIGMOID, bias, groups, top_groups, renormalize != 0,
                                                 scale, ids, weights, stream));
}

int64_t clq_expert_plan_rows(int64_t T, int64_t top_k, int64_t experts) {
    if (check_plan(T, top_k, experts) != CLQ_OK) return 0;
    return 32 * clq::plan_max_units(T * top_k, experts);
}

int64_t clq_expert_plan_ints(int64_t experts) {
    if (experts < 1 || experts > kMaxExperts) return 0;
    return clq::plan_info_ints(experts);
}

size_t clq_expert_plan_workspace_bytes(int64_t T, int64_t top_k, int64_t experts) {
    if (check_plan(T, top_k, experts) != CLQ_OK) return 0;
    return clq::expert_plan_workspace_bytes(T * top_k, experts);
}

clq_status clq_expert_plan(const int32_t *ids, int64_t T, int64_t top_k, int64_t experts, int32_t *tables,
                           int32_t *rows, int32_t *source, void *workspace, size_t workspace_bytes,
                           hipStream_t stream) {
    if (!ids || !tables || !rows || !source) return CLQ_ERR_NULL;
    clq_status s;
    if ((s = check_plan(T, top_k, experts)) != CLQ_OK) return s;
    const size_t need = clq::expert_plan_workspace_bytes(T * top_k, experts);
    if (need > 0 && !workspace) return CLQ_ERR_NULL;
    if (workspace_bytes < need) return CLQ_ERR_WORKSPACE;
    if (!aligned(ids, 4) || !aligned(tables, 4) || !aligned(rows, 4) || !aligned(source, 4) ||
        (need > 0 && !aligned(workspace, 4)))
        return CLQ_ERR_ALIGN;
    return done(stream, clq::launch_expert_plan(ids, T * top_k, (int)top_k, (int)experts, tables, rows, source,
                                                workspace, stream));
}

clq_status clq_mx4_dispatch(const void *X, clq_type type, int64_t ldx, const int32_t *perm, int64_t T, int64_t top_k,
                            int64_t experts, int64_t K, int32_t block, const int32_t *tables, const int32_t *source,
                            void *codes, void *scales, hipStream_t stream) {
    if (!X || !tables || !source || !codes || !scales) return CLQ_ERR_NULL;
    clq_status s;
    if ((s = check_plan(T, top_k, experts)) != CLQ_OK) return s;
    if (!aligned(tables, 4) || !aligned(source, 4)) return CLQ_ERR_ALIGN;
    return quantize(X, type, ldx, perm, T, K, block, source, tables + clq::plan_table_offset(experts, 0) + experts,
                    clq::plan_max_units(T * top_k, experts), codes, scales, stream);
}

clq_status clq_mx4_experts(const void *Xq, const void *Xs, const int32_t *tables, int64_t T, int64_t top_k,
                           int64_t experts, const void *Wq, const void *Ws, const void *bias, clq_type bias_type,
                           int64_t N, int64_t K, clq_type type, void *Y, int64_t ldy, hipStream_t stream) {
    if (!Xq || !Xs || !tables || !Wq || !Ws || !Y) return CLQ_ERR_NULL;
    clq::MxGemmArgs g;
    clq_status s;
    if ((s = product(Xq, Xs, Wq, Ws, bias, bias_type, experts, N, K, g)) != CLQ_OK ||
        (s = plan_rows(g, tables, T, top_k, experts)) != CLQ_OK || (s = plain_output(g, type, Y, ldy)) != CLQ_OK)
        return s;
    return done(stream, clq::launch_mx_gemm(g, stream));
}

clq_status clq_mx4_experts_mx4(const void *Xq, const void *Xs, const int32_t *tables, int64_t T, int64_t top_k,
                               int64_t experts, const void *Wq, const void *Ws, const void *bias, clq_type bias_type,
                               int64_t N, int64_t K, clq_act act, int32_t block, void *codes, void *scales,
                               hipStream_t stream) {
    if (!Xq || !Xs || !tables || !Wq || !Ws || !codes || !scales) return CLQ_ERR_NULL;
    clq::MxGemmArgs g;
    clq_status s;
    if ((s = product(Xq, Xs, Wq, Ws, bias, bias_type, experts, N, K, g)) != CLQ_OK ||
        (s = plan_rows(g, tables, T, top_k, experts)) != CLQ_OK ||
        (s = mx4_output(g, act, block, codes, scales)) != CLQ_OK)
        return s;
    return done(stream, clq::launch_mx_gemm(g, stream));
}

clq_status clq_expert_combine(const void *Y, clq_type type, int64_t ldy, const int32_t *rows, const float *weights,
                              int64_t T, int64_t top_k, int64_t experts, int64_t N, void *out, clq_type out_type,
                              int64_t ldo, hipStream_t stream) {
    if (!Y || !rows || !weights || !out) return CLQ_ERR_NULL;
    clq_status s;
    if (!is_type(type) || !is_type(out_type)) return CLQ_ERR_ARG;
    if ((s = check_plan(T, top_k, experts)) != CLQ_OK || (s = check_rows(N)) != CLQ_OK) return s;
    if (ldy < N || ldo < N || ldy % 8 != 0 || ldo % 8 != 0) return CLQ_ERR_SHAPE;
    if (!aligned(Y, 16) || !aligned(out, 16) || !aligned(rows, 4) || !aligned(weights, 4)) return CLQ_ERR_ALIGN;
    return done(stream, clq::launch_expert_combine(Y, mx_type(type), ldy, rows, weights, T, (int)top_k, N,
                                                   clq_expert_plan_rows(T, top_k, experts), out, mx_type(out_type), ldo,
                                                   stream));
}

}  // extern "C"
