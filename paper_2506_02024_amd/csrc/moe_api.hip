// C ABI of a mixture of experts (router, experts of a few tokens): argument validation, workspace layout and dispatch.  See
// include/nestedfp.h for the contract of every entry point.
#include "../../include/nestedfp.h"
#include "nfp_host.h"

#include <math.h>
#include <string.h>

namespace nfp {

static inline bool at_multiple(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kWidest = (int64_t)1 << 21;          // columns and strides

static int check_route(int64_t M, int64_t experts, int64_t K) {
    if (M < 0 || experts <= 0 || K <= 0) return kErrArg;
    return M > 0x3fffffff || experts > 512 || K > kWidest || (K & 15) != 0 ? kErrShape : kOk;
}

static int check_experts(const nestedfp_experts *e, int64_t M, int64_t top_k) {
    if (e == nullptr || e->experts <= 0 || e->hidden <= 0 || e->ffn <= 0 || M < 0 || top_k <= 0) return kErrArg;
    if (e->activation < 0 || e->activation >= kNumActivations) return kErrArg;
    if ((e->hidden & 15) != 0 || (e->ffn & 15) != 0 || e->hidden > kWidest || e->ffn > kWidest) return kErrShape;
    return experts_supported(e->experts, e->hidden, e->ffn, M, top_k) ? kOk : kErrShape;
}

}  // namespace nfp

using namespace nfp;

extern "C" {

size_t nestedfp_moe_route_workspace_size(int64_t M, int64_t experts, int64_t K) {
    if (check_route(M, experts, K) != kOk || M == 0) return 0;
    return kCounterBytes + route_logit_bytes(M, experts, K);
}

int nestedfp_moe_route(const uint16_t *X, int64_t M, int64_t K, int64_t ldx, const uint16_t *R, int64_t experts, int64_t ldr,
                       int64_t top_k, int scoring, int renormalize, float factor, const float *bias, int32_t *ids, float *weights,
                       void *workspace, size_t workspace_bytes, void *stream) {
    const int st = check_route(M, experts, K);
    if (st != kOk) return st;
    if (top_k <= 0 || (scoring != NESTEDFP_SCORE_SOFTMAX && scoring != NESTEDFP_SCORE_SIGMOID) || !isfinite(factor)) return NESTEDFP_ERR_ARG;
    if (top_k > 32 || top_k > experts) return NESTEDFP_ERR_SHAPE;
    if (M == 0) return NESTEDFP_OK;
    if (X == nullptr || R == nullptr || ids == nullptr || weights == nullptr) return NESTEDFP_ERR_ARG;
    for (const int64_t ld : {ldx, ldr})
        if (ld < K || ld > kWidest || (ld & 7) != 0) return NESTEDFP_ERR_SHAPE;
    if (!at_multiple(X, 16) || !at_multiple(R, 16) || !at_multiple(ids, 4) || !at_multiple(weights, 4) || !at_multiple(bias, 4)) return NESTEDFP_ERR_SHAPE;
    const size_t need = kCounterBytes + route_logit_bytes(M, experts, K);
    if (workspace == nullptr || workspace_bytes < need || !at_multiple(workspace, 16)) return NESTEDFP_ERR_WORKSPACE;
    RouteArgs a;
    memset(&a, 0, sizeof(a));
    a.X = X;  a.R = R;  a.ldx = ldx;  a.ldr = ldr;  a.M = M;  a.K = K;
    a.experts = (int32_t)experts;  a.top_k = (int32_t)top_k;
    a.sigmoid = scoring == NESTEDFP_SCORE_SIGMOID;  a.renormalize = renormalize != 0;
    a.factor = factor;  a.bias = bias;  a.ids = ids;  a.weights = weights;
    a.counters = static_cast<uint32_t *>(workspace);
    a.logits = reinterpret_cast<double *>(static_cast<uint8_t *>(workspace) + kCounterBytes);
    return launch_route(a, static_cast<hipStream_t>(stream));
}

size_t nestedfp_moe_workspace_size(int64_t M, const nestedfp_experts *experts_host, int64_t top_k) {
    if (check_experts(experts_host, M, top_k) != kOk || M == 0) return 0;
    return kCounterBytes + experts_workspace_bytes(experts_host->experts, experts_host->hidden, experts_host->ffn, M, top_k);
}

int nestedfp_moe(const uint16_t *X, int64_t M, int64_t ldx, const nestedfp_experts *experts_host, int mode, const int32_t *ids,
                 const float *weights, int64_t top_k, const uint16_t *residual, int64_t ldr, uint16_t *Y, int64_t ldy,
                 void *workspace, size_t workspace_bytes, void *stream) {
    const int st = check_experts(experts_host, M, top_k);
    if (st != kOk) return st;
    if (mode != NESTEDFP_MODE_FP16 && mode != NESTEDFP_MODE_FP8) return NESTEDFP_ERR_ARG;
    if (M == 0) return NESTEDFP_OK;
    const nestedfp_experts &e = *experts_host;
    const bool nested = !e.is_exception && mode == NESTEDFP_MODE_FP16;
    if (X == nullptr || Y == nullptr || ids == nullptr || weights == nullptr || e.up_upper == nullptr || e.down_upper == nullptr) return NESTEDFP_ERR_ARG;
    if (nested && (e.up_lower == nullptr || e.down_lower == nullptr)) return NESTEDFP_ERR_ARG;
    if (ldx < e.hidden || ldx > kWidest || (ldx & 7) != 0 || ldy < e.hidden || ldy > ((int64_t)1 << 31) || !at_multiple(X, 16) || !at_multiple(Y, 2)) return NESTEDFP_ERR_SHAPE;
    if (residual != nullptr && (ldr < e.hidden || ldr > ((int64_t)1 << 31) || !at_multiple(residual, 2))) return NESTEDFP_ERR_SHAPE;
    for (const void *w : {e.up_upper, e.down_upper, nested ? e.up_lower : e.up_upper, nested ? e.down_lower : e.down_upper})
        if (!at_multiple(w, 16)) return NESTEDFP_ERR_SHAPE;
    if (!at_multiple(ids, 4) || !at_multiple(weights, 4)) return NESTEDFP_ERR_SHAPE;
    const size_t need = kCounterBytes + experts_workspace_bytes(e.experts, e.hidden, e.ffn, M, top_k);
    if (workspace == nullptr || workspace_bytes < need || !at_multiple(workspace, 16)) return NESTEDFP_ERR_WORKSPACE;
    ExpertArgs a;
    memset(&a, 0, sizeof(a));
    a.X = X;  a.ldx = ldx;  a.M = M;  a.K = e.hidden;  a.ffn = e.ffn;
    a.up0 = static_cast<const uint8_t *>(e.up_upper);
    a.up1 = nested ? static_cast<const uint8_t *>(e.up_lower) : a.up0;
    a.down0 = static_cast<const uint8_t *>(e.down_upper);
    a.down1 = nested ? static_cast<const uint8_t *>(e.down_lower) : a.down0;
    a.ids = ids;  a.weights = weights;  a.residual = residual;  a.ldr = ldr;  a.Y = Y;  a.ldy = ldy;
    a.counters = static_cast<uint32_t *>(workspace);
    a.experts = (int32_t)e.experts;  a.top_k = (int32_t)top_k;  a.act = e.activation;
    a.vec = ((ldr & 3) == 0 && at_multiple(residual, 8) ? 1 : 0) | ((ldy & 3) == 0 && at_multiple(Y, 8) ? 2 : 0);
    return launch_experts_layer(e.is_exception ? kPlainF16 : (nested ? kNestedF16Row : kE4M3Row), a,
                                static_cast<uint8_t *>(workspace) + kCounterBytes, static_cast<hipStream_t>(stream));
}

}  // extern "C"
