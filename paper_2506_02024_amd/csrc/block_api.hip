// C ABI of what stands around a layer's linears (norm, rotary cache write, paged attention): argument validation, workspace
// layout and dispatch.  See include/nestedfp.h for the contract of every entry point.
#include "../../include/nestedfp.h"
#include "nfp_host.h"

#include <math.h>

namespace nfp {

static inline bool on(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMaxWidth = (int64_t)1 << 21;        // columns of a row
constexpr int64_t kMaxRows = 0x3fffffff;
constexpr int64_t kMaxStride = (int64_t)1 << 31;

// a matrix of `cols` 16-bit columns
static int check_rows(const void *p, int64_t cols, int64_t ld, uintptr_t alignment = 16) {
    if (p == nullptr) return kErrArg;
    return ld < cols || ld > kMaxStride || (ld & 7) != 0 || !on(p, alignment) ? kErrShape : kOk;
}

static int check_cache(const nestedfp_kv_cache *c) {
    if (c == nullptr || c->pages < 0 || c->kv_heads <= 0) return kErrArg;
    if (c->type != NESTEDFP_CACHE_FP16 && c->type != NESTEDFP_CACHE_E4M3) return kErrArg;
    const int p = c->page_tokens, d = c->head_dim;
    if (p < 16 || p > 256 || (p & (p - 1)) != 0 || (d != 64 && d != 96 && d != 128 && d != 256)) return kErrShape;
    if (c->pages > 0x7fffffff / p || c->kv_heads > 65535 || c->pages * p >= ((int64_t)1 << 35) / c->kv_heads) return kErrShape;
    return kOk;
}

// what the kernels need in memory
static int check_storage(const nestedfp_kv_cache *c) {
    if (c->k == nullptr || c->v == nullptr) return kErrArg;
    if (c->type == NESTEDFP_CACHE_FP16 && (c->k_scale != nullptr || c->v_scale != nullptr)) return kErrArg;      // (nothing multiplies by them)
    return on(c->k, 16) && on(c->v, 16) && on(c->k_scale, 4) && on(c->v_scale, 4) ? kOk : kErrShape;
}

static int page_shift(const nestedfp_kv_cache *c) {
    int shift = 0;
    while ((16 << shift) < c->page_tokens) ++shift;
    return shift;
}

// The shape of a paged attention; kErrArg, kErrShape for one that there is no launch for.
static int attention_shape(int64_t tokens, int64_t batch, int64_t heads, const nestedfp_kv_cache *c, int64_t max_new,
                           int64_t max_len, int64_t window, int64_t sinks, AttentionShape &s) {
    if (tokens < 0 || batch < 0 || heads <= 0 || max_new < 0 || max_len < 0 || window < 0 || sinks < 0) return kErrArg;
    const int st = check_cache(c);
    if (st != kOk) return st;
    if (heads % c->kv_heads != 0 || heads > 65535) return kErrShape;
    // (rows of a sequence, new tokens times heads, are counted in 31 bits)
    if (tokens > kMaxRows / heads || batch > 0xfffff || max_len > 0x7fffffff - 256) return kErrShape;
    s.tokens = tokens;
    s.batch = batch;
    s.kv_heads = c->kv_heads;
    s.group = heads / c->kv_heads;
    s.D = c->head_dim;
    s.max_new = max_new < tokens ? max_new : tokens;
    s.max_len = max_len;
    // (a window that reaches further than any sequence is none)
    s.window = window < 0x7fffffff ? window : 0;
    s.sinks = sinks < 0x7ffffff0 ? sinks : 0x7ffffff0;
    s.fp8 = c->type == NESTEDFP_CACHE_E4M3;
    s.ragged = tokens != batch * s.max_new;                          // (else every sequence has max_new)
    return kOk;
}

}  // namespace nfp

using namespace nfp;

extern "C" {

int nestedfp_add_rms_norm(const uint16_t *X, int64_t M, int64_t K, int64_t ldx, const uint16_t *residual, int64_t ldr,
                          const uint16_t *weight, float eps, uint16_t *sum, int64_t lds, uint16_t *Y, int64_t ldy,
                          uint8_t *Xq, float *scales, void *stream) {
    if (M < 0 || K <= 0 || !(eps >= 0.0f) || isinf(eps)) return NESTEDFP_ERR_ARG;
    if ((K & 15) != 0 || K > kMaxWidth || M > kMaxRows) return NESTEDFP_ERR_SHAPE;
    if (M == 0) return NESTEDFP_OK;
    if (weight == nullptr || (Y == nullptr && Xq == nullptr) || (Xq != nullptr && scales == nullptr)) return NESTEDFP_ERR_ARG;
    int st = check_rows(X, K, ldx);
    if (st == kOk && residual != nullptr) st = check_rows(residual, K, ldr);
    if (st == kOk && sum != nullptr) st = check_rows(sum, K, lds);
    if (st == kOk && Y != nullptr) st = check_rows(Y, K, ldy);
    if (st != kOk) return st;
    if (!on(weight, 16) || !on(Xq, 16) || !on(scales, 4)) return NESTEDFP_ERR_SHAPE;
    NormArgs a;
    a.X = X;  a.ldx = ldx;  a.R = residual;  a.ldr = ldr;  a.weight = weight;  a.eps = eps;  a.K = K;
    a.sum = sum;  a.lds = lds;  a.Y = Y;  a.ldy = ldy;  a.Xq = Xq;  a.scales = scales;
    return launch_add_rms_norm(a, M, static_cast<hipStream_t>(stream));
}

size_t nestedfp_kv_cache_bytes(const nestedfp_kv_cache *c) {
    if (check_cache(c) != kOk) return 0;
    return (size_t)c->pages * (size_t)c->page_tokens * (size_t)c->kv_heads * (size_t)c->head_dim *
           (c->type == NESTEDFP_CACHE_FP16 ? 2 : 1);
}

int nestedfp_rope_append(const uint16_t *Q, int64_t ldq, const uint16_t *K, int64_t ldk, const uint16_t *V, int64_t ldv,
                         int64_t M, int64_t heads, const float *cos_table, const float *sin_table, int64_t max_positions,
                         int64_t rotary_dim, const int32_t *positions, const int32_t *slots, uint16_t *Qout, int64_t ldqo,
                         const nestedfp_kv_cache *c, void *stream) {
    if (M < 0 || heads <= 0 || rotary_dim < 0 || max_positions < 0) return NESTEDFP_ERR_ARG;
    int st = check_cache(c);
    if (st != kOk) return st;
    if (heads % c->kv_heads != 0 || heads + 2 * (int64_t)c->kv_heads > 65535 || M > kMaxRows) return NESTEDFP_ERR_SHAPE;
    if ((rotary_dim & 15) != 0 || rotary_dim > c->head_dim || max_positions > 0x7fffffff) return NESTEDFP_ERR_SHAPE;
    if (M == 0) return NESTEDFP_OK;
    if (slots == nullptr || (rotary_dim > 0 && (positions == nullptr || cos_table == nullptr || sin_table == nullptr))) return NESTEDFP_ERR_ARG;
    const int64_t q_cols = heads * c->head_dim, kv_cols = (int64_t)c->kv_heads * c->head_dim;
    if ((st = check_rows(Q, q_cols, ldq)) != kOk || (st = check_rows(K, kv_cols, ldk)) != kOk || (st = check_rows(V, kv_cols, ldv)) != kOk ||
        (st = check_rows(Qout, q_cols, ldqo)) != kOk || (st = check_storage(c)) != kOk)
        return st;
    if (!on(slots, 4) || !on(positions, 4) || !on(cos_table, 4) || !on(sin_table, 4)) return NESTEDFP_ERR_SHAPE;
    AppendArgs a;
    a.q = Q;  a.new_k = K;  a.new_v = V;  a.ldq = ldq;  a.ldk = ldk;  a.ldv = ldv;  a.M = M;
    a.cos = cos_table;  a.sin = sin_table;  a.positions = positions;  a.slots = slots;
    a.positions_known = (int32_t)max_positions;  a.slot_count = (int32_t)(c->pages * c->page_tokens);
    a.out = Qout;  a.ldo = ldqo;
    a.k = static_cast<uint8_t *>(c->k);  a.v = static_cast<uint8_t *>(c->v);  a.k_scale = c->k_scale;  a.v_scale = c->v_scale;
    a.heads = (int32_t)heads;  a.kv_heads = c->kv_heads;  a.D = c->head_dim;  a.rotary = (int32_t)rotary_dim;
    a.page_shift = page_shift(c);  a.fp8 = c->type == NESTEDFP_CACHE_E4M3;
    a.group = 0;
    return launch_rope_append(a, static_cast<hipStream_t>(stream));
}

size_t nestedfp_paged_attention_workspace_size(int64_t tokens, int64_t batch, int64_t heads, const nestedfp_kv_cache *c,
                                               int64_t max_new, int64_t max_len, int64_t window, int64_t sinks) {
    AttentionShape s;
    if (attention_shape(tokens, batch, heads, c, max_new, max_len, window, sinks, s) != kOk) return 0;
    if (tokens == 0 || batch == 0 || s.max_new == 0) return 0;
    const size_t bytes = attention_plan(s).partial_bytes;
    return bytes > 0 ? kCounterBytes + round256(bytes) : 0;
}

int nestedfp_paged_attention(const uint16_t *Q, int64_t tokens, int64_t ldq, int64_t heads, const nestedfp_kv_cache *c,
                             const int32_t *table, int64_t ld_table, int64_t table_columns, const int32_t *lens,
                             int64_t batch, const int32_t *starts, int64_t max_new, int64_t max_len, float scale,
                             int64_t window, int64_t sinks, uint16_t *O, int64_t ldo, void *workspace,
                             size_t workspace_bytes, void *stream) {
    AttentionShape s;
    int st = attention_shape(tokens, batch, heads, c, max_new, max_len, window, sinks, s);
    if (st != kOk) return st;
    if (table_columns < 0 || ld_table < table_columns || table_columns > 0x7fffffff || !(fabsf(scale) < INFINITY)) return NESTEDFP_ERR_ARG;
    if (tokens == 0) return NESTEDFP_OK;
    if (batch == 0 || s.max_new == 0) return NESTEDFP_ERR_ARG;            // new tokens of no sequence
    if (lens == nullptr || (table == nullptr && table_columns > 0)) return NESTEDFP_ERR_ARG;
    if (starts == nullptr && (tokens % batch != 0 || tokens / batch > s.max_new)) return NESTEDFP_ERR_ARG;
    const int64_t cols = heads * c->head_dim;
    if ((st = check_rows(Q, cols, ldq)) != kOk || (st = check_rows(O, cols, ldo, 8)) != kOk || (st = check_storage(c)) != kOk) return st;
    if (!on(table, 4) || !on(lens, 4) || !on(starts, 4)) return NESTEDFP_ERR_SHAPE;
    const AttentionPlan plan = attention_plan(s);
    AttentionArgs a;
    a.partials = nullptr;  a.counters = nullptr;
    if (plan.partial_bytes > 0) {
        if (workspace == nullptr || workspace_bytes < kCounterBytes + round256(plan.partial_bytes) || !on(workspace, 16)) return NESTEDFP_ERR_WORKSPACE;
        a.counters = static_cast<uint32_t *>(workspace);
        a.partials = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + kCounterBytes);
    }
    a.Q = Q;  a.ldq = ldq;  a.O = O;  a.ldo = ldo;
    a.k = static_cast<const uint8_t *>(c->k);  a.v = static_cast<const uint8_t *>(c->v);  a.k_scale = c->k_scale;  a.v_scale = c->v_scale;
    a.table = table;  a.ld_table = ld_table;  a.columns = (int32_t)table_columns;  a.lens = lens;  a.starts = starts;
    a.scale = scale;
    a.tokens = (int32_t)tokens;  a.batch = (int32_t)batch;  a.per = (int32_t)(tokens / batch);  a.max_new = (int32_t)s.max_new;
    a.kv_heads = c->kv_heads;  a.group = (int32_t)s.group;  a.pages = (int32_t)c->pages;  a.page_shift = page_shift(c);
    a.window = (int32_t)s.window;  a.sinks = (int32_t)s.sinks;
    return launch_attention(s, plan, a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
