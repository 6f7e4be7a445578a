// A mixture of experts on a few tokens (1 ... 64), in two launches: gate and up products with the activation, down products with the
// weighted sum.  Bound by the bytes of the experts that the tokens have chosen; everything here is arranged around streaming
// those once.  Which experts these are the kernels find out themselves from the tokens' choices, which lie in device memory.
//
// As in the streaming linears, weight rows are the MFMA's first operand (row-major, fetched in pieces of 16 rows x 128 bytes and
// regrouped through 2 KB of LDS per wave) and tokens the second; activations are FP16 in both modes.  FP8 mode expands the upper
// plane's bytes to FP16 (weight times 1, exactly: see expand16), because with so few tokens only the weights' bytes count and E4M3
// activations would cost accuracy and a pass over them for nothing.
#include <algorithm>

#include "gemm_small_kernels.h"

namespace nfp {

constexpr int kNone = 255;                             // a token that has not chosen the expert
// The activated products between the two launches are kept as two FP16 terms, h = high + low: rounded to one, their error is as large as the
// output's own rounding.
constexpr int kTerms = 2;

// E4M3 bytes as FP16 words: sign, four bits of exponent and three of mantissa at the same places below FP16's exponent MSB read as the value times
// 2^-8 (subnormals too), which is the weight that the upper plane stands for (Sec. 4.1).
__device__ __forceinline__ uint32_t expand2(uint32_t u, uint32_t sel) {
    const uint32_t x = byte_perm(0u, u, sel);          // the bytes in the upper halves of the words
    return (x & 0x80008000u) | ((x >> 1) & 0x3f803f80u);
}
__device__ __forceinline__ void expand16(const u32x4 &u, u32x4 &lo, u32x4 &hi) {
    constexpr uint32_t first = 0x010c000cu, second = 0x030c020cu;      // (selector 12: a zero byte)
    lo = u32x4{expand2(u.x, first), expand2(u.x, second), expand2(u.y, first), expand2(u.y, second)};
    hi = u32x4{expand2(u.z, first), expand2(u.z, second), expand2(u.w, first), expand2(u.w, second)};
}

// Kinds: kNestedF16Row (FP16 mode), kE4M3Row (FP8 mode, the upper plane), kPlainF16 (weights that are kept in FP16).
template <int KIND, int STEPS, int POL>
__device__ __forceinline__ void load_pieces(WItem (&w)[STEPS], __amdgpu_buffer_rsrc_t r0, __amdgpu_buffer_rsrc_t r1, uint32_t lo,
                                            uint32_t hi, const bool (&kv)[STEPS]) {
    if constexpr (KIND == kE4M3Row) {
#pragma unroll
        for (int q = 0; q < STEPS / 2; ++q) {
            w[2 * q].a = __builtin_amdgcn_raw_buffer_load_b128(r0, (kv[q] ? lo : kDead) + q * 128, 0, POL);
            w[2 * q + 1].a = __builtin_amdgcn_raw_buffer_load_b128(r0, (kv[q] ? hi : kDead) + q * 128, 0, POL);
        }
    } else {
        load_rows<KIND, STEPS, POL>(w, r0, r1, lo, hi, kv);
    }
}
// pieces into operand order
template <int KIND, int STEPS>
__device__ __forceinline__ void regroup_pieces(WItem (&w)[STEPS], const Regroup<KIND == kPlainF16> &rw) {
    if constexpr (KIND == kPlainF16) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) rw.run(w[s].a, w[s].b);
    } else {
#pragma unroll
        for (int s = 0; s < STEPS; s += 2) rw.run(w[s].a, w[s + 1].a);
        if constexpr (KIND == kNestedF16Row) {
#pragma unroll
            for (int s = 0; s < STEPS; s += 2) rw.run(w[s].b, w[s + 1].b);
        }
    }
}
template <int KIND>
__device__ __forceinline__ void operand(const WItem &w, u32x4 &lo, u32x4 &hi) {
    if constexpr (KIND == kNestedF16Row) merge16(w.a, w.b, lo, hi);
    else if constexpr (KIND == kE4M3Row) expand16(w.a, lo, hi);
    else { lo = w.a;  hi = w.b; }
}

// Who has chosen whom, worked out by every workgroup from the ids (a few thousand at most): the experts that any token has chosen, in rising order, and
// for each the place of every token's choice, kNone without one.  A token that names an expert twice has one place, with the sum of both
// weights.  Ids outside the experts are nobody's.
struct Choices {
    uint16_t *rank;                                    // [experts] place among the chosen ones
    uint16_t *chosen;                                  // [chosen] the experts
    uint32_t *units;                                   // [chosen + 1] running sum of the experts' work (up kernel)
    int16_t *ids;                                      // [tokens * top_k]
    float *weights;                                    // the same (down kernel)
    uint8_t *place;                                    // [chosen][tokens_padded]
    int count, padded;
};
constexpr int kMostExperts = 512, kMostTokens = 64, kMostTop = 32;
static inline size_t choices_bytes(const ExpertArgs &a) {
    const size_t chosen = (size_t)std::min<int64_t>(a.experts, a.M * a.top_k), padded = (size_t)((a.M + 15) & ~(int64_t)15), n = (size_t)(a.M * a.top_k);
    return ((a.experts * 2 + 15) & ~(size_t)15) + ((chosen * 2 + 15) & ~(size_t)15) + ((chosen * 4 + 4 + 15) & ~(size_t)15) + ((n * 2 + 15) & ~(size_t)15) +
           ((n * 4 + 15) & ~(size_t)15) + chosen * padded;
}

__device__ __forceinline__ Choices choices_of(const ExpertArgs &a, uint8_t *at, bool want_weights) {
    const int n = (int)(a.M * a.top_k), chosen = min((int)a.experts, n);
    const int t = threadIdx.x, threads = blockDim.x, lane = t & 63;
    Choices c;
    c.padded = ((int)a.M + 15) & ~15;
    auto take = [&](int bytes) {
        uint8_t *p = at;
        at += (bytes + 15) & ~15;
        return p;
    };
    c.rank = reinterpret_cast<uint16_t *>(take((int)a.experts * 2));
    c.chosen = reinterpret_cast<uint16_t *>(take(chosen * 2));
    c.units = reinterpret_cast<uint32_t *>(take(chosen * 4 + 4));
    c.ids = reinterpret_cast<int16_t *>(take(n * 2));
    c.weights = reinterpret_cast<float *>(take(n * 4));
    c.place = at;
    for (int i = t; i < a.experts; i += threads) c.rank[i] = 0;
    for (int i = t; i < chosen * c.padded / 4; i += threads) reinterpret_cast<uint32_t *>(c.place)[i] = 0xffffffffu;
    __syncthreads();
    for (int i = t; i < n; i += threads) {
        const int e = a.ids[i];
        const bool ok = e >= 0 && e < a.experts;
        c.ids[i] = (int16_t)(ok ? e : -1);
        if (ok) c.rank[e] = 1;
        if (want_weights) c.weights[i] = a.weights[i];
    }
    __syncthreads();
    // (every wave counts by itself; the first one writes)
    int count = 0;
    for (int base = 0; base < a.experts; base += 64) {
        const bool in = base + lane < a.experts && c.rank[min(base + lane, (int)a.experts - 1)] != 0;
        const uint64_t mask = __ballot(in);
        if (t < 64 && in) c.chosen[count + __popcll(mask & ((1ull << lane) - 1))] = (uint16_t)(base + lane);
        count += __popcll(mask);
    }
    c.count = count;
    __syncthreads();
    for (int i = t; i < count; i += threads) c.rank[c.chosen[i]] = (uint16_t)i;
    __syncthreads();
    if (t < a.M) {                                     // (at most 64 tokens: lanes of the first wave)
        const int16_t *const mine = c.ids + t * a.top_k;
        for (int j = (int)a.top_k - 1; j >= 0; --j)
            if (mine[j] >= 0) c.place[c.rank[mine[j]] * c.padded + t] = (uint8_t)j;
        if (want_weights)
            for (int j = 1; j < a.top_k; ++j)
                if (mine[j] >= 0) {
                    const int first = c.place[c.rank[mine[j]] * c.padded + t];
                    if (first != j) c.weights[t * a.top_k + first] += c.weights[t * a.top_k + j];
                }
    }
    __syncthreads();
    return c;
}

__device__ __forceinline__ void lds_barrier() {
    // (loads from memory stay in flight, which the compiler's barrier would wait for)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// ---- gate and up products --------------------------------------------------------------------------
// The weight rows of an expert are gate and up rows in turn, so that a lane's four sums of a 16-row tile are two gated pairs.  A unit of work is two
// such tiles (16 columns of ffn) for one expert and up to 16 MT of its tokens; all units stand in one row, expert by expert, and every
// workgroup takes an equal stretch.  Its waves share K (slices of SPW steps of 64 columns, in several passes where K is longer) and keep the
// tokens of their slice in registers; tile t + 1 is loaded while tile t is multiplied, across units and experts; sums meet in
// LDS, one barrier per unit.
// Up to 16 tokens stand in the columns as they are (`gather` 0), and are loaded once.  Of more tokens the columns are those that have chosen
// the expert, loaded anew with every expert, so that 48 tokens over many experts take the time of a few.
// (with four token tiles the sums of one unit are all that the LDS has room for: a second barrier)
template <int MT> constexpr int kSumRegions = MT == 4 ? 1 : 2;
template <int KIND, int MT, int SPW, bool PASSES, int POL>
__global__ void __launch_bounds__(MT == 1 && !PASSES ? 1024 : 512)
experts_up_kernel(ExpertArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t shared[];
    constexpr int KSTEP = 64, EB = kind_elem_bytes(KIND), PIECES = row_pieces<KIND == kPlainF16 ? kPlainF16 : kNestedF16Row, SPW>();
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int g = lane >> 4, r16 = lane & 15;
    constexpr int SUMS = kSumRegions<MT> * 2 * MT * 1024;      // bytes of sums per wave
    floatx4 *const slots = reinterpret_cast<floatx4 *>(shared);                // [regions][2 tiles][wave][MT][64]
    const uint32_t own = (uint32_t)(waves * SUMS + wave * 2048);
    uint8_t *const list = shared + waves * (SUMS + 2048) + wave * 64;          // the columns' tokens
    const Choices c = choices_of(a, shared + waves * (SUMS + 2048 + 64), false);
    const int per_expert = (int)(a.ffn >> 4);
    // the running sum of the units: one chunk of columns for every 16 MT tokens
    if (threadIdx.x < 64) {
        uint32_t sum = 0;
        for (int base = 0; base < c.count; base += 64) {
            const int r = base + lane;
            uint32_t tokens = c.padded;                // (places are below 128)
            if (a.gather && r < c.count)
                for (int q = 0; q < c.padded / 4; ++q) tokens -= __popc(reinterpret_cast<const uint32_t *>(c.place + r * c.padded)[q] & 0x80808080u);
            uint32_t mine = r < c.count ? (a.gather ? (tokens + 16 * MT - 1) / (16 * MT) : 1u) * (uint32_t)per_expert : 0u;
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t before = __shfl_up(mine, d);
                if (lane >= d) mine += before;
            }
            if (r < c.count) c.units[r + 1] = sum + mine;
            sum += __shfl(mine, 63);
        }
        if (lane == 0) c.units[0] = 0;
    }
    __syncthreads();
    const uint32_t total = c.units[c.count];
    const uint32_t first = (uint32_t)((uint64_t)total * blockIdx.x / gridDim.x), end = (uint32_t)((uint64_t)total * (blockIdx.x + 1) / gridDim.x);
    if (first >= end) return;
    // Where a unit lies: the expert's place among the chosen ones, the chunk of its tokens, the columns of ffn.
    struct At { int r, chunk, f; };
    At at = {0, 0, 0};
    for (int base = 0; base < c.count; base += 64)
        at.r += __popcll(__ballot(base + lane < c.count && c.units[min(base + lane, c.count - 1) + 1] <= first));
    at.r = __builtin_amdgcn_readfirstlane(at.r);
    {
        const uint32_t inside = first - c.units[at.r];
        at.chunk = __builtin_amdgcn_readfirstlane(inside / (uint32_t)per_expert);
        at.f = __builtin_amdgcn_readfirstlane((int)(inside - (uint32_t)at.chunk * (uint32_t)per_expert));
    }
    auto step = [&](At &x) {
        if (++x.f < per_expert) return;
        x.f = 0;
        ++x.chunk;
        const uint32_t of = __builtin_amdgcn_readfirstlane(c.units[x.r + 1] - c.units[x.r]);
        if ((uint32_t)x.chunk * (uint32_t)per_expert >= of) { x.chunk = 0;  ++x.r; }
    };

    const uint32_t row_bytes = (uint32_t)a.K * EB;
    const int64_t expert_bytes = 2 * a.ffn * (int64_t)row_bytes;
    // (rows of a multiple of 4 KB put the 16 rows of a slice on the same memory channels: the slices are rotated from workgroup to workgroup)
    const int ks = a.rotate ? (int)((wave + (blockIdx.x >> 3) * 5u) % (unsigned)waves) : wave;
    const Regroup<true> rx(shared, own, lane);
    const Regroup<KIND == kPlainF16> rw(shared, own, lane);
    u32x4 xa[SPW][MT], xb[SPW][MT];
    int row[MT];                                       // the column's row of the products between the launches, or -1
    uint32_t x_a[MT], x_b[MT];                         // where the activations lie that the lane loads: rows 0 .. 7, 8 .. 15 of the columns
    const __amdgpu_buffer_rsrc_t rsx = weight_rsrc(reinterpret_cast<const uint8_t *>(a.X), (uint32_t)(((a.M - 1) * a.ldx + a.K) * 2));
    auto x_at = [&](int token, int l) { return token >= 0 ? (uint32_t)token * (uint32_t)(2 * a.ldx) + (l & 7) * 16u : kDead; };
    int k_slice = 0;
    auto k_of = [&](int pass) { return (pass * waves + ks) * (SPW * KSTEP); };

    auto columns = [&](const At &x) {
        const uint8_t *const place = c.place + x.r * c.padded;
        int l = lane;                                  // (what follows from the lane is worked out anew: kept across the loop it costs registers that are spilled)
        asm volatile("" : "+v"(l));
        const int col = l & 15;
        if (!a.gather) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int m = 16 * i + col, p = m < a.M ? place[m] : kNone;
                row[i] = p == kNone ? -1 : m * (int)a.top_k + p;
            }
            return;
        }
        const bool in = l < a.M && place[min(l, (int)a.M - 1)] != kNone;
        const uint64_t mask = __ballot(in);
        const int n = __popcll(mask);
        if (in) list[__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = (uint8_t)l;
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int at0 = 16 * (x.chunk * MT + i);
            auto token = [&](int q) { return q < n ? (int)list[min(q, 63)] : -1; };
            const int m = token(at0 + col);
            row[i] = m < 0 ? -1 : m * (int)a.top_k + place[m];
            x_a[i] = x_at(token(at0 + (l >> 3)), l);
            x_b[i] = x_at(token(at0 + 8 + (l >> 3)), l);
        }
        asm volatile("" ::: "memory");
    };
    auto load_tokens = [&](int pass) {
        const int k0 = k_of(pass);
#pragma unroll
        for (int s = 0; s < SPW; ++s)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const bool in = k0 + s * KSTEP + (lane & 7) * 8 < a.K;
                xa[s][i] = __builtin_amdgcn_raw_buffer_load_b128(rsx, (in ? x_a[i] + 2u * k0 : kDead) + 2 * KSTEP * s, 0, 0);
                xb[s][i] = __builtin_amdgcn_raw_buffer_load_b128(rsx, (in ? x_b[i] + 2u * k0 : kDead) + 2 * KSTEP * s, 0, 0);
            }
#pragma unroll
        for (int s = 0; s < SPW; ++s)
#pragma unroll
            for (int i = 0; i < MT; ++i) rx.run(xa[s][i], xb[s][i]);
    };
    auto fetch = [&](WItem (&w)[SPW], const At &x, int tile, int pass, bool live) {
        const int64_t base = live ? (int64_t)c.chosen[x.r] * expert_bytes : 0;
        const int64_t off = ((int64_t)__builtin_amdgcn_readfirstlane((int)(base >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)base);
        const __amdgpu_buffer_rsrc_t r0 = weight_rsrc(a.up0 + off, (uint32_t)expert_bytes);
        const __amdgpu_buffer_rsrc_t r1 = weight_rsrc(KIND == kNestedF16Row ? a.up1 + off : a.up0 + off, (uint32_t)expert_bytes);
        const int kb = k_of(pass) * EB + (lane & 7) * 16;
        const uint32_t lo = live ? (uint32_t)((2 * x.f + tile) * 16 + (lane >> 3)) * row_bytes + (uint32_t)kb : kDead;
        bool kv[SPW];
#pragma unroll
        for (int q = 0; q < SPW; ++q) kv[q] = q < PIECES && kb + 128 * q < a.K * EB;
        load_pieces<KIND, SPW, POL>(w, r0, r1, lo, lo + 8u * row_bytes, kv);
    };
    int region = 0;
    auto consume = [&](WItem (&w)[SPW], int tile, int pass) {
        floatx4 *const slot = slots + ((region * 2 + tile) * waves + ks) * MT * 64 + lane;
        floatx4 sum[MT];
        regroup_pieces<KIND, SPW>(w, rw);
#pragma unroll
        for (int i = 0; i < MT; ++i) sum[i] = PASSES && pass > 0 ? slot[i * 64] : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < SPW; ++s) {
            u32x4 w_lo, w_hi;
            operand<KIND>(w[s], w_lo, w_hi);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half8(w_lo), as_half8(xa[s][i]), sum[i], 0, 0, 0);
                sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half8(w_hi), as_half8(xb[s][i]), sum[i], 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) slot[i * 64] = sum[i];
    };

    if (!a.gather) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            x_a[i] = x_at(16 * i + (lane >> 3) < a.M ? 16 * i + (lane >> 3) : -1, lane);
            x_b[i] = x_at(16 * i + 8 + (lane >> 3) < a.M ? 16 * i + 8 + (lane >> 3) : -1, lane);
        }
    }
    WItem buf0[SPW], buf1[SPW];
    const int passes = PASSES ? a.passes : 1;
    columns(at);
    fetch(buf0, at, 0, 0, true);
    load_tokens(0);
    for (uint32_t u = first; u < end; ++u) {
        At next = at;
        step(next);
        for (int pass = 0; pass < passes; ++pass) {
            if (PASSES && (pass > 0 || u > first)) load_tokens(pass);
            fetch(buf1, at, 1, pass, true);
            __builtin_amdgcn_sched_barrier(0);
            consume(buf0, 0, pass);
            __builtin_amdgcn_sched_barrier(0);
            if (pass + 1 < passes) fetch(buf0, at, 0, pass + 1, true);
            else fetch(buf0, next, 0, 0, u + 1 < end);
            __builtin_amdgcn_sched_barrier(0);
            consume(buf1, 1, pass);
            __builtin_amdgcn_sched_barrier(0);
        }
        lds_barrier();
        // The waves take turns with the sums.  (They are written again two units later, behind the next barrier.)
        for (int item = 0; item < 2 * MT; ++item) {
            if ((int)((u * (2 * MT) + item) % (unsigned)waves) != wave) continue;
            const int t = item / MT, i = item - t * MT;
            floatx4 sum = slots[(((region * 2 + t) * waves) * MT + i) * 64 + lane];
#pragma unroll 4
            for (int w = 1; w < waves; ++w) {
                const floatx4 v = slots[(((region * 2 + t) * waves + w) * MT + i) * 64 + lane];
                sum.x += v.x;  sum.y += v.y;  sum.z += v.z;  sum.w += v.w;
            }
            int to = row[0];
#pragma unroll
            for (int q = 1; q < MT; ++q) to = i == q ? row[q] : to;
            if (to < 0) continue;
            const float h0 = activate(sum.x, a.act) * sum.y, h1 = activate(sum.z, a.act) * sum.w;
            const int f = 16 * at.f + 8 * t + 2 * g;
            uint16_t *const dst = a.H + (int64_t)to * kTerms * a.ffn + f;
            const uint32_t high = float2_to_half2_bits(h0, h1);
            *reinterpret_cast<uint32_t *>(dst) = high;
            if constexpr (kTerms == 2) {
                // (an infinite first term has no rest)
                const float l0 = h0 - half_bits_to_float(high & 0xffffu), l1 = h1 - half_bits_to_float(high >> 16);
                *reinterpret_cast<uint32_t *>(dst + a.ffn) =
                    float2_to_half2_bits((high & 0x7fffu) == 0x7c00u ? 0.0f : l0, (high & 0x7fff0000u) == 0x7c000000u ? 0.0f : l1);
            }
        }
        if constexpr (kSumRegions<MT> == 2) region ^= 1;
        else lds_barrier();
        if (u + 1 < end && (next.r != at.r || next.chunk != at.chunk)) {
            columns(next);
            if (!PASSES && a.gather) load_tokens(0);
        }
        at = next;
    }
}

// ---- down products ---------------------------------------------------------------------------------
// A workgroup owns 16 rows of the output for all tokens and walks over all chosen experts, so that the sum over a token's experts stays in its
// registers: no second pass, no order that depends on timing.  Work is cut into items of 128 columns of one expert; wave w takes items
// w, w + 8, ...; weights are loaded DEPTH items ahead, the activated products (from L2) where they are used.  Columns are the tokens as they are; a
// token tile that has not chosen the expert is skipped.
template <int KIND, int MT, int POL>
__global__ void __launch_bounds__(512)
experts_down_kernel(ExpertArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t shared[];
    constexpr int EB = kind_elem_bytes(KIND), DEPTH = KIND == kE4M3Row ? 4 : 3, PIECES = KIND == kPlainF16 ? 2 : 1;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int g = lane >> 4, r16 = lane & 15;
    floatx4 *const slots = reinterpret_cast<floatx4 *>(shared);                // [wave][MT][64]
    const uint32_t own = (uint32_t)(waves * MT * 1024 + wave * 2048);
    const Choices c = choices_of(a, shared + waves * (MT * 1024 + 2048), true);
    const Regroup<KIND == kPlainF16> rw(shared, own, lane);
    const uint32_t row_bytes = (uint32_t)a.ffn * EB;
    const int64_t expert_bytes = a.K * (int64_t)row_bytes;
    const int per_expert = (int)((a.ffn + 127) >> 7);
    struct At { int r, q; };
    auto forward = [&](At &x, int by) {
        x.q += by;
        while (x.q >= per_expert) { x.q -= per_expert;  ++x.r; }
    };
    WItem buf[DEPTH][2];
    auto fetch = [&](WItem (&w)[2], const At &x) {
        const bool live = x.r < c.count;
        const int64_t base = live ? (int64_t)c.chosen[x.r] * expert_bytes : 0;
        const int64_t off = ((int64_t)__builtin_amdgcn_readfirstlane((int)(base >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)base);
        const __amdgpu_buffer_rsrc_t r0 = weight_rsrc(a.down0 + off, (uint32_t)expert_bytes);
        const __amdgpu_buffer_rsrc_t r1 = weight_rsrc(KIND == kNestedF16Row ? a.down1 + off : a.down0 + off, (uint32_t)expert_bytes);
        const int kb = x.q * 128 * EB + (lane & 7) * 16;
        const uint32_t lo = live ? (uint32_t)(blockIdx.x * 16 + (lane >> 3)) * row_bytes + (uint32_t)kb : kDead;
        bool kv[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) kv[q] = q < PIECES && kb + 128 * q < a.ffn * EB;
        load_pieces<KIND, 2, POL>(w, r0, r1, lo, lo + 8u * row_bytes, kv);
    };
    floatx4 total[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) total[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto consume = [&](WItem (&w)[2], const At &x) {
        regroup_pieces<KIND, 2>(w, rw);
        u32x4 w_lo[2], w_hi[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) operand<KIND>(w[s], w_lo[s], w_hi[s]);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = 16 * i + r16;
            const int p = m < a.M ? c.place[x.r * c.padded + m] : kNone;
            if (!__any(p != kNone)) continue;
            const int at = m * (int)a.top_k + p;
            floatx4 sum = {0.f, 0.f, 0.f, 0.f};
            const uint16_t *const src = a.H + (int64_t)at * kTerms * a.ffn + x.q * 128 + 16 * g;
            u32x4 h[kTerms][2][2];
#pragma unroll
            for (int term = 0; term < kTerms; ++term)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const bool ok = p != kNone && x.q * 128 + 64 * s + 16 * g < a.ffn;
                    const u32x4 zero = {0u, 0u, 0u, 0u};
                    h[term][s][0] = ok ? *reinterpret_cast<const u32x4 *>(src + term * a.ffn + 64 * s) : zero;
                    h[term][s][1] = ok ? *reinterpret_cast<const u32x4 *>(src + term * a.ffn + 64 * s + 8) : zero;
                }
#pragma unroll
            for (int term = kTerms - 1; term >= 0; --term)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half8(w_lo[s]), as_half8(h[term][s][0]), sum, 0, 0, 0);
                    sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half8(w_hi[s]), as_half8(h[term][s][1]), sum, 0, 0, 0);
                }
            if (p != kNone) {
                const float weight = c.weights[at];
                total[i].x = __builtin_fmaf(weight, sum.x, total[i].x);
                total[i].y = __builtin_fmaf(weight, sum.y, total[i].y);
                total[i].z = __builtin_fmaf(weight, sum.z, total[i].z);
                total[i].w = __builtin_fmaf(weight, sum.w, total[i].w);
            }
        }
    };
    At at = {0, 0}, ahead = {0, 0};
    forward(at, wave);
    ahead = at;
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
        fetch(buf[d], ahead);
        forward(ahead, waves);
    }
    while (at.r < c.count) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (at.r < c.count) consume(buf[d], at);
            __builtin_amdgcn_sched_barrier(0);
            fetch(buf[d], ahead);
            __builtin_amdgcn_sched_barrier(0);
            forward(at, waves);
            forward(ahead, waves);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) slots[(wave * MT + i) * 64 + lane] = total[i];
    __syncthreads();
    for (int i = wave; i < MT; i += waves) {
        floatx4 sum = slots[i * 64 + lane];
        for (int w = 1; w < waves; ++w) {
            const floatx4 v = slots[(w * MT + i) * 64 + lane];
            sum.x += v.x;  sum.y += v.y;  sum.z += v.z;  sum.w += v.w;
        }
        const int m = 16 * i + r16, n = blockIdx.x * 16 + 4 * g;
        if (m >= a.M) continue;
        if (a.residual) {
            const floatx4 r = four_halves(a.residual + (int64_t)m * a.ldr + n, a.vec & 1, 4);
            sum.x += r.x;  sum.y += r.y;  sum.z += r.z;  sum.w += r.w;
        }
        u32x2 o;
        o.x = float2_to_half2_bits(sum.x, sum.y);
        o.y = float2_to_half2_bits(sum.z, sum.w);
        uint16_t *const dst = a.Y + (int64_t)m * a.ldy + n;
        if (a.vec & 2) *reinterpret_cast<u32x2 *>(dst) = o;
        else
#pragma unroll
            for (int q = 0; q < 4; ++q) dst[q] = (uint16_t)((q < 2 ? o.x : o.y) >> (16 * (q & 1)));
    }
}

// ---- host --------------------------------------------------------------------------------------------
size_t experts_product_bytes(int64_t M, int64_t top_k, int64_t ffn) { return (size_t)(M * top_k) * kTerms * (size_t)ffn * 2; }

bool experts_supported(int64_t experts, int64_t hidden, int64_t ffn, int64_t M, int64_t top_k) {
    // an expert's matrix is addressed with 31 bits
    return experts <= kMostExperts && M <= kMostTokens && top_k <= kMostTop && 2 * ffn * hidden * 2 + 64 * std::max(hidden, ffn) < ((int64_t)1 << 31);
}

template <typename Kernel>
static int launch_experts(Kernel kern, std::atomic<bool> &ready, unsigned grid, unsigned threads, size_t lds, const ExpertArgs &a, hipStream_t stream) {
    if (lds > 160 * 1024) return kErrShape;
    if (!ready.load(std::memory_order_acquire)) {
        (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        ready.store(true, std::memory_order_release);
    }
    kern<<<grid, threads, lds, stream>>>(a);
    return hip_ok(hipGetLastError());
}

template <int KIND, int MT, int SPW, int POL>
static int launch_up(ExpertArgs a, hipStream_t stream) {
    const int slices = (int)((a.K + SPW * 64 - 1) / (SPW * 64));
    const int most = MT == 1 && slices <= 16 ? 16 : 8;         // waves, as the registers allow
    a.passes = (slices + most - 1) / most;
    const int waves = (slices + a.passes - 1) / a.passes;
    a.rotate = (a.K * kind_elem_bytes(KIND)) % 4096 == 0 ? 1 : 0;
    const size_t lds = (size_t)waves * (kSumRegions<MT> * 2 * MT * 1024 + 2048 + 64) + choices_bytes(a);
    const int64_t units = std::min<int64_t>(a.experts, a.M * a.top_k) * (a.ffn / 16);
    const int64_t fit = 256 * std::max<int64_t>(1, std::min<int64_t>(16 / waves, (int64_t)(160 * 1024 / lds)));
    static std::atomic<bool> ready{false};
    static std::atomic<bool> ready_passes{false};
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min(units, fit));
    return a.passes > 1 ? launch_experts(experts_up_kernel<KIND, MT, SPW, true, POL>, ready_passes, grid, (unsigned)waves * 64, lds, a, stream)
                        : launch_experts(experts_up_kernel<KIND, MT, SPW, false, POL>, ready, grid, (unsigned)waves * 64, lds, a, stream);
}
template <int KIND, int MT, int POL>
static int launch_down(const ExpertArgs &a, hipStream_t stream) {
    static std::atomic<bool> ready{false};
    return launch_experts(experts_down_kernel<KIND, MT, POL>, ready, (unsigned)(a.K / 16), 512, 8 * (MT * 1024 + 2048) + choices_bytes(a), a, stream);
}

template <int KIND, int POL>
static int launch_kind(const ExpertArgs &a, bool up, hipStream_t stream) {
    if (!up) return a.M <= 16 ? launch_down<KIND, 1, POL>(a, stream) : (a.M <= 32 ? launch_down<KIND, 2, POL>(a, stream) : launch_down<KIND, 4, POL>(a, stream));
    if (a.M <= 16 || 2 * a.M * a.top_k <= 16 * a.experts) return launch_up<KIND, 1, 4, POL>(a, stream);
    return a.M <= 32 || a.M * a.top_k <= 16 * a.experts ? launch_up<KIND, 2, 4, POL>(a, stream) : launch_up<KIND, 4, 2, POL>(a, stream);
}

template <int KIND>
static int launch_lines(const ExpertArgs &a, bool up, hipStream_t stream) {
    const int64_t row = (up ? a.K : a.ffn) * kind_elem_bytes(KIND);
    const uintptr_t at = reinterpret_cast<uintptr_t>(up ? a.up0 : a.down0) | reinterpret_cast<uintptr_t>(up ? a.up1 : a.down1);
    return (row & 127) == 0 && (at & 127) == 0 ? launch_kind<KIND, kStream>(a, up, stream) : launch_kind<KIND, kCached>(a, up, stream);
}

int launch_experts_layer(int kind, ExpertArgs a, hipStream_t stream) {
    a.gather = a.M > 16 ? 1 : 0;
    for (const bool up : {true, false}) {
        const int st = kind == kPlainF16 ? launch_lines<kPlainF16>(a, up, stream)
                                         : (kind == kE4M3Row ? launch_lines<kE4M3Row>(a, up, stream) : launch_lines<kNestedF16Row>(a, up, stream));
        if (st != kOk) return st;
    }
    return kOk;
}

}  // namespace nfp
