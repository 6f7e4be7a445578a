// A mixture of experts on a few tokens (1 ... 64), in two launches of one kernel, gate and up products with the activation and down products, and the weighted sum, of few choices in the second
// launch, of more in a third.  Bound by the bytes of the experts that the tokens have chosen; everything here is arranged around streaming
// those once.  Which experts these are the first launch finds out itself from the tokens' choices, which lie in device memory.
//
// As in the streaming linears, weight rows are the MFMA's first operand (row-major, fetched in pieces of 16 rows x 128 bytes and
// regrouped through 2 KB of LDS per wave) and tokens the second; activations are FP16 in both modes.  FP8 mode expands the upper
// plane's bytes to FP16 (weight times 1, exactly: see expand16), because with so few tokens only the weights' bytes count and E4M3
// activations would cost accuracy and a pass over them for nothing.
#include <algorithm>

#include "gemm_small_kernels.h"

namespace nfp {

// The activated products between the two launches are kept as two FP16 terms, h = high + 2^-11 low: rounded to one, their error is as large as the
// output's own rounding.  The second term is the rest, at most half a step of the first, times 2^11, and so no larger than the first and a normal number wherever 2^-22 of h matters:
// together they are off by 2^-22 of h, by 2^-36 below 2^-14 (where the first term is subnormal).  Unscaled, the rest was subnormal from h = 1/4 down: off by 2^-25, of products of 1e-4 2^-12.5.
// Its products have a sum of their own, multiplied back once.
constexpr int kTerms = 2;
constexpr float kLowScale = 0x1p11f;

// E4M3 bytes as FP16 words: sign, four bits of exponent and three of mantissa at the same places below FP16's exponent MSB read as the value times
// 2^-8 (subnormals too), which is the weight that the upper plane stands for (Sec. 4.1).  (The conversion instruction, two bytes at a time and then a
// place for each word: up products 90.8 us for 91.5, down products 67.4 for 61.7 with 16 tokens and 64 experts of 1408.)
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

constexpr int kMostExperts = 512, kMostTokens = 64, kMostTop = 32;

// ---- who has chosen whom -----------------------------------------------------------------------------
// The experts that any token has chosen, in rising order, and for each the choices that name it, as rows of the products between the launches (token *
// top_k + place), in the tokens' order: workgroups that share a crowded expert have to agree on who is among its first sixteen.  A token that names
// an expert twice counts once, with the sum of both weights.  Ids outside the experts are nobody's.
// One wave of every workgroup of the first launch works this out (a chain of LDS accesses, which a wave's LDS serves in order, without barriers), the
// first workgroup leaves it in the workspace, and the second launch copies it from there.
struct ChoiceHead { uint32_t count, chunks;  uint32_t pad[2]; };      // experts chosen; work of all of them in chunks of 16 MT choices
struct Choices {
    ChoiceHead *head;
    u32x4 *info;                                       // [chosen + 1]: expert, first choice | number << 16, chunks before it
    u32x2 *entry;                                      // [tokens * top_k]: row | token << 16 of the choices, expert by expert
    float *share;                                      // [row] weight
    uint32_t *used;                                    // a bit per row: first choice of an expert there is
    uint8_t *scratch;                                  // first launch
};
static __host__ __device__ __forceinline__ int round16(int bytes) { return (bytes + 15) & ~15; }
static __host__ __device__ __forceinline__ int choice_most(int experts, int n) { return experts < n ? experts : n; }
// bytes that both launches share; the first one's scratch (counts and ranks of the experts, ids, unsorted choices, sizes)
static __host__ __device__ __forceinline__ int choices_shared(int experts, int n) {
    return 16 + 16 * (choice_most(experts, n) + 1) + round16(8 * n) + round16(4 * n) + round16((n + 31) / 32 * 4);
}
static __host__ __device__ __forceinline__ int choices_scratch(int experts, int n) {
    return round16(4 * experts) + 2 * round16(2 * n) + round16(4 * choice_most(experts, n));
}
__device__ __forceinline__ Choices choices_at(uint8_t *at, int experts, int n) {
    Choices c;
    auto take = [&](int bytes) {
        uint8_t *p = at;
        at += round16(bytes);
        return p;
    };
    c.head = reinterpret_cast<ChoiceHead *>(take(16));
    c.info = reinterpret_cast<u32x4 *>(take(16 * (choice_most(experts, n) + 1)));
    c.entry = reinterpret_cast<u32x2 *>(take(8 * n));
    c.share = reinterpret_cast<float *>(take(4 * n));
    c.used = reinterpret_cast<uint32_t *>(take((n + 31) / 32 * 4));
    c.scratch = at;
    return c;
}
// Sum over the lanes before this one, by DPP moves within rows of 16 and from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t add_from(uint32_t v) {
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t &all) {
    uint32_t upto = add_from<0x111, 0xf>(v);           // lane - 1
    upto = add_from<0x112, 0xf>(upto);                 // lane - 2
    upto = add_from<0x114, 0xf>(upto);
    upto = add_from<0x118, 0xf>(upto);
    upto = add_from<0x142, 0xa>(upto);                 // last lane of the row before, rows 1 and 3
    upto = add_from<0x143, 0xc>(upto);                 // lane 31, rows 2 and 3
    all = __builtin_amdgcn_readlane(upto, 63);
    return upto - v;
}
__device__ __forceinline__ int lanes_before(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

__device__ __forceinline__ void find_choices(const ExpertArgs &a, const Choices &c, int lane, int columns, bool shares) {
    const int experts = a.experts, top_k = a.top_k, n = (int)a.M * top_k;
    uint8_t *at = c.scratch;
    uint32_t *const of = reinterpret_cast<uint32_t *>(at);             // choices of an expert; then its place among the chosen ones
    at += round16(4 * experts);
    int16_t *const ids = reinterpret_cast<int16_t *>(at);
    at += round16(2 * n);
    uint16_t *const unsorted = reinterpret_cast<uint16_t *>(at);
    at += round16(2 * n);
    uint32_t *const size = reinterpret_cast<uint32_t *>(at);
    auto ordered = [] { asm volatile("" ::: "memory"); };            // (in program order; the LDS keeps a wave's accesses so)
    const int first_id = lane < n ? a.ids[lane] : -1;
    const float first_share = shares && lane < n ? a.weights[lane] : 0.0f;
    for (int e = lane; e < experts; e += 64) of[e] = 0;
    for (int w = lane; w < (n + 31) / 32; w += 64) c.used[w] = 0;
    ordered();
    for (int i = lane; i < n; i += 64) {
        const int e = i == lane ? first_id : a.ids[i];
        const bool ok = e >= 0 && e < experts;
        ids[i] = (int16_t)(ok ? e : -1);
        unsorted[i] = 0xffff;
        if (ok) atomicAdd(&of[e], 1u);
        if (shares) c.share[i] = i == lane ? first_share : a.weights[i];
    }
    ordered();
    int count = 0;
    uint32_t begin = 0;
    for (int base = 0; base < experts; base += 64) {
        const int e = base + lane;
        const uint32_t own = e < experts ? of[e] : 0u;
        const uint64_t mask = __ballot(own != 0);
        if (mask == 0) continue;
        uint32_t all;
        const uint32_t before = sum_before(own, all);
        if (own != 0) {
            const int r = count + lanes_before(mask);
            c.info[r] = u32x4{(uint32_t)e, begin + before, 0u, 0u};
            size[r] = 0;
            of[e] = (uint32_t)r;
        }
        begin += all;
        count += __popcll(mask);
    }
    ordered();
    for (int i = lane; i < n; i += 64) {
        const int e = ids[i], m = i / top_k, j = i - m * top_k;
        if (e < 0) continue;
        const int16_t *const others = ids + m * top_k;
        bool again = false;
        for (int q = 0; q < j; ++q) again |= others[q] == e;
        if (again) continue;
        if (shares) {                                  // (a choice that repeats an earlier one keeps its weight: only first ones are written)
            float w = c.share[i];
            for (int q = j + 1; q < top_k; ++q)
                if (others[q] == e) w += c.share[m * top_k + q];
            c.share[i] = w;
        }
        const uint32_t r = of[e];
        unsorted[c.info[r].y + atomicAdd(&size[r], 1u)] = (uint16_t)i;
        atomicOr(&c.used[i >> 5], 1u << (i & 31));
    }
    ordered();
    for (int s = lane; s < n; s += 64) {
        const int i = unsorted[s];
        if (i == 0xffff) continue;
        const uint32_t r = of[ids[i]];
        const int start = (int)c.info[r].y, of_r = (int)size[r];
        int place = start;
        for (int q = 0; q < of_r; ++q) place += unsorted[start + q] < i;
        c.entry[place] = u32x2{(uint32_t)i | (uint32_t)(i / top_k) << 16, 0u};
    }
    ordered();
    uint32_t chunks = 0;
    for (int base = 0; base < count; base += 64) {
        const int r = base + lane;
        const uint32_t of_r = r < count ? size[r] : 0u;
        uint32_t all;
        const uint32_t before = sum_before((of_r + columns - 1) / (uint32_t)columns, all);
        if (r < count) {
            const u32x4 v = c.info[r];
            c.info[r] = u32x4{v.x, v.y | of_r << 16, chunks + before, 0u};
        }
        chunks += all;
    }
    if (lane == 0) {
        c.info[count] = u32x4{0u, 0u, chunks, 0u};
        *c.head = ChoiceHead{(uint32_t)count, chunks, {0u, 0u}};
    }
}

__device__ __forceinline__ void lds_barrier() {
    // (loads from memory stay in flight, which the compiler's barrier would wait for)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// ---- the sum over a token's choices -------------------------------------------------------------------
constexpr int kThrough = 1 | 16;                       // sc0 | sc1: every XCD has an L2 of its own
__device__ __forceinline__ __amdgpu_buffer_rsrc_t products_rsrc(const ExpertArgs &a) {
    return weight_rsrc(reinterpret_cast<const uint8_t *>(a.products), (uint32_t)(a.M * a.top_k * a.K * 4));
}
// Four outputs of token m, its choices in their order.
__device__ __forceinline__ void join_four(const ExpertArgs &a, const Choices &c, __amdgpu_buffer_rsrc_t rsp, int m, int col) {
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < a.top_k; j0 += 8) {          // (eight loads under way at a time)
        u32x4 v[8];
        float share[8];
        uint32_t used[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = m * a.top_k + min(j0 + j, a.top_k - 1);
            v[j] = __builtin_amdgcn_raw_buffer_load_b128(rsp, j0 + j < a.top_k ? (uint32_t)(((int64_t)r * a.K + col) * 4) : 0xfffffff0u, 0, kThrough);
            used[j] = c.used[r >> 5] >> (r & 31) & 1u;
            share[j] = c.share[r];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {                  // (what nobody has written, or repeats an earlier choice, is not added, whatever it holds)
            const bool in = j0 + j < a.top_k && used[j] != 0;
            share[j] = in ? share[j] : 0.0f;
            v[j] = in ? v[j] : u32x4{0u, 0u, 0u, 0u};
            sum.x = __builtin_fmaf(share[j], __uint_as_float(v[j].x), sum.x);
            sum.y = __builtin_fmaf(share[j], __uint_as_float(v[j].y), sum.y);
            sum.z = __builtin_fmaf(share[j], __uint_as_float(v[j].z), sum.z);
            sum.w = __builtin_fmaf(share[j], __uint_as_float(v[j].w), sum.w);
        }
    }
    if (a.residual) {
        const floatx4 v = four_halves(a.residual + (int64_t)m * a.ldr + col, a.vec & 1, 4);
        sum.x += v.x;  sum.y += v.y;  sum.z += v.z;  sum.w += v.w;
    }
    u32x2 o;
    o.x = float2_to_half2_bits(sum.x, sum.y);
    o.y = float2_to_half2_bits(sum.z, sum.w);
    uint16_t *const dst = a.Y + (int64_t)m * a.ldy + col;
    if (a.vec & 2) *reinterpret_cast<u32x2 *>(dst) = o;
    else
#pragma unroll
        for (int p = 0; p < 4; ++p) dst[p] = (uint16_t)((p < 2 ? o.x : o.y) >> (16 * (p & 1)));
}

// Many choices are joined by a launch of their own: joined by the wave with a block's last unit, they keep that wave's workgroup waiting.  us of the down products that join, and without
// plus this launch (4.6): 48 tokens, top_k 6, 5120 outputs 311 and 259; 16, 6, 4096 62 and 56; 8, 8, 2048 26.5 and 17.6; 12, 4, 2048 27.5 and 19.8; 8, 4, 4096 35.4 and 31.3; 4, 6, 4096 28.5 and
// 27.0; 1, 8, 2048 10.4 and 7.7.
__global__ void __launch_bounds__(256)
join_choices_kernel(ExpertArgs a) {
    const Choices c = choices_at(a.choices, a.experts, (int)a.M * a.top_k);
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x, across = a.K >> 2;
    if (item < a.M * across) join_four(a, c, products_rsrc(a), (int)(item / across), (int)(item % across) * 4);
}

// ---- the kernel ---------------------------------------------------------------------------------------
// Rows of weights: gate and up rows in turn (first launch, !DOWN), so that a lane's four sums of a 16-row tile are two gated pairs; rows of the output (DOWN).
// A unit of work is two (or four) such tiles of one expert for up to 16 MT of its choices.  All units stand in one row, expert by expert, and every
// workgroup takes an equal stretch.  Its waves share K (slices of SPW steps of 64 columns, in several passes where K is longer) and keep
// the columns' values of their slice in registers: tokens, or the products of the first launch in two terms.  Tile t + 1 is loaded while tile t is multiplied,
// across units and experts; sums meet in LDS, one barrier per unit.
// Columns are the choices of the expert, loaded anew with every expert, so that 48 tokens over many experts take the time of a few; in the first launch up
// to 16 tokens stand in the columns as they are (`gather` 0) and are loaded once.
// The second launch leaves the product of every choice in memory, 32 bits each.  A wave of every workgroup that streams nothing adds up its units' sums and
// stores them past the caches.  Of few choices (`join`) it counts the units per block of output rows a unit later, when they have arrived; where it has the last of them, it adds up the rows'
// choices, token by token in their order, so that the result does not depend on timing.  More are added up by a third launch, in the same order.  (Counted by the workgroup at its end, the last workgroups
// to end had all their rows to add up, 10 to 17 us.)
// (Tried for the second launch: a workgroup for 16 output rows that walks over all experts and needs no memory in between.  Each of its waves has to fetch
// the products of every expert anew for 16 rows of weights: 16 tokens, 64 experts of 1408, FP8 mode 80 us; 48 tokens, 96 experts of 1520, FP16 mode 478 us.)
// TILES: 4 where K takes several passes and there are units enough: the columns' values are loaded anew for every unit and pass, which two tiles pay
// for badly (FP8 mode, 16 tokens, 64 experts of 4096: down products 231 us with two, 193 with four; but 4 tokens, 8 experts of 14336, 320 units of four for 256
// workgroups: 113 and 128).
// (with many sums those of one unit are all that the LDS has room for: a second barrier)
constexpr int sum_regions(int MT, int TILES) { return MT * TILES > 4 ? 1 : 2; }
template <int KIND, int MT, int SPW, bool PASSES, int POL, bool DOWN, int TILES>
__global__ void __launch_bounds__(MT == 1 && !PASSES ? (DOWN && SPW > 2 ? 576 : 1024) : 512)
experts_kernel(ExpertArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t shared[];
    constexpr int KSTEP = 64, EB = kind_elem_bytes(KIND), PIECES = row_pieces<KIND == kPlainF16 ? kPlainF16 : kNestedF16Row, SPW>();
    constexpr int TERMS = DOWN ? kTerms : 1;
    static_assert(PIECES > 0, "whole pieces");
    constexpr int REGIONS = sum_regions(MT, TILES);
    constexpr int SUMS = REGIONS * TILES * MT * 1024;      // bytes of sums per wave
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = (blockDim.x >> 6) - (DOWN ? 1 : 0);       // (waves that stream)
    const int g = lane >> 4, n = (int)a.M * a.top_k;
    const int64_t K = DOWN ? a.ffn : a.K;
    const int tiles = (int)((DOWN ? a.K : 2 * a.ffn) >> 4), per_expert = (tiles + TILES - 1) / TILES;
    floatx4 *const slots = reinterpret_cast<floatx4 *>(shared);                // [regions][tiles][wave][MT][64]
    const uint32_t own = (uint32_t)(waves * SUMS + wave * 2048);
    uint16_t *const list = reinterpret_cast<uint16_t *>(shared + waves * (SUMS + 2048) + wave * 32);       // the columns' rows
    const Choices c = choices_at(shared + waves * (SUMS + 2048 + 32), a.experts, n);

    const uint32_t row_bytes = (uint32_t)K * EB;
    const int64_t expert_bytes = tiles * 16 * (int64_t)row_bytes;
    const uint8_t *const w0 = DOWN ? a.down0 : a.up0, *const w1 = DOWN ? a.down1 : a.up1;
    const Regroup<true> rx(shared, own, lane);
    const Regroup<KIND == kPlainF16> rw(shared, own, lane);
    u32x4 xa[SPW][MT][TERMS], xb[SPW][MT][TERMS];
    int row[MT];                                       // the column's choice, or -1
    uint32_t x_a[MT], x_b[MT];                         // where the values lie that the lane loads: columns 0 .. 7, 8 .. 15
    const uint32_t x_row = DOWN ? (uint32_t)(kTerms * 2 * a.ffn) : (uint32_t)(2 * a.ldx);
    const __amdgpu_buffer_rsrc_t rsx = DOWN ? weight_rsrc(reinterpret_cast<const uint8_t *>(a.H), (uint32_t)n * x_row)
                                            : weight_rsrc(reinterpret_cast<const uint8_t *>(a.X), (uint32_t)(((a.M - 1) * a.ldx + a.K) * 2));
    auto x_at = [&](int which, int l) { return which >= 0 ? (uint32_t)which * x_row + (l & 7) * 16u : kDead; };
    auto k_of = [&](int pass) { return (pass * waves + wave) * (SPW * KSTEP); };
    auto request = [&](int pass) {
        const int k0 = k_of(pass);
#pragma unroll
        for (int s = 0; s < SPW; ++s)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const bool in = k0 + s * KSTEP + (lane & 7) * 8 < K;
#pragma unroll
                for (int t = 0; t < TERMS; ++t) {
                    xa[s][i][t] = __builtin_amdgcn_raw_buffer_load_b128(rsx, (in ? x_a[i] + 2u * k0 + (uint32_t)(t * 2 * K) : kDead) + 2 * KSTEP * s, 0, 0);
                    xb[s][i][t] = __builtin_amdgcn_raw_buffer_load_b128(rsx, (in ? x_b[i] + 2u * k0 + (uint32_t)(t * 2 * K) : kDead) + 2 * KSTEP * s, 0, 0);
                }
            }
    };
    auto regroup = [&] {
#pragma unroll
        for (int s = 0; s < SPW; ++s)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int t = 0; t < TERMS; ++t) rx.run(xa[s][i][t], xb[s][i][t]);
    };

    const bool in_place = !DOWN && !a.gather;          // the tokens in their places (MT is 1)
    if (in_place) {
        x_a[0] = x_at((lane >> 3) < a.M ? lane >> 3 : -1, lane);
        x_b[0] = x_at(8 + (lane >> 3) < a.M ? 8 + (lane >> 3) : -1, lane);
        request(0);
    }
    if constexpr (DOWN) {
        const u32x4 *const from = reinterpret_cast<const u32x4 *>(a.choices);
        for (int i = threadIdx.x; i < choices_shared(a.experts, n) / 16; i += blockDim.x) reinterpret_cast<u32x4 *>(c.head)[i] = from[i];
    } else if (wave == 0) {
        find_choices(a, c, lane, 16 * MT, blockIdx.x == 0);
    }
    lds_barrier();
    if (!DOWN && blockIdx.x == 0) {
        u32x4 *const to = reinterpret_cast<u32x4 *>(a.choices);
        for (int i = threadIdx.x; i < choices_shared(a.experts, n) / 16; i += blockDim.x) to[i] = reinterpret_cast<const u32x4 *>(c.head)[i];
    }
    const int count = __builtin_amdgcn_readfirstlane(c.head->count);
    const uint32_t chunks = __builtin_amdgcn_readfirstlane(c.head->chunks), total = chunks * (uint32_t)per_expert;
    const uint32_t first = (uint32_t)((uint64_t)total * blockIdx.x / gridDim.x), end = (uint32_t)((uint64_t)total * (blockIdx.x + 1) / gridDim.x);

    // Where a unit lies: the expert's place among the chosen ones, the chunk of its choices, the two tiles; the expert.
    struct At { int r, chunk, f, expert; };
    At at = {0, 0, 0, 0};
    auto scalar = [](uint32_t v) { return (int)__builtin_amdgcn_readfirstlane(v); };
    auto step = [&](At &x) {
        if (++x.f < per_expert) return;
        x.f = 0;
        ++x.chunk;
        if (x.chunk == scalar(c.info[x.r + 1].z - c.info[x.r].z)) { x.chunk = 0;  ++x.r; }
        x.expert = x.r < count ? scalar(c.info[x.r].x) : 0;
    };
    auto columns = [&](const At &x) {
        int l = lane;                                  // (what follows from the lane is worked out anew: kept across the loop it costs registers that are spilled)
        asm volatile("" : "+v"(l));
        const int col = l & 15;
        const uint32_t places = c.info[x.r].y;
        const int start = (int)(places & 0xffffu), size = (int)(places >> 16);
        if (in_place) {
            if (l < 16) list[l] = 0xffff;
            asm volatile("" ::: "memory");
            if (l < size) {
                const uint32_t e = c.entry[start + l].x;
                list[e >> 16] = (uint16_t)e;
            }
            asm volatile("" ::: "memory");
            row[0] = list[col] == 0xffff ? -1 : (int)list[col];
            asm volatile("" ::: "memory");
            return;
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int at0 = 16 * (x.chunk * MT + i);
            auto of = [&](int q) { return q < size ? (DOWN ? (int)(c.entry[start + q].x & 0xffffu) : (int)(c.entry[start + q].x >> 16)) : -1; };
            row[i] = at0 + col < size ? (int)(c.entry[start + at0 + col].x & 0xffffu) : -1;
            x_a[i] = x_at(of(at0 + (l >> 3)), l);
            x_b[i] = x_at(of(at0 + 8 + (l >> 3)), l);
        }
    };
    auto fetch = [&](WItem (&w)[SPW], const At &x, int tile, int pass, bool live) {
        live = live && TILES * x.f + tile < tiles;
        const int64_t off = (int64_t)x.expert * expert_bytes;
        const __amdgpu_buffer_rsrc_t r0 = weight_rsrc(w0 + off, (uint32_t)expert_bytes);
        const __amdgpu_buffer_rsrc_t r1 = weight_rsrc(KIND == kNestedF16Row ? w1 + off : w0 + off, (uint32_t)expert_bytes);
        const int kb = k_of(pass) * EB + (lane & 7) * 16;
        const uint32_t lo = live ? (uint32_t)((TILES * x.f + tile) * 16 + (lane >> 3)) * row_bytes + (uint32_t)kb : kDead;
        bool kv[SPW];
#pragma unroll
        for (int q = 0; q < SPW; ++q) kv[q] = q < PIECES && kb + 128 * q < K * EB;
        load_pieces<KIND, SPW, POL>(w, r0, r1, lo, lo + 8u * row_bytes, kv);
    };
    int region = 0;
    auto consume = [&](WItem (&w)[SPW], int tile, int pass) {
        floatx4 *const slot = slots + ((region * TILES + tile) * waves + wave) * MT * 64 + lane;
        floatx4 sum[MT][TERMS];
        regroup_pieces<KIND, SPW>(w, rw);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            sum[i][0] = PASSES && pass > 0 ? slot[i * 64] : floatx4{0.f, 0.f, 0.f, 0.f};
            if constexpr (TERMS == 2) sum[i][1] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int s = 0; s < SPW; ++s) {
            u32x4 w_lo, w_hi;
            operand<KIND>(w[s], w_lo, w_hi);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t) {
                    sum[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half8(w_lo), as_half8(xa[s][i][t]), sum[i][t], 0, 0, 0);
                    sum[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half8(w_hi), as_half8(xb[s][i][t]), sum[i][t], 0, 0, 0);
                }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            floatx4 all = sum[i][0];
            if constexpr (TERMS == 2) {
                all.x = __builtin_fmaf(sum[i][1].x, 1.0f / kLowScale, all.x);
                all.y = __builtin_fmaf(sum[i][1].y, 1.0f / kLowScale, all.y);
                all.z = __builtin_fmaf(sum[i][1].z, 1.0f / kLowScale, all.z);
                all.w = __builtin_fmaf(sum[i][1].w, 1.0f / kLowScale, all.w);
            }
            slot[i * 64] = all;
        }
    };
    auto add_up = [&](int t, int i) {
        floatx4 sum = slots[(((region * TILES + t) * waves) * MT + i) * 64 + lane];
#pragma unroll 4
        for (int w = 1; w < waves; ++w) {
            const floatx4 v = slots[(((region * TILES + t) * waves + w) * MT + i) * 64 + lane];
            sum.x += v.x;  sum.y += v.y;  sum.z += v.z;  sum.w += v.w;
        }
        return sum;
    };
    if (first < end) {
        const uint32_t chunk0 = first / (uint32_t)per_expert;
        for (int base = 0; base < count; base += 64)
            at.r += __popcll(__ballot(base + lane < count && c.info[min(base + lane, count - 1) + 1].z <= chunk0));
        at.r = scalar((uint32_t)at.r);
        at.chunk = scalar(chunk0 - c.info[at.r].z);
        at.f = scalar(first - chunk0 * (uint32_t)per_expert);
        at.expert = scalar(c.info[at.r].x);
    }
    if constexpr (DOWN) {
        if (wave == waves) {
            // products of the choices: written through, read back past the caches (every XCD has an L2 of its own)
            const __amdgpu_buffer_rsrc_t rsp = products_rsrc(a);
            auto join = [&](int f) {
                for (int i = lane; i < a.M * (4 * TILES); i += 64) {
                    const int m = i / (4 * TILES), col = 16 * TILES * f + 4 * (i % (4 * TILES));
                    if (col < a.K) join_four(a, c, rsp, m, col);
                }
            };
            if (total == 0 && a.join)                  // nobody has chosen anything: the rows are shared out
                for (int f = blockIdx.x; f < per_expert; f += gridDim.x) join(f);
            if (first >= end) return;
            auto count_unit = [&](int f) {             // (behind a wait for the unit's products)
                uint32_t before = 0;
                if (lane == 0) before = __hip_atomic_fetch_add(&a.counters[f], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                return before;
            };
            auto finish = [&](int f, uint32_t before) {
                if ((uint32_t)scalar(before) != chunks - 1) return;
                if (lane == 0) __hip_atomic_store(&a.counters[f], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                join(f);
            };
            columns(at);
            int f_before = -1;
            for (uint32_t u = first; u < end; ++u) {
                lds_barrier();
                uint32_t before = 0;
                if (f_before >= 0 && a.join) {
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the products of the unit before
                    before = count_unit(f_before);
                }
                floatx4 sum[TILES][MT];
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int i = 0; i < MT; ++i) sum[t][i] = add_up(t, i);
                if constexpr (REGIONS == 2) region ^= 1;
                else lds_barrier();
                if (f_before >= 0 && a.join) finish(f_before, before);
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        if (row[i] < 0 || TILES * at.f + t >= tiles) continue;
                        const uint32_t off = (uint32_t)(((int64_t)row[i] * a.K + 16 * (TILES * at.f + t) + 4 * g) * 4);
                        __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(sum[t][i].x), __float_as_uint(sum[t][i].y), __float_as_uint(sum[t][i].z),
                                                                     __float_as_uint(sum[t][i].w)}, rsp, off, 0, kThrough);
                    }
                f_before = at.f;
                At next = at;
                step(next);
                if (u + 1 < end && (next.r != at.r || next.chunk != at.chunk)) columns(next);
                at = next;
            }
            if (!a.join) return;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            finish(f_before, count_unit(f_before));
            return;
        }
    }

    if (first < end) {
        WItem buf0[SPW], buf1[SPW];
        const int passes = PASSES ? a.passes : 1;
        fetch(buf0, at, 0, 0, true);
        columns(at);
        if (!in_place) request(0);
        regroup();
        for (uint32_t u = first; u < end; ++u) {
            At next = at;
            step(next);
            for (int pass = 0; pass < passes; ++pass) {
                if (PASSES && (pass > 0 || u > first)) {
                    request(pass);
                    regroup();
                }
#pragma unroll
                for (int t = 0; t < TILES; t += 2) {
                    fetch(buf1, at, t + 1, pass, true);
                    __builtin_amdgcn_sched_barrier(0);
                    consume(buf0, t, pass);
                    __builtin_amdgcn_sched_barrier(0);
                    if (t + 2 < TILES) fetch(buf0, at, t + 2, pass, true);
                    else if (pass + 1 < passes) fetch(buf0, at, 0, pass + 1, true);
                    else fetch(buf0, next, 0, 0, u + 1 < end);
                    __builtin_amdgcn_sched_barrier(0);
                    consume(buf1, t + 1, pass);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            lds_barrier();
            // The waves take turns with the sums.  (They are written again two units later, behind the next barrier.)
            if constexpr (!DOWN) {
                for (int item = 0; item < TILES * MT; ++item) {
                    if ((int)((u * (TILES * MT) + item) % (unsigned)waves) != wave) continue;
                    const int t = item / MT, i = item - t * MT;
                    const floatx4 sum = add_up(t, i);
                    int to = row[0];
#pragma unroll
                    for (int q = 1; q < MT; ++q) to = i == q ? row[q] : to;
                    if (to < 0 || TILES * at.f + t >= tiles) continue;
                    const float h0 = activate(sum.x, a.act) * sum.y, h1 = activate(sum.z, a.act) * sum.w;
                    const int f = 8 * (TILES * at.f + t) + 2 * g;
                    uint16_t *const dst = a.H + (int64_t)to * kTerms * a.ffn + f;
                    const uint32_t high = float2_to_half2_bits(h0, h1);
                    *reinterpret_cast<uint32_t *>(dst) = high;
                    if constexpr (kTerms == 2) {
                        // (an infinite first term has no rest)
                        const float l0 = kLowScale * (h0 - half_bits_to_float(high & 0xffffu)), l1 = kLowScale * (h1 - half_bits_to_float(high >> 16));
                        *reinterpret_cast<uint32_t *>(dst + a.ffn) =
                            float2_to_half2_bits((high & 0x7fffu) == 0x7c00u ? 0.0f : l0, (high & 0x7fff0000u) == 0x7c000000u ? 0.0f : l1);
                    }
                }
            }
            if constexpr (REGIONS == 2) region ^= 1;
            else lds_barrier();
            if (u + 1 < end && (next.r != at.r || next.chunk != at.chunk)) {
                columns(next);
                if (!PASSES && !in_place) {
                    request(0);
                    regroup();
                }
            }
            at = next;
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------
// The workspace behind its counters: the choices, the activated products, the products of the choices.
static size_t choices_bytes(int64_t experts, int64_t n) { return round256((size_t)choices_shared((int)experts, (int)n)); }
static size_t activated_bytes(int64_t n, int64_t ffn) { return round256((size_t)n * kTerms * (size_t)ffn * 2); }
size_t experts_workspace_bytes(int64_t experts, int64_t hidden, int64_t ffn, int64_t M, int64_t top_k) {
    return choices_bytes(experts, M * top_k) + activated_bytes(M * top_k, ffn) + (size_t)(M * top_k) * (size_t)hidden * 4;
}

bool experts_supported(int64_t experts, int64_t hidden, int64_t ffn, int64_t M, int64_t top_k) {
    // an expert's matrix and the products between the launches are addressed with 31 bits, and every 32 output rows have a counter
    constexpr int64_t limit = (int64_t)1 << 31;
    if (experts > kMostExperts || M > kMostTokens || top_k > kMostTop || hidden > 32 * kMaxCounters) return false;
    return 2 * ffn * hidden * 2 + 64 * std::max(hidden, ffn) < limit && (int64_t)activated_bytes(M * top_k, ffn) + 4096 < limit &&
           M * top_k * hidden * 4 + 4096 < limit;
}

template <int KIND, int MT, int SPW, bool PASSES, int POL, bool DOWN, int TILES>
static int launch_experts_t(const ExpertArgs &a, int waves, hipStream_t stream) {
    auto kern = experts_kernel<KIND, MT, SPW, PASSES, POL, DOWN, TILES>;
    static std::atomic<bool> ready{false};
    if (!ready.load(std::memory_order_acquire)) {
        (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        ready.store(true, std::memory_order_release);
    }
    const int n = (int)(a.M * a.top_k);
    const size_t lds = (size_t)waves * (sum_regions(MT, TILES) * TILES * MT * 1024 + 2048 + 32) + choices_shared(a.experts, n) +
                       (DOWN ? 0 : choices_scratch(a.experts, n));
    if (lds > 160 * 1024) return kErrShape;
    const int64_t tiles = (DOWN ? a.K : 2 * a.ffn) / 16, units = choice_most(a.experts, n) * ((tiles + TILES - 1) / TILES);
    // waves that a CU holds, by registers
    const int held = MT > 1 ? 8 : (DOWN ? (PASSES ? 8 : (SPW == 2 ? 16 : 12)) : (PASSES ? 12 : 16));
    const int all = waves + (DOWN ? 1 : 0);
    const int per_cu = std::max(1, std::min(held / all, (int)(160 * 1024 / lds)));
    kern<<<(unsigned)std::max<int64_t>(1, std::min<int64_t>(units, 256 * per_cu)), (unsigned)all * 64, lds, stream>>>(a);
    return hip_ok(hipGetLastError());
}

template <int KIND, int MT, int SPW, int POL, bool DOWN>
static int launch_slices(ExpertArgs a, hipStream_t stream) {
    const int64_t K = DOWN ? a.ffn : a.K, tiles = (DOWN ? a.K : 2 * a.ffn) / 16;
    const int slices = (int)((K + SPW * 64 - 1) / (SPW * 64));
    const int one_pass = MT == 1 ? (DOWN ? (SPW == 2 ? 15 : 8) : 16) : (DOWN ? 7 : 8);         // waves that stream, as the registers allow
    const int most = slices <= one_pass ? one_pass : (DOWN ? 7 : 8);
    a.passes = (slices + most - 1) / most;
    const int waves = (slices + a.passes - 1) / a.passes;
    if (a.passes == 1) return launch_experts_t<KIND, MT, SPW, false, POL, DOWN, 2>(a, waves, stream);
    if constexpr (MT < 4) {
        // (at least four units of four tiles for each of 256 workgroups, if the tokens' choices differ)
        if (choice_most(a.experts, (int)(a.M * a.top_k)) * tiles >= 4 * 4 * 256) return launch_experts_t<KIND, MT, SPW, true, POL, DOWN, 4>(a, waves, stream);
    }
    return launch_experts_t<KIND, MT, SPW, true, POL, DOWN, 2>(a, waves, stream);
}

template <int KIND, int POL, bool DOWN>
static int launch_columns(const ExpertArgs &a, hipStream_t stream) {
    // both launches alike: the chunks of an expert's choices are counted once
    if (a.M <= 16 || 2 * a.M * a.top_k <= 16 * a.experts) {
        // Twice as many waves on half as long slices: for gate and up where there are few units, that is little more than one unit's latency (1 token, hidden 1040, 2 experts of 528:
        // 7.4 -> 7.2 us; 4 tokens, 16 experts of 768 x 2048: 22.1 -> 19.6; but 16 tokens, 52 of these, FP8 mode: 32.1 and 34.1), for down wherever one pass takes all of K
        // (1 token, 528: 7.0 -> 6.2 us; 16 tokens, 50 experts of 1408 x 4096, FP8 mode: 57 -> 52; 48 tokens, 92 of 1520 x 5120: 259 and 257; 16 tokens, 52 of 768 x 2048: 29.4 and 30.0).
        const int64_t K = DOWN ? a.ffn : a.K, tiles = 2 * a.ffn / 16;
        if (DOWN ? K <= 15 * 128 : K <= 16 * 128 && choice_most(a.experts, (int)(a.M * a.top_k)) * tiles <= 8 * 256) return launch_slices<KIND, 1, 2, POL, DOWN>(a, stream);
        return launch_slices<KIND, 1, 4, POL, DOWN>(a, stream);
    }
    return a.M <= 32 || a.M * a.top_k <= 16 * a.experts ? launch_slices<KIND, 2, 4, POL, DOWN>(a, stream) : launch_slices<KIND, 4, 2, POL, DOWN>(a, stream);
}

template <int KIND, bool DOWN>
static int launch_lines(const ExpertArgs &a, hipStream_t stream) {
    const int64_t row = (DOWN ? a.ffn : a.K) * kind_elem_bytes(KIND);
    const uintptr_t at = reinterpret_cast<uintptr_t>(DOWN ? a.down0 : a.up0) | reinterpret_cast<uintptr_t>(DOWN ? a.down1 : a.up1);
    return (row & 127) == 0 && (at & 127) == 0 ? launch_columns<KIND, kStream, DOWN>(a, stream) : launch_columns<KIND, kCached, DOWN>(a, stream);
}

template <int KIND>
static int launch_both(const ExpertArgs &a, hipStream_t stream) {
    int st = launch_lines<KIND, false>(a, stream);
    if (st == kOk) st = launch_lines<KIND, true>(a, stream);
    if (st != kOk || a.join) return st;
    join_choices_kernel<<<(unsigned)((a.M * (a.K >> 2) + 255) / 256), 256, 0, stream>>>(a);
    return hip_ok(hipGetLastError());
}

int launch_experts_layer(int kind, ExpertArgs a, uint8_t *room, hipStream_t stream) {
    a.choices = room;
    a.H = reinterpret_cast<uint16_t *>(room + choices_bytes(a.experts, a.M * a.top_k));
    a.products = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(a.H) + activated_bytes(a.M * a.top_k, a.ffn));
    a.gather = a.M > 16 ? 1 : 0;
    a.join = a.M * a.top_k <= 32 ? 1 : 0;
    return kind == kPlainF16 ? launch_both<kPlainF16>(a, stream) : (kind == kE4M3Row ? launch_both<kE4M3Row>(a, stream) : launch_both<kNestedF16Row>(a, stream));
}

}  // namespace nfp
