// Attention of new tokens over a paged cache:  o = sum_t p_t v_t / sum_t p_t,  p_t = exp(c q.k_t - m),  over the tokens t
// of the sequence that a new token at position `pos` sees:  t <= pos and (no window, or t > pos - window, or t < sinks).
//
// Rows.  The new tokens of a sequence and the query heads that share a key/value head are the rows of one small matrix:
// row r is new token r / group, head r % group.  A tile of rows reads every key and value once for all of them.
// Both products are transposed: S^T = K Q^T and O^T = V^T P^T, so that a lane holds one row's scores, the statistics of a
// row lie in one column of lanes, and P^T becomes the operand of the second product by exchanging registers between groups of 16 lanes.
//
// The visible tokens are walked in blocks of 16 (a block lies in one page): first the blocks of the sinks, then those of the
// window; pages outside are never looked at.
#include "nfp_device.h"
#include "nfp_host.h"

#include <algorithm>

namespace nfp {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_inff();
// Probabilities are at most 2^kShift instead of 1: FP16 has normal numbers down to 2^-14, so that what counts as subnormal
// starts 2^-26 below the row's maximum.  Sums carry the same factor, which the division takes out.
constexpr float kShift = 12.0f;

// ---- exchanges between the four groups of 16 lanes ------------------------------------------------------------------------
// swap32: upper half of a with lower half of b; swap16: odd groups of a with even groups of b.
__device__ __forceinline__ void swap32(uint32_t &a, uint32_t &b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
__device__ __forceinline__ void swap16(uint32_t &a, uint32_t &b) {
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
__device__ __forceinline__ float max_of_groups(float v) {
    uint32_t a = __float_as_uint(v), b = a;
    swap32(a, b);
    v = fmaxf(__uint_as_float(a), __uint_as_float(b));
    a = b = __float_as_uint(v);
    swap16(a, b);
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ float sum_of_groups(float v) {
    uint32_t a = __float_as_uint(v), b = a;
    swap32(a, b);
    v = __uint_as_float(a) + __uint_as_float(b);
    a = b = __float_as_uint(v);
    swap16(a, b);
    return __uint_as_float(a) + __uint_as_float(b);
}

// 16 E4M3 codes -> 16 FP16 values (every code is one)
__device__ __forceinline__ void widen(const u32x4 &v, half8 &lo, half8 &hi) {
    typedef _Float16 half2v __attribute__((ext_vector_type(2)));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    half2v h[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false);
        h[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true);
    }
    lo = half8{h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
    hi = half8{h[4][0], h[4][1], h[5][0], h[5][1], h[6][0], h[6][1], h[7][0], h[7][1]};
}

// Values that are not finite.  Their products with a probability of zero are NaN, also where the probability is zero because
// the row does not see the token, and so is the product with the rest of a probability.  The loops therefore run on
// the values as they come; sums that are not finite at the end are made again without those values, and what they add
// to the rows that do see them is found by itself: counts of +Inf, -Inf and NaN per row and column.
enum { kPlusInf = 0, kMinusInf = 1, kNaN = 2 };
template <bool FP8>
__device__ __forceinline__ u32x4 only_finite(const u32x4 &v) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FP8) {
#pragma unroll
            for (int j = 0; j < 32; j += 8) w[i] = (w[i] >> j & 0x7fu) == 0x7fu ? w[i] & ~(0xffu << j) : w[i];
        } else {
            w[i] = (w[i] & 0x7c00u) == 0x7c00u ? w[i] & 0xffff0000u : w[i];
            w[i] = (w[i] & 0x7c000000u) == 0x7c000000u ? w[i] & 0xffffu : w[i];
        }
    }
    return u32x4{w[0], w[1], w[2], w[3]};
}
// 1 where an FP16 value is of a kind, 0 elsewhere: bits from `low` to `high` without the sign bits that `sign` clears
__device__ __forceinline__ half8 of_kind(half8 v, int kind) {
    const u32x4 b = __builtin_bit_cast(u32x4, v);
    const uint32_t w[4] = {b.x, b.y, b.z, b.w};
    const uint32_t sign = kind == kNaN ? 0x7fffu : 0xffffu, low = kind == kPlusInf ? 0x7c00u : kind == kMinusInf ? 0xfc00u : 0x7c01u;
    const uint32_t span = kind == kNaN ? 0x3feu : 0u;
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[i] = (w[i] & sign) - low <= span ? 0x3c00u : 0u;
        r[i] |= (w[i] >> 16 & sign) - low <= span ? 0x3c000000u : 0u;
    }
    return __builtin_bit_cast(half8, u32x4{r[0], r[1], r[2], r[3]});
}
__device__ __forceinline__ float of_kind_value(int kind) {
    return kind == kPlusInf ? -kNegInf : kind == kMinusInf ? kNegInf : __builtin_nanf("");
}
__device__ __forceinline__ bool not_finite(const floatx4 &v) {
    // (a difference with itself is zero for finite values alone)
    const floatx4 z = v - v;
    return !(z[0] == 0.0f && z[1] == 0.0f && z[2] == 0.0f && z[3] == 0.0f);
}

// What a sequence's place in the batch and in the cache comes down to; lengths and starts that do not fit the arrays
// they index are cut off, so that nothing outside is read.  `fresh` are the new tokens that get an output, cut off at max_new and at the
// end of Q; `past`, the position of the first of them, follows from all that the sequence has, so that a cut moves no position.
struct Sequence { int first, fresh, past; };
__device__ __forceinline__ Sequence sequence(const AttentionArgs &p, int b) {
    Sequence s;
    const int length = max(0, min(p.lens[b], (int)min((int64_t)0x7fffffff, (int64_t)p.columns << (p.page_shift + 4))));
    if (p.starts) {
        const int from = p.starts[b], to = p.starts[b + 1], begin = max(0, from);
        s.first = min(begin, p.tokens);
        s.fresh = max(0, min(min(to, p.tokens) - s.first, p.max_new));
        if (from < 0) s.fresh = 0;
        s.past = length - (max(to, begin) - begin);
    } else {
        s.first = b * p.per;
        s.fresh = p.per;
        s.past = length - p.per;
    }
    return s;
}

// The last token before the window of a row at `pos` (-1: there is none), and whether a row with these two sees a token.
__device__ __forceinline__ int before(const AttentionArgs &p, int pos) {
    return p.window > 0 && pos >= p.window ? pos - p.window : -1;
}
__device__ __forceinline__ bool sees(int t, int pos, int low, int sinks) { return t <= pos && (t > low || t < sinks); }

// Blocks that the rows of new tokens i0 ... i1 see, in the order in which they are walked.
struct Walk {
    int sink_blocks, low_block, blocks;              // blocks in all: sink_blocks from 0, the rest from low_block
    __device__ __forceinline__ int block(int v) const { return v < sink_blocks ? v : v - sink_blocks + low_block; }
};
__device__ __forceinline__ Walk walk(const AttentionArgs &p, int low_pos, int high_pos) {
    Walk w;
    const int high_block = high_pos < 0 ? 0 : (high_pos >> 4) + 1;
    w.low_block = min((before(p, low_pos) + 1) >> 4, high_block);
    w.sink_blocks = p.window > 0 ? min((int)(((int64_t)p.sinks + 15) >> 4), w.low_block) : 0;
    w.blocks = w.sink_blocks + high_block - w.low_block;
    return w;
}
// ---- sequences split over workgroups -----------------------------------------------------------------------------------------
// A workgroup's sums lie in the workspace as [tile][chunk][row]: D sums, then the maximum and the sum of the row's
// probabilities.  They are stored past the caches (every XCD has an L2 of its own) before the tile's ticket is drawn;
// the workgroup with the last ticket joins the chunks in a fixed order and leaves the counter cleared.  Nobody waits for anybody.
// The joining workgroup has many loads under way, groups of its lanes take every so many chunks each: one after the other, 64 chunks took
// about 40 us.
__device__ __forceinline__ float2 pair_of(unsigned long long x) { return {__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32))}; }
__device__ __forceinline__ unsigned long long past_caches(const float *p) {
    return __hip_atomic_load(reinterpret_cast<const unsigned long long *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void past_caches(float *p, float a, float b) {
    __hip_atomic_store(reinterpret_cast<unsigned long long *>(p), (unsigned long long)__float_as_uint(a) | (unsigned long long)__float_as_uint(b) << 32,
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <int D, int THREADS>
__device__ __forceinline__ void join(const AttentionArgs &p, int thread, int tile, int chunks, const Sequence &sq, int row0, int row1, int past, int head,
                                     float v_scale, float *room, int *last) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (thread == 0) {
        const uint32_t ticket = __hip_atomic_fetch_add(p.counters + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *last = ticket == (uint32_t)chunks - 1;
        if (*last) __hip_atomic_store(p.counters + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!*last) return;
    const int items = (row1 - row0 + 1) * (D / 4);     // four columns of a row
    constexpr int stride = D + 2;
    const float *parts = p.partials + (int64_t)tile * p.chunks * p.part_rows * stride;
    const int64_t next = (int64_t)p.part_rows * stride;
    const int groups = max(1, min(THREADS / items, chunks));
    for (int base = 0; base < items; base += THREADS) {
        const int group = groups > 1 ? thread / items : 0, item = base + (groups > 1 ? thread - group * items : thread);
        const int r = min(item, items - 1) / (D / 4), d = 4 * (min(item, items - 1) - r * (D / 4));
        const float *src = parts + r * stride;
        float top = kNegInf, sum = 0.0f;
        floatx4 acc = floatx4{0, 0, 0, 0};
        constexpr int N = 8;
        for (int c = group; c < chunks && group < groups; c += N * groups) {
            float2 stat[N], a[N], b[N];
            float now = top;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float *at = src + min(c + i * groups, chunks - 1) * next;
                stat[i] = pair_of(past_caches(at + D));
                a[i] = pair_of(past_caches(at + d));
                b[i] = pair_of(past_caches(at + d + 2));
            }
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (c + i * groups < chunks) now = fmaxf(now, stat[i].x);
            const float ref = fmaxf(now, -1e30f), f = __builtin_amdgcn_exp2f(fmaxf(top, -1e30f) - ref);
            sum *= f;
            acc *= f;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (c + i * groups < chunks) {
                    const float g = __builtin_amdgcn_exp2f(fmaxf(stat[i].x, -1e30f) - ref);
                    sum += stat[i].y * g;
                    acc += floatx4{a[i].x, a[i].y, b[i].x, b[i].y} * g;
                }
            top = now;
        }
        if (groups > 1) {                              // (then one round of the loop has all items)
            if (group < groups) {
                *reinterpret_cast<floatx4 *>(room + 8 * thread) = acc;
                room[8 * thread + 4] = top;
                room[8 * thread + 5] = sum;
            }
            __syncthreads();
            if (group > 0) continue;
            for (int i = 1; i < groups; ++i) {
                const float *other = room + 8 * (thread + i * items);
                const float now = fmaxf(top, other[4]), ref = fmaxf(now, -1e30f);
                const float f = __builtin_amdgcn_exp2f(fmaxf(top, -1e30f) - ref), g = __builtin_amdgcn_exp2f(fmaxf(other[4], -1e30f) - ref);
                sum = sum * f + other[5] * g;
                acc = acc * f + *reinterpret_cast<const floatx4 *>(other) * g;
                top = now;
            }
        }
        if (item >= items) continue;
        const int i = (row0 + r) / p.group, g = row0 + r - i * p.group;
        const float f = v_scale / sum;
        *reinterpret_cast<u32x2 *>(p.O + (int64_t)(sq.first + i) * p.ldo + (int64_t)(head * p.group + g) * D + d) = past + i < 0 ? u32x2{0u, 0u} :
            u32x2{float2_to_half2_bits(acc[0] * f, acc[1] * f), float2_to_half2_bits(acc[2] * f, acc[3] * f)};
    }
}

// ---- who does what --------------------------------------------------------------------------------------------------------------
// The host does not know the sequences' lengths (a captured graph is replayed as they grow), so every workgroup of the streaming
// kernel works out the same schedule from them: the blocks of all tiles of rows in one row, of which each workgroup takes a stretch of
// the same length, which may end one tile and begin the next.  Equal shares for two workgroups per CU: with three, loads wait for each other
// (7 us instead of 2), and so does every step of the prologue and of the join; with one launch of all stretches that the
// largest length would have, those that turn out empty cost 1 to 2 us for every few hundred.
constexpr int kScan = 256;
template <int CTRL, int ROWS>
__device__ __forceinline__ int plus_before(int v) {
    return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
// the sum over this lane and those before it
__device__ __forceinline__ int sum_to_lane(int v) {
    v = plus_before<0x111, 0xf>(v);                    // the lane 1, 2, 4, 8 before, in its row of 16
    v = plus_before<0x112, 0xf>(v);
    v = plus_before<0x114, 0xf>(v);
    v = plus_before<0x118, 0xf>(v);
    v = plus_before<0x142, 0xa>(v);                    // the last lane of the row before
    return plus_before<0x143, 0xc>(v);                 // lane 31
}
struct Schedule {
    int begin[kScan / 64];                             // of sequence 64 i + lane in the row of all blocks
    int all, share;                                    // blocks, and of them a workgroup's
};
__device__ __forceinline__ int up_to(int v, int multiple) { return (v + multiple - 1) / multiple * multiple; }
// blocks that a tile of a sequence's rows has in the row: whole steps
__device__ __forceinline__ int padded_blocks(const AttentionArgs &p, const Sequence &sq, int least) {
    return up_to(max(1, walk(p, sq.past, sq.past + sq.fresh - 1).blocks), least);
}
__device__ __forceinline__ Schedule schedule(const AttentionArgs &p, int tile_rows, int least) {
    constexpr int N = kScan / 64;
    const int lane = threadIdx.x & 63;
    Schedule plan;
    plan.all = 0;
    uint32_t longest = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        plan.begin[i] = 0x7fffffff;
        if (64 * i >= p.batch) continue;
        const int t = 64 * i + lane;
        const Sequence sq = sequence(p, min(t, p.batch - 1));
        const int rows = sq.fresh * p.group;
        int blocks = 0;
        if (t < p.batch && rows > 0 && !(p.few > 0 && rows > p.few)) {
            const int each = padded_blocks(p, sq, least);
            longest = max(longest, (uint32_t)each);
            blocks = each * ((rows + tile_rows - 1) / tile_rows * p.kv_heads);
        }
        const int sum = sum_to_lane(blocks);
        plan.begin[i] = plan.all + sum - blocks;
        plan.all += __builtin_amdgcn_readlane(sum, 63);
    }
    plan.share = p.chunk_blocks;
    if (!p.fixed) plan.share = max(plan.share, (plan.all + (int)gridDim.x - 1) / (int)gridDim.x);
    // (a tile's parts have to fit the workspace, also where a sequence is longer than the launch was sized for)
    plan.share = up_to(max(plan.share, ((int)max_of_wave(longest) + p.chunks - 2) / max(p.chunks - 1, 1)), least);
    return plan;
}
// the sequence that a block of the row belongs to, and the block's place among the sequence's
__device__ __forceinline__ int place_of(const Schedule &plan, int x, int batch, int &b) {
    int at = -1, first = 0;
#pragma unroll
    for (int i = 0; i < kScan / 64; ++i) at += __builtin_popcountll(__builtin_amdgcn_ballot_w64(plan.begin[i] <= x));
    b = min(at, batch - 1);                            // (lanes behind the last sequence begin where it ends)
#pragma unroll
    for (int i = 0; i < kScan / 64; ++i)
        if (b >> 6 == i) first = __builtin_amdgcn_readlane(plan.begin[i], b & 63);
    return x - first;
}

// ---- streaming kernel -------------------------------------------------------------------------------------------------------
// For few rows: bound by the bytes of the cache.  A workgroup of four waves takes 16 * RT rows and a stretch of the
// sequence's blocks; a wave loads keys and values of 32 tokens (64 in E4M3) straight into registers, in operand order, every
// load instruction whole lines.  The waves' sums meet in LDS; where a sequence takes more than one workgroup, each leaves its sums
// in the workspace and the one that comes last joins them in order.
// P is carried as two FP16 terms (its FP16 rounding and the rest): the second product costs nothing here, and the
// result then has the precision of the 32-bit sums.
// Measured (128 dims, 8 key/value heads; a read-only stream reaches 7.15 TB/s): 768 equal tiles of 1600 tokens 96 us (6.6 TB/s), one token over
// 131072 84 us (6.4), 32 sequences of 500 ... 8192 tokens 67 us (5.5), 48 of 1000 ... 20000 in E4M3 113 us (5.6), one of 613 8.9 us.  Beside
// the bytes a call costs about 9 us: launch, lengths, page numbers and first keys one after the other, at the end sums, ticket
// and join.
// Tried and dropped: the next step's loads under way during the work on one (two steps of registers, 113 -> 122 us on the 48 sequences);
// loads that stay in L2 (130); three workgroups per CU (115 us, and 101 instead of 90 on the one long sequence).
template <int D, bool FP8, int RT>
__global__ void __launch_bounds__(256, D <= 128 && RT == 1 ? 3 : 2)
attention_stream_kernel(AttentionArgs p) {
    constexpr int NT = FP8 ? 4 : 2;                    // blocks per step
    constexpr int BLOCK = 16 * D * (FP8 ? 1 : 2);      // bytes of a block
    constexpr int KL = (BLOCK + 1023) / 1024;          // 16-byte loads per lane for the keys of a block
    constexpr int QS = FP8 ? 2 * KL : KL;              // operands of 32 dims
    constexpr int DB = D / 16;
    constexpr int LD = D + 4;
    // the waves' sums on their way together, then the groups' of the join (8 words for every lane)
    __shared__ __align__(16) float shared[4 * 16 * RT * LD];
    static_assert(4 * 16 * RT * LD >= 8 * 256, "");
    float (*part)[16 * RT][LD] = reinterpret_cast<float (*)[16 * RT][LD]>(shared);
    __shared__ float stat[4][2][16 * RT];
    __shared__ int last;

    constexpr int LEAST = 4 * NT;                      // blocks: one step of each wave
    Schedule plan;
    if (p.scan) plan = schedule(p, 16 * RT, LEAST);
    else plan.all = gridDim.x, plan.share = 1;
    // (without a schedule: a workgroup is a chunk of a tile)
    for (int first = blockIdx.x; (int64_t)first * plan.share < plan.all; first += gridDim.x) {
        for (int x = first * plan.share, end = min(plan.all, x + plan.share); x < end;) {
            __syncthreads();
            // (hidden from the compiler, which otherwise works out before the loop what every lane needs in it, and keeps it in 40 registers)
            int thread = threadIdx.x;
            asm volatile("" : "+v"(thread));
            const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6), group = lane >> 4, col = lane & 15;
            int chunk, rt0, head, b, offset_in_tile, here;        // (blocks of the tile before this stretch, and in it)
            Sequence sq;
            if (p.scan) {
                const int mine = place_of(plan, x, p.batch, b);
                sq = sequence(p, b);
                const int each = padded_blocks(p, sq, LEAST), index = mine / each;
                offset_in_tile = mine - index * each;
                here = min(end - x, each - offset_in_tile);
                head = index % p.kv_heads;
                rt0 = index / p.kv_heads;
                chunk = x / plan.share - (x - offset_in_tile) / plan.share;
            } else {
                const int tiles = p.batch * p.kv_heads * p.row_tiles;
                chunk = x / tiles;
                head = x % p.kv_heads;
                rt0 = x % tiles / p.kv_heads % p.row_tiles;
                b = x % tiles / p.kv_heads / p.row_tiles;
                sq = sequence(p, b);
                offset_in_tile = chunk * p.chunk_blocks;
                here = 1;
            }
            const int start_of_tile = x - offset_in_tile;
            x += here;
            const int tile = (b * p.row_tiles + rt0) * p.kv_heads + head;
            const int rows = sq.fresh * p.group, row0 = rt0 * 16 * RT;
            if (row0 >= rows || (p.few > 0 && rows > p.few)) continue;   // (the tile kernel's)
            const int row1 = min(rows, row0 + 16 * RT) - 1;
            const int past = sq.past;
            const int low_pos = past + row0 / p.group, high_pos = past + row1 / p.group;
            const Walk w = walk(p, low_pos, high_pos);
            int chunks, v1;
            const int v0 = offset_in_tile;
            if (p.scan) {
                chunks = (start_of_tile + max(w.blocks, 1) - 1) / plan.share - start_of_tile / plan.share + 1;
                v1 = min(w.blocks, v0 + here);
            } else {
                // (a sequence longer than the launch was sized for: its last workgroup takes what is left)
                chunks = min(p.chunks, max(1, (w.blocks + p.chunk_blocks - 1) / p.chunk_blocks));
                v1 = chunk == chunks - 1 ? w.blocks : v0 + p.chunk_blocks;
            }
            if (chunk >= chunks) continue;

            // queries, as the second operand: column = row, dims in the order in which the keys' chunks come
            int row[RT], pos[RT], low[RT];
            half8 q[RT][QS];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                row[r] = row0 + 16 * r + col;
                const int i = min(row[r], row1) / p.group, g = min(row[r], row1) - i * p.group;
                pos[r] = past + i;
                low[r] = before(p, pos[r]);
                const uint16_t *src = p.Q + (int64_t)(sq.first + i) * p.ldq + (int64_t)(head * p.group + g) * D;
#pragma unroll
                for (int s = 0; s < QS; ++s) {
                    const int dim = FP8 ? 16 * (4 * (s >> 1) + group) + 8 * (s & 1) : 8 * (4 * s + group);
                    q[r][s] = dim < D ? *reinterpret_cast<const half8 *>(src + dim) : half8{};
                }
            }
            floatx4 acc[RT][DB];
            float top[RT], total[RT];
            const float scale = p.scale * kLog2e * (FP8 && p.k_scale ? p.k_scale[head] : 1.0f);
            const int in_page = (1 << p.page_shift) - 1;

            // this wave's blocks of the 256 from `base`: step j takes blocks base + NT (4 j + wave) ...; lane NT j + k has the page of the k-th of step j
            const auto pages_from = [&](int base) {
                const int v = base + NT * (4 * (lane / NT) + wave) + lane % NT;
                return v < v1 ? p.table[(int64_t)b * p.ld_table + (w.block(v) >> p.page_shift)] : 0;
            };
            const auto offset = [&](int block, int pg, bool valid) {
                return ((((int64_t)(valid ? pg : 0) * p.kv_heads + head) << p.page_shift) + (valid ? block & in_page : 0)) * BLOCK;
            };
            // this lane's values: of its group's block, 8 (16 in E4M3) tokens of dims 16 d + col
            const int mine_in_block = (FP8 ? 0 : (group & 1) * D * 16) + col * 16, mine_first = FP8 ? 0 : 8 * (group & 1);
            const int first_low = before(p, low_pos), last_low = before(p, high_pos);

            bool clean = false;
            for (;;) {
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    top[r] = kNegInf;
                    total[r] = 0.0f;
#pragma unroll
                    for (int d = 0; d < DB; ++d) acc[r][d] = floatx4{0, 0, 0, 0};
                }
                for (int base = v0; base < v1; base += 64 * 4) {
                    const int page = pages_from(base);
                    for (int j = 0; j < 64 / NT; ++j) {
                        const int v = base + NT * (4 * j + wave);
                        if (v >= v1) break;
                        u32x4 kk[NT][KL], vv[DB];
                        int t0[NT];
                        bool plain = true;
                        uint32_t missing = 0;                      // blocks of this step that are not there
                        const uint8_t *mine = nullptr;             // of this lane's block of values
#pragma unroll
                        for (int k = 0; k < NT; ++k) {
                            const int block = w.block(min(v + k, v1 - 1)), pg = __builtin_amdgcn_readlane(page, NT * j + k);
                            const bool there = v + k < v1;
                            const bool valid = (uint32_t)pg < (uint32_t)p.pages;
                            t0[k] = there ? block * 16 : 0x7ffffff0;          // (nothing sees those)
                            if (there && !valid) missing |= 1u << k;
                            plain &= there && valid && t0[k] + 15 <= low_pos && (t0[k] > last_low || t0[k] + 15 < p.sinks);
                            const int64_t at = offset(block, pg, valid && there);
                            const uint8_t *kb = p.k + at, *vb = p.v + at;
#pragma unroll
                            for (int s = 0; s < KL; ++s) {
                                int off = s * 1024 + lane * 16;
                                if (BLOCK % 1024 != 0 && off >= BLOCK) off -= 512;           // (those dims are multiplied by zero)
                                kk[k][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kb + off));
                            }
                            if ((FP8 ? group : group >> 1) == k) mine = vb;
                        }
                        mine += mine_in_block;
#pragma unroll
                        for (int d = 0; d < DB; ++d) vv[d] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(mine + d * 256));
                        // scores, in units of log 2
                        floatx4 s4[RT][NT];
#pragma unroll
                        for (int k = 0; k < NT; ++k)
#pragma unroll
                            for (int r = 0; r < RT; ++r) {
                                floatx4 s = floatx4{0, 0, 0, 0};
#pragma unroll
                                for (int i = 0; i < KL; ++i) {
                                    if constexpr (FP8) {
                                        half8 lo, hi;
                                        widen(kk[k][i], lo, hi);
                                        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, q[r][2 * i], s, 0, 0, 0);
                                        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, q[r][2 * i + 1], s, 0, 0, 0);
                                    } else {
                                        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, kk[k][i]), q[r][i], s, 0, 0, 0);
                                    }
                                }
                                s4[r][k] = s * scale;
                            }
                        if (!plain) {
#pragma unroll
                            for (int k = 0; k < NT; ++k)
#pragma unroll
                                for (int r = 0; r < RT; ++r)
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {
                                        if (missing >> k & 1) s4[r][k][i] = __builtin_nanf("");
                                        if (!sees(t0[k] + 4 * group + i, pos[r], low[r], p.sinks)) s4[r][k][i] = kNegInf;
                                        // (an entry outside the cache gives NaN where a token is seen, nothing elsewhere)
                                    }
                            // values that no row sees may be anything: memory that was never written, another sequence's
                            int t = mine_first;
#pragma unroll
                            for (int k = 0; k < NT; ++k)
                                if ((FP8 ? group : group >> 1) == k) t += t0[k];
                            uint32_t keep[4] = {0, 0, 0, 0};
#pragma unroll
                            for (int i = 0; i < (FP8 ? 16 : 8); ++i)
                                if (sees(t + i, high_pos, first_low, p.sinks)) keep[FP8 ? i >> 2 : i >> 1] |= FP8 ? 0xffu << (8 * (i & 3)) : 0xffffu << (16 * (i & 1));
#pragma unroll
                            for (int d = 0; d < DB; ++d) vv[d] &= u32x4{keep[0], keep[1], keep[2], keep[3]};
                        }
                        if (clean)
#pragma unroll
                            for (int d = 0; d < DB; ++d) vv[d] = only_finite<FP8>(vv[d]);
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            float m = top[r];
#pragma unroll
                            for (int k = 0; k < NT; ++k) m = fmaxf(fmaxf(fmaxf(m, s4[r][k][0]), fmaxf(s4[r][k][1], s4[r][k][2])), s4[r][k][3]);
                            m = max_of_groups(m);
                            const float from = fmaxf(m, -1e30f) - kShift;        // (a row that has seen nothing yet)
                            const float shrink = __builtin_amdgcn_exp2f(fmaxf(top[r], -1e30f) - fmaxf(m, -1e30f));
                            top[r] = m;
                            uint32_t hi[NT][2], lo[NT][2];
                            float sum = 0.0f;
#pragma unroll
                            for (int k = 0; k < NT; ++k) {
                                float e[4], rest[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    e[i] = __builtin_amdgcn_exp2f(s4[r][k][i] - from);
                                    sum += e[i];
                                    rest[i] = e[i] - (float)(_Float16)e[i];
                                }
                                hi[k][0] = float2_to_half2_bits(e[0], e[1]);
                                hi[k][1] = float2_to_half2_bits(e[2], e[3]);
                                lo[k][0] = float2_to_half2_bits(rest[0], rest[1]);
                                lo[k][1] = float2_to_half2_bits(rest[2], rest[3]);
                            }
                            total[r] = total[r] * shrink + sum;
                            if (__builtin_amdgcn_ballot_w64(shrink != 1.0f)) {
#pragma unroll
                                for (int d = 0; d < DB; ++d) acc[r][d] *= shrink;
                            }
                            // from (block, tokens 4 group ...) to (group, the tokens that this group's values are of)
                            half8 ph[NT / 2], pl[NT / 2];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                if constexpr (FP8) {
                                    swap32(hi[0][i], hi[2][i]);  swap32(hi[1][i], hi[3][i]);
                                    swap16(hi[0][i], hi[1][i]);  swap16(hi[2][i], hi[3][i]);
                                    swap32(lo[0][i], lo[2][i]);  swap32(lo[1][i], lo[3][i]);
                                    swap16(lo[0][i], lo[1][i]);  swap16(lo[2][i], lo[3][i]);
                                } else {
                                    swap32(hi[0][i], hi[1][i]);  swap16(hi[0][i], hi[1][i]);
                                    swap32(lo[0][i], lo[1][i]);  swap16(lo[0][i], lo[1][i]);
                                }
                            }
#pragma unroll
                            for (int k = 0; k < NT / 2; ++k) {
                                ph[k] = __builtin_bit_cast(half8, u32x4{hi[2 * k][0], hi[2 * k][1], hi[2 * k + 1][0], hi[2 * k + 1][1]});
                                pl[k] = __builtin_bit_cast(half8, u32x4{lo[2 * k][0], lo[2 * k][1], lo[2 * k + 1][0], lo[2 * k + 1][1]});
                            }
#pragma unroll
                            for (int d = 0; d < DB; ++d) {
                                if constexpr (FP8) {
                                    half8 va, vb;
                                    widen(vv[d], va, vb);
                                    acc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, ph[0], acc[r][d], 0, 0, 0);
                                    acc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vb, ph[1], acc[r][d], 0, 0, 0);
                                    acc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, pl[0], acc[r][d], 0, 0, 0);
                                    acc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vb, pl[1], acc[r][d], 0, 0, 0);
                                } else {
                                    const half8 va = __builtin_bit_cast(half8, vv[d]);
                                    acc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, ph[0], acc[r][d], 0, 0, 0);
                                    acc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, pl[0], acc[r][d], 0, 0, 0);
                                }
                            }
                        }
                    }
                }
                bool bad = false;
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int d = 0; d < DB; ++d) bad |= not_finite(acc[r][d]);
                if (clean || !__builtin_amdgcn_ballot_w64(bad)) break;
                clean = true;
            }
            if (clean) {
                for (int kind = kPlusInf; kind <= kNaN; ++kind) {
                    floatx4 count[RT][DB];
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int d = 0; d < DB; ++d) count[r][d] = floatx4{0, 0, 0, 0};
                    for (int base = v0; base < v1; base += 64 * 4) {
                        const int page = pages_from(base);
                        for (int j = 0; j < 64 / NT; ++j) {
                            const int v = base + NT * (4 * j + wave);
                            if (v >= v1) break;
                            const int k = FP8 ? group : group >> 1;
                            const bool there = v + k < v1;
                            const int block = w.block(min(v + k, v1 - 1)), pg = __shfl(page, NT * j + k);
                            const bool valid = there && (uint32_t)pg < (uint32_t)p.pages;
                            const int t = valid ? block * 16 + mine_first : 0x7ffffff0;
                            const uint8_t *mine = p.v + offset(block, pg, valid) + mine_in_block;
                            half8 seen[RT][NT / 2];
#pragma unroll
                            for (int r = 0; r < RT; ++r)
#pragma unroll
                                for (int i = 0; i < 4 * NT; ++i) seen[r][i >> 3][i & 7] = sees(t + i, pos[r], low[r], p.sinks) ? (_Float16)1.0f : (_Float16)0.0f;
#pragma unroll
                            for (int d = 0; d < DB; ++d) {
                                const u32x4 vv = *reinterpret_cast<const u32x4 *>(mine + d * 256);
                                half8 part_of[NT / 2];
                                if constexpr (FP8) widen(vv, part_of[0], part_of[1]);
                                else part_of[0] = __builtin_bit_cast(half8, vv);
#pragma unroll
                                for (int i = 0; i < NT / 2; ++i)
#pragma unroll
                                    for (int r = 0; r < RT; ++r)
                                        count[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(of_kind(part_of[i], kind), seen[r][i], count[r][d], 0, 0, 0);
                            }
                        }
                    }
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int d = 0; d < DB; ++d)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (count[r][d][i] > 0.0f) acc[r][d][i] += of_kind_value(kind);
                }
            }

            // the four waves' sums: statistics first, then each wave's sums relative to the largest maximum; of rows that there are
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                total[r] = sum_of_groups(total[r]);
                if (group == 0) {
                    stat[wave][0][16 * r + col] = top[r];
                    stat[wave][1][16 * r + col] = total[r];
                }
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float m = kNegInf;
#pragma unroll
                for (int i = 0; i < 4; ++i) m = fmaxf(m, stat[i][0][16 * r + col]);
                const float f = __builtin_amdgcn_exp2f(fmaxf(top[r], -1e30f) - fmaxf(m, -1e30f));
                if (row[r] <= row1) {
#pragma unroll
                    for (int d = 0; d < DB; ++d) *reinterpret_cast<floatx4 *>(&part[wave][16 * r + col][16 * d + 4 * group]) = acc[r][d] * f;
                }
            }
            __syncthreads();
            const float v_scale = FP8 && p.v_scale ? p.v_scale[head] : 1.0f;
            for (int at = thread; at < (row1 - row0 + 1) * (D / 4); at += 256) {
                const int r = at / (D / 4), d = 4 * (at - r * (D / 4));
                float m = kNegInf, sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) m = fmaxf(m, stat[i][0][r]);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += stat[i][1][r] * __builtin_amdgcn_exp2f(fmaxf(stat[i][0][r], -1e30f) - fmaxf(m, -1e30f));
                floatx4 o = *reinterpret_cast<const floatx4 *>(&part[0][r][d]);
#pragma unroll
                for (int i = 1; i < 4; ++i) o += *reinterpret_cast<const floatx4 *>(&part[i][r][d]);
                if (chunks == 1) {
                    const int i = (row0 + r) / p.group, g = row0 + r - i * p.group;
                    const float f = v_scale / sum;
                    // a row that sees nothing is zero
                    *reinterpret_cast<u32x2 *>(p.O + (int64_t)(sq.first + i) * p.ldo + (int64_t)(head * p.group + g) * D + d) = past + i < 0 ? u32x2{0u, 0u} :
                        u32x2{float2_to_half2_bits(o[0] * f, o[1] * f), float2_to_half2_bits(o[2] * f, o[3] * f)};
                } else {
                    float *dst = p.partials + (((int64_t)tile * p.chunks + chunk) * p.part_rows + r) * (D + 2);
                    past_caches(dst + d, o[0], o[1]);
                    past_caches(dst + d + 2, o[2], o[3]);
                    if (d == 0) past_caches(dst + D, m, sum);
                }
            }
            if (chunks == 1) continue;
            join<D, 256>(p, thread, tile, chunks, sq, row0, row1, past, head, v_scale, shared, &last);
        }
    }
}

// ---- tile kernel --------------------------------------------------------------------------------------------------------------
// For many rows: bound by the matrix pipe and the exponentials.  A workgroup of NW waves takes 32 * NW rows, a wave 32 of them; keys and
// values of TK tokens at a time go through two buffers of LDS, which all waves read, in the storage's own order: a wave's operand reads
// are contiguous, nothing is transposed.  E4M3 codes become FP16 on their way into LDS, once for all rows.
// A row's probabilities are taken relative to a maximum that follows the true one only when that is 2^kLag larger, so that
// the sums are rarely rescaled.  P is rounded to FP16, as much as the output's own rounding, and its sum is that of the rounded values.  The
// output is then 2.5e-4 to 2.9e-4 off (2-norm, against 64 bits) where the rounding of the output alone is 2.0e-4.  With P as two terms, as in the
// streaming kernel, it is 2.0e-4, and a prompt of 8192 takes 786 us instead of 583, one of 2048 at 256 dims 110 / 90, 512 tokens after
// 8192 116 / 89, two chunks of 600 beside decoding sequences 204 / 168, 777 tokens of 64 dims 18.1 / 17.1: half as many products
// again and the vector work that makes the second term, which the streaming kernel has for nothing.
// 32 rows per wave: a wave's operand reads from LDS then take as long as its products.
// Measured: a prompt of 8192 tokens (32 query heads, 128 dims; 16, 256 dims alike) 583-600 us, 915-945 TFLOP/s; a large matrix product of the
// vendor's library reaches 1336 on this card, the matrix pipe alone 1580 under the power limit.  By the counters a step of 64 tokens takes 2240
// cycles of a SIMD for each of its two waves: the matrix pipe is busy for 1024 of them (46 %), vector instructions issue for 917 (41 %; 160 beside the
// 32 products, 32 exponentials among them), so that the two hardly overlap.
// Tried and dropped: scores one step ahead of their use (692 us), with an order of instructions given (643, 660); halves of the waves
// taking turns at the pipe with two barriers per step (688, with raised priority 677).
constexpr float kLag = 8.0f;
constexpr float kTileShift = 4.0f;                     // probabilities up to 2^(kLag + kTileShift)

// The sequence that the t-th tile of rows belongs to, and which of its tiles it is; b < 0: there are not so many.  Sequences of few rows have
// none (the streaming kernel's), the others one for every `tile_rows` rows.
struct TileOf { int b, index; };
__device__ __forceinline__ TileOf tile_of(const AttentionArgs &p, int t, int tile_rows) {
    if (!p.starts) {
        if (p.per * p.group <= p.few) return {-1, 0};
        const int each = (p.per * p.group + tile_rows - 1) / tile_rows, b = t / each;
        return {b < p.batch ? b : -1, t - b * each};
    }
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < p.batch; base += 64) {
        int mine = 0;
        if (base + lane < p.batch) {
            const int rows = sequence(p, base + lane).fresh * p.group;
            mine = rows > p.few ? (rows + tile_rows - 1) / tile_rows : 0;
        }
        int sum = mine;                                // of this lane's sequence and those before it
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
            const int other = __shfl_up(sum, i);
            if (lane >= i) sum += other;
        }
        const uint64_t past = __builtin_amdgcn_ballot_w64(t < sum);
        if (past) {
            const int at = __builtin_ctzll(past);
            return {base + at, t - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(mine, at))};
        }
        t -= __builtin_amdgcn_readlane(sum, 63);
    }
    return {-1, 0};
}

// v *= f where any bit of `mask` is set.  The branch is inside the statement: around a product in C++ the compiler keeps the sums in
// two sets of registers and copies one to the other in every step, 64 moves and 64 registers at 128 dims.  (The values come from
// matrix instructions that `f` depends on having ended; the waits are for `f`, an exponential, and for those that read the values next.)
__device__ __forceinline__ void scale_if(uint64_t mask, float f, floatx16 &v) {
#pragma unroll
    for (int i = 0; i < 16; i += 8) {
        float a = v[i], b = v[i + 1], c = v[i + 2], d = v[i + 3], e = v[i + 4], g = v[i + 5], h = v[i + 6], j = v[i + 7];
        asm("s_cmp_eq_u64 %9, 0\n\ts_cbranch_scc1 .Lscaled%=\n\ts_nop 1\n\t"
            "v_mul_f32 %0, %8, %0\n\tv_mul_f32 %1, %8, %1\n\tv_mul_f32 %2, %8, %2\n\tv_mul_f32 %3, %8, %3\n\t"
            "v_mul_f32 %4, %8, %4\n\tv_mul_f32 %5, %8, %5\n\tv_mul_f32 %6, %8, %6\n\tv_mul_f32 %7, %8, %7\n\ts_nop 1\n"
            ".Lscaled%=:"
            : "+v"(a), "+v"(b), "+v"(c), "+v"(d), "+v"(e), "+v"(g), "+v"(h), "+v"(j) : "v"(f), "s"(mask) : "scc");
        v[i] = a;  v[i + 1] = b;  v[i + 2] = c;  v[i + 3] = d;  v[i + 4] = e;  v[i + 5] = g;  v[i + 6] = h;  v[i + 7] = j;
    }
}

// What a workgroup of the tile kernel has to do; rows1 < 0: nothing.
struct TilePlace {
    int head, b, row0, row1, past, chunks;
    Sequence sq;
    Walk w;
};
__device__ __forceinline__ TilePlace tile_place(const AttentionArgs &p, int tile, int tile_rows) {
    TilePlace o;
    o.row1 = -1;
    o.head = tile % p.kv_heads;
    const TileOf at = tile_of(p, tile / p.kv_heads, tile_rows);
    if (at.b < 0) return o;
    o.b = at.b;
    o.sq = sequence(p, o.b);
    const int rows = o.sq.fresh * p.group, row_tiles = (rows + tile_rows - 1) / tile_rows;
    o.row0 = (row_tiles - 1 - at.index) * tile_rows;       // rows of late tokens, which see most, first
    o.row1 = min(rows, o.row0 + tile_rows) - 1;
    o.past = o.sq.past;
    o.w = walk(p, o.past + o.row0 / p.group, o.past + o.row1 / p.group);
    // (the workspace has room for the parts of the first split_tiles alone)
    o.chunks = tile / p.kv_heads < p.split_tiles ? min(p.chunks, max(1, (o.w.blocks + p.chunk_blocks - 1) / p.chunk_blocks)) : 1;
    return o;
}

template <int D, bool FP8, int NW, int TK>
__global__ void __launch_bounds__(64 * NW, D > 128 && NW == 4 ? 1 : 2)
attention_tile_kernel(AttentionArgs p) {
    constexpr int T = 64 * NW, NB = TK / 16, HB = TK / 32;       // threads, blocks and halves (of 32 tokens) of a tile of tokens
    constexpr int CB = FP8 ? D : 2 * D;                          // 16-byte chunks of a block in memory
    constexpr int CHUNKS = NB * CB, PER = (CHUNKS + T - 1) / T;  // of a tile, and per lane
    constexpr int KS = D / 16, DB = D / 32;
    extern __shared__ u32x4 lds[];                               // [2][keys, values][NB][2 D] chunks of FP16
    constexpr int HALF = NB * 2 * D, BUFFER = 2 * HALF;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    // the heads of a sequence on different XCDs
    const int tiles = p.kv_heads * p.row_tiles;
    const int chunk = blockIdx.x / tiles, tile = blockIdx.x - chunk * tiles;
    const TilePlace place = tile_place(p, tile, 32 * NW);
    if (place.row1 < 0 || chunk >= place.chunks) return;
    const int head = place.head, b = place.b, row0 = place.row0, row1 = place.row1, past = place.past, chunks = place.chunks;
    const Sequence sq = place.sq;
    const Walk w = place.w;
    const int low_pos = past + row0 / p.group, high_pos = past + row1 / p.group;
    const int v0 = chunk * p.chunk_blocks, v1 = chunk == chunks - 1 ? w.blocks : v0 + p.chunk_blocks;
    const int steps = (v1 - v0 + NB - 1) / NB;
    const int first_low = before(p, low_pos);

    // this wave's rows
    const int wave_row0 = row0 + 32 * wave;
    const bool idle = wave_row0 > row1;
    const int clamped = min(wave_row0 + col, row1), token = clamped / p.group, g = clamped - token * p.group;
    const int pos = past + token, low = before(p, pos);
    const int wave_low = past + min(wave_row0, row1) / p.group, wave_high = past + min(wave_row0 + 31, row1) / p.group;
    const int wave_last_low = before(p, wave_high);
    half8 q[KS];
    {
        const uint16_t *src = p.Q + (int64_t)(sq.first + token) * p.ldq + (int64_t)(head * p.group + g) * D + 8 * h;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const half8 *>(src + 16 * s);
    }
    // (a negative scale turns the queries round, so that the largest product has the largest score)
    float scale = p.scale * kLog2e * (FP8 && p.k_scale ? p.k_scale[head] : 1.0f);
    if (scale < 0.0f) {
        scale = -scale;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = -q[s];
    }
    scale = scale < 1e-30f ? 1e-30f : scale;                     // (zero: a masked score has to stay -Inf; a NaN stays one)
    const int in_page = (1 << p.page_shift) - 1;
    // the row of S^T that this lane's operand of K holds is one of these tokens of a half: with it the lane's scores are those of the 8
    // tokens that its operand of V holds (8 h ... of each block)
    const int k_token = 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
    const int k_chunk = (col >> 4) * 2 * D + h * 16 + k_token, v_chunk = h * D + col;

    int page = 0, page_base = v0 - 64;                           // pages of the 64 blocks from page_base, a lane each
    u32x4 kreg[PER], vreg[PER];

    // where a block of the walk lies: -1 if it is not in the cache (blocks behind the last one: some block's place)
    const auto offset_of = [&](int v) -> int64_t {
        v = min(v, v1 - 1);
        const int pg = __builtin_amdgcn_readlane(page, v - page_base);
        const int64_t at = ((((int64_t)pg * p.kv_heads + head) << p.page_shift) + (w.block(v) & in_page)) * (CB * 16);
        return (uint32_t)pg < (uint32_t)p.pages ? at : -1;
    };
    // Steps from `from` to `to` see nothing but tokens that the rows from position low to high (and windows from after first to after
    // last) see whole, one block behind the other.
    struct Span { int from, to; };
    const auto whole = [&](int low_pos, int last_low) {
        const int behind = max(w.sink_blocks, w.sink_blocks + ((last_low + 16) >> 4) - w.low_block);    // the first block of the walk that starts after last_low
        const int until = min(v1, w.sink_blocks + ((low_pos + 1) >> 4) - w.low_block);                  // blocks before it end by low_pos
        return Span{max(0, behind - v0 + NB - 1) / NB, until > v0 ? (until - v0) / NB : 0};
    };
    const Span staged = whole(high_pos, first_low), plain_steps = whole(wave_low, wave_last_low);

    bool holes = false;                                          // some block so far is not in the cache
    const auto load = [&](int step) {
        const int v = v0 + step * NB;
        if (v >= page_base + 64) {
            page_base = v;
            page = v + lane < v1 ? p.table[(int64_t)b * p.ld_table + (w.block(v + lane) >> p.page_shift)] : 0;
            holes |= __builtin_amdgcn_ballot_w64((uint32_t)page >= (uint32_t)p.pages && v + lane < v1) != 0;
        }
        // (not known to be the same in every step: addresses per lane, kept over the loop, would be 64 bits each)
        uint32_t thread = threadIdx.x;
        if constexpr (D > 128) asm volatile("" : "+v"(thread));
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int id = thread + i * T, first = (64 * wave + i * T) / CB;
            if (CHUNKS % T != 0 && 64 * wave + i * T >= CHUNKS) break;
            int64_t from = max(offset_of(v + first), (int64_t)0);
            int block = first;
            if (CB % 64 != 0) {                                  // (64 chunks from two blocks)
                const int64_t next = max(offset_of(v + first + 1), (int64_t)0);
                block = id / CB;
                from = block == first ? from : next;
            }
            const uint32_t place = (uint32_t)(id - block * CB) * 16;
            kreg[i] = *reinterpret_cast<const u32x4 *>(p.k + from + place);
            vreg[i] = *reinterpret_cast<const u32x4 *>(p.v + from + place);
        }
    };
    const auto first_token = [&](int v) { return v < v1 ? w.block(v) * 16 : 0x7ffffff0; };     // (nothing sees those)
    const auto store = [&](int step, int buffer) {
        const int v = v0 + step * NB;
        const bool plain = step >= staged.from && step < staged.to;
        u32x4 *keys = lds + buffer * BUFFER, *values = keys + HALF;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int id = threadIdx.x + i * T;
            if (CHUNKS % T != 0 && 64 * wave + i * T >= CHUNKS) break;
            const int block = CB % 64 ? id / CB : (64 * wave + i * T) / CB, place = id - block * CB;
            u32x4 vv = vreg[i];
            if (!plain) {
                // values that no row sees may be anything: memory that was never written, another sequence's
                int at = place;                                  // (as in `load`)
                if constexpr (D > 128) asm volatile("" : "+v"(at));
                const int t = first_token(v + block) + (FP8 ? 0 : at >= D ? 8 : 0);
                uint32_t keep[4] = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < (FP8 ? 16 : 8); ++j)
                    if (sees(t + j, high_pos, first_low, p.sinks)) keep[FP8 ? j >> 2 : j >> 1] |= FP8 ? 0xffu << (8 * (j & 3)) : 0xffffu << (16 * (j & 1));
                vv &= u32x4{keep[0], keep[1], keep[2], keep[3]};
            }
            if constexpr (FP8) {
                half8 lo, hi;
                widen(kreg[i], lo, hi);
                const int k_at = block * 2 * D + (place >> 4) * 32 + (place & 15), v_at = block * 2 * D + place;
                keys[k_at] = __builtin_bit_cast(u32x4, lo);
                keys[k_at + 16] = __builtin_bit_cast(u32x4, hi);
                widen(vv, lo, hi);
                values[v_at] = __builtin_bit_cast(u32x4, lo);
                values[v_at + D] = __builtin_bit_cast(u32x4, hi);
            } else {
                keys[id] = kreg[i];
                values[id] = vv;
            }
        }
    };

    floatx16 acc[DB];
    float top, total;
    top = kNegInf;
    total = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
    if (steps > 0) {
        load(0);
        store(0, 0);
        if (steps > 1) load(1);
    }
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
        const u32x4 *keys = lds + (step & 1) * BUFFER, *values = keys + HALF;
        floatx16 s[HB];
#pragma unroll
        for (int t = 0; t < HB; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k)
                s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, keys[t * 4 * D + k * 32 + k_chunk]), q[k], s[t], 0, 0, 0);
        }
        if (step + 1 < steps) store(step + 1, (step + 1) & 1);
        if (step + 2 < steps) load(step + 2);
        if (holes || step < plain_steps.from || step >= plain_steps.to) {
            const int v = v0 + step * NB;
#pragma unroll
            for (int k = 0; k < NB; ++k) {
                const int t = first_token(v + k) + 8 * h;
                bool there = true;
                if (holes) there = (uint32_t)p.table[(int64_t)b * p.ld_table + (w.block(min(v + k, v1 - 1)) >> p.page_shift)] < (uint32_t)p.pages;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    // (an entry outside the cache gives NaN where a token is seen, nothing elsewhere)
                    const float x = there ? s[k >> 1][8 * (k & 1) + i] : __builtin_nanf("");
                    s[k >> 1][8 * (k & 1) + i] = sees(t + i, pos, low, p.sinks) ? x : kNegInf;
                }
            }
        }
        float m = kNegInf;
#pragma unroll
        for (int t = 0; t < HB; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 2) m = fmaxf(fmaxf(m, s[t][i]), s[t][i + 1]);
        {
            uint32_t x = __float_as_uint(m), y = x;
            swap32(x, y);
            m = fmaxf(__uint_as_float(x), __uint_as_float(y));
        }
        m *= scale;
        // (also where the first score is seen: top is -Inf until then)
        const uint64_t behind = __builtin_amdgcn_ballot_w64(m > top + kLag);
        const float next = behind ? fmaxf(top, m) : top;
        const float shrink = __builtin_amdgcn_exp2f(fmaxf(top, -1e30f) - fmaxf(next, -1e30f));
        top = next;
        total *= shrink;
#pragma unroll
        for (int d = 0; d < DB; ++d) scale_if(behind, shrink, acc[d]);
        const float from = kTileShift - fmaxf(top, -1e30f);
        half8 pr[2 * HB];
#pragma unroll
        for (int t = 0; t < HB; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) pr[2 * t + (i >> 3)][i & 7] = (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], scale, from));
        typedef _Float16 half2v __attribute__((ext_vector_type(2)));
        const half2v ones = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
        for (int k = 0; k < 2 * HB; ++k)
#pragma unroll
            for (int i = 0; i < 8; i += 2) total = __builtin_amdgcn_fdot2(half2v{pr[k][i], pr[k][i + 1]}, ones, total, false);
#pragma unroll
        for (int k = 0; k < 2 * HB; ++k)
#pragma unroll
            for (int d = 0; d < DB; ++d)
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, values[k * 2 * D + d * 32 + v_chunk]), pr[k], acc[d], 0, 0, 0);
        __syncthreads();
    }
    bool bad = false;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) bad |= not_finite(floatx4{acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]});
    if (__builtin_amdgcn_ballot_w64(bad && !idle)) {
        // this wave's rows again, straight from memory and by itself: first without the values that are not finite ...
        const auto refresh = [&](int v) {
            if (((v - v0) & 63) == 0) {
                page_base = v;
                page = v + lane < v1 ? p.table[(int64_t)b * p.ld_table + (w.block(v + lane) >> p.page_shift)] : 0;
            }
        };
        const auto values_of = [&](int64_t at, int d) {
            if constexpr (FP8) {
                half8 lo, hi;
                widen(*reinterpret_cast<const u32x4 *>(p.v + at + (d * 32 + col) * 16), lo, hi);
                return h ? hi : lo;
            } else {
                return *reinterpret_cast<const half8 *>(p.v + at + (d * 32 + v_chunk) * 16);
            }
        };
        top = kNegInf;
        total = 0.0f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
        for (int v = v0; v < v1; v += 2) {
            refresh(v);
            const int64_t first = offset_of(v), second = offset_of(v + 1), mine = (col >> 4) ? second : first;
            const uint8_t *keys = p.k + max(mine, (int64_t)0);
            floatx16 s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                half8 x;
                if constexpr (FP8) {
                    half8 lo, hi;
                    widen(*reinterpret_cast<const u32x4 *>(keys + (k * 16 + k_token) * 16), lo, hi);
                    x = h ? hi : lo;
                } else {
                    x = *reinterpret_cast<const half8 *>(keys + (k * 32 + h * 16 + k_token) * 16);
                }
                s = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, q[k], s, 0, 0, 0);
            }
            float m = top;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int t = first_token(v + (i >> 3)) + 8 * h + (i & 7);
                s[i] = (i >> 3 ? second : first) < 0 ? __builtin_nanf("") : s[i] * scale;
                if (!sees(t, pos, low, p.sinks)) s[i] = kNegInf;
                m = fmaxf(m, s[i]);
            }
            uint32_t x = __float_as_uint(m), y = x;
            swap32(x, y);
            m = fmaxf(__uint_as_float(x), __uint_as_float(y));
            const float shrink = __builtin_amdgcn_exp2f(fmaxf(top, -1e30f) - fmaxf(m, -1e30f)), from = fmaxf(m, -1e30f) - kTileShift;
            top = m;
            total *= shrink;
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] *= shrink;
            half8 pr[2];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = __builtin_amdgcn_exp2f(s[i] - from);
                total += e;
                pr[i >> 3][i & 7] = (_Float16)e;
            }
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int64_t at = k ? second : first;
                    const u32x4 vv = only_finite<false>(__builtin_bit_cast(u32x4, values_of(max(at, (int64_t)0), d)));
                    acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, vv), pr[k], acc[d], 0, 0, 0);
                }
        }
        // ... then what these add to the rows that do see them
#pragma unroll
        for (int d = 0; d < DB; ++d) {
#pragma unroll 1
            for (int kind = kPlusInf; kind <= kNaN; ++kind) {
                floatx16 count;
#pragma unroll
                for (int i = 0; i < 16; ++i) count[i] = 0.0f;
#pragma unroll 1
                for (int v = v0; v < v1; ++v) {
                    refresh(v);
                    const int64_t at = offset_of(v);
                    if (at < 0) continue;
                    const int t = w.block(v) * 16 + 8 * h;
                    half8 seen;
#pragma unroll
                    for (int i = 0; i < 8; ++i) seen[i] = sees(t + i, pos, low, p.sinks) ? (_Float16)1.0f : (_Float16)0.0f;
                    count = __builtin_amdgcn_mfma_f32_32x32x16_f16(of_kind(values_of(at, d), kind), seen, count, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (count[i] > 0.0f) acc[d][i] += of_kind_value(kind);
            }
        }
    }
    {
        uint32_t x = __float_as_uint(total), y = x;
        swap32(x, y);
        total = __uint_as_float(x) + __uint_as_float(y);
    }
    const float v_scale = FP8 && p.v_scale ? p.v_scale[head] : 1.0f;
    if (chunks == 1) {
        // (the row's place is worked out again: over the loop it would cost registers)
        int again = lane;
        asm volatile("" : "+v"(again));
        const int row = wave_row0 + (again & 31), token = row / p.group, g = row - token * p.group;
        if (row > row1) return;
        uint16_t *dst = p.O + (int64_t)(sq.first + token) * p.ldo + (int64_t)(head * p.group + g) * D + 4 * (again >> 5);
        const float f = v_scale / total;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<u32x2 *>(dst + 32 * d + 2 * i) = past + token < 0 ? u32x2{0u, 0u} :
                    u32x2{float2_to_half2_bits(acc[d][i] * f, acc[d][i + 1] * f), float2_to_half2_bits(acc[d][i + 2] * f, acc[d][i + 3] * f)};
        return;
    }
    int again = lane;
    asm volatile("" : "+v"(again));
    // this wave's part: the sums as its lanes hold them, then the rows' maxima and sums of probabilities
    float *part = p.partials + (((int64_t)tile * p.chunks + chunk) * NW + wave) * (32 * (D + 2));
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<floatx4 *>(part + ((d * 4 + (i >> 2)) * 64 + again) * 4) = floatx4{acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
    if (again < 32) {
        part[32 * D + 2 * again] = top;
        part[32 * D + 2 * again + 1] = total;
    }
}

// Joins the parts of split tiles, in order: a launch of its own, since a tile's parts are hundreds of kilobytes and all of the chip can
// read them then, where the last workgroup of a tile would read them alone (64 tokens after 16384, 4 query heads to a key/value head: 287
// us in all that way).  A workgroup has the 32 rows of one wave and DN dims,
// and the loads of several parts
// under way (17 parts of 256 rows of 256 dims 42 us with one at a time and all dims, now 7.6).  Few tiles: 32 dims each, to fill the chip
// (22 parts of 256 rows of 128 dims, 8 tiles 11.8 -> 7.6); where there are many it costs, all of them look their tile up (1216 waves' rows 19.4 against 12.7).
template <int D, int DN>
__global__ void __launch_bounds__(256)
attention_join_kernel(AttentionArgs p, int waves, const float *v_scales) {
    constexpr int DB = DN / 32, SPLIT = D / DN, AHEAD = DB == 1 ? 8 : 4;
    const int of_tile = waves * SPLIT, tile = blockIdx.x / of_tile, rest = blockIdx.x - tile * of_tile, wave = rest / SPLIT, d0 = (rest - wave * SPLIT) * DB;
    const TilePlace place = tile_place(p, tile, 32 * waves);
    const int lane = threadIdx.x & 63, col = lane & 31, i4 = threadIdx.x >> 6;
    const int row = place.row0 + 32 * wave + col;
    if (place.row1 < 0 || place.chunks <= 1 || place.row0 + 32 * wave > place.row1) return;
    const float *part = p.partials + ((int64_t)tile * p.chunks * waves + wave) * (32 * (D + 2));
    const int64_t next = (int64_t)waves * (32 * (D + 2));
    float top = kNegInf, total = 0.0f;
    floatx4 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = floatx4{0, 0, 0, 0};
    for (int c = 0; c < place.chunks; c += AHEAD) {
        float m[AHEAD], l[AHEAD];
        floatx4 o[AHEAD][DB];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float *from = part + min(c + i, place.chunks - 1) * next;      // (behind the last part: that one again, left out below)
            m[i] = from[32 * D + 2 * col];
            l[i] = from[32 * D + 2 * col + 1];
#pragma unroll
            for (int d = 0; d < DB; ++d) o[i][d] = *reinterpret_cast<const floatx4 *>(from + (((d0 + d) * 4 + i4) * 64 + lane) * 4);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const bool there = c + i < place.chunks;
            const float mine = there ? m[i] : kNegInf, now = fmaxf(top, mine), ref = fmaxf(now, -1e30f);
            const float f = __builtin_amdgcn_exp2f(fmaxf(top, -1e30f) - ref), g = __builtin_amdgcn_exp2f(fmaxf(mine, -1e30f) - ref);
            top = now;
            total = total * f + (there ? l[i] : 0.0f) * g;
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] = acc[d] * f + (there ? o[i][d] : floatx4{0, 0, 0, 0}) * g;
        }
    }
    if (row > place.row1) return;
    const int token = row / p.group, g = row - token * p.group;
    uint16_t *dst = p.O + (int64_t)(place.sq.first + token) * p.ldo + (int64_t)(place.head * p.group + g) * D + 32 * d0 + 8 * i4 + 4 * (lane >> 5);
    const float f = (v_scales ? v_scales[place.head] : 1.0f) / total;
#pragma unroll
    for (int d = 0; d < DB; ++d)
        *reinterpret_cast<u32x2 *>(dst + 32 * d) = place.past + token < 0 ? u32x2{0u, 0u} :
            u32x2{float2_to_half2_bits(acc[d][0] * f, acc[d][1] * f), float2_to_half2_bits(acc[d][2] * f, acc[d][3] * f)};
}

// ---- launch shapes ----------------------------------------------------------------------------------------------------------

// Blocks that a tile of `rows` rows sees at most.
static int64_t blocks_seen(const AttentionShape &s, int64_t rows) {
    int64_t blocks = (s.max_len + 15) / 16;
    if (s.window > 0) {
        const int64_t near = (s.window + rows / s.group + 17) / 16 + 1 + (s.sinks + 15) / 16;
        if (near < blocks) blocks = near;
    }
    return blocks < 1 ? 1 : blocks;
}

// `busy`: tiles among a.tiles that are expected to have work; `wanted`: workgroups that fill the chip; `least`: blocks below
// which a workgroup has too little to do; `tickets`: the parts are joined by the last workgroup of a tile, which takes a counter.
static void plan_launch(AttentionLaunch &a, const AttentionShape &s, int64_t tile_rows, int64_t busy, int64_t least, int64_t wanted, bool tickets) {
    const int64_t blocks = blocks_seen(s, tile_rows);
    int64_t chunk = (blocks * busy + wanted - 1) / wanted, step = least;
    if (!tickets && wanted >= 2 * busy) {
        // equal parts, all in one round: 76 tiles of 4600 tokens and 256 dims in three 130 us, in three and a remainder, which waits for a
        // free CU, 156; 32 tiles of 8320 tokens (128 dims) 36.9 against 39.3.  (Between one and two rounds the remainder pays: 152 tiles of
        // 5800 tokens 167 us, whole 238.)
        chunk = (blocks + wanted / busy - 1) / (wanted / busy);
        step = 4;
    }
    if (tuning().attn_chunk > 0) chunk = tuning().attn_chunk / 16;
    if (chunk < least) chunk = least;
    chunk = (chunk + step - 1) / step * step;
    if (tickets && a.tiles > kMaxCounters) chunk = (blocks + least - 1) / least * least;
    a.chunk_blocks = chunk;
    a.chunks = (blocks + chunk - 1) / chunk;
    a.partial_bytes = a.chunks > 1 ? (size_t)a.tiles * (size_t)a.chunks * (size_t)a.part_rows * (size_t)(s.D + 2) * sizeof(float) : 0;
}

constexpr size_t kMostPartBytes = (size_t)256 << 20;   // parts of the tile kernel; a full chip's are 68 MB at 256 dims

AttentionPlan attention_plan(const AttentionShape &s) {
    AttentionPlan a;
    const int64_t rows = s.max_new * s.group, stream_rows = s.D > 128 ? 16 : 32;      // (two tiles of 256 dims do not fit the registers)
    a.few = 0;
    a.scan = false;
    a.stream.tiles = a.tile.tiles = a.stream.split_tiles = a.tile.split_tiles = 0;
    a.stream.partial_bytes = a.tile.partial_bytes = 0;
    const bool many = tuning().attn_tiles >= 0 ? tuning().attn_tiles > 0 : rows > stream_rows;
    if (many) {
        // sequences of few rows beside the others: none if all have as many new tokens
        a.few = s.ragged && rows > stream_rows && s.group <= stream_rows ? stream_rows : 0;
        const int64_t total = s.tokens * s.group;
        // 128-row tiles where 256-row tiles would leave CUs without work, unless the sequences are long, whose keys and values are then
        // read twice as often: 777 tokens of 64 dims 16.7 against 18.3 us, a prompt of 2048 68.2 / 69.7; 512 tokens after 8192
        // 104 against 91.  256 dims: 16 query heads, 512 tokens 30 / 35, 1000 51 / 46, 2048 134 / 89 (four waves fill the registers of
        // a CU, one to a SIMD, so that nothing runs beside a wave's exponentials; with eight the compiler keeps a wave in 256).
        a.waves = tuning().attn_waves > 0 ? tuning().attn_waves :
                  (total + 255) / 256 * s.kv_heads >= (s.D > 128 ? 64 : 512) || s.max_len >= 4096 ? 8 : 4;
        const int64_t tile_rows = 32 * a.waves;
        int64_t most = s.batch * ((rows + tile_rows - 1) / tile_rows), likely = most;
        if (s.ragged) {
            // rows lie in whole tiles, but for the last one of every sequence that has any
            const int64_t with = s.tokens / (a.few / s.group + 1);
            const int64_t bound = total / tile_rows + (with < s.batch ? with : s.batch);
            if (bound < most) most = bound;
            likely = (total + tile_rows - 1) / tile_rows;
            if (likely > most) likely = most;
        }
        a.tile.row_tiles = most;
        a.tile.tiles = most * s.kv_heads;
        a.tile.part_rows = tile_rows;
        plan_launch(a.tile, s, tile_rows, likely * s.kv_heads, s.D > 128 ? 8 : 16, a.waves == 8 || s.D > 128 ? 256 : 512, false);
        // Where every sequence may have a tile that it does not fill there can be many times the likely tiles: room for the parts of all of
        // them, up to a bound (it would be 1.7 GB for 1600 tokens in 1000 sequences at 256 dims).  Tiles behind it are whole; so many fill the
        // chip as they are.  Room for twice the likely ones and 8 more instead: 85 sequences of 9 tokens before 512 tokens after
        // 16384, whose tiles are the last, 540 us instead of 385 (102 MB instead of 224).
        const size_t each = (size_t)(s.kv_heads * a.tile.chunks * tile_rows * (s.D + 2)) * sizeof(float);
        const size_t split = std::min((size_t)most, kMostPartBytes / each);
        if (split == 0) a.tile.chunks = 1;
        a.tile.split_tiles = (int64_t)split;
        a.tile.partial_bytes = a.tile.chunks > 1 ? split * each : 0;
    }
    if (!many || a.few > 0) {
        const int64_t most = many ? a.few / s.group * s.group : rows;
        // (beside prompt chunks most sequences have one new token; the others read their keys and values twice)
        a.rt = most <= 16 || many || s.D > 128 ? 1 : 2;
        a.stream.row_tiles = (most + 16 * a.rt - 1) / (16 * a.rt);
        a.stream.tiles = s.batch * s.kv_heads * a.stream.row_tiles;
        a.stream.part_rows = most < 16 * a.rt ? most : 16 * a.rt;
        plan_launch(a.stream, s, 16 * a.rt, a.stream.tiles, s.fp8 ? 16 : 8, s.batch <= kScan ? 4096 : 1536, true);
        // a schedule worked out by the workgroups, unless there is nothing to share out; its parts of a tile are one more, since a tile
        // may begin anywhere in a stretch
        AttentionLaunch &l = a.stream;
        a.scan = s.batch <= kScan && l.chunks > 1;
        if (a.scan) {
            l.chunks += 1;
            l.partial_bytes = (size_t)l.tiles * (size_t)l.chunks * (size_t)l.part_rows * (size_t)(s.D + 2) * sizeof(float);
        }
    }
    a.partial_bytes = a.stream.partial_bytes > a.tile.partial_bytes ? a.stream.partial_bytes : a.tile.partial_bytes;
    return a;
}

static bool shape_of(const AttentionLaunch &l, AttentionArgs &a, dim3 &grid) {
    const int64_t groups = l.tiles * l.chunks;
    if (groups > 0xfffffff) return false;
    a.row_tiles = (int)l.row_tiles;
    a.part_rows = (int)l.part_rows;
    a.chunk_blocks = (int)l.chunk_blocks;
    a.chunks = (int)l.chunks;
    a.split_tiles = (int)l.split_tiles;
    grid = dim3((unsigned)groups);
    return true;
}

template <int D, bool FP8>
static void launch_stream(int64_t rt, const AttentionArgs &a, dim3 grid, hipStream_t stream) {
    if constexpr (D <= 128) {
        if (rt == 2) {
            attention_stream_kernel<D, FP8, 2><<<grid, 256, 0, stream>>>(a);
            return;
        }
    }
    attention_stream_kernel<D, FP8, 1><<<grid, 256, 0, stream>>>(a);
}

template <int D, bool FP8>
static int launch_tile(int64_t waves, const AttentionArgs &a, dim3 grid, hipStream_t stream) {
    constexpr int TK = D <= 128 ? 64 : 32, LDS = 8 * TK * D;         // two buffers of keys and values in FP16
    static_assert(LDS <= 65536, "");
    if (waves == 8) attention_tile_kernel<D, FP8, 8, TK><<<grid, 512, LDS, stream>>>(a);
    if (waves == 4) attention_tile_kernel<D, FP8, 4, TK><<<grid, 256, LDS, stream>>>(a);
    const int st = hip_ok(hipGetLastError());
    if (a.chunks == 1 || st != kOk) return st;
    const int64_t groups = grid.x / a.chunks * waves;
    if (groups <= 256) attention_join_kernel<D, 32><<<dim3(groups * (D / 32)), 256, 0, stream>>>(a, (int)waves, FP8 ? a.v_scale : nullptr);
    else attention_join_kernel<D, D <= 128 ? D : 128><<<dim3(groups * (D <= 128 ? 1 : 2)), 256, 0, stream>>>(a, (int)waves, FP8 ? a.v_scale : nullptr);
    return hip_ok(hipGetLastError());
}

int launch_attention(const AttentionShape &s, const AttentionPlan &plan, AttentionArgs a, hipStream_t stream) {
    dim3 grid;
    a.few = (int)plan.few;
    int st = kOk;
#define NFP_FOR_D(CALL)                                                     \
    switch (s.D) {                                                          \
        case 64: if (s.fp8) { CALL(64, true); } else { CALL(64, false); } break;    \
        case 96: if (s.fp8) { CALL(96, true); } else { CALL(96, false); } break;    \
        case 128: if (s.fp8) { CALL(128, true); } else { CALL(128, false); } break; \
        default: if (s.fp8) { CALL(256, true); } else { CALL(256, false); } break;  \
    }
    if (plan.tile.tiles > 0) {
        if (!shape_of(plan.tile, a, grid)) return kErrShape;
#define NFP_TILE(D, FP8) st = launch_tile<D, FP8>(plan.waves, a, grid, stream)
        NFP_FOR_D(NFP_TILE)
#undef NFP_TILE
        if (st != kOk) return st;
    }
    if (plan.stream.tiles > 0) {
        if (!shape_of(plan.stream, a, grid)) return kErrShape;
        // (the lengths are bounded by the table alone, and the blocks of all tiles are counted in 31 bits)
        a.scan = plan.scan && plan.stream.tiles * (((int64_t)a.columns << a.page_shift) + 16) < (int64_t)1 << 30;
        a.fixed = tuning().attn_chunk > 0;
        // 256 workgroups up to 128 tiles, 512 above (microseconds with 256 / 512: one sequence of 8192 15.4 / 21.7, of 131072 84.3 / 90.5, 8 of 4096
        // 26.7 / 27.8, 12 with a window of 4096, 120 tiles, 50.9 / 52.9): of 512 more share a tile, and meet in its join
        if (a.scan) grid = dim3((unsigned)std::min<int64_t>(grid.x, tuning().attn_groups > 0 ? tuning().attn_groups : plan.stream.tiles <= 128 ? 256 : 512));
#define NFP_STREAM(D, FP8) launch_stream<D, FP8>(plan.rt, a, grid, stream)
        NFP_FOR_D(NFP_STREAM)
#undef NFP_STREAM
        st = hip_ok(hipGetLastError());
    }
#undef NFP_FOR_D
    return st;
}

}  // namespace nfp
