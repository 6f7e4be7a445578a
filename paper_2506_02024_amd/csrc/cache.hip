// Rotary positions on the queries and keys of new tokens, and the write of keys and values into the paged cache.
// Cache storage (include/nestedfp.h): blocks of 16 tokens; with E elements in 16 bytes a key block is
// [D / E][16 tokens][E dims], a value block [16 / E][D][E tokens], which is the order in which lanes of the
// attention kernels hold matrix operands.
// HBM-bound: 2 bytes read per value of q, k and v, 2 (q) and 2 or 1 (k, v) written; the tables come from the caches.  Measured (8 key/value heads
// of 128 dims, 32 query heads): 4101 tokens into FP16 24.2 us (4.2 TB/s; a large copy reaches 4.9), 8192 into E4M3 55 us (3.4 TB/s),
// 16 tokens 4.7 us (loads one after the other: position, then angles).  In the second of these the vector unit issues 37 % of the cycles, LDS is
// active in 2 %, waves wait for memory in 55 % of theirs; 103 MB are read and 88 written, where 103 and 84 have to be: short workgroups,
// whose loads and stores do not overlap much.
#include "nfp_device.h"
#include "nfp_host.h"

#include <algorithm>

namespace nfp {

constexpr int kAppendThreads = 256;

// byte offset of the block that holds a slot
__device__ __forceinline__ int64_t block_offset(const AppendArgs &p, int slot, int head) {
    const int block = slot >> 4, page = block >> p.page_shift, in_page = block & ((1 << p.page_shift) - 1);
    return ((((int64_t)page * p.kv_heads + head) << p.page_shift) + in_page) * (16 * p.D * (p.fp8 ? 1 : 2));
}

__device__ __forceinline__ void unpack8(const u32x4 &v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = half_bits_to_float(w[i] & 0xffffu);
        f[2 * i + 1] = half_bits_to_float(w[i] >> 16);
    }
}
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
    return u32x4{float2_to_half2_bits(f[0], f[1]), float2_to_half2_bits(f[2], f[3]),
                 float2_to_half2_bits(f[4], f[5]), float2_to_half2_bits(f[6], f[7])};
}
// Codes are rounded once, from the 32-bit value, and saturate at +-448 (a NaN stays one).  The quotient by the caller's scale is
// the correctly rounded one: by its reciprocal and the remainder for scales far inside the binary32 range, by a division for others.
struct Divisor {
    float s, y;
    bool quick;
    __device__ __forceinline__ explicit Divisor(float scale) : s(scale), y(1.0f / scale), quick(scale > 1e-30f && scale < 1e30f) {}
    __device__ __forceinline__ float quotient(float x) const {
        float q;
        if (quick) {
            const float first = x * y;
            q = __builtin_fmaf(__builtin_fmaf(-first, s, x), y, first);
            q = fabsf(first) < __builtin_inff() ? __builtin_copysignf(q, x) : first;
        } else {
            q = x / s;
        }
        return q != q ? q : clamp448(q);
    }
};
__device__ __forceinline__ u32x2 codes8(const float (&f)[8], const Divisor &s) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = s.quotient(f[i]);
    return u32x2{e4m3x4_from_float_hw(q[0], q[1], q[2], q[3]), e4m3x4_from_float_hw(q[4], q[5], q[6], q[7])};
}

// Many tokens: what is written is far larger than the caches, and written past them (4101 tokens 32 -> 26 us).
template <bool MANY, typename T>
__device__ __forceinline__ void put(T *to, const T &v) {
    if (MANY) __builtin_nontemporal_store(v, to);
    else *to = v;
}

// 8 dims from `dim` (a multiple of 8) of one token's query or key
template <bool MANY>
__device__ __forceinline__ void put8(const AppendArgs &p, bool query, int head, int64_t m, int slot, int dim, const float (&f)[8]) {
    if (query) {
        put<MANY>(reinterpret_cast<u32x4 *>(p.out + m * p.ldo + (int64_t)head * p.D + dim), pack8(f));
        return;
    }
    if (slot < 0) return;
    uint8_t *block = p.k + block_offset(p, slot, head);
    const int token = slot & 15;
    if (p.fp8)
        put<MANY>(reinterpret_cast<u32x2 *>(block + ((dim >> 4) * 16 + token) * 16 + (dim & 8)), codes8(f, Divisor(p.k_scale ? p.k_scale[head] : 1.0f)));
    else
        put<MANY>(reinterpret_cast<u32x4 *>(block + ((dim >> 3) * 16 + token) * 16), pack8(f));
}

// Queries and keys of HEADS heads: a lane has 8 dims and their 8 partners (or 8 dims that are not rotated) of one token, in every
// head, with the token's angles in registers (with one head to a lane the tables were read 48 times over).
template <int HEADS>
__device__ __forceinline__ void rotate(const AppendArgs &p, int first_head) {
    const int r = p.rotary / 2, turns = r / 8, items = turns + (p.D - p.rotary) / 8;
    const int token = threadIdx.x / items, item = threadIdx.x - token * items;
    const int64_t m = (int64_t)blockIdx.x * p.group + token;
    if (token >= p.group || m >= p.M) return;
    const bool turned = item < turns, odd = item & 1;
    // chunks of 16 codes: dims of two items each, where both halves of a head begin at a chunk (items of a token are even in number then)
    const bool pairs = p.fp8 && r % 16 == 0;
    const int lo_dim = turned ? 8 * item : p.rotary + 8 * (item - turns), hi_dim = lo_dim + r;
    u32x4 lo[HEADS], hi[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int head = min(first_head + i, p.heads + p.kv_heads - 1);
        const uint16_t *x = head < p.heads ? p.q + m * p.ldq + (int64_t)head * p.D : p.new_k + m * p.ldk + (int64_t)(head - p.heads) * p.D;
        lo[i] = *reinterpret_cast<const u32x4 *>(x + lo_dim);
        if (turned) hi[i] = *reinterpret_cast<const u32x4 *>(x + hi_dim);
    }
    int slot = -1;
    if (first_head + HEADS > p.heads) {
        slot = p.slots[m];
        if (slot >= p.slot_count) slot = -1;
    }
    float c[8], s[8];
    if (turned) {
        const int position = p.positions[m];
        const bool known = position >= 0 && position < p.positions_known;
        const int64_t at = (known ? (int64_t)position : 0) * r + 8 * item;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // a position that the tables do not have gives NaN, not another position's angles
            c[i] = known ? p.cos[at + i] : __builtin_nanf("");
            s[i] = known ? p.sin[at + i] : __builtin_nanf("");
        }
    }
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int head = first_head + i;
        if (head >= p.heads + p.kv_heads) break;
        const bool query = head < p.heads;
        const int h = query ? head : head - p.heads;
        float a[8];
        unpack8(lo[i], a);
        if (!turned) {
            put8<(HEADS > 1)>(p, query, h, m, slot, lo_dim, a);
            continue;
        }
        float b[8], x[8], y[8];
        unpack8(hi[i], b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = __builtin_fmaf(a[j], c[j], -(b[j] * s[j]));
            y[j] = __builtin_fmaf(b[j], c[j], a[j] * s[j]);
        }
        if (!query && pairs) {
            // neighbouring lanes have the two halves of the same chunks of codes: one writes the first dims' chunk, the other the partners'
            const Divisor scale(p.k_scale ? p.k_scale[h] : 1.0f);
            const u32x2 first = codes8(x, scale), other = codes8(y, scale), give = odd ? first : other, keep = odd ? other : first;
            const u32x2 got = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)give.x, 0xb1, 0xf, 0xf, false),
                               (uint32_t)__builtin_amdgcn_update_dpp(0, (int)give.y, 0xb1, 0xf, 0xf, false)};      // (lane ^ 1)
            if (slot >= 0)
                put<(HEADS > 1)>(reinterpret_cast<u32x4 *>(p.k + block_offset(p, slot, h) + (((odd ? hi_dim : lo_dim) >> 4) * 16 + (slot & 15)) * 16),
                                 odd ? u32x4{got.x, got.y, keep.x, keep.y} : u32x4{keep.x, keep.y, got.x, got.y});
            continue;
        }
        put8<(HEADS > 1)>(p, query, h, m, slot, lo_dim, x);
        put8<(HEADS > 1)>(p, query, h, m, slot, hi_dim, y);
    }
}

// Values of one head: E tokens of a dim are 16 bytes of the cache, so the tokens of a workgroup are turned in LDS.  A lane then has
// one dim of a run of tokens that end where a chunk of the cache ends; a whole chunk is one store, lines are written whole by
// neighbouring lanes.  (Value by value, each lane waiting for its own, 4101 tokens took 64 us in all.)
constexpr int kMaxTokens = 64;                         // tokens of a workgroup
template <bool MANY>
__device__ __forceinline__ void turn_values(const AppendArgs &p, int h, uint16_t *lds, int *slots) {
    const int64_t first = (int64_t)blockIdx.x * p.group;
    const int count = (int)min((int64_t)p.group, p.M - first), pieces = p.D / 8, ld = p.D + 8;
    uint8_t *bytes = reinterpret_cast<uint8_t *>(lds);
    const Divisor scale(p.fp8 && p.v_scale ? p.v_scale[h] : 1.0f);
    for (int i = threadIdx.x; i < count * pieces; i += kAppendThreads) {
        const int token = i / pieces, piece = i - token * pieces;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(p.new_v + (first + token) * p.ldv + (int64_t)h * p.D + 8 * piece);
        if (p.fp8) {
            float f[8];
            unpack8(v, f);
            *reinterpret_cast<u32x2 *>(bytes + token * ld + 8 * piece) = codes8(f, scale);
        } else {
            *reinterpret_cast<u32x4 *>(lds + token * ld + 8 * piece) = v;
        }
    }
    if ((int)threadIdx.x < count) slots[threadIdx.x] = p.slots[first + threadIdx.x];
    __syncthreads();
    const int chunk = p.fp8 ? 16 : 8, lead = slots[0] & (chunk - 1);         // the first run ends at a chunk's end
    const int runs = (lead + count + chunk - 1) / chunk;
    for (int i = threadIdx.x; i < runs * p.D; i += kAppendThreads) {
        const int run = i / p.D, d = i - run * p.D;
        const int from = max(run * chunk - lead, 0), to = min((run + 1) * chunk - lead, count);
        const int start = slots[from];
        bool whole = to - from == chunk && (start & (chunk - 1)) == 0 && start >= 0 && start < p.slot_count;
        for (int t = from; whole && t < to; ++t) whole = slots[t] == start + t - from;
        if (p.fp8 && whole) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint8_t *at = bytes + (from + 4 * k) * ld + d;
                w[k] = at[0] | (uint32_t)at[ld] << 8 | (uint32_t)at[2 * ld] << 16 | (uint32_t)at[3 * ld] << 24;
            }
            put<MANY>(reinterpret_cast<u32x4 *>(p.v + block_offset(p, start, h) + d * 16), u32x4{w[0], w[1], w[2], w[3]});
        } else if (p.fp8) {
            for (int t = from; t < to; ++t) {
                const int slot = slots[t];
                if (slot >= 0 && slot < p.slot_count) p.v[block_offset(p, slot, h) + d * 16 + (slot & 15)] = bytes[t * ld + d];
            }
        } else if (whole) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = lds[(from + 2 * k) * ld + d] | (uint32_t)lds[(from + 2 * k + 1) * ld + d] << 16;
            put<MANY>(reinterpret_cast<u32x4 *>(p.v + block_offset(p, start, h) + (((start >> 3) & 1) * p.D + d) * 16), u32x4{w[0], w[1], w[2], w[3]});
        } else {
            for (int t = from; t < to; ++t) {
                const int slot = slots[t];
                if (slot < 0 || slot >= p.slot_count) continue;
                reinterpret_cast<uint16_t *>(p.v + block_offset(p, slot, h))[(((slot >> 3) & 1) * p.D + d) * 8 + (slot & 7)] = lds[t * ld + d];
            }
        }
    }
}

// grid: (groups of tokens, heads of the values, then groups of heads of queries and keys)
template <int HEADS>
__global__ void __launch_bounds__(kAppendThreads)
rope_append_kernel(AppendArgs p) {
    __shared__ u32x4 lds[(16 * kAppendThreads + 8 * kMaxTokens) / 8];     // (16 dims to a lane at most, and 8 more for every token)
    __shared__ int slots[kMaxTokens];
    if ((int)blockIdx.y < p.kv_heads) turn_values<(HEADS > 1)>(p, blockIdx.y, reinterpret_cast<uint16_t *>(lds), slots);
    else rotate<HEADS>(p, (blockIdx.y - p.kv_heads) * HEADS);
}

int launch_rope_append(AppendArgs a, hipStream_t stream) {
    const int items = a.rotary / 16 + (a.D - a.rotary) / 8;
    a.group = std::min(kAppendThreads / items, kMaxTokens);
    const int heads = a.heads + a.kv_heads;
    const int64_t groups = (a.M + a.group - 1) / a.group;
    // four heads to a lane from about 400 tokens of 40 heads on: 500 tokens 8.6 -> 7.7 us, 2000 24.3 -> 17.1
    if (groups * heads >= 512) {
        rope_append_kernel<4><<<dim3((unsigned)groups, (unsigned)(a.kv_heads + (heads + 3) / 4)), kAppendThreads, 0, stream>>>(a);
    } else {
        rope_append_kernel<1><<<dim3((unsigned)groups, (unsigned)(a.kv_heads + heads)), kAppendThreads, 0, stream>>>(a);
    }
    return hip_ok(hipGetLastError());
}

}  // namespace nfp
