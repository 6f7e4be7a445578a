// Rotary positions on the queries and keys of new tokens, and the write of keys and values into the paged cache.
// Cache storage (include/nestedfp.h): blocks of 16 tokens; with E elements in 16 bytes a key block is
// [D / E][16 tokens][E dims], a value block [16 / E][D][E tokens], which is the order in which lanes of the
// attention kernels hold matrix operands.
#include "nfp_device.h"
#include "nfp_host.h"

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
// Codes are rounded once, from the 32-bit value, and saturate at +-448 (a NaN stays one): the quotient by the caller's
// scale is a division, whatever that scale is.
__device__ __forceinline__ float quotient(float x, float s) {
    const float q = x / s;
    return q != q ? q : clamp448(q);
}
__device__ __forceinline__ u32x2 codes8(const float (&f)[8], float s) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = quotient(f[i], s);
    return u32x2{e4m3x4_from_float_hw(q[0], q[1], q[2], q[3]), e4m3x4_from_float_hw(q[4], q[5], q[6], q[7])};
}

// 8 dims from `dim` (a multiple of 8) of one token's query or key
__device__ __forceinline__ void put8(const AppendArgs &p, bool query, int head, int64_t m, int slot, int dim, const float (&f)[8]) {
    if (query) {
        *reinterpret_cast<u32x4 *>(p.out + m * p.ldo + (int64_t)head * p.D + dim) = pack8(f);
        return;
    }
    if (slot < 0) return;
    uint8_t *block = p.k + block_offset(p, slot, head);
    const int token = slot & 15;
    if (p.fp8)
        *reinterpret_cast<u32x2 *>(block + ((dim >> 4) * 16 + token) * 16 + (dim & 8)) = codes8(f, p.k_scale ? p.k_scale[head] : 1.0f);
    else
        *reinterpret_cast<u32x4 *>(block + ((dim >> 3) * 16 + token) * 16) = pack8(f);
}

// grid: (groups of tokens, heads of q, then of k, then of v).  Queries and keys: a lane has 8 dims and their 8 partners
// (or 8 dims that are not rotated) of one token.  Values: a lane has one dim, of one token after the other.
__global__ void __launch_bounds__(kAppendThreads)
rope_append_kernel(AppendArgs p) {
    const int head = blockIdx.y;
    if (head < p.heads + p.kv_heads) {
        const bool query = head < p.heads;
        const int h = query ? head : head - p.heads;
        const int r = p.rotary / 2, turns = r / 8, items = turns + (p.D - p.rotary) / 8;
        const int token = threadIdx.x / items, item = threadIdx.x - token * items;
        const int64_t m = (int64_t)blockIdx.x * p.group + token;
        if (token >= p.group || m >= p.M) return;
        int slot = -1;
        if (!query) {
            slot = p.slots[m];
            if (slot >= p.slot_count) slot = -1;
        }
        const uint16_t *x = (query ? p.q + m * p.ldq : p.new_k + m * p.ldk) + (int64_t)h * p.D;
        float a[8];
        if (item >= turns) {
            const int dim = p.rotary + 8 * (item - turns);
            unpack8(*reinterpret_cast<const u32x4 *>(x + dim), a);
            put8(p, query, h, m, slot, dim, a);
            return;
        }
        float b[8], c[8], s[8], lo[8], hi[8];
        unpack8(*reinterpret_cast<const u32x4 *>(x + 8 * item), a);
        unpack8(*reinterpret_cast<const u32x4 *>(x + r + 8 * item), b);
        const int position = p.positions[m];
        const bool known = position >= 0 && position < p.positions_known;
        const int64_t at = (known ? (int64_t)position : 0) * r + 8 * item;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // a position that the tables do not have gives NaN, not another position's angles
            c[i] = known ? p.cos[at + i] : __builtin_nanf("");
            s[i] = known ? p.sin[at + i] : __builtin_nanf("");
            lo[i] = __builtin_fmaf(a[i], c[i], -(b[i] * s[i]));
            hi[i] = __builtin_fmaf(b[i], c[i], a[i] * s[i]);
        }
        put8(p, query, h, m, slot, 8 * item, lo);
        put8(p, query, h, m, slot, r + 8 * item, hi);
        return;
    }
    const int h = head - p.heads - p.kv_heads;
    const float scale = p.fp8 && p.v_scale ? p.v_scale[h] : 1.0f;
    const int64_t first = (int64_t)blockIdx.x * p.group;
    const int count = (int)min((int64_t)p.group, p.M - first);
    for (int i = threadIdx.x; i < count * p.D; i += kAppendThreads) {
        const int token = i / p.D, d = i - token * p.D;
        const int slot = p.slots[first + token];
        if (slot < 0 || slot >= p.slot_count) continue;
        const uint16_t v = p.new_v[(first + token) * p.ldv + (int64_t)h * p.D + d];
        uint8_t *block = p.v + block_offset(p, slot, h);
        const int t = slot & 15;
        if (p.fp8) {
            const float q = quotient(half_bits_to_float(v), scale);
            block[d * 16 + t] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(q, q, 0, false);
        } else {
            reinterpret_cast<uint16_t *>(block)[((t >> 3) * p.D + d) * 8 + (t & 7)] = v;
        }
    }
}

int launch_rope_append(AppendArgs a, hipStream_t stream) {
    const int items = a.rotary / 16 + (a.D - a.rotary) / 8;
    a.group = kAppendThreads / items;
    const dim3 grid((unsigned)((a.M + a.group - 1) / a.group), (unsigned)(a.heads + 2 * a.kv_heads));
    rope_append_kernel<<<grid, kAppendThreads, 0, stream>>>(a);
    return hip_ok(hipGetLastError());
}

}  // namespace nfp
