// The router of a mixture of experts: logits, scores, the chosen experts and their weights.
//
// Which experts are the largest must not depend on the order of a sum, so the logits are worked out in binary64: products of FP16 values are exact
// there, and v_mfma_f64_16x16x4 adds them up.  Small batches are bound by a chain of latencies, larger ones by the matrix pipe's 64-bit
// rate, 1 / 32 of the FP16 one; where there are many logits, they are worked out in binary32 first, and again only those that may be among the
// largest.
#include <algorithm>
#include <type_traits>

#include "nfp_device.h"

namespace nfp {

typedef double doublex4 __attribute__((ext_vector_type(4)));
constexpr int kRouteWaves = 8, kMostSlices = 8, kMostTop = 32;
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

// Tokens of a launch: as many tiles as there are counters, and 32 MiB of logits (of 256 experts 16384 tokens, whose products take 0.4 ms).
static __host__ __device__ int64_t route_tokens(int64_t M, int64_t experts) {
    const int64_t most = min((int64_t)16 * kMaxCounters, (((int64_t)1 << 22) / experts) & ~(int64_t)31);
    return min(M, most);
}

// Orders doubles as unsigned numbers: larger numbers above smaller ones, NaN below all, zero below NaN (for what has been taken or lies outside).
__device__ __forceinline__ uint64_t sortable(double x) {
    if (x != x) return 1;
    const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);          // (-0 is 0)
    return b ^ ((b >> 63) != 0 ? ~0ull : 1ull << 63);
}
__device__ __forceinline__ double unsorted(uint64_t key) {
    return key == 1 ? __longlong_as_double(0x7ff8000000000000ll) : __longlong_as_double((long long)(key ^ ((key >> 63) != 0 ? 1ull << 63 : ~0ull)));
}
// Largest value and sum of the lanes of a group, in all of them.
template <int GROUP>
__device__ __forceinline__ uint32_t max_of_group(uint32_t v) {
    if (GROUP == 64) return max_of_wave(v);
    v = max_of_16_lanes(v);
    return GROUP == 32 ? max(v, (uint32_t)__shfl_xor((int)v, 16)) : v;
}
template <int GROUP>
__device__ __forceinline__ double sum_of_group(double v) {
#pragma unroll
    for (int d = 1; d < GROUP; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// The choice of one token by a group of lanes; lane `sub` of the group holds experts sub, sub + GROUP, ....  Groups of a wave choose side by side (what is longest, the
// search for the largest one top_k times, is the same work for one token as for four); `live`: the group has a token.  Scores of all experts are worked out only
// where they matter: for a bias, or for the sum of a softmax that is not divided out again.
template <int GROUP, int VALUES>
__device__ __forceinline__ void choose(const RouteArgs &a, const double (&logit)[VALUES], int64_t token, int lane, bool live) {
    const int sub = lane & (GROUP - 1);
    uint64_t key[VALUES];
    double score[VALUES];
    double most = 0.0, sum = 1.0;
    uint32_t strange = 0;                              // a NaN among the logits
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        key[v] = sub + GROUP * v < a.experts ? sortable(logit[v]) : 0;
        strange |= key[v] == 1 ? 1u : 0u;
        score[v] = 0.0;
    }
    if (!a.sigmoid) {
        uint64_t best = key[0];
#pragma unroll
        for (int v = 1; v < VALUES; ++v) best = max(best, key[v]);
        const uint32_t high = max_of_group<GROUP>((uint32_t)(best >> 32)), low = max_of_group<GROUP>((uint32_t)(best >> 32) == high ? (uint32_t)best : 0u);
        most = unsorted(((uint64_t)high << 32) | low);
        if (a.bias || !a.renormalize) {
            sum = 0.0;
#pragma unroll
            for (int v = 0; v < VALUES; ++v) {
                score[v] = sub + GROUP * v < a.experts ? exp(logit[v] - most) : 0.0;
                sum += score[v];
            }
            sum = sum_of_group<GROUP>(sum);
        }
        if (max_of_group<GROUP>(strange)) sum = __longlong_as_double(0x7ff8000000000000ll);
    }
    auto of = [&](double l) { return a.sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - most) / sum; };
    if (a.bias) {
#pragma unroll
        for (int v = 0; v < VALUES; ++v) {
            const int e = sub + GROUP * v;
            score[v] = a.sigmoid ? of(logit[v]) : score[v] / sum;
            key[v] = e < a.experts ? sortable(score[v] + (double)a.bias[e]) : 0;
        }
    }
    // the largest, top_k times; the lowest index of equal ones.  Lane j keeps the j-th (and the one GROUP further on)
    constexpr int KEPT = GROUP < 32 ? 2 : 1;           // (top_k is 32 at most)
    double mine[KEPT];
    int id[KEPT];
#pragma unroll
    for (int q = 0; q < KEPT; ++q) { mine[q] = 0.0;  id[q] = 0; }
    for (int j = 0; j < a.top_k; ++j) {
        uint64_t best = key[0];
        int at = sub;
#pragma unroll
        for (int v = 1; v < VALUES; ++v)
            if (key[v] > best) { best = key[v];  at = sub + GROUP * v; }
        const uint32_t high = max_of_group<GROUP>((uint32_t)(best >> 32));
        const bool in = (uint32_t)(best >> 32) == high;
        const uint32_t low = max_of_group<GROUP>(in ? (uint32_t)best : 0u);
        const int first = (int)~max_of_group<GROUP>(in && (uint32_t)best == low ? ~(uint32_t)at : 0u);
        double value;
        if (a.bias) {                                  // the score itself
            double s = score[0];
#pragma unroll
            for (int v = 1; v < VALUES; ++v) s = first == sub + GROUP * v ? score[v] : s;
            value = __shfl(s, (lane & ~(GROUP - 1)) | (first & (GROUP - 1)));
        } else {
            value = unsorted(((uint64_t)high << 32) | low);
        }
#pragma unroll
        for (int v = 0; v < VALUES; ++v)
            if (first == sub + GROUP * v) key[v] = 0;
#pragma unroll
        for (int q = 0; q < KEPT; ++q)
            if (j == sub + GROUP * q) { mine[q] = value;  id[q] = first; }
    }
    double all = 0.0;
#pragma unroll
    for (int q = 0; q < KEPT; ++q) {
        if (!a.bias) mine[q] = of(mine[q]);
        all += sub + GROUP * q < a.top_k ? mine[q] : 0.0;
    }
    if (a.renormalize) all = sum_of_group<GROUP>(all);
#pragma unroll
    for (int q = 0; q < KEPT; ++q) {
        const int j = sub + GROUP * q;
        if (!live || j >= a.top_k) continue;
        a.ids[token * a.top_k + j] = id[q];
        a.weights[token * a.top_k + j] = (float)((a.renormalize ? mine[q] / all : mine[q]) * (double)a.factor);
    }
}

// (What each kernel here reads, 35 MB at 4000 tokens and 256 experts of 4096 columns, takes 7 us; the products 107 us at the matrix pipe's 64-bit rate.)
// Workgroup (x, y, z): 16 T experts, 16 T tokens, one slice of K, which its eight waves share (each holds 8 consecutive columns of a row per lane and step: the sum
// does not care which four columns a MFMA takes, so its step j takes the j-th of each lane's eight).  The logits go to memory past the caches; the
// workgroup that takes the token tile's last ticket adds the slices in order and chooses, a token for every GROUP lanes.
// T: 2 on large batches, where the conversions to 64 bits, half as many per product, take as long as the products (4000 tokens, 256 experts, 4096 columns: 255 us
// with 1).
template <int GROUP, int VALUES, int T>
__global__ void __launch_bounds__(64 * kRouteWaves)
route_kernel(RouteArgs a) {
    __shared__ doublex4 sums[kRouteWaves][64];
    __shared__ uint32_t ticket;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r16 = lane & 15;
    const int tile = blockIdx.y, slice = blockIdx.z;
    const int64_t token0 = (int64_t)a.token0 + tile * (16 * T);
    const int e0 = blockIdx.x * (16 * T);
    const int steps = (int)((a.K + 31) >> 5), per = (steps + a.slices - 1) / a.slices;
    const int begin = slice * per, end = min(begin + per, steps);
    const uint16_t *re[T], *xm[T];
    bool has_e[T], has_m[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        has_e[t] = e0 + 16 * t + r16 < a.experts;
        has_m[t] = token0 + 16 * t + r16 < a.M;
        re[t] = a.R + (int64_t)(has_e[t] ? e0 + 16 * t + r16 : 0) * a.ldr + 8 * g;
        xm[t] = a.X + (has_m[t] ? token0 + 16 * t + r16 : 0) * a.ldx + 8 * g;
    }
    doublex4 acc[T][T];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j) acc[i][j] = doublex4{0.0, 0.0, 0.0, 0.0};
    struct Step { u32x4 w[T], x[T]; };
    auto load = [&](Step &v, int s) {
        const u32x4 zero = {0u, 0u, 0u, 0u};
        const bool in = s < end && 32 * s + 8 * g < a.K;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            v.w[t] = in && has_e[t] ? *reinterpret_cast<const u32x4 *>(re[t] + 32 * s) : zero;
            v.x[t] = in && has_m[t] ? *reinterpret_cast<const u32x4 *>(xm[t] + 32 * s) : zero;
        }
    };
    Step v[2];
    load(v[0], begin + wave);
    load(v[1], begin + wave + kRouteWaves);
    for (int s = begin + wave; s < end; s += 2 * kRouteWaves) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const Step now = v[b];
            load(v[b], s + (2 + b) * kRouteWaves);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t half = 16u * (j & 1);
                double w[T], x[T];
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    w[t] = (double)half_bits_to_float((now.w[t][j >> 1] >> half) & 0xffffu);
                    x[t] = (double)half_bits_to_float((now.x[t][j >> 1] >> half) & 0xffffu);
                }
#pragma unroll
                for (int i = 0; i < T; ++i)
#pragma unroll
                    for (int q = 0; q < T; ++q) acc[i][q] = __builtin_amdgcn_mfma_f64_16x16x4f64(w[i], x[q], acc[i][q], 0, 0, 0);
            }
        }
    }
    constexpr int kThrough = 1 | 16;                   // sc0 | sc1: every XCD has an L2 of its own
    const int tokens = (int)min((int64_t)gridDim.y * (16 * T), a.M - a.token0);         // of this launch
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        a.logits, 0, (uint32_t)((int64_t)a.slices * tokens * a.experts * 8), 0x00020000);
    // the waves' sums, 16 x 16 at a time; rows of a block: expert g + 4 v of lane group g, column: token r16
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int q = 0; q < T; ++q) {
            if (i + q > 0) __syncthreads();
            sums[wave][lane] = acc[i][q];
            __syncthreads();
            if (threadIdx.x < 256) {
                const int row = threadIdx.x >> 6, e = e0 + 16 * i + g + 4 * row, m = tile * (16 * T) + 16 * q + r16;
                double sum = sums[0][lane][row];
#pragma unroll
                for (int w = 1; w < kRouteWaves; ++w) sum += sums[w][lane][row];
                const uint64_t bits = (uint64_t)__double_as_longlong(sum);
                if (e < a.experts && m < tokens)
                    __builtin_amdgcn_raw_buffer_store_b64(u32x2{(uint32_t)bits, (uint32_t)(bits >> 32)}, rs,
                                                          (uint32_t)((((int64_t)slice * tokens + m) * a.experts + e) * 8), 0, kThrough);
            }
        }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this lane's stores have reached memory
    __syncthreads();
    if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add(&a.counters[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (ticket != gridDim.x * gridDim.z - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store(&a.counters[tile], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    constexpr int AT_ONCE = 64 / GROUP;                // tokens of a wave
    const int sub = lane & (GROUP - 1);
    for (int q = wave * AT_ONCE; q < 16 * T && tile * (16 * T) + q < tokens; q += kRouteWaves * AT_ONCE) {
        const int m = tile * (16 * T) + q + lane / GROUP;
        const bool live = m < tokens;
        double logit[VALUES];
#pragma unroll
        for (int i = 0; i < VALUES; ++i) logit[i] = 0.0;
        auto add = [&](auto count, int s0) {           // so many slices under way at a time
            u32x2 bits[decltype(count)::value][VALUES];
#pragma unroll
            for (int s = 0; s < decltype(count)::value; ++s)
#pragma unroll
                for (int i = 0; i < VALUES; ++i)
                    bits[s][i] = __builtin_amdgcn_raw_buffer_load_b64(
                        rs, live && s0 + s < a.slices && sub + GROUP * i < a.experts
                                ? (uint32_t)((((int64_t)(s0 + s) * tokens + m) * a.experts + sub + GROUP * i) * 8) : 0xfffffff0u, 0, kThrough);
#pragma unroll
            for (int s = 0; s < decltype(count)::value; ++s)
#pragma unroll
                for (int i = 0; i < VALUES; ++i)
                    if (s0 + s < a.slices) logit[i] += __longlong_as_double((long long)(((uint64_t)bits[s][i].y << 32) | bits[s][i].x));
        };
        if (T > 1 || a.slices == 1) add(std::integral_constant<int, 1>{}, 0);
        else
            for (int s0 = 0; s0 < a.slices; s0 += 32 / VALUES) add(std::integral_constant<int, 32 / VALUES>{}, s0);
        choose<GROUP, VALUES>(a, logit, (int64_t)a.token0 + m, lane, live);
    }
}

// ---- many logits --------------------------------------------------------------------------------------
// Two launches: all logits with FP16 matrix instructions and what they may be off by; then, token by token, the experts that may be among the top_k largest by that, their logits
// again in binary64, and the choice among these.  Where choices differ by more than the sums' error, as nearly always, that is top_k logits of a token, or one more.
//
// A sum of n terms whose every addition loses at most a step of the largest magnitude met is off by n 2^-23 sum |x r| <= n 2^-23 |x| |r|; taken twice.  A wave adds up an eighth
// of the columns, and the eight sums are added up.  (Measured: at most 0.6 % of this, of large values that cancel, outliers, subnormal numbers and sums of one sign as of normal numbers.)
constexpr int kNear = 64;                              // tokens and experts of a workgroup
__device__ __forceinline__ float near_error(int64_t K) {
    return 2.0f * (float)((K + 64 * kRouteWaves - 1) / (64 * kRouteWaves) * 64 + kRouteWaves) * 0x1p-23f * 1.01f;         // (1 %: the norms' own rounding)
}
static __host__ __device__ __forceinline__ int near_stride(int experts) { return (experts + 3) & ~3; }

__global__ void __launch_bounds__(64 * kRouteWaves)
route_near_kernel(RouteArgs a) {
    constexpr int T = kNear / 16;
    __shared__ floatx4 parts[kRouteWaves][T][64];
    __shared__ float norms[kRouteWaves][2 * kNear];
    __shared__ __attribute__((aligned(16))) uint8_t room[kRouteWaves * 2048];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r16 = lane & 15;
    const int tokens = (int)min(route_tokens(a.M, a.experts), a.M - a.token0), tiles = (a.experts + kNear - 1) / kNear;
    // (workgroups go to the eight XCDs in turn; those of the same tokens to the same one, whose L2 fetches them once)
    const int in_xcd = blockIdx.x >> 3, m0 = ((blockIdx.x & 7) + in_xcd / tiles * 8) * kNear, e0 = in_xcd % tiles * kNear;
    if (m0 >= tokens) return;
    // (rows behind the last one and columns behind the last one read as zero)
    auto from = [&](const uint16_t *first, int64_t ld, int rows) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(first), 0, (uint32_t)(((int64_t)(rows - 1) * ld + a.K) * 2), 0x00020000);
    };
    const __amdgpu_buffer_rsrc_t rsr = from(a.R + (int64_t)e0 * a.ldr, a.ldr, min(kNear, a.experts - e0));
    const __amdgpu_buffer_rsrc_t rsx = from(a.X + (a.token0 + m0) * a.ldx, a.ldx, min(kNear, tokens - m0));
    // (rows are fetched in pieces of 8 x 128 bytes and put into operand order through LDS: fetched in operand order, 16 rows at a time, 34 us for 4000 tokens)
    const uint32_t row_r = (uint32_t)(2 * a.ldr), row_x = (uint32_t)(2 * a.ldx), at = 16 * (lane & 7);
    const Regroup<true> order(room, (uint32_t)(wave * 2048), lane);
    floatx4 acc[T][T];
    float rr[T], xx[T];
#pragma unroll
    for (int i = 0; i < T; ++i) {
        rr[i] = xx[i] = 0.0f;
#pragma unroll
        for (int q = 0; q < T; ++q) acc[i][q] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    struct Step { u32x4 w[T][2], x[T][2]; };           // 64 columns
    auto load = [&](Step &v, int k0) {
        const bool in = 2 * k0 + at < 2 * a.K;
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t row = 16 * t + 8 * h + (lane >> 3);
                v.w[t][h] = __builtin_amdgcn_raw_buffer_load_b128(rsr, in ? row * row_r + 2 * k0 + at : 0xfffffff0u, 0, 0);
                v.x[t][h] = __builtin_amdgcn_raw_buffer_load_b128(rsx, in ? row * row_x + 2 * k0 + at : 0xfffffff0u, 0, 0);
            }
    };
    auto square = [](const u32x4 &v, float s) {
        const half8v h = __builtin_bit_cast(half8v, v);        // (of the whole: __builtin_bit_cast of one element of a vector takes its first)
        s = __builtin_amdgcn_fdot2(half2v{h[0], h[1]}, half2v{h[0], h[1]}, s, false);
        s = __builtin_amdgcn_fdot2(half2v{h[2], h[3]}, half2v{h[2], h[3]}, s, false);
        s = __builtin_amdgcn_fdot2(half2v{h[4], h[5]}, half2v{h[4], h[5]}, s, false);
        return __builtin_amdgcn_fdot2(half2v{h[6], h[7]}, half2v{h[6], h[7]}, s, false);
    };
    auto multiply = [&](Step &v) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
            order.run(v.w[t][0], v.w[t][1]);
            order.run(v.x[t][0], v.x[t][1]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int q = 0; q < T; ++q)
                    acc[i][q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, v.w[i][h]), __builtin_bit_cast(half8v, v.x[q][h]), acc[i][q], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < T; ++i) {
                rr[i] = square(v.w[i][h], rr[i]);
                xx[i] = square(v.x[i][h], xx[i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int STRIDE = 64 * kRouteWaves;
    Step v0, v1;
    const int K = (int)a.K;
    int k0 = 64 * wave;
    load(v0, k0);
    for (; k0 < K; k0 += 2 * STRIDE) {
        load(v1, k0 + STRIDE);
        __builtin_amdgcn_sched_barrier(0);
        multiply(v0);
        load(v0, k0 + 2 * STRIDE);
        __builtin_amdgcn_sched_barrier(0);
        multiply(v1);
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
        rr[t] += __shfl_xor(rr[t], 16);
        rr[t] += __shfl_xor(rr[t], 32);
        xx[t] += __shfl_xor(xx[t], 16);
        xx[t] += __shfl_xor(xx[t], 32);
        if (g == 0) {
            norms[wave][16 * t + r16] = rr[t];
            norms[wave][kNear + 16 * t + r16] = xx[t];
        }
    }
    float *const logits = reinterpret_cast<float *>(a.logits), *const errors = logits + (int64_t)tokens * near_stride(a.experts);
    // the waves' sums, 16 experts at a time; rows of a block: expert 4 g + v of lane group g, column: token r16
#pragma unroll
    for (int i = 0; i < T; ++i) {
        if (i > 0) __syncthreads();
#pragma unroll
        for (int q = 0; q < T; ++q) parts[wave][q][lane] = acc[i][q];
        __syncthreads();
        if (threadIdx.x < 64 * T) {
            const int q = threadIdx.x >> 6, e = e0 + 16 * i + 4 * g, m = m0 + 16 * q + r16;
            floatx4 sum = parts[0][q][lane];
#pragma unroll
            for (int w = 1; w < kRouteWaves; ++w) sum += parts[w][q][lane];
            if (m < tokens && e < a.experts) *reinterpret_cast<floatx4 *>(logits + (int64_t)m * near_stride(a.experts) + e) = sum;
        }
    }
    if (wave == 0) {
        float r = 0.0f, x = 0.0f;
        for (int w = 0; w < kRouteWaves; ++w) {
            r += norms[w][lane];
            x += norms[w][kNear + lane];
        }
        r = __uint_as_float(max_of_wave(__float_as_uint(r) & 0x7fffffffu));        // (of a NaN among them: a NaN)
        if (m0 + lane < tokens) errors[(int64_t)(m0 + lane) * tiles + e0 / kNear] = near_error(a.K) * sqrtf(r) * sqrtf(x);
    }
}

// A wave for each token: bounds and border 9 of 31 us (4000 tokens, top_k 8 of 256, 4096 columns), the rest rows of experts from the L2 (0.3 GB) and their products, as many with sums
// in binary32 (28 us).
constexpr int kChoosers = 4;
template <int VALUES>
__global__ void __launch_bounds__(64 * kChoosers)
route_near_choose_kernel(RouteArgs a) {
    __shared__ uint16_t named[kChoosers][64 * VALUES];
    __shared__ double exact[kChoosers][64 * VALUES];
    __shared__ uint64_t keys[kChoosers][64 * VALUES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tiles = (a.experts + kNear - 1) / kNear;
    const int tokens = (int)min(route_tokens(a.M, a.experts), a.M - a.token0);
    const int m = blockIdx.x * kChoosers + wave;
    if (m >= tokens) return;
    auto ordered = [] { asm volatile("" ::: "memory"); };              // (a wave's LDS accesses stay in order)
    const float *const logits = reinterpret_cast<const float *>(a.logits), *const errors = logits + (int64_t)tokens * near_stride(a.experts);
    const float error = __uint_as_float(max_of_wave(lane < tiles ? __float_as_uint(errors[(int64_t)m * tiles + lane]) & 0x7fffffffu : 0u));
    const bool sure = error < __builtin_inff();
    // Every expert's choice lies between `least` and `upper`; whose upper bound lies below the top_k-th largest lower bound is not among the top_k.
    uint32_t least[VALUES];
    float upper[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        const int e = lane + 64 * v;
        least[v] = 0;
        upper[v] = 0.0f;
        if (e >= a.experts) continue;
        float c = logits[(int64_t)m * near_stride(a.experts) + e], off = error;
        if (a.bias) {                                  // (sigmoid: a slope of 1/4 at most; eight roundings)
            c = 1.0f / (1.0f + __expf(-c)) + a.bias[e];
            off = __builtin_isinf(c) ? 0.0f : 0.25f * error + 0x1p-20f + 0x1p-22f * fabsf(c);
        }
        const float low = sure && c == c ? c - off : -__builtin_inff();
        upper[v] = !sure ? __builtin_inff() : (c == c ? c + off : -__builtin_inff());
        const uint32_t b = __float_as_uint(low);
        least[v] = b ^ ((b >> 31) != 0 ? ~0u : 1u << 31);
    }
    uint32_t left = (uint32_t)a.top_k, border = 0, rest[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) rest[v] = least[v];
    while (left > 0) {                                 // (top_k is no more than the experts: there is one left)
        uint32_t best = rest[0];
#pragma unroll
        for (int v = 1; v < VALUES; ++v) best = max(best, rest[v]);
        border = max_of_wave(best);
        bool gone = false;
#pragma unroll
        for (int v = 0; v < VALUES; ++v) {
            const bool it = !gone && rest[v] == border;
            gone |= it;
            rest[v] = it ? 0u : rest[v];
        }
        left -= min(left, (uint32_t)__popcll(__ballot(gone)));
    }
    const float floor_value = __uint_as_float(border ^ ((border >> 31) != 0 ? 1u << 31 : ~0u));
    int count = 0;
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        const bool in = lane + 64 * v < a.experts && !(upper[v] < floor_value);
        const uint64_t mask = __ballot(in);
        if (in) named[wave][count + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = (uint16_t)(lane + 64 * v);
        count += __popcll(mask);
    }
    const uint16_t *const x = a.X + (a.token0 + m) * a.ldx;
    // A row of zeros (padding) among finite experts: all logits are zero.  Without a bias they all tie and would all be summed again, 540 us in place of 53 for 4000 such tokens
    // (256 experts, 4096 columns); the first top_k are the choice (34 us).  (A bound of zero alone is not enough: squares of the smallest numbers may be lost on the way to it.)
    bool zeros = error == 0.0f && !a.bias;
    if (zeros) {
        u32x4 any = {0u, 0u, 0u, 0u};
        for (int64_t k = 8 * lane; k < a.K; k += 512) any |= *reinterpret_cast<const u32x4 *>(x + k);
        zeros = __ballot(((any.x | any.y | any.z | any.w) & 0x7fff7fffu) != 0) == 0;
        if (zeros) {
            if (lane < a.top_k) {
                named[wave][lane] = (uint16_t)lane;
                exact[wave][lane] = 0.0;
            }
            count = a.top_k;
        }
    }
    ordered();
    // their logits: products of FP16 values, exact in binary32, added up in binary64
    auto dots = [&](auto width, int at) {
        constexpr int W = decltype(width)::value;
        const uint16_t *row[W];
        double sum[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            row[i] = a.R + (int64_t)__builtin_amdgcn_readfirstlane(named[wave][min(at + i, count - 1)]) * a.ldr;
            sum[i] = 0.0;
        }
        struct Columns { u32x4 x, w[W]; };
        auto load = [&](Columns &c, int64_t at) {      // (behind the last column the last ones again)
            c.x = *reinterpret_cast<const u32x4 *>(x + min(at, a.K - 8));
#pragma unroll
            for (int i = 0; i < W; ++i) c.w[i] = *reinterpret_cast<const u32x4 *>(row[i] + min(at, a.K - 8));
        };
        auto half = [](const u32x4 &v, int j) { return (float)__builtin_bit_cast(half8v, v)[j]; };
        Columns next;
        load(next, 8 * lane);
        for (int64_t k = 8 * lane; k < a.K; k += 512) {
            const Columns c = next;
            load(next, k + 512);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < W; ++i) sum[i] += (double)__builtin_fmaf(half(c.x, j), half(c.w[i], j), 0.0f);
            __builtin_amdgcn_sched_barrier(0);
        }
        // (lanes that differ in the lowest bits take over one sum each)
#pragma unroll
        for (int d = 1; d < W; d <<= 1)
#pragma unroll
            for (int i = 0; i < W / (2 * d); ++i) {
                const bool odd = (lane & d) != 0;
                sum[i] = (odd ? sum[2 * i + 1] : sum[2 * i]) + __shfl_xor(odd ? sum[2 * i] : sum[2 * i + 1], d);
            }
#pragma unroll
        for (int d = W; d < 64; d <<= 1) sum[0] += __shfl_xor(sum[0], d);
        if (lane < W && at + lane < count) exact[wave][at + lane] = sum[0];
    };
    // (eight rows at a time: level; the rows come from the L2, 8 KB each at 4096 columns, and that is what these take)
    int at = zeros ? count : 0;
    for (; at + 4 <= count; at += 4) dots(std::integral_constant<int, 4>{}, at);
    for (; at < count; at += 2) dots(std::integral_constant<int, 2>{}, at);
    ordered();
    auto sigmoid = [](double l) { return 1.0 / (1.0 + exp(-l)); };
    double most = 0.0;
    uint32_t strange = 0;
    uint64_t high = 0;
    for (int i = lane; i < count; i += 64) {
        const double l = exact[wave][i];
        strange |= l != l ? 1u : 0u;
        const uint64_t key = a.bias ? sortable(sigmoid(l) + (double)a.bias[named[wave][i]]) : sortable(l);
        keys[wave][i] = key;
        high = max(high, key);
    }
    ordered();
    if (!a.sigmoid) {
        const uint32_t up = max_of_wave((uint32_t)(high >> 32)), low = max_of_wave((uint32_t)(high >> 32) == up ? (uint32_t)high : 0u);
        most = max_of_wave(strange) ? __longlong_as_double(0x7ff8000000000000ll) : unsorted(((uint64_t)up << 32) | low);
    }
    // the place of each: how many are larger, or as large and before it
    double score[VALUES], all = 0.0;
    int place[VALUES];
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        const int i = lane + 64 * v;
        place[v] = kMostTop;
        score[v] = 0.0;
        if (64 * v >= count) continue;
        if (i < count) {
            const uint64_t key = keys[wave][i];
            int before = 0;
            for (int q = 0; q < count; ++q) {
                const uint64_t other = keys[wave][q];
                before += other > key || (other == key && q < i) ? 1 : 0;
            }
            if (before < a.top_k) {
                place[v] = before;
                score[v] = a.sigmoid ? sigmoid(exact[wave][i]) : exp(exact[wave][i] - most);
                all += score[v];
            }
        }
    }
    if (a.renormalize) all = sum_of_group<64>(all);
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        if (place[v] >= a.top_k) continue;
        const int64_t to = (a.token0 + m) * a.top_k + place[v];
        a.ids[to] = named[wave][lane + 64 * v];
        a.weights[to] = (float)((a.renormalize ? score[v] / all : score[v]) * (double)a.factor);
    }
}

static bool route_pairs(int64_t M, int64_t experts) { return ((M + 31) / 32) * ((experts + 31) / 32) >= 512; }       // two workgroups per CU
// Slices of K: enough workgroups for the chip, at least a step of every wave's each.
static int route_slices(int64_t M, int64_t experts, int64_t K) {
    const int64_t tiles = ((experts + 15) / 16) * ((M + 15) / 16), steps = (K + 31) / 32;
    return (int)std::max<int64_t>(1, std::min<int64_t>({kMostSlices, 256 / tiles, steps / kRouteWaves}));
}
// Room for M tokens and for any fewer, whose logits can take more of it in more slices (256 experts of 2048 columns: 32 tokens 8 slices and 512 KiB, 33 tokens 5 and 330 KiB): a
// program shares the workspace of its largest batch.
size_t route_logit_bytes(int64_t M, int64_t experts, int64_t K) {
    const int64_t tokens = route_tokens(M, experts), across = (experts + 15) / 16;
    int64_t rows = tokens;                             // slices * tokens, at most
    for (int64_t s = 2; s <= std::min<int64_t>(kMostSlices, (K + 31) / 32 / kRouteWaves); ++s)
        rows = std::max(rows, s * std::min(tokens, 256 / (s * across) * 16));          // (the most tokens that take s slices)
    return (size_t)rows * (size_t)experts * 8;
}

template <int T, int GROUP>
static void launch_route_t(const RouteArgs &a, int64_t tokens, hipStream_t stream) {
    const dim3 grid((unsigned)((a.experts + 16 * T - 1) / (16 * T)), (unsigned)((tokens + 16 * T - 1) / (16 * T)), (unsigned)a.slices);
    if (a.experts <= 64) route_kernel<GROUP, 64 / GROUP, T><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
    else if (a.experts <= 128) route_kernel<GROUP, 128 / GROUP, T><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
    else if (a.experts <= 256) route_kernel<GROUP, 256 / GROUP, T><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
    else route_kernel<GROUP < 32 ? 32 : GROUP, GROUP < 64 ? 16 : 8, T><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
}

// Where a choice depends on one logit each, and there are many: us in binary64 and this way, columns 2048 / 7168:
// 65536 logits (256 tokens, 256 experts) 17.3 and 19.5 / 33.9 and 41.8, 131072 (512, 256) 24.7 and 19.4 / 55.5 and 44.0, (2048, 64) 21.7 and 19.7 / 52.8 and 45.2,
// 2^20 (4096, 256) 100 and 27 / 283 and 66.  (Scores of a softmax that is not divided out again, or with a bias, need all logits in binary64.)
static bool route_near(const RouteArgs &a, int64_t tokens) {
    return (a.sigmoid || (a.renormalize && !a.bias)) && a.experts >= 16 && tokens * a.experts >= ((int64_t)1 << 17);
}
static void launch_near(const RouteArgs &a, int64_t tokens, hipStream_t stream) {
    route_near_kernel<<<(unsigned)((a.experts + kNear - 1) / kNear * ((tokens + 8 * kNear - 1) / (8 * kNear)) * 8), 64 * kRouteWaves, 0, stream>>>(a);
    const unsigned groups = (unsigned)((tokens + kChoosers - 1) / kChoosers);
    if (a.experts <= 64) route_near_choose_kernel<1><<<groups, 64 * kChoosers, 0, stream>>>(a);
    else if (a.experts <= 128) route_near_choose_kernel<2><<<groups, 64 * kChoosers, 0, stream>>>(a);
    else if (a.experts <= 256) route_near_choose_kernel<4><<<groups, 64 * kChoosers, 0, stream>>>(a);
    else route_near_choose_kernel<8><<<groups, 64 * kChoosers, 0, stream>>>(a);
}

int launch_route(RouteArgs a, hipStream_t stream) {
    const int64_t tokens = route_tokens(a.M, a.experts);
    a.slices = route_slices(tokens, a.experts, a.K);
    for (int64_t m = 0; m < a.M; m += tokens) {
        a.token0 = m;
        const int64_t some = std::min(tokens, a.M - m);
        // (a token per wave, two or four: as many waves as a tile has)
        if (route_near(a, some)) launch_near(a, some, stream);
        else if (a.slices == 1 && route_pairs(some, a.experts)) launch_route_t<2, 16>(a, some, stream);
        else if (some <= kRouteWaves) launch_route_t<1, 64>(a, some, stream);
        else launch_route_t<1, 32>(a, some, stream);
        if (hipGetLastError() != hipSuccess) return kErrHip;
    }
    return kOk;
}

}  // namespace nfp
