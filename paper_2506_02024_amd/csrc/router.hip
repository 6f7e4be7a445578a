// The router of a mixture of experts: logits, scores, the chosen experts and their weights.
//
// Which experts are the largest must not depend on the order of a sum, so the logits are worked out in binary64: products of FP16 values are exact
// there, and v_mfma_f64_16x16x4 adds them up.  That is also what bounds the kernel on large batches (the matrix pipe's 64-bit rate, 1 / 32 of
// the FP16 one); small ones are bound by a chain of latencies.
#include <algorithm>
#include <type_traits>

#include "nfp_device.h"

namespace nfp {

typedef double doublex4 __attribute__((ext_vector_type(4)));
constexpr int kRouteWaves = 8, kMostSlices = 8;

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

// Tokens of a launch: as many tiles as there are counters, and 32 MiB of logits (of 256 experts 16384 tokens, whose products take 0.4 ms).
static int64_t route_tokens(int64_t M, int64_t experts) {
    const int64_t most = std::min<int64_t>(16 * kMaxCounters, (((int64_t)1 << 22) / experts) & ~(int64_t)31);
    return std::min(M, most);
}
static bool route_pairs(int64_t M, int64_t experts) { return ((M + 31) / 32) * ((experts + 31) / 32) >= 512; }       // two workgroups per CU
// Slices of K: enough workgroups for the chip, at least a step of every wave's each.
static int route_slices(int64_t M, int64_t experts, int64_t K) {
    const int64_t tiles = ((experts + 15) / 16) * ((M + 15) / 16), steps = (K + 31) / 32;
    return (int)std::max<int64_t>(1, std::min<int64_t>({kMostSlices, 256 / tiles, steps / kRouteWaves}));
}
size_t route_logit_bytes(int64_t M, int64_t experts, int64_t K) {
    const int64_t tokens = route_tokens(M, experts);
    return (size_t)route_slices(tokens, experts, K) * (size_t)tokens * (size_t)experts * 8;
}

template <int T, int GROUP>
static void launch_route_t(const RouteArgs &a, int64_t tokens, hipStream_t stream) {
    const dim3 grid((unsigned)((a.experts + 16 * T - 1) / (16 * T)), (unsigned)((tokens + 16 * T - 1) / (16 * T)), (unsigned)a.slices);
    if (a.experts <= 64) route_kernel<GROUP, 64 / GROUP, T><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
    else if (a.experts <= 128) route_kernel<GROUP, 128 / GROUP, T><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
    else if (a.experts <= 256) route_kernel<GROUP, 256 / GROUP, T><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
    else route_kernel<GROUP < 32 ? 32 : GROUP, GROUP < 64 ? 16 : 8, T><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
}

int launch_route(RouteArgs a, hipStream_t stream) {
    const int64_t tokens = route_tokens(a.M, a.experts);
    a.slices = route_slices(tokens, a.experts, a.K);
    for (int64_t m = 0; m < a.M; m += tokens) {
        a.token0 = m;
        const int64_t some = std::min(tokens, a.M - m);
        // (a token per wave, two or four: as many waves as a tile has)
        if (a.slices == 1 && route_pairs(some, a.experts)) launch_route_t<2, 16>(a, some, stream);
        else if (some <= kRouteWaves) launch_route_t<1, 64>(a, some, stream);
        else launch_route_t<1, 32>(a, some, stream);
        if (hipGetLastError() != hipSuccess) return kErrHip;
    }
    return kOk;
}

}  // namespace nfp
