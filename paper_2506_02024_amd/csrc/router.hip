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
constexpr int kRouteWaves = 8;

// Orders doubles as unsigned numbers: larger numbers above smaller ones, NaN below all, zero below NaN (for what has been taken or lies outside).
__device__ __forceinline__ uint64_t sortable(double x) {
    if (x != x) return 1;
    const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);          // (-0 is 0)
    return b ^ ((b >> 63) != 0 ? ~0ull : 1ull << 63);
}
__device__ __forceinline__ double sum_of_wave(double v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// One token's choice by one wave; lane l holds experts l, l + 64, ....  VALUES: of 64 experts each.
template <int VALUES>
__device__ __forceinline__ void choose(const RouteArgs &a, const double (&logit)[VALUES], int64_t token, int lane) {
    double score[VALUES];
    uint64_t key[VALUES];
    if (a.sigmoid) {
#pragma unroll
        for (int v = 0; v < VALUES; ++v) score[v] = 1.0 / (1.0 + exp(-logit[v]));
    } else {
        uint64_t best = 0;
#pragma unroll
        for (int v = 0; v < VALUES; ++v) best = max(best, lane + 64 * v < a.experts ? sortable(logit[v]) : 0);
        const uint32_t high = max_of_wave((uint32_t)(best >> 32)), low = max_of_wave((uint32_t)(best >> 32) == high ? (uint32_t)best : 0u);
        const uint64_t b = ((uint64_t)high << 32) | low;
        const double most = __longlong_as_double((long long)(b ^ ((b >> 63) != 0 ? 1ull << 63 : ~0ull)));       // (of NaN alone: some NaN)
        double sum = 0.0;
#pragma unroll
        for (int v = 0; v < VALUES; ++v) {
            score[v] = lane + 64 * v < a.experts ? exp(logit[v] - most) : 0.0;
            sum += score[v];
        }
        sum = sum_of_wave(sum);
#pragma unroll
        for (int v = 0; v < VALUES; ++v) score[v] /= sum;
    }
#pragma unroll
    for (int v = 0; v < VALUES; ++v) {
        const int e = lane + 64 * v;
        key[v] = e < a.experts ? sortable(a.bias ? score[v] + (double)a.bias[e] : logit[v]) : 0;
    }
    // the largest, top_k times; the lowest index of equal ones
    double mine = 0.0;                                 // lane j: the score of the j-th choice
    int id = 0;
    for (int j = 0; j < a.top_k; ++j) {
        uint64_t best = key[0];
        int at = lane;
#pragma unroll
        for (int v = 1; v < VALUES; ++v)
            if (key[v] > best) { best = key[v];  at = lane + 64 * v; }
        const uint32_t high = max_of_wave((uint32_t)(best >> 32));
        const bool in = (uint32_t)(best >> 32) == high;
        const uint32_t low = max_of_wave(in ? (uint32_t)best : 0u);
        const uint32_t first = ~max_of_wave(in && (uint32_t)best == low ? ~(uint32_t)at : 0u);
        const int owner = (int)(first & 63u), which = (int)(first >> 6);
        double s = score[0];
#pragma unroll
        for (int v = 1; v < VALUES; ++v) s = which == v ? score[v] : s;
        s = __shfl(s, owner);
#pragma unroll
        for (int v = 0; v < VALUES; ++v)
            if (lane == owner && which == v) key[v] = 0;
        if (lane == j) { mine = s;  id = (int)first; }
    }
    if (a.renormalize) {
        const double sum = sum_of_wave(lane < a.top_k ? mine : 0.0);
        mine /= sum;
    }
    if (lane < a.top_k) {
        a.ids[token * a.top_k + lane] = id;
        a.weights[token * a.top_k + lane] = (float)(mine * (double)a.factor);
    }
}

// Workgroup (x, y, z): 16 experts, 16 tokens, one slice of K, which its eight waves share (each holds 8 consecutive columns of a row per lane and step: the sum
// does not care which four columns a MFMA takes, so its step j takes the j-th of each lane's eight).  The logits go to memory past the caches; the
// workgroup that takes the token tile's last ticket adds the slices in order and chooses, two tokens per wave.
template <int VALUES>
__global__ void __launch_bounds__(64 * kRouteWaves)
route_kernel(RouteArgs a) {
    __shared__ doublex4 sums[kRouteWaves][64];
    __shared__ uint32_t ticket;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r16 = lane & 15;
    const int tile = blockIdx.y, slice = blockIdx.z;
    const int64_t token0 = (int64_t)(a.tile0 + tile) * 16;
    const int e0 = blockIdx.x * 16;
    const int steps = (int)((a.K + 31) >> 5), per = (steps + a.slices - 1) / a.slices;
    const int begin = slice * per, end = min(begin + per, steps);
    const bool has_e = e0 + r16 < a.experts, has_m = token0 + r16 < a.M;
    const uint16_t *const re = a.R + (int64_t)(e0 + r16) * a.ldr + 8 * g, *const xm = a.X + (token0 + r16) * a.ldx + 8 * g;
    doublex4 acc = {0.0, 0.0, 0.0, 0.0};
    auto load = [&](u32x4 &w, u32x4 &x, int s) {
        const u32x4 zero = {0u, 0u, 0u, 0u};
        const bool in = s < end && 32 * s + 8 * g < a.K;
        w = in && has_e ? *reinterpret_cast<const u32x4 *>(re + 32 * s) : zero;
        x = in && has_m ? *reinterpret_cast<const u32x4 *>(xm + 32 * s) : zero;
    };
    u32x4 w[2], x[2];
    load(w[0], x[0], begin + wave);
    load(w[1], x[1], begin + wave + kRouteWaves);
    for (int s = begin + wave; s < end; s += 2 * kRouteWaves) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const u32x4 wn = w[b], xn = x[b];
            load(w[b], x[b], s + (2 + b) * kRouteWaves);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t half = 16u * (j & 1);
                acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)half_bits_to_float((wn[j >> 1] >> half) & 0xffffu),
                                                           (double)half_bits_to_float((xn[j >> 1] >> half) & 0xffffu), acc, 0, 0, 0);
            }
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    // rows of the result: expert g + 4 v of lane group g, column: token r16
    constexpr int kThrough = 1 | 16;                   // sc0 | sc1: every XCD has an L2 of its own
    const int tokens = (int)min((int64_t)gridDim.y * 16, a.M - (int64_t)a.tile0 * 16);          // of this launch
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        a.logits, 0, (uint32_t)((int64_t)a.slices * tokens * a.experts * 8), 0x00020000);
    if (threadIdx.x < 256) {
        const int v = threadIdx.x >> 6, e = e0 + g + 4 * v, m = tile * 16 + r16;
        double sum = sums[0][lane][v];
#pragma unroll
        for (int q = 1; q < kRouteWaves; ++q) sum += sums[q][lane][v];
        const uint64_t bits = (uint64_t)__double_as_longlong(sum);
        if (e < a.experts && m < tokens)
            __builtin_amdgcn_raw_buffer_store_b64(u32x2{(uint32_t)bits, (uint32_t)(bits >> 32)}, rs,
                                                  (uint32_t)((((int64_t)slice * tokens + m) * a.experts + e) * 8), 0, kThrough);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this lane's stores have reached memory
    __syncthreads();
    if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add(&a.counters[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (ticket != gridDim.x * gridDim.z - 1) return;
    for (int q = wave; q < 16 && tile * 16 + q < tokens; q += kRouteWaves) {
        const int m = tile * 16 + q;
        double logit[VALUES];
#pragma unroll
        for (int v = 0; v < VALUES; ++v) logit[v] = 0.0;
        for (int s = 0; s < a.slices; ++s) {
            u32x2 bits[VALUES];
#pragma unroll
            for (int v = 0; v < VALUES; ++v)
                bits[v] = __builtin_amdgcn_raw_buffer_load_b64(
                    rs, lane + 64 * v < a.experts ? (uint32_t)((((int64_t)s * tokens + m) * a.experts + lane + 64 * v) * 8) : 0xfffffff0u, 0, kThrough);
#pragma unroll
            for (int v = 0; v < VALUES; ++v) logit[v] += __longlong_as_double((long long)(((uint64_t)bits[v].y << 32) | bits[v].x));
        }
        choose<VALUES>(a, logit, (int64_t)a.tile0 * 16 + m, lane);
    }
    if (threadIdx.x == 0) __hip_atomic_store(&a.counters[tile], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Tokens of a launch: as many tiles as there are counters, and 32 MiB of logits (of 256 experts 16384 tokens, whose products take 0.4 ms).
static int64_t route_tokens(int64_t M, int64_t experts) {
    const int64_t most = std::min<int64_t>(16 * kMaxCounters, (((int64_t)1 << 22) / experts) & ~(int64_t)15);
    return std::min(M, most);
}
// Slices of K: enough workgroups for the chip, at least a step of every wave's each.
static int route_slices(int64_t M, int64_t experts, int64_t K) {
    const int64_t tiles = ((experts + 15) / 16) * ((M + 15) / 16), steps = (K + 31) / 32;
    return (int)std::max<int64_t>(1, std::min<int64_t>({16, 256 / tiles, steps / kRouteWaves}));
}
size_t route_logit_bytes(int64_t M, int64_t experts, int64_t K) {
    const int64_t tokens = route_tokens(M, experts);
    return (size_t)route_slices(tokens, experts, K) * (size_t)tokens * (size_t)experts * 8;
}

int launch_route(RouteArgs a, hipStream_t stream) {
    const int64_t tokens = route_tokens(a.M, a.experts);
    a.slices = route_slices(tokens, a.experts, a.K);
    for (int64_t m = 0; m < a.M; m += tokens) {
        a.tile0 = (int32_t)(m / 16);
        const dim3 grid((unsigned)((a.experts + 15) / 16), (unsigned)((std::min(tokens, a.M - m) + 15) / 16), (unsigned)a.slices);
        if (a.experts <= 64) route_kernel<1><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
        else if (a.experts <= 128) route_kernel<2><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
        else if (a.experts <= 256) route_kernel<4><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
        else route_kernel<8><<<grid, 64 * kRouteWaves, 0, stream>>>(a);
        if (hipGetLastError() != hipSuccess) return kErrHip;
    }
    return kOk;
}

}  // namespace nfp
