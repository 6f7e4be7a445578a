// The residual's addition and the root-mean-square norm in front of a layer's linears, with the E4M3 codes that FP8 mode
// takes:  h = fp16(x + r),  y = h / sqrt(mean(h^2) + eps) * w,  scale = max|y| / 448,  code = E4M3(y / scale).
// HBM-bound: 2 + 2 bytes read and 2 + 2 (FP16) or 2 + 1 (codes) written per element.  A row stays in the registers of one
// workgroup from its only read to its last write; the two statistics (sum of squares, largest magnitude) each cost
// one exchange between its waves.  As many lanes as the row has chunks of 8 values, so that a few rows take one load's latency.
// Measured: 8192 rows of 4096 to codes 42.6 us (5.5 TB/s; a large copy reaches 4.9), 48 of 5120 to both 4.2 us, one of 1040 2.0 us
// (of which an empty kernel takes 1.5).  The counters of the large case read 134 and write 101 MB: nothing twice.
#include "nfp_device.h"
#include "nfp_host.h"

namespace nfp {

// Sum over the 64 lanes in all of them, in a fixed order.
template <int CTRL>
__device__ __forceinline__ float plus_lane(float v) {
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}
__device__ __forceinline__ float sum_of_wave(float v) {
    v = plus_lane<0x140>(plus_lane<0x141>(plus_lane<0x4e>(plus_lane<0xb1>(v))));
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

struct Eight { float f[8]; };
__device__ __forceinline__ Eight halves(const u32x4 &v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e.f[2 * i] = half_bits_to_float(w[i] & 0xffffu);
        e.f[2 * i + 1] = half_bits_to_float(w[i] >> 16);
    }
    return e;
}
__device__ __forceinline__ u32x4 to_halves(const Eight &e) {
    return u32x4{float2_to_half2_bits(e.f[0], e.f[1]), float2_to_half2_bits(e.f[2], e.f[3]),
                 float2_to_half2_bits(e.f[4], e.f[5]), float2_to_half2_bits(e.f[6], e.f[7])};
}

// 8 consecutive values of h from x and r; the sum is rounded to FP16 because that is what the next layer adds to and
// what is normalised here
__device__ __forceinline__ u32x4 add_halves(const u32x4 &x, const u32x4 &r) {
    const Eight a = halves(x), b = halves(r);
    Eight e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.f[i] = a.f[i] + b.f[i];
    return to_halves(e);
}
__device__ __forceinline__ float squares(const u32x4 &h) {
    const Eight e = halves(h);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf(e.f[i], e.f[i], s);
    return s;
}
__device__ __forceinline__ Eight normed(const u32x4 &h, const u32x4 &w, float inv) {
    Eight e = halves(h);
    const Eight g = halves(w);
#pragma unroll
    for (int i = 0; i < 8; ++i) e.f[i] = e.f[i] * inv * g.f[i];
    return e;
}
__device__ __forceinline__ uint32_t largest(const Eight &e, uint32_t top) {
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(e.f[i]) & 0x7fffffffu);
    return top;
}
// The codes come from y in 32 bits, not from its FP16 rounding: one rounding less, and the scale is that of the values
// themselves.  (y and the scale are far inside the binary32 range, see div_by_scale.)
__device__ __forceinline__ u32x2 codes(const Eight &e, float s, float y) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = clamp448(div_by_scale(e.f[i], s, y));
    return u32x2{e4m3x4_from_float_hw(q[0], q[1], q[2], q[3]), e4m3x4_from_float_hw(q[4], q[5], q[6], q[7])};
}

__device__ __forceinline__ float sum_of_workgroup(float v, float *red, int waves) {
    v = sum_of_wave(v);
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
    for (int i = 0; i < waves; ++i) s += red[i];
    return s;
}
__device__ __forceinline__ uint32_t max_of_workgroup(uint32_t v, uint32_t *red, int waves) {
    v = max_of_wave(v);
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int i = 0; i < waves; ++i) v = max(v, red[i]);
    return v;
}

// CPT > 0: a lane keeps CPT chunks of 8 values in registers.  CPT == 0, for rows that do not fit (above 32768 columns): three
// passes over the row, h from x and r each time (x and r are not changed: a sum written over one of them is written in the
// last pass, after the lane's own last read of that chunk).
template <int CPT>
__global__ void __launch_bounds__(1024)
add_rms_norm_kernel(NormArgs p) {
    const int64_t m = blockIdx.x;
    const u32x4 *x = reinterpret_cast<const u32x4 *>(p.X + m * p.ldx);
    const u32x4 *r = p.R ? reinterpret_cast<const u32x4 *>(p.R + m * p.ldr) : nullptr;
    u32x4 *sum = p.sum ? reinterpret_cast<u32x4 *>(p.sum + m * p.lds) : nullptr;
    const u32x4 *w = reinterpret_cast<const u32x4 *>(p.weight);
    u32x4 *out = p.Y ? reinterpret_cast<u32x4 *>(p.Y + m * p.ldy) : nullptr;
    u32x2 *code = p.Xq ? reinterpret_cast<u32x2 *>(p.Xq + m * p.K) : nullptr;
    const int chunks = (int)(p.K / 8), waves = blockDim.x >> 6, threads = blockDim.x;
    __shared__ float red_sum[16];
    __shared__ uint32_t red_max[16];
    float total = 0.0f;
    uint32_t top = 0;
    if constexpr (CPT > 0) {
        u32x4 h[CPT], g[CPT];
        Eight y[CPT];
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const int c = threadIdx.x + i * threads;
            h[i] = c < chunks ? x[c] : u32x4{0u, 0u, 0u, 0u};
            g[i] = c < chunks ? w[c] : u32x4{0u, 0u, 0u, 0u};
        }
        if (r) {
            u32x4 add[CPT];
#pragma unroll
            for (int i = 0; i < CPT; ++i) {
                const int c = threadIdx.x + i * threads;
                add[i] = c < chunks ? r[c] : u32x4{0u, 0u, 0u, 0u};
            }
#pragma unroll
            for (int i = 0; i < CPT; ++i) h[i] = add_halves(h[i], add[i]);
        }
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const int c = threadIdx.x + i * threads;
            if (sum && c < chunks) sum[c] = h[i];
            total += squares(h[i]);
        }
        const float inv = rsqrtf(sum_of_workgroup(total, red_sum, waves) / (float)p.K + p.eps);
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const int c = threadIdx.x + i * threads;
            y[i] = normed(h[i], g[i], inv);
            if (out && c < chunks) out[c] = to_halves(y[i]);
            top = largest(y[i], top);
        }
        if (!code) return;
        const float amax = __uint_as_float(max_of_workgroup(top, red_max, waves));
        const float s = amax == 0.0f ? 1.0f : amax / 448.0f, back = 1.0f / s;
        if (threadIdx.x == 0) p.scales[m] = s;
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const int c = threadIdx.x + i * threads;
            if (c < chunks) code[c] = codes(y[i], s, back);
        }
    } else {
        for (int c = threadIdx.x; c < chunks; c += threads) total += squares(r ? add_halves(x[c], r[c]) : x[c]);
        const float inv = rsqrtf(sum_of_workgroup(total, red_sum, waves) / (float)p.K + p.eps);
        float s = 1.0f, back = 1.0f;
        if (code) {
            for (int c = threadIdx.x; c < chunks; c += threads) top = largest(normed(r ? add_halves(x[c], r[c]) : x[c], w[c], inv), top);
            const float amax = __uint_as_float(max_of_workgroup(top, red_max, waves));
            s = amax == 0.0f ? 1.0f : amax / 448.0f;
            back = 1.0f / s;
            if (threadIdx.x == 0) p.scales[m] = s;
        }
        for (int c = threadIdx.x; c < chunks; c += threads) {
            const u32x4 h = r ? add_halves(x[c], r[c]) : x[c];
            const Eight y = normed(h, w[c], inv);
            if (sum) sum[c] = h;
            if (out) out[c] = to_halves(y);
            if (code) code[c] = codes(y, s, back);
        }
    }
}

int launch_add_rms_norm(const NormArgs &a, int64_t M, hipStream_t stream) {
    const int64_t chunks = a.K / 8;
    const dim3 grid((unsigned)M);
    if (chunks > 4096) {
        add_rms_norm_kernel<0><<<grid, 1024, 0, stream>>>(a);
        return hip_ok(hipGetLastError());
    }
    const int cpt = chunks <= 1024 ? 1 : (chunks <= 2048 ? 2 : 4);
    const int threads = (int)(((chunks + cpt - 1) / cpt + 63) / 64 * 64);
    if (cpt == 1) add_rms_norm_kernel<1><<<grid, threads, 0, stream>>>(a);
    else if (cpt == 2) add_rms_norm_kernel<2><<<grid, threads, 0, stream>>>(a);
    else add_rms_norm_kernel<4><<<grid, threads, 0, stream>>>(a);
    return hip_ok(hipGetLastError());
}

}  // namespace nfp
