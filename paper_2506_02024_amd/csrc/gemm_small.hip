// Streaming GEMM for decode-sized batches (M <= 64): which launch shape a problem takes, the launch, and the reduction of K splits.  The
// kernel is in gemm_small_kernels.h.
#include <algorithm>
#include <cmath>

#include "gemm_small_kernels.h"

namespace nfp {

struct NoEpilogue {};
template <int EPI> using ReducedEpilogue = std::conditional_t<EPI == kEpiNone, NoEpilogue, Epilogue>;

// Sums the S split-K partials (rows of ldp floats) in slice order, four columns per lane, applies the
// FP8-mode scale, writes fp16.  VEC: 8-byte stores (N % 4 == 0 and 8-byte aligned output rows; gated: 4-byte
// stores).
template <int EPI, bool VEC>
__global__ void __launch_bounds__(256)
splitk_reduce_kernel(const float *__restrict__ partials, int S, int M, int N, int ldp, const float *scales,
                     float w_scale, uint16_t *Y, int64_t ldy, ReducedEpilogue<EPI> epi) {
    const int64_t total = (int64_t)M * ldp;
    const int64_t idx = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (idx >= total) return;
    const int m = (int)(idx / ldp), n = (int)(idx - (int64_t)m * ldp);
    // (what is added to the sums is under way while they are loaded)
    floatx4 bias = {0.f, 0.f, 0.f, 0.f};
    u32x2 add = {0u, 0u};
    if constexpr (EPI != kEpiNone) {
        bias = bias4(epi, n, N);
        add = residual4<EPI>(epi, m, n, N);
    }
    floatx4 v = *reinterpret_cast<const floatx4 *>(partials + idx);
    for (int s = 1; s < S; ++s) {
        const floatx4 u = *reinterpret_cast<const floatx4 *>(partials + (int64_t)s * total + idx);
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    if (scales) {
        const float sc = scales[m] * w_scale;
        v.x = scale_f32(v.x, sc); v.y = scale_f32(v.y, sc); v.z = scale_f32(v.z, sc); v.w = scale_f32(v.w, sc);
    }
    if constexpr (EPI != kEpiNone) v = epilogue4<EPI>(v, bias, add, epi.act);
    if constexpr (EPI == kEpiGated) {
        uint16_t *to = Y + (int64_t)m * ldy + (n >> 1);
        const uint32_t o = float2_to_half2_bits(v.x, v.y);
        if (VEC) {
            *reinterpret_cast<uint32_t *>(to) = o;
        } else {
            to[0] = (uint16_t)o;
            if (n + 2 < N) to[1] = (uint16_t)(o >> 16);
        }
        return;
    }
    uint16_t *dst = Y + (int64_t)m * ldy + n;
    if (VEC) {
        u32x2 o;
        o.x = float2_to_half2_bits(v.x, v.y);
        o.y = float2_to_half2_bits(v.z, v.w);
        *reinterpret_cast<u32x2 *>(dst) = o;
    } else {
        const float x[4] = {v.x, v.y, v.z, v.w};
        for (int q = 0; q < 4 && n + q < N; ++q) {
            union { _Float16 f; uint16_t u; } c;
            c.f = (_Float16)x[q];
            dst[q] = c.u;
        }
    }
}

template <int EPI>
static void launch_reduce_t(const float *partials, int S, int64_t M, int64_t N, const float *scales, float w_scale, uint16_t *Y, int64_t ldy,
                            const ReducedEpilogue<EPI> &epi, hipStream_t stream) {
    const int64_t ldp = partial_ld(N), total = M * ldp;
    const int64_t piece = EPI == kEpiGated ? 2 : 4;            // outputs of a lane
    const bool vec = (N & 3) == 0 && ldy % piece == 0 && (reinterpret_cast<uintptr_t>(Y) & (2 * piece - 1)) == 0;
    const unsigned blocks = (unsigned)((total / 4 + 255) / 256);
    if (vec) splitk_reduce_kernel<EPI, true><<<blocks, 256, 0, stream>>>(partials, S, (int)M, (int)N, (int)ldp, scales, w_scale, Y, ldy, epi);
    else splitk_reduce_kernel<EPI, false><<<blocks, 256, 0, stream>>>(partials, S, (int)M, (int)N, (int)ldp, scales, w_scale, Y, ldy, epi);
}

int launch_splitk_reduce(const float *partials, int S, int64_t M, int64_t N, const float *scales,
                         float w_scale, uint16_t *Y, int64_t ldy, const Epilogue &epi, hipStream_t stream) {
    if (epi.kind == kEpiNone) launch_reduce_t<kEpiNone>(partials, S, M, N, scales, w_scale, Y, ldy, NoEpilogue(), stream);
    else if (epi.kind == kEpiFull) launch_reduce_t<kEpiFull>(partials, S, M, N, scales, w_scale, Y, ldy, epi, stream);
    else launch_reduce_t<kEpiGated>(partials, S, M, N, scales, w_scale, Y, ldy, epi, stream);
    return hip_ok(hipGetLastError());
}

// ---- host-side configuration ---------------------------------------------------------
// Launch shapes of the streaming kernel that were timed faster than what the cost model below chooses, on the
// layer shapes of the models the paper evaluates (Sec. 5.1), for batches of up to 16 tokens.
struct TunedSmall { int cls, N, K, spw, split, tiles; };
static const TunedSmall kTunedSmall[] = {
#include "tuned_small.inc"
    {-1, 0, 0, 0, 0, 0},
};

// What a launch costs, in microseconds.  Fitted by fit_costs.py to 129 000 timings: 72 layer shapes of 0.3 to
// 500 Mi weights x 1, 8, 16, 24, 32 and 64 tokens x both storage orders of the planes and FP16 weights x
// every K split, slice length and tile count; weights cold, replayed graphs.  On those the cheapest candidate
// is 1 % behind the fastest launch on average, 5-6 % at the 95th percentile.  What it says: a K split
// costs about 1 us and 0.7 us per slice (the last workgroup's three trips to memory), more than it gives
// on small layers, where eight slices took 10 us against 4.3 for one ((1560, 1040), 1 token); a CU takes in
// weights at 40 GB/s at most, and at 27 if its workgroups have a single tile each, whose look-ahead then has
// nothing to fetch: (2432, 7104) at 1 token 13.4 us on 152 workgroups of one tile, 10.6 on 228 of two.
struct SmallCost {
    double base;            // launch, first load, reduction over the waves
    double chip_rate, cu_rate;      // bytes per microsecond of the weight stream: whole chip, one CU
    double single;          // a CU's time with one tile per workgroup, against several
    double four;            // a CU's time with four token tiles, against one or two
    double split, slice;    // K split: once, per slice
    double x_rate;          // bytes per microsecond at which a CU fetches activations
    double round;           // workgroups beyond what fits the chip at a time, per round
    double part_rate;       // bytes per microsecond of partial sums
    double pass;            // a further pass over K
};
static const SmallCost kSmallCost[2] = {
    // FP16 mode; plain FP16 too (fitted together), so that the same knobs give both the same launch shape
    {2.90, 8.08e6, 40.4e3, 1.47, 1.25, 0.57, 0.67, 110e3, 2.37, 1.11e6, 1.24},
    {2.99, 8.01e6, 40.6e3, 1.48, 1.34, 0.35, 0.73, 137e3, 1.58, 0.98e6, 1.23},      // E4M3
};

static double price_small(int kind, const SmallConfig &c, int64_t M, int64_t N, int64_t K) {
    const bool fp8 = kind_is_fp8(kind);
    const SmallCost &k = kSmallCost[fp8 ? 1 : 0];
    const double wb = fp8 ? 1.0 : 2.0;                            // bytes per weight, and per activation
    const int64_t tiles = (N + 15) / 16;
    const int64_t wgs = ((tiles + c.tiles_per_wg - 1) / c.tiles_per_wg) * c.split;
    const int64_t lds = (int64_t)((c.tiles_per_wg + 1) & ~1) * c.waves * c.mt * 1024 + c.waves * 2048;
    const int waves_cu = c.mt == 1 ? (c.spw == 2 ? 28 : (c.spw == 4 ? 16 : 8)) : (c.mt == 2 ? 20 : 16);   // by registers
    const int64_t slots = std::max<int64_t>(1, std::min<int64_t>(160 * 1024 / lds, waves_cu / c.waves));
    const double k_wg = (double)c.waves * c.passes * c.spw * (fp8 ? 128 : 64);      // columns of a workgroup
    const double wg_cu = (double)((wgs + 255) / 256);             // workgroups of the busiest CU
    const double chip = (double)N * (double)K * wb / k.chip_rate;
    const double cu = wg_cu * c.tiles_per_wg * 16.0 * std::min(k_wg, (double)K) * wb / k.cu_rate *
                      (c.tiles_per_wg == 1 ? k.single : 1.0) * (c.mt == 4 ? k.four : 1.0);
    const double a = chip * chip, b = cu * cu;
    double t = k.base + std::sqrt(std::sqrt(a * a + b * b));
    t += wg_cu * (double)std::min<int64_t>(M, 16 * c.mt) * k_wg * wb / k.x_rate;
    t += k.round * (double)((wgs + 256 * slots - 1) / (256 * slots) - 1) + k.pass * (c.passes - 1);
    if (c.split > 1) t += k.split + k.slice * c.split + (double)c.split * (double)M * (double)N * 4.0 / k.part_rate;
    return t;
}

static SmallConfig compute_small(int kind, int64_t M, int64_t N, int64_t K) {
    const Tuning &t = tuning();
    const int mt = M <= 16 ? 1 : (M <= 32 ? 2 : 4);
    // knobs first; with none set, the table of timed shapes; otherwise the cheapest candidate
    int64_t k_spw = t.small_spw, k_split = t.small_split, k_tiles = t.small_tiles;
    if (k_spw <= 0 && k_split <= 0 && k_tiles <= 0 && t.tuned_table != 0 && mt == 1) {
        for (const TunedSmall &e : kTunedSmall)
            if (e.cls == kind_class(kind) && e.N == N && e.K == K) {
                k_spw = e.spw;  k_split = e.split;  k_tiles = e.tiles;
                break;
            }
    }
    const bool fp8 = kind_is_fp8(kind);
    const int kstep = fp8 ? 128 : 64;
    const int steps = (int)((K + kstep - 1) / kstep);
    // K-steps per wave: 2 or 4; 2 with several token tiles (their activations need the registers); 8 where
    // it is asked for and exists (row-major weights of a long K: 512 bytes or more of each row)
    const bool can_long = (kind == kPlainF16 || kind == kNestedF16Row) && mt == 1 && (K + 63) / 64 >= 64;
    int spws[2] = {2, 4}, n_spw = 2;
    if (mt > 1) n_spw = 1;
    else if (k_spw == 2 || k_spw == 4 || (k_spw == 8 && can_long)) { spws[0] = (int)k_spw;  n_spw = 1; }
    else if (k_spw == 8) { spws[0] = 4;  n_spw = 1; }
    SmallConfig best;
    best.cost = 1e30;
    for (int q = 0; q < n_spw; ++q) {
        SmallConfig c;
        c.mt = mt;
        c.spw = spws[q];
        const int max_waves = (mt == 4 || c.spw == 8) ? 8 : 16;   // (these need up to 256 VGPRs per wave)
        const int slices = (steps + c.spw - 1) / c.spw;           // wave-sized K slices
        const int rounds = (slices + max_waves - 1) / max_waves;
        for (int split : {1, 2, 3, 4, 6, 8}) {
            if (k_split > 0) split = (int)std::min<int64_t>(k_split, slices);
            // a split's scratch has to leave room in the fixed scratch of nestedfp_gemm_static, which takes
            // every problem that fits it unsplit
            else if (split > 1 && (split > slices || (double)split * (double)M * (double)N * 4.0 +
                                                     (fp8 ? (double)M * (double)K : 0.0) > 30.0 * 1024 * 1024)) break;
            // what the waves of all grid slices do not cover at once is walked in passes
            c.split = split;
            c.passes = (rounds + split - 1) / split;
            c.waves = (slices + split * c.passes - 1) / (split * c.passes);
            // a workgroup keeps a kilobyte of partial sums per tile, token tile and wave in LDS (an even
            // number of tiles, 128 KB at most)
            int per_max = (128 / (c.waves * mt)) & ~1;
            per_max = std::max(1, std::min(per_max, 16));
            for (int per = 1; per <= per_max; ++per) {
                c.tiles_per_wg = k_tiles > 0 ? (int)std::min<int64_t>(k_tiles, per_max) : per;
                c.cost = price_small(kind, c, M, N, K);
                if (c.cost < best.cost) best = c;
                if (k_tiles > 0) break;
            }
            if (k_split > 0) break;
        }
    }
    return best;
}

static SmallConfig choose_small(int kind, int64_t M, int64_t N, int64_t K) {
    static thread_local PlanCache<SmallConfig> cache;
    // (row-major planes can take 8 K-steps where packed ones cannot)
    return cache.get(kind == kNestedF16Row ? 3 : kind_class(kind), M, N, K, [&] { return compute_small(kind, M, N, K); });
}

double small_gemm_cost(int kind, int64_t M, int64_t N, int64_t K) { return choose_small(kind, M, N, K).cost; }

bool small_gemm_supports(int kind, int64_t M, int64_t N, int64_t K, int64_t ldw) {
    // the weight array must be addressable with 31-bit byte offsets (bit 31 marks a load as dead),
    // a few tiles of slack included
    (void)M;
    return weight_array_bytes(kind, N + 48, K, ldw) < ((int64_t)1 << 31);
}

size_t small_gemm_partial_bytes(int kind, int64_t M, int64_t N, int64_t K) {
    SmallConfig c = choose_small(kind, M, N, K);
    return c.split > 1 ? (size_t)c.split * (size_t)M * (size_t)partial_ld(N) * sizeof(float) : 0;
}

// Whether the streaming kernel quantises the activations itself: one token tile, all of K in the workgroup.  What it saves
// is a launch (1.3 us in a graph, 3 us of host time outside one); what it costs is that every workgroup waits for
// its M x K activations, their row maxima and 3 VALU instructions per value before it multiplies, while two weight
// tiles are on their way.  Up to 8 tokens (half the lanes' rows) that pays where a workgroup has further tiles or the
// rows are short (us with the launch of its own / fused): (1024, 1024) 5.2 / 4.0, (12288, 3072) 10.9 / 9.8, (8192, 5120) 11.6 / 11.0,
// (8192, 8192) 15.7 / 14.9; with one tile (4096, 4096) takes 8.5 / 8.5 and (3072, 7168) 10.5 / 11.3.  With 16 rows to convert it pays
// on short rows, 16 tokens on (1024, 1280) 5.8 / 5.5, and up to 3584 columns from three tiles on: (12288, 2048) 9.6 / 9.0,
// (32768, 2048) 15.2 / 14.7, (16384, 3584) 14.2 / 13.7 at 9 tokens and level at 16, (6144, 2560) with two 8.0 / 8.4, (4096, 4096) 8.7 / 10.5.
bool small_gemm_fuses_quant(int64_t M, int64_t N, int64_t K) {
    const int64_t knob = tuning().small_fuse_quant;
    if (knob == 0) return false;
    const SmallConfig c = choose_small(kE4M3, M, N, K);
    if (c.mt != 1 || c.split != 1 || c.passes != 1 || (c.spw != 2 && M > 8) || small_lds(c) > (size_t)kQuantLds) return false;
    return knob > 0 || (M <= 8 ? (c.tiles_per_wg > 1 || K <= 3072) : (K <= 1280 || (K <= 3584 && c.tiles_per_wg > 2)));
}

int launch_small_gemm(int kind, const GemmArgs &a, hipStream_t stream) {
    SmallConfig c = choose_small(kind, a.M, a.N, a.K);
    FusedSmallParams p;
    p.X = static_cast<const uint8_t *>(a.X);
    p.x_row_bytes = (kind == kE4M3 || kind == kE4M3Row) ? a.ldx : 2 * a.ldx;
    p.scales = a.scales;
    p.static_scale = a.static_scale;
    p.quant_hw = tuning().quant_hw != 0 ? 1 : 0;
    p.w_scale = a.w_scale;
    p.W0 = static_cast<const uint8_t *>(a.W0);
    p.W1 = static_cast<const uint8_t *>(a.W1);
    if (kind_is_packed(kind)) {
        // 16 rows of a tile take 16 * Kp contiguous elements (Kp = K rounded up to 64)
        p.w_row_bytes = 0;
        p.tile_bytes = (uint32_t)(((a.K + 63) / 64) * 1024 * kind_elem_bytes(kind));
    } else {
        p.w_row_bytes = (uint32_t)(kind == kPlainF16 ? 2 * a.ldw : a.K);
        p.tile_bytes = 16u * p.w_row_bytes;
    }
    p.w_bytes = (uint32_t)weight_array_bytes(kind, a.N, a.K, a.ldw);
    p.M = (int)a.M;  p.N = (int)a.N;  p.K = (int)a.K;
    p.Y = a.Y;  p.ldy = a.ldy;
    p.partials = a.partials;
    p.ldp = (int)partial_ld(a.N);
    p.tiles_per_wg = c.tiles_per_wg;
    const int64_t tiles = (a.N + 15) / 16;
    const unsigned grid_x = (unsigned)((tiles + c.tiles_per_wg - 1) / c.tiles_per_wg);
    // the last workgroup of a tile column sums the K slices itself where there is a counter for it
    const bool fused_reduce = c.split > 1 && a.counters != nullptr && grid_x <= (unsigned)kMaxCounters &&
                              (int64_t)c.split * a.M * partial_ld(a.N) * 4 < ((int64_t)1 << 32) && tuning().fused_reduce != 0;
    p.counters = fused_reduce ? a.counters : nullptr;
    p.k_passes = c.passes;
    p.tile_stride = (tuning().small_interleave != 0 && c.tiles_per_wg > 1) ? (int)grid_x : 1;
    // Rows that are a multiple of 4 KB long put the 16 rows of a slice on the same memory channels, and as
    // the workgroups start together, wave by wave, the whole chip asks for one group of channels after
    // the other; with the slices rotated from workgroup to workgroup of an XCD it does not (16 tokens,
    // FP16 mode: (28672, 4096) 44.2 -> 39.5 us, (57344, 8192) 174 -> 154 us).  Other row lengths lose up to
    // 3 % by it, and plain FP16 weights, whose slices are a kilobyte long, gain only from rows of 16 KB on
    // ((57344, 8192) 172 -> 150 us, (28672, 4096) 37.2 -> 38.4 us).
    const uint32_t channels = kind == kPlainF16 ? 16384u : 4096u;
    p.rotate = !kind_is_packed(kind) && p.w_row_bytes % channels == 0 ? 1 : 0;
    p.vec_store = ((a.N & 3) == 0 && (a.ldy & 3) == 0 && (reinterpret_cast<uintptr_t>(a.Y) & 7) == 0) ? 1 : 0;
    if (a.epi.kind == kEpiGated) p.vec_store = ((a.N & 3) == 0 && (a.ldy & 1) == 0 && (reinterpret_cast<uintptr_t>(a.Y) & 3) == 0) ? 1 : 0;
    if (c.split > 1 && (a.partials == nullptr ||
                        a.partial_bytes < (size_t)c.split * a.M * partial_ld(a.N) * sizeof(float)))
        return kErrWorkspace;
    dim3 grid(grid_x, (unsigned)c.split);
    if (kind_quantizes(kind) && !(c.mt == 1 && c.split == 1 && c.passes == 1)) return kErrArg;   // caller checks first
    p.epi = a.epi;
    if (kind < 0 || kind >= kNumKinds) return kErrArg;
    if (a.epi.kind == kEpiNone) launch_stream_t<kEpiNone>(kind, p, c, grid, stream);
    else if (a.epi.kind == kEpiFull) launch_stream_full(kind, p, c, grid, stream);
    else launch_stream_gated(kind, p, c, grid, stream);
    if (hipGetLastError() != hipSuccess) return kErrHip;
    if (c.split > 1 && !fused_reduce)
        return launch_splitk_reduce(a.partials, c.split, a.M, a.N, kind_is_fp8(kind) ? a.scales : nullptr,
                                    a.w_scale, a.Y, a.ldy, a.epi, stream);
    return kOk;
}

}  // namespace nfp
