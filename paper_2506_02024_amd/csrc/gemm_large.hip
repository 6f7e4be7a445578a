// LDS-tiled MFMA GEMMs for prefill-sized batches: which launch shape a problem takes, and the launch.  The kernels are in
// gemm_large_kernels.h.
#include "gemm_large_kernels.h"

namespace nfp {


static const int kSplits[] = {1, 2, 3, 4, 6, 8};

// split-K cost: the reduction kernel's launch plus its traffic
static double split_cost(int64_t M, int64_t N, int slices, double launch_us, double bytes_per_us) {
    return launch_us + 8.0 * (double)M * (double)N * slices / bytes_per_us;
}

// At most 64 tokens: one 64 x 128 tile shape per weight kind and only the split to choose.  Such a
// launch is bound by the weight stream, whose rate depends on how many workgroups pull on it.
// Constants from timings of the four splits on six layer shapes at M = 64, packed planes.  Row-major planes
// share them, so that both storage orders launch alike and give the same bits, though by pairs of K-tiles
// (BypassKernel::PAIR) they hold one workgroup per CU: over 72 layer shapes at 20 ... 64 tokens the choice is
// 1.7 % (packed) and 2.3 % (row-major) behind the best split on average, 25 and 36 % at worst.
struct Tile64Cost {
    double tk, tfix;        // microseconds per K-tile and per workgroup
    int slots;              // workgroups the chip holds at a time
    double rate, rate512;   // bytes per microsecond of the weight stream (from 512 workgroups on)
    double few;             // exponent of the rate's fall below 256 workgroups
};
static const Tile64Cost kTile64Cost[3] = {
    {0.7, 0.4, 512, 4.5e6, 5.5e6, 0.5},       // plain FP16 (LDS kernel, three workgroups per CU)
    {0.466, 0.4, 512, 5.25e6, 5.5e6, 0.5},    // NestedFP16 (register path; packed planes: two per CU)
    {0.35, 0.4, 256, 5.5e6, 5.5e6, 0.3},      // E4M3 (register path, one per CU)
};
static LargeConfig choose_tile64(int cls, int64_t M, int64_t N, int64_t K, int max_split = 8) {
    const int kt = (int)(((cls == 2 ? K : 2 * K) + 127) / 128);
    const Tuning &t = tuning();
    const Tile64Cost &tc = kTile64Cost[cls];
    LargeConfig c;
    c.tm = 64;  c.tn = 128;  c.split = 1;  c.deep = 0;  c.height = 64;
    const int64_t tiles = ((M + 63) / 64) * ((N + 127) / 128);
    double best = 1e30;
    // A split stays inside the scratch of the entry point without a workspace wherever the problem does: the
    // streaming kernel, which may run the same layer, never needs more.  It bars splits of very wide layers only, which
    // fill the chip without: (57344, 8192) in FP16 mode at 64 tokens 199 us in the four slices the model
    // would take, 159 unsplit.  (Plain FP16 weights have no such entry point.)
    const bool bounded = cls != 0 && static_scratch_holds(1, M, N, K, cls == 2, partial_ld(N));
    for (int split : {1, 2, 3, 4, 6, 8}) {
        if (t.large_split > 0) split = (int)(t.large_split < kt ? t.large_split : kt);
        else if (split > 1 && (split > kt / 4 || split > max_split)) break;
        else if (bounded && !static_scratch_holds(split, M, N, K, cls == 2, partial_ld(N))) break;
        const int per = (kt + split - 1) / split;
        const int slices = (kt + per - 1) / per;
        const int64_t wgs = tiles * slices;
        const int64_t rounds = (wgs + tc.slots - 1) / tc.slots;
        double time = (double)rounds * (tc.tfix + per * tc.tk);
        double floor_t = (double)N * (double)kt * 128.0 / (wgs < 512 ? tc.rate : tc.rate512);
        if (wgs < 256) floor_t *= std::pow(256.0 / (double)wgs, tc.few);
        // the weight stream is shared per CU: workgroups beyond one per CU that do not make a whole
        // further round leave most CUs waiting for a few (measured: 320 workgroups take 1.3-1.5 times
        // as long as 240 with the same bytes)
        if (wgs > 256) floor_t *= (double)(((wgs + 255) / 256) * 256) / (double)wgs;
        if (time < floor_t) time = floor_t;
        if (slices > 1) time += split_cost(M, N, slices, 4.56, 4.24e6);
        if (time < best) { best = time;  c.split = split; }
        if (t.large_split > 0) break;
    }
    c.cost = best;
    // (a split whose scratch the padding of the rows has pushed past the fixed one: the best smaller split)
    if (t.large_split <= 0 && !padded_split_fits(c.split, M, N, K, cls == 2)) return choose_tile64(cls, M, N, K, c.split - 1);
    return c;
}

Tile64Plan tile64_plan(int kind, int64_t M, int64_t N, int64_t K) {
    static thread_local PlanCache<Tile64Plan> cache;
    return cache.get(kind_class(kind), M, N, K, [&] {
        const LargeConfig c = choose_tile64(kind_class(kind), M, N, K);
        return Tile64Plan{c.cost, c.split};
    });
}

// Token tiles of 256 exist cut down to 160, 192 and 224 tokens as well, all of a launch alike: register-path tiles and the
// 256 x 256 tiles of plain FP16 and E4M3.  The sums are the same at every height.
static bool cuts_tiles(int cls, int tn) { return cls == 1 || tn == 256; }
// Up to 256 tokens, and for timed launch shapes: the height that the batch needs, as many tiles as of 256 without the
// rows that only padding would fill.  777 tokens are four tiles of 224 instead of three of 256 and one of 9.  (28672, 4096),
// FP16 mode: 150 tokens 83.6 -> 66.9 us (row-major planes), 300 tokens 120 -> 96 us; FP8 mode gains 1-8 %.
static int token_tile(int cls, int tm, int tn, int64_t M) {
    if (tm != 256 || !cuts_tiles(cls, tn)) return tm;
    const int64_t tiles = (M + 255) / 256;
    const int h = (int)(((M + tiles - 1) / tiles + 31) / 32 * 32);
    return h < 160 ? 160 : h;
}
// the knob large_height instead, where there are such tiles
static int knob_height(int cls, int tm, int tn) {
    const int64_t want = tuning().large_height;
    return tm == 256 && cuts_tiles(cls, tn) && want >= 160 && want <= 256 && want % 32 == 0 ? (int)want : 0;
}

// Launch shapes that were timed faster than the cost model's choice, for the layer shapes of the
// models the paper evaluates (Sec. 5.1).  An entry tuned at M tokens serves the batches of more than
// 3 M / 4 (M / 2 up to 64 tokens) and at most M tokens that give the same number of token tiles.
// An entry holds no height of the token tiles: up to 256 tokens that is token_tile's, with the tile pinned for a timing as
// in the launch it stands for; above, the model would choose it, and the entry would be launched at another one than it was timed at.
struct TunedTile { int cls, N, K, M, tm, tn, split, deep; };
static constexpr TunedTile kTunedTiles[] = {
#include "tuned_tiles.inc"
    {-1, 0, 0, 0, 0, 0, 0, 0},
};
static constexpr bool tuned_up_to(int tokens) {
    for (const TunedTile &e : kTunedTiles)
        if (e.M > tokens) return false;
    return true;
}
static_assert(tuned_up_to(256), "timed launch shapes of more than 256 tokens need their height");

static bool tuned_large(int cls, int64_t M, int64_t N, int64_t K, LargeConfig &c) {
    for (const TunedTile &e : kTunedTiles) {
        if (e.cls != cls || e.N != N || e.K != K) continue;
        // (batches of up to 64 tokens are one 64-token tile whatever their size; above, a shape timed
        // at M tokens is trusted down to three quarters of M)
        if (M > e.M || (e.M <= 64 ? 2 * M <= e.M : 4 * M <= 3 * e.M)) continue;
        if ((M + e.tm - 1) / e.tm != (e.M + e.tm - 1) / e.tm) continue;
        c.tm = e.tm;  c.tn = e.tn;  c.split = e.split;  c.deep = e.deep;  c.height = token_tile(cls, e.tm, e.tn, M);
        return true;
    }
    return false;
}

// 65 ... 256 tokens of the two classes whose tiles of 256 tokens are cut down: every tile shape, the 64-token tiles
// included, priced by what was found to add up -- the rounds of workgroups, the weights, what all workgroups take in
// from L2 (weights and tokens) and what the busiest CU does.  Taken from timings of every shape and split (and both
// pipeline depths of E4M3, of which the deeper one is all that is left).  On the 82 000 launches that fit_costs.py times for them (weights
// cold, 70 layers of 0.8 to 500 Mi weights, twelve batch sizes, both storage orders) the choice is 2.2 % (FP16 mode) and 2.0 % (FP8
// mode) behind the fastest launch on average, 12-13 % at the 95th percentile; the model below, which knows neither the 64-token
// tiles nor the newer kernels, was 7-10 % behind.  Constants fitted to these timings are at 1.7 and 1.6 %, but take 40 to 90
// launches that lose more than 6 %; one launch timed twice differs by up to as much.
struct ShortShape { int tm, tn, deep; double tk, tfix, tk160, tfix160; };      // microseconds per K-tile and per workgroup; at a height of 160
struct ShortCost {
    ShortShape shape[5];
    double pair128, pair64;             // workgroups of a CU that run together
    double base, w_rate, l2_rate, cu_rate, split, split_rate;
};
static const ShortCost kShortCost[2] = {
    // FP16 operands through registers
    {{{256, 256, 0, 0.725, 6.05, 0.556, 3.47}, {256, 128, 0, 0.421, 2.63, 0.314, 1.28}, {128, 256, 0, 0.500, 2.61, 0, 0},
      {128, 128, 0, 0.2785, 0.83, 0, 0}, {64, 128, 0, 0.271, 0.51, 0, 0}}, 1.045, 1.045, 3.0, 15.2e6, 219e6, 167e3, 3.45, 5.28e6},
    // E4M3
    {{{256, 256, 0, 0.6255, 3.16, 0.378, 3.16}, {256, 128, 1, 0.319, 2.41, 0.319, 2.41}, {128, 256, 1, 0.334, 2.71, 0, 0},
      {128, 128, 1, 0.2136, 1.73, 0, 0}, {64, 128, 0, 0.183, 1.54, 0, 0}}, 1.0, 1.10, 2.0, 10.4e6, 1e15, 144e3, 3.28, 4.68e6},
};
// Splits whose partial sums outgrow the fixed scratch of nestedfp_gemm_static are left to FP16 mode, where they are priced 4 %
// cheaper than what fits: (17616, 5872) at 256 tokens in three slices of 18 MB 81 us (packed) and 93 (row-major), unsplit 103 and 111.
// (At 1-3 % they gain and lose by 10 %; in FP8 mode (8192, 28672) would gain 5-13 %, (5120, 32768) lose 12-21 %.)  That entry
// point takes what fits (bounded).
// E4M3 weights on 64-token tiles: the weight tiles past a multiple of eight (see tile_of_block) are fetched by each token tile on
// another XCD, from memory once the plane is larger than the L2s: with three and four token tiles such launches take 10-30 % longer than
// priced ((5840, 5840) at 144 tokens 29 us against 20.6 in two slices of 128 x 128), the others what they are priced at.
static LargeConfig choose_short(int cls, int64_t M, int64_t N, int64_t K, bool bounded) {
    const bool fp8 = cls == 2;
    const ShortCost &m = kShortCost[fp8 ? 1 : 0];
    const Tuning &t = tuning();
    const int kt = (int)(((fp8 ? K : 2 * K) + 127) / 128);
    const bool limited = static_scratch_holds(1, M, N, K, fp8, partial_ld(N));
    const int want_m = (t.large_bm == 128 || t.large_bm == 256) ? (int)t.large_bm : 0;
    const int want_n = (t.large_bn == 128 || t.large_bn == 256) ? (int)t.large_bn : want_m;
    LargeConfig c;
    c.tm = 128;  c.tn = 128;  c.split = 1;  c.deep = 0;  c.height = 128;
    double best = 1e30;
    for (const ShortShape &e : m.shape) {
        if (want_m && want_m != e.tm) continue;
        if (want_n && want_n != e.tn) continue;
        const int height = token_tile(cls, e.tm, e.tn, M);
        const int64_t tiles = ((M + e.tm - 1) / e.tm) * ((N + e.tn - 1) / e.tn);
        double tk = e.tk, tfix = e.tfix;
        if (e.tm == 256) {
            const double f = (height - 160) / 96.0;
            tk = e.tk160 + f * (e.tk - e.tk160);
            tfix = e.tfix160 + f * (e.tfix - e.tfix160);
        }
        for (int split : kSplits) {
            if (t.large_split > 0) split = (int)(t.large_split < kt ? t.large_split : kt);
            else if (split > 1 && split > kt / 4) break;
            const bool fits = t.large_split > 0 || !limited || static_scratch_holds(split, M, N, K, fp8, partial_ld(N));
            if (!fits && (fp8 || bounded || !padded_split_fits(split, M, N, K, fp8))) break;
            const int per = (kt + split - 1) / split;
            const int slices = (kt + per - 1) / per;
            const double wgs = (double)(tiles * slices), rounds = (double)((tiles * slices + 255) / 256);
            double time = rounds * (tfix + per * tk);
            if (rounds > 1 && e.tn == 128 && e.tm <= 128) time /= e.tm == 64 ? m.pair64 : m.pair128;
            time += m.base + (double)N * (double)K * (fp8 ? 1.0 : 2.0) / m.w_rate + wgs * per * (height + e.tn) * 128.0 / m.l2_rate +
                    rounds * per * (double)(std::min<int64_t>(height, M) + e.tn) * 128.0 / m.cu_rate;
            if (slices > 1) time += split_cost(M, N, slices, m.split, m.split_rate);
            if (!fits) time /= 0.96;
            if (fp8 && e.tm == 64 && M > 128 && (((N + 127) / 128) & 7) != 0 && N * K >= ((int64_t)24 << 20)) time *= 1.1;
            if (time < best) { best = time;  c.tm = e.tm;  c.tn = e.tn;  c.split = split;  c.deep = e.deep;  c.height = height; }
            if (t.large_split > 0) break;
        }
    }
    c.cost = best;
    return c;
}

// More than 256 tokens: tile shape, height of the token tiles and K split by the rounds of
// workgroups over 256 CUs, each a fixed time and a time per K-tile, the operands that all workgroups take in from L2,
// and what a split costs.  What is won over tiles of 256 tokens is the last round: (5888, 5888) at 1645 tokens is 161 tiles of
// 256 or 253 of 160, (6144, 4096) at 2048 tokens 192 or 240 of 224.  The constants were fitted to 112 000 timings of every shape,
// height and split worth one on 150 layers of 1 to 300 Mi weights at 272 to 8192 tokens, both storage orders, and to 40 000 more
// of FP8 mode with padded rows of codes (fit_costs.py time-tall and fit-tall take such timings and fit them).  Long K loops of the
// smaller tiles take more than their share (tk2): E4M3 on 128 x 128 tiles 13 % more at 100 K-tiles; (4064, 12208) at 589 tokens
// 73 us so, 60 in slices.  On the layers of the fit, and some left out of it, the choice was 0.5 to 0.6 % behind the fastest launch on
// average and 3.3 to 4.4 % at the 95th percentile; timed again on 159 layers, half of them drawn at random (114 000 timings of
// 4560 problems), 1.0 % (FP16 mode), 0.8 % (E4M3) and 1.1 % (plain FP16), and 6 to 9 %.  The model before it, which knew no
// heights, is 3.9, 4.3 and 4.5 % behind there, 16 to 19 %, but ahead by more than 3 % on 3 to 6 % of the problems, mostly small
// ones.  Constants fitted to these timings, with a term for rows that start inside lines, won 0.0 to 0.2 % on 855 further layers and slowed
// down as many calls as they sped up: not taken.
// Tiles of 128 tokens that all run at once, unsplit, read the same 128 bytes of K at the same time, and wait for memory
// together; a last token tile of few rows, which has half as much to load, runs ahead of the others and fetches their weights.
// Plain (2560, 2560) takes 28.5 us at 504 tokens, 28.9 at 767, but 21.5 at 649 and 776; in three and two slices, which start at
// other columns, 20.2 and 24.3.  Hence their price (lone, lone256; 2/5 is where the residuals of the prices part).  Timed with
// and without, weights cold, on 5622 problems drawn at 257 to 8192 tokens: behind the fastest launch 0.59 instead of 0.72 %
// (FP16 mode), 0.44 and 0.51 % (E4M3), 0.78 and 1.20 % (plain FP16), at the 95th percentile 4.0 and 4.8, 3.1 and 3.3, 5.4 and
// 8.0 %; slower by more than 3 % than the model without heights on 1.7 instead of 2.6, 0.9 and 1.3, 3.3 and 5.7 % of them.  The
// 140 problems whose launch it changes take 0.94 of the time; 22 of them are slower by 3 to 18 %, 90 faster by 3 to 22 %.
// That model still serves plain FP16 weights at 65 to 256 tokens, with the weights' one pass over the memory bus as a floor.  Launches
// that the floor prices alike are taken in the table's order, the larger tile first: (16142, 8128) at 125 tokens 80.7 us on 256 x 128
// tiles, 96.0 on 128 x 128 ones, and 12 to 25 % on 26 more of 65 to 128 tokens.
struct TallShape { int tm, tn, deep; double tk, tfix, tk160, tfix160, tk2; };       // as ShortShape; tk2: per K-tile squared
struct TallCost {
    int shapes;
    TallShape shape[7];
    double pair;                        // 128 x 128 workgroups of a CU that run together, from the second round on
    double l2_rate, split, split_rate;  // (no l2_rate: operands from L2 are not priced)
    double odd;                         // register path, rows on lines: slices of an odd number of K-tiles (see rows_through_lds)
    double lone, lone256;               // unsplit on 128 x 128 and 128 x 256 tiles, at most one workgroup per CU, the last token tile more than 2/5 full
    double floor_rate, floor_rate512;   // of the memory bus, slower while the chip is not full (from 512 workgroups on)
    bool both_depths;                   // every tile below 256 x 256 is priced in both pipelines, not 128 x 128 alone
};
static const TallCost kTallCost[4] = {
    // plain FP16 of up to 256 tokens
    {7, {{256, 256, 0, 1.353, 0, 1.353, 0, 0}, {256, 128, 0, 1.053, 0.07, 0, 0, 0}, {256, 128, 1, 0.863, 1.56, 0, 0, 0}, {128, 256, 0, 1.098, 0, 0, 0, 0},
         {128, 256, 1, 0.900, 1.71, 0, 0, 0}, {128, 128, 0, 0.848, 0, 0, 0, 0}, {128, 128, 1, 0.585, 2.50, 0, 0, 0}}, 1.58, 0, 3.18, 4.44e6, 1.0, 1.0, 1.0, 4.57e6, 4.44e6, true},
    // FP16 operands through registers
    {4, {{256, 256, 0, 1.11, 8.54, 0.773, 6.36, 0}, {256, 128, 0, 0.573, 6.03, 0.351, 5.53, 0.309e-3}, {128, 256, 0, 0.634, 6.39, 0, 0, 0.103e-3},
         {128, 128, 0, 0.285, 4.28, 0, 0, 0.466e-3}}, 1.0, 28.3e6, 2.98, 6.93e6, 1.05, 1.07, 1.0, 0, 0, false},
    // E4M3
    {5, {{256, 256, 0, 0.951, 9.83, 0.653, 7.57, 0}, {256, 128, 1, 0.445, 7.46, 0, 0, 0.502e-3}, {128, 256, 1, 0.598, 5.27, 0, 0, 0.026e-3},
         {128, 128, 0, 0.515, 4.75, 0, 0, 1.88e-3}, {128, 128, 1, 0.247, 5.41, 0, 0, 1.19e-3}}, 1.83, 50.5e6, 2.14, 5.55e6, 1.0, 1.09, 1.0, 0, 0, false},
    // plain FP16 above
    {5, {{256, 256, 0, 1.04, 7.72, 0.716, 5.68, 0}, {256, 128, 1, 0.466, 7.05, 0, 0, 0.286e-3}, {128, 256, 1, 0.578, 4.71, 0, 0, 0.168e-3},
         {128, 128, 0, 0.432, 4.88, 0, 0, 1.34e-3}, {128, 128, 1, 0.223, 4.69, 0, 0, 1.00e-3}}, 1.70, 34.3e6, 2.61, 6.13e6, 1.0, 1.12, 1.05, 0, 0, false},
};
// A split whose partial sums outgrow the fixed scratch of nestedfp_gemm_static is taken where it is priced 4 % below what fits,
// and by that entry point (bounded) nowhere: FP16 mode is 0.5 % behind the fastest launch so, 0.9 % if nothing beyond
// the scratch is taken.
static LargeConfig choose_tall(int cls, int64_t M, int64_t N, int64_t K, bool bounded) {
    const bool fp8 = cls == 2;
    const TallCost &m = kTallCost[cls == 0 && M > 256 ? 3 : cls];
    const Tuning &t = tuning();
    const int kt = (int)(((fp8 ? K : 2 * K) + 127) / 128);
    const bool limited = cls != 0 && static_scratch_holds(1, M, N, K, fp8, partial_ld(N));
    const int want_m = (t.large_bm == 128 || t.large_bm == 256) ? (int)t.large_bm : 0;
    const int want_n = (t.large_bn == 128 || t.large_bn == 256) ? (int)t.large_bn : want_m;
    LargeConfig c;
    c.tm = 128;  c.tn = 128;  c.split = 1;  c.deep = 0;  c.height = 128;
    double best = 1e30;
    for (int i = 0; i < m.shapes; ++i) {
        const TallShape &e = m.shape[i];
        if (want_m && want_m != e.tm) continue;
        if (want_n && want_n != e.tn) continue;
        int deep = e.deep;
        if (t.large_deep >= 0 && cls != 1 && !(e.tm == 256 && e.tn == 256)) {
            deep = t.large_deep > 0 ? 1 : 0;
            if (((e.tm == 128 && e.tn == 128) || m.both_depths) && deep != e.deep) continue;
        }
        const int pinned = knob_height(cls, e.tm, e.tn);
        const bool cut = e.tm == 256 && cuts_tiles(cls, e.tn);
        const int least = pinned ? pinned : (M <= 256 ? token_tile(cls, e.tm, e.tn, M) : (cut ? 160 : e.tm));
        const int most = pinned || M <= 256 ? least : e.tm;
        for (int height = least; height <= most; height += 32) {
            const double f = cut ? (height - 160) / 96.0 : 1.0;
            const double tk = e.tk160 + f * (e.tk - e.tk160), tfix = e.tfix160 + f * (e.tfix - e.tfix160);
            const int64_t tiles = ((M + height - 1) / height) * ((N + e.tn - 1) / e.tn);
            for (int split : kSplits) {
                if (t.large_split > 0) split = (int)(t.large_split < kt ? t.large_split : kt);
                else if (split > 1 && split > kt / 4) break;
                const bool fits = t.large_split > 0 || !limited || static_scratch_holds(split, M, N, K, fp8, partial_ld(N));
                if ((!fits && bounded) || (t.large_split <= 0 && !padded_split_fits(split, M, N, K, fp8))) break;
                const int per = (kt + split - 1) / split;                     // K-tiles per workgroup
                const int slices = (kt + per - 1) / per;
                const int64_t wgs = tiles * slices, rounds = (wgs + 255) / 256;
                double time = (double)rounds * (tfix + per * tk);
                if (rounds > 1 && e.tm == 128 && e.tn == 128 && !deep) time /= m.pair;
                time += (double)rounds * per * per * e.tk2;
                if (M <= 256 && cls == 0) {
                    double floor_t = (double)N * (double)K * 2.0 / (wgs < 512 ? m.floor_rate : m.floor_rate512);
                    if (wgs < 256) floor_t *= std::sqrt(256.0 / (double)wgs);
                    if (time < floor_t) time = floor_t;
                }
                if (m.l2_rate > 0) time += (double)wgs * per * (height + e.tn) * 128.0 / m.l2_rate;
                if (slices > 1) {
                    time += split_cost(M, N, slices, m.split, m.split_rate);
                    if ((per & 1) && (K & 127) == 0) time *= m.odd;
                } else if (e.tm == 128 && wgs <= 256 && 5 * ((M - 1) % 128 + 1) > 2 * 128) {
                    time *= e.tn == 128 ? m.lone : m.lone256;
                }
                if (!fits) time /= 0.96;
                if (time < best) { best = time;  c.tm = e.tm;  c.tn = e.tn;  c.split = split;  c.deep = deep;  c.height = height; }
                if (t.large_split > 0) break;
            }
        }
    }
    c.cost = best;
    return c;
}

static LargeConfig compute_large(int cls, int64_t M, int64_t N, int64_t K, bool bounded) {
    LargeConfig c;
    c.cost = 0.0;
    const Tuning &t = tuning();
    if (t.tuned_table != 0 && t.large_bm < 0 && t.large_bn < 0 && t.large_split <= 0 && t.large_deep < 0 && t.large_height < 0 &&
        tuned_large(cls, M, N, K, c))
        return c;
    if (t.large_bm == 64 || (M <= 64 && t.large_bm < 0 && t.large_bn < 0)) return choose_tile64(cls, M, N, K);
    const bool pinned = t.large_bm > 0 || t.large_bn > 0 || t.large_split > 0;
    if (M <= 256 && t.large_height < 0 && ((cls == 1 && t.large_deep <= 0) || (cls == 2 && t.large_deep < 0 && !pinned)))
        return choose_short(cls, M, N, K, bounded);
    return choose_tall(cls, M, N, K, bounded);
}

static LargeConfig choose_large(int kind, int64_t M, int64_t N, int64_t K, bool bounded) {
    static thread_local PlanCache<LargeConfig> cache;
    return cache.get(kind_class(kind) + (bounded ? 3 : 0), M, N, K, [&] { return compute_large(kind_class(kind), M, N, K, bounded); });
}

static size_t partial_bytes(const LargeConfig &c, int64_t M, int64_t N) {
    return c.split > 1 ? (size_t)c.split * (size_t)M * (size_t)partial_ld(N) * sizeof(float) : 0;
}
size_t large_gemm_partial_bytes(int kind, int64_t M, int64_t N, int64_t K) { return partial_bytes(choose_large(kind, M, N, K, false), M, N); }
size_t large_gemm_bounded_bytes(int kind, int64_t M, int64_t N, int64_t K) { return partial_bytes(choose_large(kind, M, N, K, true), M, N); }
int large_gemm_height(int kind, int64_t M, int64_t N, int64_t K) { return choose_large(kind, M, N, K, false).height; }

// Row-major planes on the 64-token tiles and in the deeper pipeline of 128 tokens, 128 weight rows per tile: by pairs of K-tiles
// (see BypassKernel::PAIR; up to 45 % faster) where the longer look-ahead pays.  Timed both ways on 2760 launches (26 values
// of K from 512 to 17344, four N, twelve batch sizes, every split; tiles of 256 tokens among them): the rule was 0.4 % behind
// the faster way on average and at most 8 % behind unpaired loads (the rule "12 K-tiles per slice" 1.3 % and 23 %).
//  - Rows that start on lines: a dozen K-tiles per slice (64 tokens per tile 1.07-1.12 x at 12 K-tiles and 1.2 x at
//    24, 128 tokens 1.01 and 1.07); but not where the slices of a split have an odd number of K-tiles: every
//    second slice then starts in the middle of a line, its pieces take two lines each, and K-tile by K-tile
//    is 4-8 % faster.
//  - Rows that start inside lines: 14 K-tiles per slice, 6 Mi weights (smaller planes stay in the caches: K = 2064
//    at 100 tokens 0.97 x with N = 2048, 1.20 x with N = 5632), and longer rows the more token tiles read them
//    ((12288, 1600) at 128 tokens per tile: 1.11 x with one, 0.90 x with three).
bool rows_by_pairs(int tm, int64_t M, int64_t N, int64_t K, int64_t row_bytes, int split) {
    const int64_t kt = (K + 63) / 64, per = (kt + split - 1) / split, tiles_m = (M + tm - 1) / tm;
    const int64_t weights = N * K, mi = (int64_t)1 << 20;
    if ((row_bytes & 127) == 0) return per >= 12 && (per >= kt || (per & 1) == 0);
    if (per < 14) return false;
    if (tiles_m == 1) return weights >= (kt >= 24 ? 6 : 10) * mi;
    return weights >= 6 * mi && kt >= (tiles_m <= 4 ? 32 : 48);
}

// Row-major planes on the other tiles: through LDS by pairs of K-tiles (RowsKernel), or straight into registers in operand
// order, K-tile by K-tile.  Timed both ways by fit_costs.py on 17600 launches at 65 ... 256 tokens (70 layers, every tile shape
// and split, weights cold): the rule is 0.6 % behind the faster way on average, 5 % at the 95th percentile (everything
// straight into registers: 12 and 32 %); on 7200 launches of 300 ... 2048 tokens 0.3 and 2 % (8 %).
//  - Rows that start on lines: through LDS (1.01-1.06 x at less than a dozen K-tiles per slice, 1.15-1.24 x from three
//    dozen on), but on 128 x 128 tiles from a dozen K-tiles on (0.99 x on average below, 0.81 x at worst).
//  - Slices with an odd number of such K-tiles: every second one starts in the middle of a line, so that its pieces take
//    two lines each, and the last pair is half empty: a dozen K-tiles, but never on 256 x 256 tiles, whose two row tiles
//    per wave copy twice as much (1.02-1.07 x the time whatever the length; (5120, 14336) at 1024 tokens in slices of 75
//    K-tiles 170.7 us against 158.7).
//  - Rows that start inside lines, where pieces share lines but unpaired loads take whole halves if the row is a multiple
//    of 64 bytes: longer slices and rows, all the more where several token tiles read them from the caches.
bool rows_through_lds(int tm, int tn, int64_t M, int64_t K, int64_t row_bytes, int split) {
    const int64_t kt = (K + 63) / 64, per = (kt + split - 1) / split, tiles_m = (M + tm - 1) / tm;
    if ((row_bytes & 127) == 0) {
        if (per < kt && (per & 1)) return per >= 12 && !(tm == 256 && tn == 256);
        return per >= 12 || tm > 128 || tn > 128;
    }
    if ((row_bytes & 63) == 0) return per >= 20 && kt >= (tiles_m == 1 ? 24 : 48);
    return per >= 14 && kt >= (tiles_m == 1 ? 20 : 36);
}

// The kernels address a tile with 32-bit byte offsets whose bit 31 marks a dead load, so 256 rows
// of any operand must stay below 2^31 bytes.
bool large_gemm_supports(int kind, int64_t K, int64_t ldx, int64_t ldw) {
    const int64_t x_row = kind_is_fp8(kind) ? ldx : 2 * ldx;
    const int64_t w_row = kind == kPlainF16 ? 2 * ldw : ((K + 63) / 64) * 64 * kind_elem_bytes(kind);
    const int64_t lim = (int64_t)1 << 31;
    return 256 * x_row + 4096 < lim && 256 * w_row + 4096 < lim;
}

int launch_large_gemm(int kind, const GemmArgs &a, hipStream_t stream) {
    if (!large_gemm_supports(kind, a.K, a.ldx, a.ldw)) return kErrShape;
    LargeConfig c = choose_large(kind, a.M, a.N, a.K, a.bounded);
    // the register-path kernels take the deeper pipeline only where it is asked for (knob) or was
    // timed faster (table), and only on the tiles of 128 tokens
    if (kind_class(kind) == 1) c.deep = (tuning().large_deep > 0 || (c.deep && tuning().large_deep != 0)) && c.tm == 128;
    // Workspaces are sized without the row stride of FP16 weights.  A matrix that spans 2 GiB or more comes here
    // with the scratch of the streaming kernel, which cannot address it: as many K slices as that holds.
    const size_t slice_bytes = (size_t)a.M * (size_t)partial_ld(a.N) * sizeof(float);
    const size_t room = a.partials != nullptr ? a.partial_bytes / slice_bytes : 0;
    if ((size_t)c.split > room) c.split = room > 1 ? (int)room : 1;
    FusedLargeParams p;
    p.X = static_cast<const uint8_t *>(a.X);
    p.x_row_bytes = kind_is_fp8(kind) ? a.ldx : 2 * a.ldx;
    p.scales = a.scales;
    p.w_scale = a.w_scale;
    p.W0 = static_cast<const uint8_t *>(a.W0);
    p.W1 = static_cast<const uint8_t *>(a.W1);
    p.w_row_bytes = (kind == kPlainF16) ? 2 * a.ldw : a.K;        // row-major kinds only
    p.M = (int)a.M;  p.N = (int)a.N;  p.K = (int)a.K;
    p.k_bytes = kind_is_fp8(kind) ? (int)a.K : (int)(2 * a.K);
    p.kblocks = (int)((a.K + 63) / 64);
    p.Y = a.Y;  p.ldy = a.ldy;
    p.partials = a.partials;
    p.ldp = (int)partial_ld(a.N);
    p.tiles_m = (int)((a.M + c.height - 1) / c.height);
    p.tiles_n = (int)((a.N + c.tn - 1) / c.tn);
    p.ktiles_total = (p.k_bytes + 127) / 128;
    p.ktiles_per_split = (p.ktiles_total + c.split - 1) / c.split;
    c.split = (p.ktiles_total + p.ktiles_per_split - 1) / p.ktiles_per_split;   // no empty slices
    p.xcd_map = (tuning().large_xcd_map != 0 && p.tiles_m >= 2 && p.tiles_m < 8) ? 1 : 0;
    p.xcd_group = 0;
    if (tuning().large_xcd_map != 0 && p.tiles_m >= 8) {
        const int groups = (p.tiles_m + 5) / 6;
        p.xcd_group = (p.tiles_m + groups - 1) / groups;
    }
    const int64_t outputs = a.epi.kind == kEpiGated ? a.N / 2 : a.N;
    p.rows_anywhere = ((outputs & 7) == 0 && (a.ldy & 7) == 0 && (reinterpret_cast<uintptr_t>(a.Y) & 15) == 0) ? 0 : 1;
    dim3 grid((unsigned)(p.tiles_m * p.tiles_n), (unsigned)c.split);
    p.epi = a.epi;
    if (kind < 0 || kind >= kNumKinds || kind_quantizes(kind)) return kErrArg;
    const bool staged = kind == kPlainF16 || kind_is_fp8(kind);
    if (a.epi.kind == kEpiNone || c.split > 1) (staged ? launch_staged_t<kEpiNone> : launch_nested_t<kEpiNone>)(kind, p, c, grid, stream);
    else if (a.epi.kind == kEpiFull) (staged ? launch_staged_full : launch_nested_full)(kind, p, c, grid, stream);
    else (staged ? launch_staged_gated : launch_nested_gated)(kind, p, c, grid, stream);
    if (hipGetLastError() != hipSuccess) return kErrHip;
    if (c.split > 1)
        return launch_splitk_reduce(a.partials, c.split, a.M, a.N, kind_is_fp8(kind) ? a.scales : nullptr,
                                    a.w_scale, a.Y, a.ldy, a.epi, stream);
    return kOk;
}

}  // namespace nfp
