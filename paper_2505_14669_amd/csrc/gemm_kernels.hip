// MXFP4 x MXFP4 -> fp32 GEMM on the gfx950 block-scaled matrix cores (Section 4.4, "Stage 2":
// D = (A x SFA)(B x SFB)^T with one E8M0 scale per 32 elements along K).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 operand layout (FP4, cbsz = blgp = 4), measured on gfx950:
//   A: lane l holds row l%16, K-elements 32*(l/16) .. +31 as 128 bits, element j in bits [4j,4j+4)
//      -- exactly the packed row-major code bytes, so a fragment is one 16-byte LDS read;
//   B: the same with the output column in place of the row;
//   scale: one byte per lane (selected by op_sel from a 32-bit register) = the E8M0 scale of that
//      lane's 32 K-elements, i.e. one MX group per lane per instruction;
//   D: lane l, register r -> row 4*(l/16) + r, column l%16.
// The 256 x 256 kernel uses it, the smaller tiles v_mfma_scale_f32_32x32x64_f8f6f4 (lane l: row or column l%32, K-elements 32*(l/32) ..
// +31; D: row 8*(r/4) + 4*(l/32) + r%4, column l%32).  Why 16 x 16 x 128 on the large tiles (same rate, same operand bytes per wave
// tile): there the chip is power-limited, and the deeper instruction reads and writes each fp32 accumulator once per 128 K-elements instead of once per 64.
// Registers only, quantized normal data, 128 x 128 wave tiles: 7.09 PFLOP/s at 1.79 GHz against 6.38 at 1.59 GHz; both give the same bits (compared over 25 binades of scales).
// The tiled scale layout (see scale_tile_offset) stores, for each block of 32 rows and 256
// K-elements, dword 32 h + row with the scales of groups h, 2 + h, 4 + h, 6 + h.  16 x 16 x 128: lane l reads the dword of its row and h =
// (l/16) % 2 once per K-quad (128 contiguous bytes twice per wave), and its group of the quad's first and second K-step is byte
// l/32 and byte 2 + l/32.  32 x 32 x 64: lane l reads dword l of the tile, byte s for K-step s.  The paper's separate scale-rearrangement step does not exist here.
//
// Kernels: gemm_mxfp4_stream_kernel (256 x 256 tiles) and gemm_mxfp4_stream_tile_kernel (128 x 256 and 128 x 128 tiles
// for small problems): one block per compute unit streams its tiles through a ring of K-quads (256 elements) in LDS, of 128 x 128 tiles
// also two (gemm_mxfp4_twin_kernel).  The wide kernels are for Hadamard blocks of 256, the past kernels for bf16 results of 256 MB and more.  All work through a batch of one or two products per launch (GemmBatch).
// What bounds them besides power is the way of the operands into the LDS: a cache line is 128 bytes, so a ring of 128-element
// stages (64 bytes of codes per row) fetched every line twice.  K-quads, whole lines, one barrier per quad and reads and loads spread
// evenly over the matrix-core instructions, 16 x 16 x 128 on the large tiles and 32 x 32 x 64 on the small ones, took against that design
// (layer steps, us): 16384 x 4096 x 11008 1434 -> 1378, 16384 x 4096 x 4096 620 -> 601, 2336 x 1376 x 3168 78.7 -> 71.5, 4096 x 2048 x 2048
// 91.2 -> 85.1, forward 1003 x 2048 x 5632 25.6 -> 23.9.  (16 x 16 x 128 on the old stages: 0-4 % slower.)
#include "block_launchers.h"
#include "gemm_common.h"
#include "gemm_stream.h"
#include "launchers.h"
#include "pair_level.h"

namespace quartet {

// Test / tuning override of the kernel choice (quartet_debug_set_gemm_plan): -1 / 0 = the size heuristics below.
static int g_forced_variant = -1;
static int g_forced_band = 0;

// quartet_profile_clock: device counters the streaming kernel adds each block's run time to (null: off)
static uint64_t* g_clock_counters = nullptr;

void set_clock_counters(uint64_t* device_counters) { g_clock_counters = device_counters; }

constexpr int kTwoPerCu = 3;          // variant: 128 x 128 tiles, two blocks per compute unit
constexpr int kTwoPerCuCode = 22;     // its number outside

void set_gemm_plan(int variant, int band_height) {
    g_forced_variant = variant == kTwoPerCuCode ? kTwoPerCu : variant;
    g_forced_band = band_height;
}

template <bool OUT_BF16, bool FUSED>
__global__ void __launch_bounds__(256)
gemm_mxfp4_stream_kernel(GemmBatch batch, uint32_t nb, uint64_t* __restrict__ clock_counters) {
    stream_large_tiles<OUT_BF16, FUSED, false>(batch, nb, clock_counters);
}

template <bool FUSED>
__global__ void __launch_bounds__(256)
gemm_mxfp4_past_kernel(GemmBatch batch, uint32_t nb, uint64_t* __restrict__ clock_counters) {
    stream_large_tiles<true, FUSED, false, true>(batch, nb, clock_counters);
}

__global__ void __launch_bounds__(256)
gemm_mxfp4_past_wide_kernel(GemmBatch batch, uint64_t* __restrict__ clock_counters) {
    stream_large_tiles<true, true, true, true>(batch, 8u, clock_counters);
}

template <bool OUT_BF16>
__global__ void __launch_bounds__(256)
gemm_mxfp4_wide_kernel(GemmBatch batch, uint64_t* __restrict__ clock_counters) {
    stream_large_tiles<OUT_BF16, true, true>(batch, 8u, clock_counters);
}

template <int TM, int TN, bool OUT_BF16, bool FUSED>
__global__ void __launch_bounds__(256)
gemm_mxfp4_stream_tile_kernel(GemmBatch batch, uint32_t nb, uint64_t* __restrict__ clock_counters) {
    stream_tiles<TM, TN, 1, OUT_BF16, FUSED>(batch, nb, clock_counters);
}

template <bool OUT_BF16>
__global__ void __launch_bounds__(256)
gemm_mxfp4_wide_tile_kernel(GemmBatch batch, uint64_t* __restrict__ clock_counters) {
    stream_tiles<2, 4, 1, OUT_BF16, true, true>(batch, 8u, clock_counters);
}

template <bool OUT_BF16, bool FUSED>
__global__ void __launch_bounds__(256, 2)
gemm_mxfp4_twin_kernel(GemmBatch batch, uint32_t nb, uint64_t* __restrict__ clock_counters) {
    stream_tiles<2, 2, 2, OUT_BF16, FUSED>(batch, nb, clock_counters);
}

template <bool FUSED>
__global__ void __launch_bounds__(256, 2)
gemm_mxfp4_past_twin_kernel(GemmBatch batch, uint32_t nb, uint64_t* __restrict__ clock_counters) {
    stream_tiles<2, 2, 2, true, FUSED, false, true>(batch, nb, clock_counters);
}

static int stream_blocks() {
    static int cus = 0;
    if (cus == 0) {
        int dev = 0, n = 0;
        if (hipGetDevice(&dev) == hipSuccess && hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n >= 8)
            cus = n & ~7;
        else
            cus = 8;
    }
    return cus;
}

// Results of a launch that the memory-side cache (256 MB) cannot hold beside its operands are stored past it: they would only push those and
// what follows out.  Less is stored through the L2 and stays there for its reader.  Through the L2 / past the cache (us), layer steps
// (tokens, in, out): fp32 16384 x 2048 x 4096 (y 256 MB) 357 / 344, 16384 x 4096 x 4096 572 / 534, 8192 x 7936 x 1024 (gradients 279 MB) 229 / 219; bf16
// 16384 x 2048 x 8192 (y 256 MB) 605 / 592, 16384 x 8192 x 1024 (gradients 272 MB) 447 / 430, 12544 x 10752 x 2048 659 / 637.  A forward pass of 256 MB that is
// repeated alone is 1-10 % slower past the cache (fp32 8192 x 2048 x 8192 107 / 117), from 264 MB on 0-6 % faster.  For bf16 on the kernels that such
// launches take; 128 x 256 tiles, which take 1 in 1000 of them, and forced 128 x 128 ones with one block per compute unit stay with the L2.
static uint32_t stored_past(const GemmBatch& batch, bool bf16) {
    const double results = (double)batch.p[0].m * batch.p[0].n + (double)batch.p[1].m * batch.p[1].n;
    return results * (bf16 ? 2.0 : 4.0) >= 256.0 * 1024.0 * 1024.0 ? 1u : 0u;
}

// tile grid and band height of one product for block tiles of bm x bn
static GemmProblem make_problem(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales,
                                int64_t m, int64_t n, int64_t k, float alpha, void* d, int64_t ldd, const uint32_t* mask,
                                int64_t bm, int64_t bn) {
    GemmProblem q;
    q.a_codes = a_codes; q.a_scales = a_scales; q.b_codes = b_codes; q.b_scales = b_scales;
    q.d = d; q.mask = mask;
    q.m = (uint32_t)m; q.n = (uint32_t)n; q.k = (uint32_t)k; q.ldd = (uint32_t)ldd;
    q.alpha = alpha;
    q.tiles_m = (uint32_t)((m + bm - 1) / bm); q.tiles_n = (uint32_t)((n + bn - 1) / bn);
    q.band_height = (bm == 256 && bn == 256 && q.tiles_n >= 40u && (q.tiles_m & 1u) == 0u) ? 2u : 4u;
    if (g_forced_band > 0) q.band_height = (uint32_t)g_forced_band;
    q.total_tiles = q.tiles_m * q.tiles_n;
    return q;
}

template <bool OUT_BF16, bool FUSED>
static void launch_stream_batch_t(const GemmBatch& batch, uint32_t nb, hipStream_t st) {
    const uint32_t total = batch.p[0].total_tiles + batch.p[1].total_tiles, cus = (uint32_t)stream_blocks();
    const dim3 grid(total < cus ? total : cus);
    if (OUT_BF16 && batch.past) hipLaunchKernelGGL((gemm_mxfp4_past_kernel<FUSED>), grid, dim3(256), 0, st, batch, nb, g_clock_counters);
    else hipLaunchKernelGGL((gemm_mxfp4_stream_kernel<OUT_BF16, FUSED>), grid, dim3(256), 0, st, batch, nb, g_clock_counters);
}

template <bool OUT_BF16, bool FUSED>
static void launch_stream_t(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes,
                            const uint8_t* b_scales, int64_t m, int64_t n, int64_t k, float alpha, void* d,
                            int64_t ldd, const uint32_t* mask, uint32_t nb, hipStream_t st) {
    GemmBatch batch;
    batch.p[0] = make_problem(a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, d, ldd, mask, 256, 256);
    batch.p[1] = GemmProblem{};      // no second product
    batch.past = stored_past(batch, OUT_BF16);
    batch.extra_tiles = batch.late = 0u;
    launch_stream_batch_t<OUT_BF16, FUSED>(batch, nb, st);
}

template <int TM, int TN, int PER_CU, bool OUT_BF16, bool FUSED>
static void launch_stream_tile_batch_t(const GemmBatch& batch, uint32_t nb, hipStream_t st) {
    const uint32_t total = batch.p[0].total_tiles + batch.p[1].total_tiles, room = PER_CU * (uint32_t)stream_blocks();
    const dim3 grid(total < room ? total : room);
    if (PER_CU == 2 && OUT_BF16 && batch.past) hipLaunchKernelGGL((gemm_mxfp4_past_twin_kernel<FUSED>), grid, dim3(256), 0, st, batch, nb, g_clock_counters);
    else if constexpr (PER_CU == 2) hipLaunchKernelGGL((gemm_mxfp4_twin_kernel<OUT_BF16, FUSED>), grid, dim3(256), 0, st, batch, nb, g_clock_counters);
    else hipLaunchKernelGGL((gemm_mxfp4_stream_tile_kernel<TM, TN, OUT_BF16, FUSED>), grid, dim3(256), 0, st, batch, nb, g_clock_counters);
}

template <int TM, int TN, int PER_CU, bool OUT_BF16, bool FUSED>
static void launch_stream_tile_t(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes,
                                 const uint8_t* b_scales, int64_t m, int64_t n, int64_t k, float alpha, void* d,
                                 int64_t ldd, const uint32_t* mask, uint32_t nb, hipStream_t st) {
    GemmBatch batch;
    batch.p[0] = make_problem(a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, d, ldd, mask, 64 * TM, 64 * TN);
    batch.p[1] = GemmProblem{};      // no second product
    batch.past = stored_past(batch, OUT_BF16);
    batch.extra_tiles = batch.late = 0u;
    launch_stream_tile_batch_t<TM, TN, PER_CU, OUT_BF16, FUSED>(batch, nb, st);
}

// Variants: 0 = 256x256 tiles (hand-scheduled K-quad), 1 = 128x256 tiles, 2 = 128x128 tiles (schedule generated from the
// tile shape), kTwoPerCu = 128x128 tiles with two blocks per compute unit; blocks stream their tiles through a ring of K-quads, two
// K-steps per trip with the scale byte picked by op_sel.  set_gemm_plan overrides the size heuristic (tests reach every variant
// through it).
// fused != 0: D = alpha * H_along_n((A B^T) . mask) with Hadamard blocks of nb = 1, 2 or 4 groups of 32 columns (mask may
// be null = all ones), n % (32 nb) == 0.
//
// The tile shape is the one with the smallest estimated time: launch and first loads, the share of the chip that starts, the
// busiest compute unit's K-quads and its tiles' epilogues (weighed with the mean: the last round runs on a chip that is partly idle), or
// what the memory takes for the results if that is more.  Fitted to the products of 330 layers' backward passes (tokens 256 .. 16384, in and
// out 256 .. 11008) and of 400 forward or serving calls (m 8 .. 16384), both result types, every shape timed behind the conversions that
// write its operands: the shape chosen costs 1.0 % (pairs) and 1.1 % (singles) more than the best one on average, 7 / 5 % at the 95th
// percentile.  Measured, 256 x 256 / 128 x 256 / 128 x 128 / 128 x 128 with two blocks per compute unit (us): pairs (dW, dx) of layers (tokens,
// in, out) 4608 x 2432 x 6016 107 / 104 / 105 / 95, 13696 x 2816 x 832 101 / 69 / 77 / 80; single products 4253 x 3648 x 5408 59.7 / 62.3 / 72.8 /
// 69.2, 2860 x 4448 x 320 18.2 / 17.2 / 16.2 / 13.2.
struct StreamCost {
    double start, per_quad, per_tile, per_fill, per_result, busiest;     // us; per_result: of 10^6 results; busiest: weight against the mean
};
static const StreamCost kStreamSingle[4] = {{1.42, 1.590, 5.39, 11.7, 0.803, 1.00}, {3.04, 0.904, 3.60, 4.40, 0.752, 1.00},
                                            {3.20, 0.609, 1.94, 1.95, 0.718, 1.00}, {1.54, 0.677, 1.03, 2.33, 0.591, 0.80}};
static const StreamCost kStreamPair[4] = {{0.00, 1.520, 10.1, 19.8, 1.505, 1.00}, {3.06, 0.897, 6.46, 2.03, 1.351, 1.00},
                                          {4.26, 0.582, 4.19, 0.00, 0.128, 0.62}, {0.00, 0.638, 0.84, 5.04, 1.247, 1.00}};
constexpr int64_t kTileM[4] = {256, 128, 128, 128}, kTileN[4] = {256, 256, 128, 128};

// *extra: the late blocks' rounds.  Two blocks b and b + half of a compute unit take turns at its matrix cores: their loads add up.
static double stream_estimate(int variant, int products, const int64_t* m, const int64_t* n, const int64_t* k, int64_t cus, int64_t* extra) {
    const StreamCost& c = (products == 1 ? kStreamSingle : kStreamPair)[variant];
    int64_t tiles[2] = {0, 0};
    double cost[2] = {0.0, 1.0}, results = 0.0, sum = 0.0;
    for (int p = 0; p < products; ++p) {
        tiles[p] = ((m[p] + kTileM[variant] - 1) / kTileM[variant]) * ((n[p] + kTileN[variant] - 1) / kTileN[variant]);
        cost[p] = c.per_quad * (double)(k[p] > 256 ? (k[p] + 255) / 256 : 1) + c.per_tile;
        sum += (double)tiles[p] * cost[p];
        results += (double)m[p] * (double)n[p];
    }
    const int64_t total = tiles[0] + tiles[1], used = total < cus ? total : cus;
    const int64_t room = variant == kTwoPerCu ? 2 * cus : cus, blocks = total < room ? total : room, half = blocks / 2;
    PairLevel l = pair_level(tiles, cost, blocks);
    *extra = l.extra;
    // Where the second product cannot fill the rounds that would level the loads, the estimate does not count on extra ones: the constants, fitted
    // so, are low for launches that few long tiles dominate.  140 such layers, every shape timed: the one chosen costs 0.6 % more than the best
    // one on average, with the extra rounds counted 1.0 % (10848 x 288 x 544: 45.1 us in place of 35.8).
    if ((int64_t)(cost[0] / cost[1]) - 1 > pair_most_extra(tiles, blocks)) l = pair_loads(tiles, cost, blocks, 0);
    double busiest = l.busiest();
    if (variant == kTwoPerCu) {
        // a tile per compute unit: the deeper ring of one block; products narrower than a tile: not measured
        if (total <= cus || n[0] < 128 || (products == 2 && n[1] < 128)) return 1e30;
        const double mixed = l.early_load + l.late_load;
        busiest = l.early == 0 ? 2.0 * l.late_load : l.early > half ? 2.0 * l.early_load : 0.0;
        if (l.early > 0 && mixed > busiest) busiest = mixed;
        if (l.early > 0 && l.early < half && 2.0 * l.late_load > busiest) busiest = 2.0 * l.late_load;
    }
    const double mean = sum / (double)used, weight = busiest > 4.0 * mean ? 1.0 : c.busiest;     // (a few long tiles alone: theirs is the time)
    const double work = weight * busiest + (1.0 - weight) * mean + c.per_fill * (double)used / (double)cus;
    const double memory = c.per_result * 1e-6 * results;
    return c.start + (work > memory ? work : memory);
}

// the variant for one product or a pair, and its estimated time
static int pick_variant(int products, const int64_t* m, const int64_t* n, const int64_t* k, int cus, double* estimate) {
    int variant = -1;
    for (int v = 0; v < 4; ++v) {
        if (g_forced_variant >= 0 && g_forced_variant != v) continue;
        int64_t extra;
        const double t = stream_estimate(v, products, m, n, k, cus, &extra);
        if (variant < 0 || t < *estimate) { *estimate = t; variant = v; }
    }
    return variant;
}

// Problems that the split kernels (gemm_split_kernels.hip) finish sooner: few rows, small layers, long inner dimensions with few
// tiles.  Compares their estimate with that of the streaming kernels, in favour of the latter by 12 % (one product, two waves) or
// 35 % (two products; four waves, whose estimate is low for 64 x 64 tiles), which cost least over the calls the estimates were fitted to.  Measured, streaming against split (us): 630 x 1312 x 2944 11.7 / 7.0;
// 2910 x 384 x 1056 7.6 / 7.2; 469 x 1792 x 1728 8.3 / 6.5; on the other side 2538 x 864 x 384 8.1 / 10.2; four waves 339 x 2624 x 5600 15.5 / 9.2 and
// 377 x 4096 x 3936 12.8 / 13.9, 950 x 1696 x 5664 16.5 / 18.1; pairs of layers 736 x 928 x 800 10.5 / 8.2, 2176 x 1024 x 864 11.8 / 14.7.  For
// one product the choice depends on m, n and k alone, so fused and plain products of one size run on the same side.
static bool use_split(int products, const int64_t* m, const int64_t* n, const int64_t* k, int cus, double streaming, int* shape) {
    if (g_forced_variant >= 0) return false;
    // A block per tile, and a launch has fewer than 2^32 threads: with 32 x 32 tiles of up to four waves, 2^24 tiles at most
    int64_t tiles = 0;
    for (int p = 0; p < products; ++p) tiles += ((m[p] + 31) / 32) * ((n[p] + 31) / 32);
    if (tiles >= ((int64_t)1 << 24)) return false;
    const bool four = split_waves(products == 2 && k[1] > k[0] ? k[1] : k[0]) == 4;
    return best_split_shape(products, m, n, k, cus, shape) < (four || products == 2 ? 0.65 : 0.88) * streaming;
}

// The kernel for one product or a pair, plain (nb = 0) or with the gradient epilogue of Hadamard blocks of nb groups.
struct GemmPlan {
    bool split;
    int shape;          // split: tile shape (see launch_gemm_split); otherwise the streaming variant
};
static GemmPlan plan_gemm(int products, const int64_t* m, const int64_t* n, const int64_t* k, uint32_t nb, int cus) {
    double estimate = 0.0;
    int shape = 0, variant = pick_variant(products, m, n, k, cus, &estimate);
    if (nb >= 4u && variant >= 2) {
        // A block of 128 columns needs the 128-column wave tile.  (256 x 256 where the estimates put it before 128 x 256 is not sooner: 40 layers
        // each with blocks of 128 and 256, 1.00 and 0.98 of its speed on average.)
        variant = 1;
        // In a pair the split kernels are weighed against the tiles that run; against those that cannot, backward passes of layers with blocks
        // of 128 took (tokens, in, out; us) 384 x 3456 x 256 21.6 for 13.9, 6016 x 384 x 640 40.2 for 26.5, 1280 x 640 x 2560 30.0 for 22.8.  One
        // product stays on the side where the plain product of its sizes runs: their results are the same bits.
        int64_t extra;
        if (products == 2) estimate = stream_estimate(1, 2, m, n, k, cus, &extra);
    }
    if (nb != 8u && use_split(products, m, n, k, cus, estimate, &shape)) return {true, split_shape_for(shape, nb)};
    return {false, variant};
}

int gemm_plan_code(int products, const int64_t* m, const int64_t* n, const int64_t* k, uint32_t nb, int cus) {
    const GemmPlan plan = plan_gemm(products, m, n, k, nb, cus);
    const int64_t k_max = products == 2 && k[1] > k[0] ? k[1] : k[0];
    return plan.split ? 100 * split_waves(k_max) + plan.shape : plan.shape == kTwoPerCu ? kTwoPerCuCode : plan.shape;
}

hipError_t launch_gemm(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes,
                       const uint8_t* b_scales, int64_t m, int64_t n, int64_t k, float alpha, void* d,
                       int d_bf16, int64_t ldd, int fused, const uint32_t* mask, uint32_t nb, hipStream_t st) {
    if (m == 0 || n == 0) return hipSuccess;
    const GemmPlan plan = plan_gemm(1, &m, &n, &k, fused ? nb : 0u, stream_blocks());
    if (plan.split) {
        const GemmArgs g = {a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, d, ldd, mask};
        return launch_gemm_split(g, nullptr, d_bf16, fused, nb, plan.shape, st);
    }
    const int variant = plan.shape;
#define QUARTET_DISPATCH(FN, ...)                                                                     \
    do {                                                                                              \
        if (d_bf16) { if (fused) FN<__VA_ARGS__ true, true>(a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, d, ldd, mask, nb, st); \
                      else FN<__VA_ARGS__ true, false>(a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, d, ldd, mask, nb, st); }   \
        else { if (fused) FN<__VA_ARGS__ false, true>(a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, d, ldd, mask, nb, st);      \
               else FN<__VA_ARGS__ false, false>(a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, d, ldd, mask, nb, st); }         \
    } while (0)
    if (variant == 1) QUARTET_DISPATCH(launch_stream_tile_t, 2, 4, 1, );
    else if (variant == 2) QUARTET_DISPATCH(launch_stream_tile_t, 2, 2, 1, );
    else if (variant == kTwoPerCu) QUARTET_DISPATCH(launch_stream_tile_t, 2, 2, 2, );
    else QUARTET_DISPATCH(launch_stream_t, );
#undef QUARTET_DISPATCH
    return hipGetLastError();
}

// Hadamard blocks of 256 columns: the kernels that apply their epilogue take whole tiles of 256 x 256 (hence of 128 x 256) only, which is
// what every layer with such blocks has, and results and masks aligned as the C entry requires them (a guard: nothing else comes here).  Against two products on the kernels that are soonest for them, fp32 results in the
// workspace and two epilogue kernels, layer steps (tokens, in, out; us): 256 x 1024 x 512 32.5 -> 24.5, 1024 x 768 x 1280 48 -> 34, 4096 x 4096 x
// 2048 145 -> 112, 8192 x 2048 x 5632 288 -> 268, 1024 x 10752 x 7936 496 -> 330, 14336 x 1792 x 7680 541 -> 499.
static bool wide_fits(const GemmArgs& g, int d_bf16) {
    return g.m % 256 == 0 && g.n % 256 == 0 && g.ldd % 4 == 0 && g.mask != nullptr && (reinterpret_cast<uintptr_t>(g.d) & (d_bf16 ? 7u : 15u)) == 0;
}
static void launch_wide(const GemmBatch& batch, bool large, int d_bf16, hipStream_t st) {
    const uint32_t total = batch.p[0].total_tiles + batch.p[1].total_tiles, cus = (uint32_t)stream_blocks();
    const dim3 grid(total < cus ? total : cus), block(256);
    if (large && d_bf16 && batch.past) hipLaunchKernelGGL(gemm_mxfp4_past_wide_kernel, grid, block, 0, st, batch, g_clock_counters);
    else if (large && d_bf16) hipLaunchKernelGGL((gemm_mxfp4_wide_kernel<true>), grid, block, 0, st, batch, g_clock_counters);
    else if (large) hipLaunchKernelGGL((gemm_mxfp4_wide_kernel<false>), grid, block, 0, st, batch, g_clock_counters);
    else if (d_bf16) hipLaunchKernelGGL((gemm_mxfp4_wide_tile_kernel<true>), grid, block, 0, st, batch, g_clock_counters);
    else hipLaunchKernelGGL((gemm_mxfp4_wide_tile_kernel<false>), grid, block, 0, st, batch, g_clock_counters);
}

// Two gradient products in one launch (both with the fused epilogue, results of one type).  One tile shape serves both.  Hadamard
// blocks of 256 columns (nb = 8): hipErrorNotSupported, and nothing is launched, for what those kernels do not take; the caller sees to it that
// there is no empty product.
hipError_t launch_gemm_grad_pair(const GemmArgs& g0, const GemmArgs& g1, int d_bf16, uint32_t nb, hipStream_t st) {
    const bool empty0 = g0.m == 0 || g0.n == 0, empty1 = g1.m == 0 || g1.n == 0;
    if (nb == 8u && (empty0 || empty1)) return hipErrorNotSupported;
    if (empty0 || empty1) {
        hipError_t e = launch_gemm(g0.a_codes, g0.a_scales, g0.b_codes, g0.b_scales, g0.m, g0.n, g0.k, g0.alpha, g0.d, d_bf16, g0.ldd,
                                   1, g0.mask, nb, st);
        if (e != hipSuccess) return e;
        return launch_gemm(g1.a_codes, g1.a_scales, g1.b_codes, g1.b_scales, g1.m, g1.n, g1.k, g1.alpha, g1.d, d_bf16, g1.ldd, 1,
                           g1.mask, nb, st);
    }
    const int64_t ms[2] = {g0.m, g1.m}, ns[2] = {g0.n, g1.n}, ks[2] = {g0.k, g1.k};
    const GemmPlan plan = plan_gemm(2, ms, ns, ks, nb, stream_blocks());
    if (nb == 8u && !(wide_fits(g0, d_bf16) && wide_fits(g1, d_bf16))) return hipErrorNotSupported;
    if (plan.split) return launch_gemm_split(g0, &g1, d_bf16, 1, nb, plan.shape, st);
    const int variant = plan.shape;
    GemmBatch batch;
    batch.p[0] = make_problem(g0.a_codes, g0.a_scales, g0.b_codes, g0.b_scales, g0.m, g0.n, g0.k, g0.alpha, g0.d, g0.ldd, g0.mask,
                              kTileM[variant], kTileN[variant]);
    batch.p[1] = make_problem(g1.a_codes, g1.a_scales, g1.b_codes, g1.b_scales, g1.m, g1.n, g1.k, g1.alpha, g1.d, g1.ldd, g1.mask,
                              kTileM[variant], kTileN[variant]);
    const int64_t cus = stream_blocks();
    const uint32_t total = batch.p[0].total_tiles + batch.p[1].total_tiles, room = (uint32_t)(variant == kTwoPerCu ? 2 * cus : cus), blocks = total < room ? total : room;
    int64_t extra;
    stream_estimate(variant, 2, ms, ns, ks, cus, &extra);
    batch.past = stored_past(batch, d_bf16 != 0);
    batch.late = blocks - batch.p[0].total_tiles % blocks;
    batch.extra_tiles = (uint32_t)extra * batch.late;
#define QUARTET_PAIR(FN, ...)                                                                           \
    do { if (d_bf16) FN<__VA_ARGS__ true, true>(batch, nb, st); else FN<__VA_ARGS__ false, true>(batch, nb, st); } while (0)
    if (nb == 8u) launch_wide(batch, variant == 0, d_bf16, st);
    else if (variant == 1) QUARTET_PAIR(launch_stream_tile_batch_t, 2, 4, 1, );
    else if (variant == 2) QUARTET_PAIR(launch_stream_tile_batch_t, 2, 2, 1, );
    else if (variant == kTwoPerCu) QUARTET_PAIR(launch_stream_tile_batch_t, 2, 2, 2, );
    else QUARTET_PAIR(launch_stream_batch_t, );
#undef QUARTET_PAIR
    return hipGetLastError();
}

// The kernel that the plain product of these sizes runs on, with the epilogue of quartet_mxfp4_gemm_act.
hipError_t launch_gemm_act(const GemmArgs& g, const GemmActArgs& act, int d_bf16, hipStream_t st) {
    if (g.m == 0 || g.n == 0) return hipSuccess;
    const GemmPlan plan = plan_gemm(1, &g.m, &g.n, &g.k, 0u, stream_blocks());
    if (plan.split) return launch_gemm_act_split(g, act, d_bf16, plan.shape, st);
    GemmBatch batch;
    batch.p[0] = make_problem(g.a_codes, g.a_scales, g.b_codes, g.b_scales, g.m, g.n, g.k, g.alpha, g.d, g.ldd, nullptr, kTileM[plan.shape], kTileN[plan.shape]);
    batch.p[1] = GemmProblem{};      // no second product
    batch.past = batch.extra_tiles = batch.late = 0u;
    const uint32_t room = (plan.shape == kTwoPerCu ? 2u : 1u) * (uint32_t)stream_blocks(), total = batch.p[0].total_tiles;
    const uint32_t blocks = total < room ? total : room;
    return d_bf16 ? launch_gemm_act_stream<true>(batch, act, plan.shape, blocks, st) : launch_gemm_act_stream<false>(batch, act, plan.shape, blocks, st);
}

}  // namespace quartet
