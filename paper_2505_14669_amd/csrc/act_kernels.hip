// Backward pass of the product's epilogue: dz = dy * multiplier * a'(z), dmul = dy * a(z), and the bias's gradient, the column sums of dz.
// Bound by memory: 2 bytes each of dy, z, the multiplier, dz and dmul per element, one pass.  A block is four waves over 512 columns of neighbouring rows (a
// lane holds eight of them: 16-byte accesses, a kilobyte per wave and row), one row a wave; with the bias's gradient four, whose sums stay in registers.
// What decides is that the blocks in flight cover neighbouring memory: 16384 x 11008, gated (1.8 GB), takes 289 us so (6.2 TB/s), 319 with two rows a wave
// and plain accesses, 381 with a stretch of 176 rows a block, and 363 where 2048 blocks go on by all their rows at a time (they drift apart).
#include "block_common.h"
#include "block_launchers.h"

namespace quartet {

namespace {

// the first `left` of eight bf16 values (8 and more: all); PAST: past the caches
template <bool PAST>
__device__ __forceinline__ uint4 load_bf16x8(const uint16_t* p, int left) {
    if (left >= 8) return PAST ? load_stream16(p) : *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < left) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool PAST>
__device__ __forceinline__ void store_bf16x8(uint16_t* p, int left, const float (&v)[8]) {
    if (left >= 8) {
        if (PAST) store_stream16(p, pack8(v));
        else store_through16(p, pack8(v));
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < left) p[i] = bf16_of(v[i]);
}

template <bool PAST>
__global__ void __launch_bounds__(256)
act_bwd_kernel(ActBwdArgs a, uint32_t col_blocks, FastDiv by_col_blocks, uint32_t rows_per_block) {
    __shared__ float4 join[4][128];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t group = fast_div(blockIdx.x, by_col_blocks), col = ((blockIdx.x - group * col_blocks) * 64u + lane) * 8u;
    const int left = (int)a.n - (int)col;
    const uint64_t row0 = (uint64_t)group * rows_per_block, row1 = row0 + rows_per_block < a.m ? row0 + rows_per_block : a.m;
    float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (left > 0) {
        for (uint64_t row = row0 + wave; row < row1; row += 4u) {
            float dy[8], z[8], mul[8], value[8], slope[8];
            unpack8(load_bf16x8<PAST>(a.dy + row * a.lddy + col, left), dy);
            if (a.pre) unpack8(load_bf16x8<PAST>(a.pre + row * a.ldpre + col, left), z);
            else for (int i = 0; i < 8; ++i) z[i] = 0.0f;
            if (a.mul) unpack8(load_bf16x8<PAST>(a.mul + row * a.ldmul + col, left), mul);
            activate_slope(z, value, slope, a.act);
            float dz[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                value[i] *= dy[i];
                dz[i] = (a.mul ? dy[i] * mul[i] : dy[i]) * slope[i];
                sum[i] += dz[i];
            }
            if (a.dz) store_bf16x8<PAST>(a.dz + row * a.lddz + col, left, dz);
            if (a.dmul) store_bf16x8<PAST>(a.dmul + row * a.lddmul + col, left, value);
        }
    }
    if (!a.partial) return;
    join[wave][lane] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    join[wave][64u + lane] = make_float4(sum[4], sum[5], sum[6], sum[7]);
    __syncthreads();
    // thread t: half t / 64 % 2 of lane t % 64's eight columns
    if (threadIdx.x < 128u) {
        float4 s = join[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            const float4 t = join[w][threadIdx.x];
            s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
        }
        const uint32_t pitch = (a.n + 7u) & ~7u;
        if (col < pitch) *reinterpret_cast<float4*>(a.partial + (size_t)group * pitch + col + (threadIdx.x >> 6) * 4u) = s;
    }
}

struct ActPlan {
    uint32_t col_blocks, groups, rows_per_block;
};
// One row a wave; with the bias's gradient four: every block leaves a row of partial sums (us, 16 / 32 / 64 / 128 rows a block: 1003 x 5632 10.7 / 11.8 / 17.1 /
// 29.5, 4096 x 5632 31.8 / 32.8 / 33.8 / 45.9, 16384 x 11008 185 / 186 / 200 / 219, 16384 x 4096 77 / 80 / 85 / 74).
ActPlan act_plan(int64_t m, int64_t n, bool sums) {
    const int64_t cb = (n + 511) / 512;
    int64_t rows = sums ? 16 : 4;
    while ((m + rows - 1) / rows * cb > ((int64_t)1 << 23) && rows < m) rows *= 2;      // a launch has fewer than 2^32 threads
    return {(uint32_t)cb, (uint32_t)((m + rows - 1) / rows), (uint32_t)rows};
}

// What the memory-side cache (256 MB) cannot hold goes past it: 16384 x 11008 without a gate 207 -> 186 us, gated 312 -> 289; below, plain loads and stores
// through the L2 are 10-15 % sooner.
bool past_cache(const ActBwdArgs& a) {
    const int matrices = 1 + (a.pre != nullptr) + (a.mul != nullptr) + (a.dz != nullptr) + (a.dmul != nullptr);
    return (double)a.m * (double)a.n * 2.0 * matrices >= 256.0 * 1024.0 * 1024.0;
}

}  // namespace

size_t act_bwd_workspace(int64_t m, int64_t n) {
    if (m <= 0 || n <= 0) return 0;
    return (size_t)act_plan(m, n, true).groups * (size_t)((n + 7) / 8 * 8) * sizeof(float);
}

hipError_t launch_act_bwd(const ActBwdArgs& args, float* dbias, float* workspace, hipStream_t st) {
    if (args.n == 0) return hipSuccess;
    if (args.m == 0) return dbias ? launch_column_sum(nullptr, 0u, 0u, args.n, dbias, st) : hipSuccess;
    ActBwdArgs a = args;
    a.partial = dbias ? workspace : nullptr;
    const ActPlan p = act_plan(a.m, a.n, dbias != nullptr);
    const dim3 grid(p.col_blocks * p.groups), block(256);
    const FastDiv by = make_fast_div(p.col_blocks);
    if (past_cache(a)) hipLaunchKernelGGL((act_bwd_kernel<true>), grid, block, 0, st, a, p.col_blocks, by, p.rows_per_block);
    else hipLaunchKernelGGL((act_bwd_kernel<false>), grid, block, 0, st, a, p.col_blocks, by, p.rows_per_block);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !dbias) return e;
    return launch_column_sum(workspace, p.groups, (a.n + 7u) & ~7u, a.n, dbias, st);
}

}  // namespace quartet
