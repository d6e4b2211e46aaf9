// The streaming MXFP4 products with bias, activation, gate and residual in their epilogue (quartet_mxfp4_gemm_act); the bodies are gemm_stream.h's.
// Two files instantiate them, one for each result type: they take longest to compile.
#pragma once
#include "block_launchers.h"
#include "gemm_stream.h"

namespace quartet {

template <bool OUT_BF16, int EXTRA>
__global__ void __launch_bounds__(256)
mxfp4_act_large_kernel(GemmBatch batch, GemmActArgs act) {
    stream_large_tiles<OUT_BF16, false, false, false, EXTRA, GemmActArgs>(batch, 1u, nullptr, act);
}

template <int TM, int TN, bool OUT_BF16, int EXTRA>
__global__ void __launch_bounds__(256)
mxfp4_act_tile_kernel(GemmBatch batch, GemmActArgs act) {
    stream_tiles<TM, TN, 1, OUT_BF16, false, false, false, EXTRA, GemmActArgs>(batch, 1u, nullptr, act);
}

template <bool OUT_BF16, int EXTRA>
__global__ void __launch_bounds__(256, 2)
mxfp4_act_twin_kernel(GemmBatch batch, GemmActArgs act) {
    stream_tiles<2, 2, 2, OUT_BF16, false, false, false, EXTRA, GemmActArgs>(batch, 1u, nullptr, act);
}

template <bool OUT_BF16, int EXTRA>
static void launch_act_variant(const GemmBatch& batch, const GemmActArgs& act, int variant, dim3 grid, hipStream_t st) {
    const dim3 block(256);
    if (variant == 0) hipLaunchKernelGGL((mxfp4_act_large_kernel<OUT_BF16, EXTRA>), grid, block, 0, st, batch, act);
    else if (variant == 1) hipLaunchKernelGGL((mxfp4_act_tile_kernel<2, 4, OUT_BF16, EXTRA>), grid, block, 0, st, batch, act);
    else if (variant == 2) hipLaunchKernelGGL((mxfp4_act_tile_kernel<2, 2, OUT_BF16, EXTRA>), grid, block, 0, st, batch, act);
    else hipLaunchKernelGGL((mxfp4_act_twin_kernel<OUT_BF16, EXTRA>), grid, block, 0, st, batch, act);
}

// variant, blocks: as launch_gemm picks them
template <bool OUT_BF16>
hipError_t launch_gemm_act_stream(const GemmBatch& batch, const GemmActArgs& act, int variant, uint32_t blocks, hipStream_t st) {
    const dim3 grid(blocks);
    if (act.mul && act.res_kind) launch_act_variant<OUT_BF16, kExtraBoth>(batch, act, variant, grid, st);
    else if (act.res_kind == 2) launch_act_variant<OUT_BF16, kExtraFp32>(batch, act, variant, grid, st);
    else if (act.mul || act.res_kind) launch_act_variant<OUT_BF16, kExtraOne>(batch, act, variant, grid, st);
    else launch_act_variant<OUT_BF16, kExtraNone>(batch, act, variant, grid, st);
    return hipGetLastError();
}

}  // namespace quartet
