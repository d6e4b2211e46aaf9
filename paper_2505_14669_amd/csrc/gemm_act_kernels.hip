// The streaming MXFP4 products with bias, activation, gate and residual in their epilogue (quartet_mxfp4_gemm_act); the bodies are gemm_stream.h's.
#include "block_launchers.h"
#include "gemm_stream.h"

namespace quartet {

template <bool OUT_BF16>
__global__ void __launch_bounds__(256)
mxfp4_act_large_kernel(GemmBatch batch, GemmActArgs act) {
    stream_large_tiles<OUT_BF16, false, false, false, GemmActArgs>(batch, 1u, nullptr, act);
}

template <int TM, int TN, bool OUT_BF16>
__global__ void __launch_bounds__(256)
mxfp4_act_tile_kernel(GemmBatch batch, GemmActArgs act) {
    stream_tiles<TM, TN, 1, OUT_BF16, false, false, false, GemmActArgs>(batch, 1u, nullptr, act);
}

template <bool OUT_BF16>
__global__ void __launch_bounds__(256, 2)
mxfp4_act_twin_kernel(GemmBatch batch, GemmActArgs act) {
    stream_tiles<2, 2, 2, OUT_BF16, false, false, false, GemmActArgs>(batch, 1u, nullptr, act);
}

// variant, blocks: as launch_gemm picks them
hipError_t launch_gemm_act_stream(const GemmBatch& batch, const GemmActArgs& act, int d_bf16, int variant, uint32_t blocks, hipStream_t st) {
    const dim3 grid(blocks), block(256);
#define QUARTET_ACT(FN, ...)                                                                            \
    do {                                                                                                \
        if (d_bf16) hipLaunchKernelGGL((FN<__VA_ARGS__ true>), grid, block, 0, st, batch, act);         \
        else hipLaunchKernelGGL((FN<__VA_ARGS__ false>), grid, block, 0, st, batch, act);               \
    } while (0)
    if (variant == 0) QUARTET_ACT(mxfp4_act_large_kernel, );
    else if (variant == 1) QUARTET_ACT(mxfp4_act_tile_kernel, 2, 4, );
    else if (variant == 2) QUARTET_ACT(mxfp4_act_tile_kernel, 2, 2, );
    else QUARTET_ACT(mxfp4_act_twin_kernel, );
#undef QUARTET_ACT
    return hipGetLastError();
}

}  // namespace quartet
