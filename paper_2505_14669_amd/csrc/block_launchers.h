// Host-side launch functions of the kernels of include/quartet_block.h (internal to the library).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "../../include/quartet_block.h"
#include "launchers.h"

namespace quartet {

struct NormFwdArgs {
    const void *x, *residual, *weight;
    void *h, *y;
    uint8_t *codes, *scales;
    uint32_t* mask;
    float* rstd;
    int64_t ldx, ldres, ldh, ldy;
    uint32_t rows, n;
    float eps;
    bool x_f32, h_f32, w_f32;
    bool by_tile, past;           // set by the launcher
    double inv_n;
};
struct NormBwdArgs {
    const void *dy, *h, *weight, *dh;
    const float* rstd;
    void *dx, *dx16;
    float* partial;               // set by the launcher
    int64_t lddy, ldh, lddh, lddx, lddx16;
    uint32_t rows, n;
    bool h_f32, w_f32;
};
hipError_t launch_rmsnorm_fwd(const NormFwdArgs& a, int format, hipStream_t st);
size_t rmsnorm_bwd_workspace(int64_t rows, int64_t n);
hipError_t launch_rmsnorm_bwd(const NormBwdArgs& a, float* dweight, float* workspace, hipStream_t st);
// out[j] = sum over the rows of partial [rows x pitch], j < n (rows = 0: zeros)
hipError_t launch_column_sum(const float* partial, uint32_t rows, uint32_t pitch, uint32_t n, float* out, hipStream_t st);

struct ActBwdArgs {
    const uint16_t *dy, *pre, *mul;
    uint16_t *dz, *dmul;
    float* partial;               // set by the launcher
    int64_t lddy, ldpre, ldmul, lddz, lddmul;
    uint32_t m, n;
    int act;
};
size_t act_bwd_workspace(int64_t m, int64_t n);
hipError_t launch_act_bwd(const ActBwdArgs& a, float* dbias, float* workspace, hipStream_t st);

constexpr uint32_t kClipPartials = 1u << 15;                                       // sums of squares, then the factor
constexpr size_t kClipWorkspaceBytes = kClipPartials * sizeof(double) + 16;
hipError_t launch_grad_clip(const quartet_grad_tensor* tensors, int64_t count, float max_norm, float* norm, double* workspace, hipStream_t st);

// the epilogue of quartet_mxfp4_gemm_act; kinds: 0 = none, 1 = bf16, 2 = fp32
struct GemmActArgs {
    const void *bias, *residual;
    const uint16_t* mul;
    uint16_t* pre;
    uint32_t ldmul, ldres, ldpre;
    uint8_t bias_kind, res_kind, act;
};
hipError_t launch_gemm_act(const GemmArgs& g, const GemmActArgs& act, int d_bf16, hipStream_t st);
hipError_t launch_gemm_act_split(const GemmArgs& g, const GemmActArgs& act, int d_bf16, int shape, hipStream_t st);

}  // namespace quartet
