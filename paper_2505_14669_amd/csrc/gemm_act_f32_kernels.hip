// quartet_mxfp4_gemm_act's streaming kernels with fp32 results
#include "gemm_act_kernels.h"

namespace quartet {

template hipError_t launch_gemm_act_stream<false>(const GemmBatch& batch, const GemmActArgs& act, int variant, uint32_t blocks, hipStream_t st);

}  // namespace quartet
