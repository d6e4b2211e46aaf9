// Host-only stand-ins for the launchers of the kernels of include/quartet_block.h (see launcher_stubs.cpp, which this is linked with): each
// counts its calls, so that a refused call can be seen to have reached none.
#include "block_launchers.h"
static int g_block_launches = 0;
extern "C" int quartet_hostcheck_block_launches(void) { return g_block_launches; }
namespace quartet {
hipError_t launch_rmsnorm_fwd(const NormFwdArgs&, int, hipStream_t) { ++g_block_launches; return hipSuccess; }
size_t rmsnorm_bwd_workspace(int64_t rows, int64_t n) { return rows ? 1024u * (size_t)((n + 7) / 8 * 8) * 4u : 0u; }
hipError_t launch_rmsnorm_bwd(const NormBwdArgs&, float*, float*, hipStream_t) { ++g_block_launches; return hipSuccess; }
size_t act_bwd_workspace(int64_t m, int64_t n) { return m > 0 && n > 0 ? (size_t)((n + 7) / 8 * 8) * 4u : 0u; }
hipError_t launch_act_bwd(const ActBwdArgs&, float*, float*, hipStream_t) { ++g_block_launches; return hipSuccess; }
hipError_t launch_grad_clip(const quartet_grad_tensor*, int64_t, float, float*, double*, hipStream_t) { ++g_block_launches; return hipSuccess; }
hipError_t launch_gemm_act(const GemmArgs&, const GemmActArgs&, int, hipStream_t) { ++g_block_launches; return hipSuccess; }
}
