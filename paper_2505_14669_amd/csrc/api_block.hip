// C ABI of include/quartet_block.h: argument validation and kernel sequencing only.
#include "../../include/quartet_block.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdlib.h>

#include <algorithm>

#include "api_common.h"
#include "block_launchers.h"

using quartet::aligned16;
using quartet::check_gemm_args;
using quartet::hip_fail;
using quartet::ProfileScope;

namespace {

constexpr int64_t kMaxNorm = 32768, kMaxActColumns = (int64_t)1 << 26;

bool is_dtype(int t) { return t == QUARTET_DTYPE_F32 || t == QUARTET_DTYPE_BF16; }
bool is_activation(int a) { return a >= QUARTET_ACT_NONE && a <= QUARTET_ACT_SILU; }

// a matrix with rows of n values 16 bytes apart at their starts; optional ones may be null
bool bad_rows(const void* p, int64_t ld, int64_t n, bool required) {
    if (!p) return required;
    return !aligned16(p) || ld < n || (ld % 8) != 0;
}

// the bytes of a gradient or of its copy; in place: of both
struct Range {
    uintptr_t begin, end;
    bool written;
};

// Whether something that is written overlaps anything else.  Sorted by address, each range is held against the furthest end of those before it.
bool overlaps(Range* r, int64_t count) {
    std::sort(r, r + count, [](const Range& a, const Range& b) { return a.begin < b.begin; });
    uintptr_t written_end = 0, read_end = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (written_end > r[i].begin || (r[i].written && read_end > r[i].begin)) return true;
        uintptr_t& end = r[i].written ? written_end : read_end;
        if (r[i].end > end) end = r[i].end;
    }
    return false;
}

}  // namespace

extern "C" {

int quartet_mxfp4_gemm_act(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales,
                           int64_t m, int64_t n, int64_t k, float alpha, const void* bias, int bias_dtype, int activation,
                           const void* multiplier_bf16, int64_t ldmul, const void* residual, int residual_dtype, int64_t ldres,
                           void* pre_bf16, int64_t ldpre, void* d, int d_dtype, int64_t ldd, void* stream) {
    int rc = check_gemm_args(a_codes, a_scales, b_codes, b_scales, m, n, k, d, d_dtype, ldd);
    if (rc) return rc;
    if (!is_activation(activation)) return QUARTET_EINVAL;
    if (bias && (!is_dtype(bias_dtype) || !aligned16(bias))) return QUARTET_EINVAL;
    if (residual && (!is_dtype(residual_dtype) || !aligned16(residual) || ldres < n)) return QUARTET_EINVAL;
    if (multiplier_bf16 && (!aligned16(multiplier_bf16) || ldmul < n)) return QUARTET_EINVAL;
    if (pre_bf16 && (!aligned16(pre_bf16) || ldpre < n)) return QUARTET_EINVAL;
    // in place: element for element
    if (pre_bf16 && (pre_bf16 == d || pre_bf16 == residual || pre_bf16 == multiplier_bf16)) return QUARTET_EINVAL;
    if (residual == d && (residual_dtype != d_dtype || ldres != ldd)) return QUARTET_EINVAL;
    if (multiplier_bf16 == d && (d_dtype != QUARTET_DTYPE_BF16 || ldmul != ldd)) return QUARTET_EINVAL;
    const int64_t most = (int64_t)1 << 21;
    if ((residual && ldres > most) || (multiplier_bf16 && ldmul > most) || (pre_bf16 && ldpre > most)) return QUARTET_ENOTSUP;
    const quartet::GemmArgs g = {a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, d, ldd, nullptr};
    auto kind = [](const void* p, int dtype) { return (uint8_t)(!p ? 0 : dtype == QUARTET_DTYPE_F32 ? 2 : 1); };
    const quartet::GemmActArgs act = {bias, residual, static_cast<const uint16_t*>(multiplier_bf16), static_cast<uint16_t*>(pre_bf16),
                                      (uint32_t)ldmul, (uint32_t)ldres, (uint32_t)ldpre, kind(bias, bias_dtype),
                                      kind(residual, residual_dtype), (uint8_t)activation};
    ProfileScope prof(QUARTET_KIND_GEMM, (hipStream_t)stream);
    const hipError_t e = quartet::launch_gemm_act(g, act, d_dtype == QUARTET_DTYPE_BF16, (hipStream_t)stream);
    return e == hipSuccess ? QUARTET_OK : hip_fail(e);
}

size_t quartet_act_bwd_workspace_bytes(int64_t m, int64_t n) {
    if (m < 0 || n < 0 || m >= ((int64_t)1 << 31) || n > kMaxActColumns) return 0;
    return quartet::act_bwd_workspace(m, n);
}

int quartet_act_bwd(const void* dy_bf16, int64_t lddy, const void* pre_bf16, int64_t ldpre, const void* multiplier_bf16, int64_t ldmul,
                    int64_t m, int64_t n, int activation, void* dz_bf16, int64_t lddz, void* dmul_bf16, int64_t lddmul, float* dbias,
                    void* workspace, size_t workspace_bytes, void* stream) {
    if (m < 0 || n < 0 || !is_activation(activation)) return QUARTET_EINVAL;
    if (!dz_bf16 && !dmul_bf16 && !dbias) return QUARTET_EINVAL;
    if (bad_rows(dy_bf16, lddy, n, true) || bad_rows(pre_bf16, ldpre, n, activation != QUARTET_ACT_NONE || dmul_bf16) ||
        bad_rows(multiplier_bf16, ldmul, n, false) || bad_rows(dz_bf16, lddz, n, false) || bad_rows(dmul_bf16, lddmul, n, false))
        return QUARTET_EINVAL;
    if (!aligned16(dbias)) return QUARTET_EINVAL;
    // in place: element for element
    if (dz_bf16 && ((dz_bf16 == dy_bf16 && lddz != lddy) || dz_bf16 == dmul_bf16 || dz_bf16 == pre_bf16 || dz_bf16 == multiplier_bf16)) return QUARTET_EINVAL;
    if (dmul_bf16 && (dmul_bf16 == dy_bf16 || (dmul_bf16 == pre_bf16 && lddmul != ldpre) || (dmul_bf16 == multiplier_bf16 && lddmul != ldmul)))
        return QUARTET_EINVAL;
    if (m >= ((int64_t)1 << 31) || n > kMaxActColumns) return QUARTET_ENOTSUP;
    const size_t need = dbias ? quartet::act_bwd_workspace(m, n) : 0;
    if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return QUARTET_EINVAL;
    const quartet::ActBwdArgs a = {static_cast<const uint16_t*>(dy_bf16), static_cast<const uint16_t*>(pre_bf16),
                                   static_cast<const uint16_t*>(multiplier_bf16), static_cast<uint16_t*>(dz_bf16),
                                   static_cast<uint16_t*>(dmul_bf16), nullptr, lddy, ldpre, ldmul, lddz, lddmul, (uint32_t)m, (uint32_t)n, activation};
    ProfileScope prof(QUARTET_KIND_ACT, (hipStream_t)stream);
    const hipError_t e = quartet::launch_act_bwd(a, dbias, static_cast<float*>(workspace), (hipStream_t)stream);
    return e == hipSuccess ? QUARTET_OK : hip_fail(e);
}

static int check_norm_sizes(int64_t rows, int64_t n) {
    if (rows < 0 || n < 1) return QUARTET_EINVAL;
    if (n > kMaxNorm || rows >= ((int64_t)1 << 31) || rows * ((n + 31) / 32) >= ((int64_t)1 << 31)) return QUARTET_ENOTSUP;
    return QUARTET_OK;
}

int quartet_rmsnorm_fwd(const void* x, int x_dtype, int64_t ldx, const void* residual, int64_t ldres, int64_t rows, int64_t n,
                        const void* weight, int weight_dtype, float eps, void* h, int h_dtype, int64_t ldh, void* y_bf16, int64_t ldy,
                        int format, uint8_t* codes, uint8_t* scales, uint32_t* mask, float* rstd, void* stream) {
    const int rc = check_norm_sizes(rows, n);
    if (rc) return rc;
    if (bad_rows(x, ldx, n, true) || bad_rows(residual, ldres, n, false) || bad_rows(h, ldh, n, false) || bad_rows(y_bf16, ldy, n, false))
        return QUARTET_EINVAL;
    if (!weight || !aligned16(weight) || !is_dtype(x_dtype) || !is_dtype(weight_dtype)) return QUARTET_EINVAL;
    if (residual ? !is_dtype(h_dtype) : h != nullptr) return QUARTET_EINVAL;
    if (!(eps >= 0.0f) || isinf(eps)) return QUARTET_EINVAL;
    if (reinterpret_cast<uintptr_t>(rstd) & 3u) return QUARTET_EINVAL;
    if (format == QUARTET_FORMAT_MXFP4 || format == QUARTET_FORMAT_MXFP8) {
        if (!codes || !scales || !aligned16(codes) || (reinterpret_cast<uintptr_t>(scales) & 3u) || (n % 32) != 0) return QUARTET_EINVAL;
        if (mask && (format != QUARTET_FORMAT_MXFP4 || !aligned16(mask))) return QUARTET_EINVAL;
    } else if (format != QUARTET_FORMAT_NONE || codes || scales || mask) {
        return QUARTET_EINVAL;
    }
    if (!h && !y_bf16 && !codes && !rstd) return QUARTET_EINVAL;
    // in place: element for element
    if (h && ((h == residual && ldh != ldres) || (h == x && (x_dtype != h_dtype || ldh != ldx)) || h == y_bf16)) return QUARTET_EINVAL;
    if (y_bf16 && (y_bf16 == x || y_bf16 == residual)) return QUARTET_EINVAL;
    const quartet::NormFwdArgs a = {x, residual, weight, h, y_bf16, codes, scales, mask, rstd, ldx, ldres, ldh, ldy, (uint32_t)rows, (uint32_t)n, eps,
                                    x_dtype == QUARTET_DTYPE_F32, residual && h_dtype == QUARTET_DTYPE_F32, weight_dtype == QUARTET_DTYPE_F32, false, false, 0.0};
    ProfileScope prof(QUARTET_KIND_NORM, (hipStream_t)stream);
    const hipError_t e = quartet::launch_rmsnorm_fwd(a, format, (hipStream_t)stream);
    return e == hipSuccess ? QUARTET_OK : hip_fail(e);
}

size_t quartet_rmsnorm_bwd_workspace_bytes(int64_t rows, int64_t n) {
    if (check_norm_sizes(rows, n) != QUARTET_OK) return 0;
    return quartet::rmsnorm_bwd_workspace(rows, n);
}

int quartet_rmsnorm_bwd(const void* dy_bf16, int64_t lddy, const void* h, int h_dtype, int64_t ldh, int64_t rows, int64_t n,
                        const void* weight, int weight_dtype, const float* rstd, const void* dh, int64_t lddh, void* dx, int64_t lddx,
                        void* dx16, int64_t lddx16, float* dweight, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_norm_sizes(rows, n);
    if (rc) return rc;
    if (!is_dtype(h_dtype) || !is_dtype(weight_dtype) || !weight || !aligned16(weight)) return QUARTET_EINVAL;
    if (!rstd || (reinterpret_cast<uintptr_t>(rstd) & 3u) || !aligned16(dweight)) return QUARTET_EINVAL;
    if (!dx && !dweight) return QUARTET_EINVAL;
    if (bad_rows(dy_bf16, lddy, n, true) || bad_rows(h, ldh, n, true) || bad_rows(dh, lddh, n, false) || bad_rows(dx, lddx, n, false) ||
        bad_rows(dx16, lddx16, n, false))
        return QUARTET_EINVAL;
    if (dx16 && (!dx || h_dtype != QUARTET_DTYPE_F32)) return QUARTET_EINVAL;
    // in place: element for element
    if (dx && ((dx == dh && lddx != lddh) || (dx == h && lddx != ldh) || dx == dx16)) return QUARTET_EINVAL;
    if (dx && dx == dy_bf16 && (h_dtype != QUARTET_DTYPE_BF16 || lddx != lddy)) return QUARTET_EINVAL;
    if (dx16 && ((dx16 == dy_bf16 && lddx16 != lddy) || dx16 == h || dx16 == dh)) return QUARTET_EINVAL;
    const size_t need = dweight ? quartet::rmsnorm_bwd_workspace(rows, n) : 0;
    if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return QUARTET_EINVAL;
    const quartet::NormBwdArgs a = {dy_bf16, h, weight, dh, rstd, dx, dx16, nullptr, lddy, ldh, lddh, lddx, lddx16, (uint32_t)rows, (uint32_t)n,
                                    h_dtype == QUARTET_DTYPE_F32, weight_dtype == QUARTET_DTYPE_F32};
    ProfileScope prof(QUARTET_KIND_NORM, (hipStream_t)stream);
    const hipError_t e = quartet::launch_rmsnorm_bwd(a, dweight, static_cast<float*>(workspace), (hipStream_t)stream);
    return e == hipSuccess ? QUARTET_OK : hip_fail(e);
}

size_t quartet_grad_clip_workspace_bytes(void) { return quartet::kClipWorkspaceBytes; }

int quartet_grad_clip(const quartet_grad_tensor* tensors, int64_t count, float max_norm, float* norm, void* workspace,
                      size_t workspace_bytes, void* stream) {
    if (count < 0 || (count > 0 && !tensors) || !norm || (reinterpret_cast<uintptr_t>(norm) & 3u)) return QUARTET_EINVAL;
    if (!(max_norm >= 0.0f)) return QUARTET_EINVAL;
    if (!workspace || !aligned16(workspace) || workspace_bytes < quartet::kClipWorkspaceBytes) return QUARTET_EINVAL;
    if (count > ((int64_t)1 << 15)) return QUARTET_ENOTSUP;       // a sum in the workspace each
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) {
        const quartet_grad_tensor& t = tensors[i];
        if (t.size < 0) return QUARTET_EINVAL;
        if (t.size == 0) continue;
        if (!t.grad || !t.out || !is_dtype(t.grad_dtype) || !is_dtype(t.out_dtype)) return QUARTET_EINVAL;
        if ((reinterpret_cast<uintptr_t>(t.grad) & (t.grad_dtype == QUARTET_DTYPE_F32 ? 3u : 1u)) ||
            (reinterpret_cast<uintptr_t>(t.out) & (t.out_dtype == QUARTET_DTYPE_F32 ? 3u : 1u)))
            return QUARTET_EINVAL;
        if (t.grad == t.out && t.grad_dtype != t.out_dtype) return QUARTET_EINVAL;
        if (t.size >= ((int64_t)1 << 43)) return QUARTET_ENOTSUP;
        total += t.size;
        if (total >= ((int64_t)1 << 43)) return QUARTET_ENOTSUP;
    }
    constexpr int64_t kHere = 256;
    Range here[2 * kHere];
    Range* ranges = count <= kHere ? here : static_cast<Range*>(malloc(sizeof(Range) * 2 * (size_t)count));
    if (!ranges) return QUARTET_ENOTSUP;
    int64_t found = 0;
    for (int64_t i = 0; i < count; ++i) {
        const quartet_grad_tensor& t = tensors[i];
        if (t.size == 0) continue;
        const uintptr_t g = reinterpret_cast<uintptr_t>(t.grad), o = reinterpret_cast<uintptr_t>(t.out);
        if (g != o) ranges[found++] = {g, g + (uintptr_t)t.size * (t.grad_dtype == QUARTET_DTYPE_F32 ? 4u : 2u), false};
        ranges[found++] = {o, o + (uintptr_t)t.size * (t.out_dtype == QUARTET_DTYPE_F32 ? 4u : 2u), true};
    }
    const bool overlap = overlaps(ranges, found);
    if (ranges != here) free(ranges);
    if (overlap) return QUARTET_EINVAL;
    ProfileScope prof(QUARTET_KIND_CLIP, (hipStream_t)stream);
    const hipError_t e = quartet::launch_grad_clip(tensors, count, max_norm, norm, static_cast<double*>(workspace), (hipStream_t)stream);
    return e == hipSuccess ? QUARTET_OK : hip_fail(e);
}

}  // extern "C"
