// Norm of all gradients of a step and their scaled copies.  Bound by memory: every gradient is read for the norm, which must be known before the
// first copy is written, and read again for its copy.  The tensors are cut into chunks of kChunk elements; the blocks take chunks b, b + B, ...
// of all tensors, so a list of many small tensors and one of a few large ones fill the chip alike.  A launch's arguments hold up to kTensors tensors;
// longer lists take more launches, each adding to the blocks' sums of squares in the workspace (in launch order: the bits do not depend on timing).
#include <math.h>

#include "block_common.h"
#include "block_launchers.h"

namespace quartet {

namespace {

constexpr uint32_t kChunk = 8192, kBlocks = 2048;
constexpr int kTensors = 80;

struct ClipTensor {
    const void* grad;
    void* out;
    uint64_t size;
    uint32_t first_chunk;         // of this launch's
    uint16_t grad_f32, out_f32;
};
struct ClipList {
    ClipTensor t[kTensors];
    uint32_t count, chunks;
};
static_assert(sizeof(ClipList) + 64 <= 4096, "a launch's arguments");

__device__ __forceinline__ const ClipTensor& tensor_of(const ClipList& l, uint32_t chunk) {
    uint32_t lo = 0u, hi = l.count;            // the last tensor whose first chunk is not behind this one
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) >> 1;
        if (l.t[mid].first_chunk <= chunk) lo = mid;
        else hi = mid;
    }
    return l.t[lo];
}

// elements at .. at + 7 of a tensor of `size` (missing ones: 0); whole: eight of them, aligned to 16 bytes
__device__ __forceinline__ void load8(const void* p, bool f32, uint64_t at, uint64_t size, bool aligned, float (&v)[8]) {
    if (aligned && at + 8u <= size) {
        if (f32) {
            const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
            const float4 a = s[0], b = s[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            unpack8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at), v);
        }
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        v[i] = 0.0f;
        if (at + i < size) v[i] = f32 ? static_cast<const float*>(p)[at + i] : bf16_lo(static_cast<const uint16_t*>(p)[at + i]);
    }
}
__device__ __forceinline__ void store8(void* p, bool f32, uint64_t at, uint64_t size, bool aligned, const float (&v)[8]) {
    if (aligned && at + 8u <= size) {
        if (f32) {
            float4* d = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
            d[0] = make_float4(v[0], v[1], v[2], v[3]);
            d[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = pack8(v);
        }
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (at + i < size) {
            if (f32) static_cast<float*>(p)[at + i] = v[i];
            else static_cast<uint16_t*>(p)[at + i] = bf16_of(v[i]);
        }
}
__device__ __forceinline__ bool is_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0u; }

// sum of a double over the block's 256 threads, in every thread
__device__ __forceinline__ double block_sum(double s, double* meet) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63u) == 0u) meet[threadIdx.x >> 6] = s;
    __syncthreads();
    return (meet[0] + meet[1]) + (meet[2] + meet[3]);
}

__global__ void __launch_bounds__(256)
grad_square_kernel(ClipList l, double* __restrict__ partial, uint32_t add) {
    __shared__ double meet[4];
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
        const ClipTensor& t = tensor_of(l, c);
        const uint64_t base = (uint64_t)(c - t.first_chunk) * kChunk, size = t.size;
        const bool aligned = is_aligned16(t.grad), f32 = t.grad_f32;
#pragma unroll
        for (uint32_t i = 0; i < kChunk / 2048u; ++i) {
            float v[8];
            load8(t.grad, f32, base + i * 2048u + threadIdx.x * 8u, size, aligned, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = __builtin_fma((double)v[e], (double)v[e], s);
        }
    }
    s = block_sum(s, meet);
    if (threadIdx.x == 0u) partial[blockIdx.x] = add ? partial[blockIdx.x] + s : s;
}

__global__ void __launch_bounds__(256)
grad_scale_kernel(ClipList l, const double* __restrict__ partial, uint32_t partials, float max_norm, float* __restrict__ norm_out) {
    __shared__ double meet[4];
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < partials; i += 256u) s += partial[i];
    const float norm = (float)__builtin_sqrt(block_sum(s, meet));
    if (blockIdx.x == 0u && threadIdx.x == 0u) *norm_out = norm;
    const float ratio = max_norm / (norm + 1e-6f);
    const float factor = norm - norm == 0.0f && ratio < 1.0f ? ratio : 1.0f;      // (a norm that is not finite: 1)
    for (uint32_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
        const ClipTensor& t = tensor_of(l, c);
        if (t.grad == t.out && factor == 1.0f) continue;
        const uint64_t base = (uint64_t)(c - t.first_chunk) * kChunk, size = t.size;
        const bool in = is_aligned16(t.grad), out = is_aligned16(t.out), in32 = t.grad_f32, out32 = t.out_f32;
#pragma unroll
        for (uint32_t i = 0; i < kChunk / 2048u; ++i) {
            const uint64_t at = base + i * 2048u + threadIdx.x * 8u;
            if (at >= size) continue;
            float v[8];
            load8(t.grad, in32, at, size, in, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= factor;
            store8(t.out, out32, at, size, out, v);
        }
    }
}

}  // namespace

hipError_t launch_grad_clip(const quartet_grad_tensor* tensors, int64_t count, float max_norm, float* norm, double* workspace, hipStream_t st) {
    auto fill = [&](ClipList& l, int64_t& at) {     // the next tensors of the list
        l.count = l.chunks = 0u;
        for (; at < count && l.count < (uint32_t)kTensors; ++at) {
            const quartet_grad_tensor& t = tensors[at];
            if (t.size <= 0) continue;
            l.t[l.count++] = {t.grad, t.out, (uint64_t)t.size, l.chunks, (uint16_t)(t.grad_dtype == QUARTET_DTYPE_F32), (uint16_t)(t.out_dtype == QUARTET_DTYPE_F32)};
            l.chunks += (uint32_t)(((uint64_t)t.size + kChunk - 1u) / kChunk);
        }
    };
    uint64_t all = 0;
    for (int64_t i = 0; i < count; ++i) all += ((uint64_t)tensors[i].size + kChunk - 1u) / kChunk;
    const uint32_t blocks = all < 1u ? 1u : all < kBlocks ? (uint32_t)all : kBlocks;
    ClipList l;
    int64_t at = 0;
    uint32_t add = 0u;
    do {
        fill(l, at);
        hipLaunchKernelGGL(grad_square_kernel, dim3(blocks), dim3(256), 0, st, l, workspace, add);
        add = 1u;
    } while (at < count);
    at = 0;
    do {
        fill(l, at);
        hipLaunchKernelGGL(grad_scale_kernel, dim3(blocks), dim3(256), 0, st, l, workspace, blocks, max_norm, norm);
    } while (at < count);
    return hipGetLastError();
}

}  // namespace quartet
