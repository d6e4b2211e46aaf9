// Norm of all gradients of a step and their scaled copies.  Bound by memory: every gradient is read for the norm, which must be known before the
// first copy is written, and read again for its copy.  The tensors are cut into chunks of kChunk elements, a block each: a list of many small tensors and
// one of a few large ones fill the chip alike, and the blocks in flight cover neighbouring memory.  Every chunk leaves its sum of squares in the workspace (in
// fixed places and added up in a fixed order: the bits do not depend on timing); where the chunks are few, every block of the second kernel adds them up for itself, otherwise a
// kernel of one block does.  A launch's arguments hold up to kTensors tensors; longer lists take more launches.
#include <math.h>

#include "block_common.h"
#include "block_launchers.h"

namespace quartet {

namespace {

constexpr uint32_t kChunk = 4096;              // (180 small tensors: 36.1 us with 8192, 31.8 with 4096; large ones alike)
constexpr uint32_t kFew = 1024;                 // chunks that every block adds up for itself
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

// The tensor of a chunk: the last one whose first chunk is not behind it.  Every lane looks at one or two, one trip to memory (a search would wait for several).
__device__ __forceinline__ const ClipTensor& tensor_of(const ClipList& l, uint32_t chunk) {
    static_assert(kTensors > 64 && kTensors <= 128, "two tensors a lane");
    const uint32_t lane = threadIdx.x & 63u, high = lane + 64u;
    const bool a = lane < l.count && l.t[lane].first_chunk <= chunk, b = high < l.count && l.t[high < (uint32_t)kTensors ? high : 0u].first_chunk <= chunk;
    const int before = __popcll(__ballot(a)) + __popcll(__ballot(b));
    return l.t[__builtin_amdgcn_readfirstlane(before) - 1];
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
// Elements at .. at + 3, aligned to their size: what the second kernel goes by.  A store instruction of a wave then writes whole lines, in fp32 too: with eight a
// lane, two stores of 16 bytes 32 apart, 202 M values from bf16 to fp32 took 352 us in place of 260.
template <bool PAST>
__device__ __forceinline__ void load4(const void* p, bool f32, uint64_t at, uint64_t size, bool aligned, float (&v)[4]) {
    if (aligned && at + 4u <= size) {
        if (f32) {
            const v4f* s = reinterpret_cast<const v4f*>(static_cast<const float*>(p) + at);
            const v4f t = PAST ? __builtin_nontemporal_load(s) : *s;
            v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
        } else {
            const v2u_t* s = reinterpret_cast<const v2u_t*>(static_cast<const uint16_t*>(p) + at);
            const v2u_t t = PAST ? __builtin_nontemporal_load(s) : *s;
            v[0] = bf16_lo(t.x); v[1] = bf16_hi(t.x); v[2] = bf16_lo(t.y); v[3] = bf16_hi(t.y);
        }
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        v[i] = 0.0f;
        if (at + i < size) v[i] = f32 ? static_cast<const float*>(p)[at + i] : bf16_lo(static_cast<const uint16_t*>(p)[at + i]);
    }
}
template <bool PAST>
__device__ __forceinline__ void store4(void* p, bool f32, uint64_t at, uint64_t size, bool aligned, const float (&v)[4]) {
    if (aligned && at + 4u <= size) {
        if (f32) {
            const v4f t = {v[0], v[1], v[2], v[3]};
            v4f* d = reinterpret_cast<v4f*>(static_cast<float*>(p) + at);
            if (PAST) __builtin_nontemporal_store(t, d);
            else *d = t;
        } else {
            const v2u_t t = {bf16_pack2(v[0], v[1]), bf16_pack2(v[2], v[3])};
            v2u_t* d = reinterpret_cast<v2u_t*>(static_cast<uint16_t*>(p) + at);
            if (PAST) __builtin_nontemporal_store(t, d);
            else *d = t;
        }
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
        if (at + i < size) {
            if (f32) static_cast<float*>(p)[at + i] = v[i];
            else static_cast<uint16_t*>(p)[at + i] = bf16_of(v[i]);
        }
}
__device__ __forceinline__ bool is_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0u; }

// sum of a double over the block's W waves, in every thread
template <int W>
__device__ __forceinline__ double block_sum(double s, double (&meet)[W]) {
    s = wave_sum64(s);
    if ((threadIdx.x & 63u) == 0u) meet[threadIdx.x >> 6] = s;
    __syncthreads();
    s = meet[0];
#pragma unroll
    for (int w = 1; w < W; ++w) s += meet[w];
    return s;
}

// chunks of kChunk << shift elements
__global__ void __launch_bounds__(256)
grad_square_kernel(ClipList l, double* __restrict__ partial, uint32_t shift) {
    __shared__ double meet[4];
    const ClipTensor& t = tensor_of(l, blockIdx.x);
    const uint64_t chunk = (uint64_t)kChunk << shift, base = (blockIdx.x - t.first_chunk) * chunk, size = t.size;
    const bool aligned = is_aligned16(t.grad), f32 = t.grad_f32;
    double s = 0.0;
    for (uint64_t at = base + threadIdx.x * 8u, end = base + chunk < size ? base + chunk : size; at < end; at += kChunk) {
        float v[kChunk / 2048u][8];
#pragma unroll
        for (uint32_t i = 0; i < kChunk / 2048u; ++i) load8(t.grad, f32, at + i * 2048u, size, aligned, v[i]);
#pragma unroll
        for (uint32_t i = 0; i < kChunk / 2048u; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s = __builtin_fma((double)v[i][e], (double)v[i][e], s);
    }
    s = block_sum(s, meet);
    if (threadIdx.x == 0u) partial[blockIdx.x] = s;
}

__device__ __forceinline__ float clip_factor(float norm, float max_norm) {
    const float ratio = max_norm / (norm + 1e-6f);
    return norm - norm == 0.0f && ratio < 1.0f ? ratio : 1.0f;      // (a norm that is not finite: 1)
}

__global__ void __launch_bounds__(1024)
grad_norm_kernel(const double* __restrict__ partial, uint32_t partials, float max_norm, float* __restrict__ norm_out, float* __restrict__ factor_out) {
    __shared__ double meet[16];
    double s = 0.0;
#pragma unroll 8
    for (uint32_t i = threadIdx.x; i < partials; i += 1024u) s += partial[i];
    const float norm = (float)__builtin_sqrt(block_sum(s, meet));
    if (threadIdx.x != 0u) return;
    *norm_out = norm;
    *factor_out = clip_factor(norm, max_norm);
}

// partials: of all chunks, if they are few; otherwise 0, and the factor is known.  The last chunks first: they are what the caches hold of the first pass.
template <bool PAST>
__global__ void __launch_bounds__(256)
grad_scale_kernel(ClipList l, const double* __restrict__ partial, uint32_t partials, float max_norm, float* __restrict__ norm_out,
                  const float* __restrict__ factor_in, uint32_t shift) {
    __shared__ double meet[4];
    float factor;
    if (partials) {
        double s = 0.0;
        for (uint32_t i = threadIdx.x; i < partials; i += 256u) s += partial[i];
        const float norm = (float)__builtin_sqrt(block_sum(s, meet));
        if (blockIdx.x == 0u && threadIdx.x == 0u) *norm_out = norm;
        factor = clip_factor(norm, max_norm);
    } else {
        factor = *factor_in;
    }
    const uint32_t c = l.chunks - 1u - blockIdx.x;
    const ClipTensor& t = tensor_of(l, c);
    if (t.grad == t.out && factor == 1.0f) return;
    const uint64_t chunk = (uint64_t)kChunk << shift, base = (c - t.first_chunk) * chunk, size = t.size;
    const bool in32 = t.grad_f32, out32 = t.out_f32;
    const bool in = (reinterpret_cast<uintptr_t>(t.grad) & (in32 ? 15u : 7u)) == 0u, out = (reinterpret_cast<uintptr_t>(t.out) & (out32 ? 15u : 7u)) == 0u;
    for (uint64_t at = base + threadIdx.x * 4u, end = base + chunk < size ? base + chunk : size; at < end; at += kChunk) {
        float v[kChunk / 1024u][4];
#pragma unroll
        for (uint32_t i = 0; i < kChunk / 1024u; ++i) load4<PAST>(t.grad, in32, at + i * 1024u, size, in, v[i]);
#pragma unroll
        for (uint32_t i = 0; i < kChunk / 1024u; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][e] *= factor;
            store4<PAST>(t.out, out32, at + i * 1024u, size, out, v[i]);
        }
    }
}

}  // namespace

hipError_t launch_grad_clip(const quartet_grad_tensor* tensors, int64_t count, float max_norm, float* norm, double* workspace, hipStream_t st) {
    uint32_t shift = 0u;
    uint64_t all = 0u;
    for (;; ++shift) {            // the smallest chunks whose sums the workspace holds
        all = 0u;
        for (int64_t i = 0; i < count; ++i) all += ((uint64_t)tensors[i].size + ((uint64_t)kChunk << shift) - 1u) / ((uint64_t)kChunk << shift);
        if (all <= kClipPartials || shift >= 40u) break;
    }
    if (all > kClipPartials) return hipErrorInvalidValue;
    auto fill = [&](ClipList& l, int64_t& at) {     // the next tensors of the list
        l.count = l.chunks = 0u;
        for (; at < count && l.count < (uint32_t)kTensors; ++at) {
            const quartet_grad_tensor& t = tensors[at];
            if (t.size <= 0) continue;
            l.t[l.count++] = {t.grad, t.out, (uint64_t)t.size, l.chunks, (uint16_t)(t.grad_dtype == QUARTET_DTYPE_F32), (uint16_t)(t.out_dtype == QUARTET_DTYPE_F32)};
            l.chunks += (uint32_t)(((uint64_t)t.size + ((uint64_t)kChunk << shift) - 1u) / ((uint64_t)kChunk << shift));
        }
    };
    float* factor = reinterpret_cast<float*>(workspace + kClipPartials);
    const bool few = all <= kFew;
    // Copies go past the memory-side cache (256 MiB) where it cannot hold them and their gradients: plain accesses would push out what the second pass still reads
    // (us, through / past: bf16 to fp32 64 + 128 MiB 48.8 / 48.8, 96 + 192 69.4 / 68.2, 128 + 256 91.5 / 86.9, 256 + 512 185 / 167; fp32 to bf16 192 + 96 81.6 / 78.7;
    // fp32 128 + 128 64.8 / 64.9).  In place nothing is pushed out, each line is written where it was read: through it at every size (fp32 32 MiB 23.0 / 27.9, 256 MiB
    // 122.9 / 127.4, 512 MiB 294 / 306, bf16 64 MiB 42.3 / 45.4).
    uint64_t copied = 0u;
    for (int64_t i = 0; i < count; ++i) {
        const quartet_grad_tensor& t = tensors[i];
        if (t.size > 0 && t.grad != t.out) copied += (uint64_t)t.size * ((t.grad_dtype == QUARTET_DTYPE_F32 ? 4u : 2u) + (t.out_dtype == QUARTET_DTYPE_F32 ? 4u : 2u));
    }
    const bool past = copied >= ((uint64_t)256 << 20);
    ClipList l;
    double* partial = workspace;
    for (int64_t at = 0; at < count; partial += l.chunks) {
        fill(l, at);
        if (l.chunks) hipLaunchKernelGGL(grad_square_kernel, dim3(l.chunks), dim3(256), 0, st, l, partial, shift);
    }
    if (!few || all == 0u) hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, st, workspace, (uint32_t)all, max_norm, norm, factor);
    for (int64_t at = 0; at < count;) {
        fill(l, at);
        if (l.chunks == 0u) continue;
        if (past) hipLaunchKernelGGL((grad_scale_kernel<true>), dim3(l.chunks), dim3(256), 0, st, l, workspace, few ? (uint32_t)all : 0u, max_norm, norm, factor, shift);
        else hipLaunchKernelGGL((grad_scale_kernel<false>), dim3(l.chunks), dim3(256), 0, st, l, workspace, few ? (uint32_t)all : 0u, max_norm, norm, factor, shift);
    }
    return hipGetLastError();
}

}  // namespace quartet
