// The epilogue of quartet_mxfp4_gemm_act on chunks of four columns: what the product kernels share.
#pragma once
#include "block_common.h"
#include "block_launchers.h"
#include "gemm_common.h"

namespace quartet {

// A chunk's residual and multiplier as they lie in memory
struct ActChunk {
    v4u_t res;     // bf16: x, y
    v2u_t mul;
};
// every chunk of every matrix starts at a multiple of its size; wave-uniform
__device__ __forceinline__ bool act_wide(const GemmActArgs& e, uint32_t ldd) {
    return ((ldd | (e.res_kind ? e.ldres : 0u) | (e.mul ? e.ldmul : 0u) | (e.pre ? e.ldpre : 0u)) & 3u) == 0u;
}
// any chunk, element by element where it is not whole; rows and columns outside the matrix: not read
__device__ __forceinline__ void load_act_chunk(ActChunk& c, const GemmActArgs& e, uint32_t row, uint32_t col, uint32_t m, uint32_t n, bool wide) {
    c.res = {0u, 0u, 0u, 0u};
    c.mul = {0u, 0u};
    if (row >= m || col >= n) return;
    const bool whole = wide && col + 4u <= n;
    const uint32_t left = n - col;
    if (e.res_kind == 2) {
        const float* p = static_cast<const float*>(e.residual) + (size_t)row * e.ldres + col;
        if (whole) c.res = *reinterpret_cast<const v4u_t*>(p);
        else
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i < left) c.res[i] = f2u(p[i]);
    } else if (e.res_kind == 1) {
        const uint16_t* p = static_cast<const uint16_t*>(e.residual) + (size_t)row * e.ldres + col;
        if (whole) {
            const v2u_t t = *reinterpret_cast<const v2u_t*>(p);
            c.res.x = t.x; c.res.y = t.y;
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i < left) c.res[i >> 1] |= (uint32_t)p[i] << (16u * (i & 1u));
        }
    }
    if (e.mul) {
        const uint16_t* p = e.mul + (size_t)row * e.ldmul + col;
        if (whole) c.mul = *reinterpret_cast<const v2u_t*>(p);
        else
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i < left) c.mul[i >> 1] |= (uint32_t)p[i] << (16u * (i & 1u));
    }
}
// the four columns' bias; columns outside the matrix: 0
__device__ __forceinline__ void load_bias(float (&b)[4], const GemmActArgs& e, uint32_t col, uint32_t n) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        b[i] = 0.0f;
        if (e.bias_kind == 2) { if (col + i < n) b[i] = static_cast<const float*>(e.bias)[col + i]; }
        else if (e.bias_kind == 1) { if (col + i < n) b[i] = bf16_lo(static_cast<const uint16_t*>(e.bias)[col + i]); }
    }
}
// gate and residual of a chunk whose activation is in v
__device__ __forceinline__ void combine_act_chunk(float (&v)[4], const ActChunk& c, const GemmActArgs& e) {
    if (e.mul) {
        v[0] *= bf16_lo(c.mul.x); v[1] *= bf16_hi(c.mul.x); v[2] *= bf16_lo(c.mul.y); v[3] *= bf16_hi(c.mul.y);
    }
    if (e.res_kind == 2) {
        v[0] += u2f(c.res.x); v[1] += u2f(c.res.y); v[2] += u2f(c.res.z); v[3] += u2f(c.res.w);
    } else if (e.res_kind == 1) {
        v[0] += bf16_lo(c.res.x); v[1] += bf16_hi(c.res.x); v[2] += bf16_lo(c.res.y); v[3] += bf16_hi(c.res.y);
    }
}
// four columns to a matrix, bf16 or fp32, whole or as far as they exist
template <bool BF16>
__device__ __forceinline__ void store_act_chunk(void* d, uint32_t ld, uint32_t row, uint32_t col, uint32_t m, uint32_t n, bool wide, const float (&v)[4]) {
    if (row >= m || col >= n) return;
    const size_t at = (size_t)row * ld + col;
    if (BF16) {
        uint16_t* p = static_cast<uint16_t*>(d) + at;
        const uint32_t lo = bf16_pack2(v[0], v[1]), hi = bf16_pack2(v[2], v[3]);
        if (wide && col + 4u <= n) {
            *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
        } else {
            p[0] = (uint16_t)lo;
            if (col + 1u < n) p[1] = (uint16_t)(lo >> 16);
            if (col + 2u < n) p[2] = (uint16_t)hi;
            if (col + 3u < n) p[3] = (uint16_t)(hi >> 16);
        }
    } else {
        float* p = static_cast<float*>(d) + at;
        if (wide && col + 4u <= n) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (col + i < n) p[i] = v[i];
        }
    }
}

}  // namespace quartet
