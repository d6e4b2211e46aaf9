// Pieces shared by the kernels of include/quartet_block.h: bf16 conversion, activations, reductions across a wave.
#pragma once
#include "device_common.h"

namespace quartet {

typedef __bf16 v2bf_t __attribute__((ext_vector_type(2)));

// two fp32 values to bf16, round to nearest even (NaN stays NaN): one instruction
__device__ __forceinline__ uint32_t bf16_pack2(float lo, float hi) {
    const v2f v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, v2bf_t));
}
__device__ __forceinline__ uint16_t bf16_of(float v) { return (uint16_t)bf16_pack2(v, v); }
__device__ __forceinline__ float bf16_lo(uint32_t w) { return u2f(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return u2f(w & 0xFFFF0000u); }
__device__ __forceinline__ void unpack8(const uint4& q, float* v) {
    v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
    v[4] = bf16_lo(q.z); v[5] = bf16_hi(q.z); v[6] = bf16_lo(q.w); v[7] = bf16_hi(q.w);
}
__device__ __forceinline__ uint4 pack8(const float* v) {
    return make_uint4(bf16_pack2(v[0], v[1]), bf16_pack2(v[2], v[3]), bf16_pack2(v[4], v[5]), bf16_pack2(v[6], v[7]));
}

// Activations (QUARTET_ACT_*).  SiLU and GELU are z s(p(z)) with s(t) = 1 / (1 + exp(-t)); exp through the hardware's 2^x and the quotient through
// its reciprocal, each good to about 1 ulp: the relative error stays near 2^-22 + |t| 2^-24, below every result's rounding but fp32's.  A gate below 2^-126 (SiLU: z
// below -87) may come out as 0: the reciprocal gives no subnormal numbers; the value is then off by less than 10^-35.
enum Act { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGelu1 = 1.5957691216057308f, kGelu3 = 0.07135481282553447f;     // 2 c and 2 c 0.044715, c = sqrt(2 / pi)

__device__ __forceinline__ float sigmoid_of_neg_log2(float t) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t)); }
// (the square is held below 10^30: times a slope that is 0 there an infinity would make a NaN)
__device__ __forceinline__ float square_bounded(float z) { return __builtin_fminf(z * z, 1e30f); }
__device__ __forceinline__ float gelu_gate(float z) {
    return sigmoid_of_neg_log2(z * __builtin_fmaf(square_bounded(z), -kGelu3 * kLog2e, -kGelu1 * kLog2e));
}
__device__ __forceinline__ float silu_gate(float z) { return sigmoid_of_neg_log2(z * -kLog2e); }

// N values through the activation; `act` is the same for the whole wave
template <int N>
__device__ __forceinline__ void activate(float (&z)[N], int act) {
    if (act == kActSilu) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] *= silu_gate(z[i]);
    } else if (act == kActGelu) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] *= gelu_gate(z[i]);
    } else if (act == kActRelu) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i];
    }
}
// value and slope
template <int N>
__device__ __forceinline__ void activate_slope(const float (&z)[N], float (&a)[N], float (&slope)[N], int act) {
    if (act == kActSilu) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float s = silu_gate(z[i]);
            a[i] = z[i] * s;
            slope[i] = __builtin_fmaf(a[i], 1.0f - s, s);
        }
    } else if (act == kActGelu) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float s = gelu_gate(z[i]);
            a[i] = z[i] * s;
            slope[i] = __builtin_fmaf(a[i] * (1.0f - s), __builtin_fmaf(square_bounded(z[i]), 3.0f * kGelu3, kGelu1), s);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            a[i] = act == kActRelu && z[i] < 0.0f ? 0.0f : z[i];
            slope[i] = act == kActRelu && z[i] <= 0.0f ? 0.0f : 1.0f;
        }
    }
}

// sum over the 64 lanes, the same bits in every lane (a butterfly: partners form the same sum)
__device__ __forceinline__ float wave_sum(float v) {
    v += lane_xor<1>(v);
    v += lane_xor<2>(v);
    v += lane_xor<4>(v);
    v += __shfl_xor(v, 8);
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    return v;
}

// value of lane (l ^ XOR) of a double
template <int XOR>
__device__ __forceinline__ double lane_xor64(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = f2u(lane_xor<XOR>(u2f((uint32_t)u))), hi = f2u(lane_xor<XOR>(u2f((uint32_t)(u >> 32))));
    return __builtin_bit_cast(double, (uint64_t)lo | ((uint64_t)hi << 32));
}
// wave_sum of a double
__device__ __forceinline__ double wave_sum64(double s) {
    s += lane_xor64<1>(s);
    s += lane_xor64<2>(s);
    s += lane_xor64<4>(s);
    s += __shfl_xor(s, 8);
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    return s;
}

}  // namespace quartet
