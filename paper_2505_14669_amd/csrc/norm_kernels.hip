// Root-mean-square norm of the residual stream, into bf16 or straight into a linear layer's MX operand, and its backward pass.
// Bound by memory: every value is read once, held in registers across the row's sum, and every result written once.
#include "block_common.h"
#include "block_launchers.h"

namespace quartet {

namespace {

constexpr int kFmtNone = 0, kFmtMx4 = 1, kFmtMx8 = 2;
typedef short v2s_t __attribute__((ext_vector_type(2)));

// four values, |v| <= 448, -> four E4M3 bytes, round to nearest even
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    v2s_t w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, 1.0f, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, 1.0f, true);
    return (uint32_t)(uint16_t)w[0] | ((uint32_t)(uint16_t)w[1] << 16);
}
// eight values -> eight E2M1 codes of v / scale, round to nearest even, saturating
__device__ __forceinline__ uint32_t e2m1x8(const float* v, float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    return c;
}

// One row of a matrix as a buffer resource over its whole chunks of eight values: a load past them gives zeros, a store past them is dropped, so
// the lanes beyond the row need no branches.  The n % 8 values behind the last whole chunk go one by one.
struct Row {
    __amdgpu_buffer_rsrc_t res;
    uint8_t* tail;            // the values behind the whole chunks
    uint32_t bytes;           // per value
};
__device__ __forceinline__ Row row_of(const void* p, bool f32, size_t at, uint32_t n) {     // n = 0: no row
    const uint32_t bytes = f32 ? 4u : 2u;
    uint8_t* base = static_cast<uint8_t*>(const_cast<void*>(p)) + at * bytes;
    return {__builtin_amdgcn_make_buffer_rsrc(base, 0, (n & ~7u) * bytes, 0x00020000), base + (size_t)(n & ~7u) * bytes, bytes};
}
__device__ __forceinline__ uint4 u4(v4u_t v) { return make_uint4(v.x, v.y, v.z, v.w); }

// eight consecutive values as they lie in memory
struct Raw8 {
    uint4 lo, hi;      // bf16: lo
};
constexpr int kNonTemporal = 2;      // cache policy of a buffer access
// PAST: past the caches
template <bool PAST = false>
__device__ __forceinline__ void load8(Raw8& r, const Row& row, bool f32, uint32_t col) {
    constexpr int policy = PAST ? kNonTemporal : 0;
    if (f32) {
        r.lo = u4(__builtin_amdgcn_raw_buffer_load_b128(row.res, (int)(col * 4u), 0, policy));
        r.hi = u4(__builtin_amdgcn_raw_buffer_load_b128(row.res, (int)(col * 4u + 16u), 0, policy));
    } else {
        r.lo = u4(__builtin_amdgcn_raw_buffer_load_b128(row.res, (int)(col * 2u), 0, policy));
    }
}
// the lane whose columns are the row's last, incomplete chunk: `left` = 1 .. 7 values (other lanes: 0)
__device__ __forceinline__ void load_tail(Raw8& r, const Row& row, bool f32, uint32_t left) {
    if (left == 0u) return;
    uint32_t w[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
#pragma unroll
    for (uint32_t i = 0; i < 7; ++i)
        if (i < left) {
            if (f32) w[i] = reinterpret_cast<const uint32_t*>(row.tail)[i];
            else w[i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(row.tail)[i] << (16u * (i & 1u));
        }
    r.lo = make_uint4(w[0], w[1], w[2], w[3]);
    r.hi = make_uint4(w[4], w[5], w[6], w[7]);
}
__device__ __forceinline__ void values8(const Raw8& r, bool f32, float* v) {
    if (f32) {
        v[0] = u2f(r.lo.x); v[1] = u2f(r.lo.y); v[2] = u2f(r.lo.z); v[3] = u2f(r.lo.w);
        v[4] = u2f(r.hi.x); v[5] = u2f(r.hi.y); v[6] = u2f(r.hi.z); v[7] = u2f(r.hi.w);
    } else {
        unpack8(r.lo, v);
    }
}
template <bool PAST>
__device__ __forceinline__ void store8(const Row& row, bool f32, uint32_t col, uint32_t tail, const float* v) {
    constexpr int policy = PAST ? kNonTemporal : 0;
    if (f32) {
        const v4u_t lo = {f2u(v[0]), f2u(v[1]), f2u(v[2]), f2u(v[3])}, hi = {f2u(v[4]), f2u(v[5]), f2u(v[6]), f2u(v[7])};
        __builtin_amdgcn_raw_buffer_store_b128(lo, row.res, (int)(col * 4u), 0, policy);
        __builtin_amdgcn_raw_buffer_store_b128(hi, row.res, (int)(col * 4u + 16u), 0, policy);
    } else {
        const uint4 q = pack8(v);
        const v4u_t d = {q.x, q.y, q.z, q.w};
        __builtin_amdgcn_raw_buffer_store_b128(d, row.res, (int)(col * 2u), 0, policy);
    }
    if (tail == 0u) return;
#pragma unroll
    for (uint32_t i = 0; i < 7; ++i)
        if (i < tail) {
            if (f32) reinterpret_cast<float*>(row.tail)[i] = v[i];
            else reinterpret_cast<uint16_t*>(row.tail)[i] = bf16_of(v[i]);
        }
}
// how many values the lane with columns col .. col + 7 has of the row's incomplete chunk
__device__ __forceinline__ uint32_t tail_of(uint32_t col, uint32_t n) { return col == (n & ~7u) ? n & 7u : 0u; }

// The scale bytes of a row's 256 columns (one per four lanes, 32 lanes) as the two dwords of its scale tile: lanes 0 and 4 of the 32 hold them afterwards.
__device__ __forceinline__ uint32_t scale_dword(uint32_t b) {
    uint32_t w = b | ((uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0x108 /* row_shl:8 */, 0xF, 0xF, true) << 8);
    return w | ((uint32_t)__shfl_down((int)w, 16) << 16);
}

// Eight columns of one row in each lane; the WPR waves of a row meet in LDS.
// sum of `part` over the row's lanes, the same bits in all of them
template <int WPR>
__device__ __forceinline__ float row_sum(float part, float* meet, uint32_t slot, uint32_t sub, uint32_t lane) {
    float s = wave_sum(part);
    if (WPR == 1) return s;
    if (lane == 0) meet[slot * WPR + sub] = s;
    __syncthreads();
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < WPR; ++w) s += meet[slot * WPR + w];
    return s;
}

// Blocks go to the XCDs in turn.  The first row of block b where the 32 rows of a scale tile are to meet in one L2: tiles t, t + 8, ... on XCD t % 8.
template <uint32_t RPB>
__device__ __forceinline__ uint32_t tile_row(uint32_t b) {
    constexpr uint32_t PER = 32u / RPB;                                  // blocks of a tile
    const uint32_t i = b >> 3;
    return ((i / PER) * 8u + (b & 7u)) * 32u + (i % PER) * RPB;
}

// The row's squares and their sum in 64 bits (no value of fp32 has a square outside them): the statistic is rounded once, to fp32.  Rounding of the values behind
// it still moves codes next to the middle of two; against the exact operand 25 of 128.6 M E2M1 codes and 370 of 671 M E4M3 codes fall otherwise (with everything in
// 32 bits, in torch's order, 70 and 488).  Beside squares in 32 bits it costs 0.5 % (16384 x 4096 into MXFP8 84.0 us for 83.0, into bf16 93.3 for 93.2).
template <int WPR>
__device__ __forceinline__ double row_sum64(double s, double* meet, uint32_t slot, uint32_t sub, uint32_t lane) {
    s = wave_sum64(s);
    if (WPR == 1) return s;
    if (lane == 0) meet[slot * WPR + sub] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < WPR; ++w) s += meet[slot * WPR + w];
    return s;
}
// 1 / sqrt(x) from the hardware's 64-bit estimate and one Newton step, rounded once (0, infinities and NaN as the estimate has them)
__device__ __forceinline__ float rsqrt_once(double x) {
    const double r = __builtin_amdgcn_rsq(x), better = r * (1.5 - 0.5 * x * r * r);
    return (float)(better == better ? better : r);
}

// A row belongs to WPR waves; lane l of wave `sub` of a row holds the columns 8 ((j WPR + sub) 64 + l) .. + 7 of chunk j < CH.
template <int WPR, int CH, int FMT>
__global__ void __launch_bounds__(WPR < 4 ? 256 : 64 * WPR)
rmsnorm_fwd_kernel(NormFwdArgs a) {
    constexpr uint32_t THREADS = WPR < 4 ? 256 : 64 * WPR, RPB = THREADS / 64 / WPR;
    __shared__ double meet[THREADS / 64];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), block = blockIdx.y * gridDim.x + blockIdx.x;
    const uint32_t slot = wave / WPR, sub = wave % WPR, row = a.by_tile ? tile_row<RPB>(block) + slot : block * RPB + slot;
    const bool in = row < a.rows;
    const uint32_t n = a.n;
    const uint32_t n_in = in ? n : 0u;
    const Row x_row = row_of(a.x, a.x_f32, (size_t)row * a.ldx, n_in), w_row = row_of(a.weight, a.w_f32, 0, n);
    const Row r_row = row_of(a.residual, a.h_f32, (size_t)row * a.ldres, a.residual ? n_in : 0u);
    const Row h_row = row_of(a.h, a.h_f32, (size_t)row * a.ldh, a.h ? n_in : 0u), y_row = row_of(a.y, false, (size_t)row * a.ldy, a.y ? n_in : 0u);
    Raw8 rx[CH], rr[CH], rw[CH];
    uint32_t col[CH], tail[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        col[j] = (((uint32_t)j * WPR + sub) * 64u + lane) * 8u;
        tail[j] = in ? tail_of(col[j], n) : 0u;
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) load8(rx[j], x_row, a.x_f32, col[j]);
    if (a.residual) {
#pragma unroll
        for (int j = 0; j < CH; ++j) load8(rr[j], r_row, a.h_f32, col[j]);
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) load8(rw[j], w_row, a.w_f32, col[j]);
    if ((n & 7u) != 0u) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            load_tail(rx[j], x_row, a.x_f32, tail[j]);
            if (a.residual) load_tail(rr[j], r_row, a.h_f32, tail[j]);
            load_tail(rw[j], w_row, a.w_f32, tail[j]);
        }
    }
    float v[CH][8];
    double part = 0.0;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        values8(rx[j], a.x_f32, v[j]);
        if (a.residual) {
            float r[8];
            values8(rr[j], a.h_f32, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] += r[i];
            if (!a.h_f32) {                   // the norm reads what the stream holds
                const uint4 q = pack8(v[j]);
                unpack8(q, v[j]);
            }
            if (a.h) store8<true>(h_row, a.h_f32, col[j], tail[j], v[j]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) part = __builtin_fma((double)v[j][i], (double)v[j][i], part);
    }
    const float rstd = rsqrt_once(row_sum64<WPR>(part, meet, slot, sub, lane) * a.inv_n + (double)a.eps);
    if (a.rstd && in && sub == 0u && lane == 0u) a.rstd[row] = rstd;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        float w[8];
        values8(rw[j], a.w_f32, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = v[j][i] * rstd * w[i];
        if (a.y) {
            if (a.past) store8<true>(y_row, false, col[j], tail[j], v[j]);
            else store8<false>(y_row, false, col[j], tail[j], v[j]);
        }
        if (FMT == kFmtNone) continue;
        // a group is four consecutive lanes; n is a multiple of 32, so it exists as a whole or not at all
        const bool there = in && col[j] < n;
        const uint32_t g = col[j] >> 5, kqs = (n + 255u) >> 8, at32 = lane & 31u;
        auto store_scale = [&](uint32_t b) __attribute__((always_inline)) {
            const uint32_t w = scale_dword(b), h = at32 >> 2;            // lanes 0 and 4: groups h, 2 + h, 4 + h, 6 + h of the K-quad
            if (!there || (at32 != 0u && at32 != 4u)) return;
            uint8_t* dst = a.scales + scale_tile_offset(row, g, kqs);
            if ((n & 255u) == 0u || (col[j] | 255u) < n) {
                *reinterpret_cast<uint32_t*>(dst) = w;
            } else {                                                     // a ragged last K-quad: bytes of groups past n are not written
                for (uint32_t i = 0; i < 4u; ++i)
                    if ((g & ~7u) + 2u * i + h < (n >> 5)) dst[i] = (uint8_t)(w >> (8u * i));
            }
        };
        if (FMT == kFmtMx8) {
            float mx = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) mx = __builtin_fmaxf(mx, __builtin_fabsf(v[j][i]));
            mx = __builtin_fmaxf(mx, lane_xor<1>(mx));
            mx = __builtin_fmaxf(mx, lane_xor<2>(mx));
            const uint32_t E = (f2u(mx) >> 23) & 0xFFu, b = E >= 8u ? E - 8u : 0u;
            const float mult = u2f((254u - b) << 23);
            float q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = __builtin_amdgcn_fmed3f(v[j][i] * mult, -448.0f, 448.0f);
            if (there) {
                const v2u_t c = {e4m3x4(q[0], q[1], q[2], q[3]), e4m3x4(q[4], q[5], q[6], q[7])};
                v2u_t* dst = reinterpret_cast<v2u_t*>(a.codes + (size_t)row * n + col[j]);
                if (a.past) __builtin_nontemporal_store(c, dst);
                else *dst = c;
            }
            store_scale(b);
        } else {
            // 32-point transform: strides 1, 2, 4 in the lane, 8 and 16 between lanes (own * t + partner: a + b below, a - b above)
#pragma unroll
            for (int h = 1; h < 8; h <<= 1)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if ((i & h) == 0) {
                        const float p = v[j][i], q = v[j][i + h];
                        v[j][i] = p + q;
                        v[j][i + h] = p - q;
                    }
            const float t8 = (lane & 1u) ? -1.0f : 1.0f, t16 = (lane & 2u) ? -1.0f : 1.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = __builtin_fmaf(v[j][i], t8, lane_xor<1>(v[j][i]));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = __builtin_fmaf(v[j][i], t16, lane_xor<2>(v[j][i]));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] *= kInvSqrt32;
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = v[j][i] * v[j][i];
            float sq = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));      // the pairwise tree of quartet_quant_fwd
            sq += lane_xor<1>(sq);
            sq += lane_xor<2>(sq);
            const uint32_t E = (f2u(sq) >> 23) & 0xFFu;
            const int e = E == 0u ? 0 : ((int)E - 133) >> 1;
            const uint32_t b = (uint32_t)(e + 127);
            const float scale = u2f(b << 23), thr = u2f(0x40C00000u + ((uint32_t)e << 23));
            uint32_t m = 0u;
#pragma unroll
            for (int i = 7; i >= 0; --i) m = (m << 1) | (__builtin_fabsf(v[j][i]) <= thr ? 1u : 0u);
            m <<= 8u * (lane & 3u);
            m |= f2u(lane_xor<1>(u2f(m)));
            m |= f2u(lane_xor<2>(u2f(m)));
            if (there) {
                uint32_t* dst = reinterpret_cast<uint32_t*>(a.codes + (size_t)row * (n >> 1) + (col[j] >> 1));
                if (a.past) store_stream4(dst, e2m1x8(v[j], scale));
                else *dst = e2m1x8(v[j], scale);
                if (a.mask && (lane & 3u) == 0u) a.mask[(size_t)row * (n >> 5) + g] = m;
            }
            store_scale(b);
        }
    }
}

// Backward: a block goes through the rows blockIdx.x RPB + slot, + gridDim.x RPB, ...; the weight and its gradient's partial sums stay in
// registers, the latter meet in LDS and go to the workspace, one row of n floats per block.
// With the next row's loads ahead of the reduction, against one row at a time (us): 16384 x 4096 bf16 111 -> 94, 4096 x 8192 57 -> 40, 8192 x 2048 fp32 59 -> 56.
// PAST: more is read than the memory-side cache holds.
template <int WPR, int CH, bool PAST>
__global__ void __launch_bounds__(WPR < 4 ? 256 : 64 * WPR)
rmsnorm_bwd_kernel(NormBwdArgs a) {
    // Rows wider than 8192: 1024 threads leave 128 registers each, too few for the values of one row beside the sums: the compiler spills 84 bytes a lane up to
    // 16384 columns and 676 beyond (us, and the bytes at 6.2 TB/s: 4096 x 11008 bf16 120 / 58, 4096 x 16384 145 / 87, 2048 x 32768 591 / 87; 4096 x 8192 54.6 / 43.3).
    constexpr bool AHEAD = WPR < 16 || CH == 1;
    constexpr uint32_t THREADS = WPR < 4 ? 256 : 64 * WPR, RPB = THREADS / 64 / WPR;
    __shared__ float meet[2][THREADS / 64];
    __shared__ float4 join[RPB > 1 ? THREADS * 2 : 1];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t slot = wave / WPR, sub = wave % WPR, n = a.n;
    uint32_t col[CH];
    float w[CH][8], dw[CH][8];
    const Row w_row = row_of(a.weight, a.w_f32, 0, n);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        col[j] = (((uint32_t)j * WPR + sub) * 64u + lane) * 8u;
        Raw8 r;
        load8(r, w_row, a.w_f32, col[j]);
        if ((n & 7u) != 0u) load_tail(r, w_row, a.w_f32, tail_of(col[j], n));
        values8(r, a.w_f32, w[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
    }
    // the next row's values are on their way while this one's sum is formed and its results leave
    Raw8 rdy[CH], rh[CH], rd[CH];
    float rstd = 0.0f;
    auto load_row = [&](uint32_t row) __attribute__((always_inline)) {
        const bool in = row < a.rows;
        const uint32_t n_in = in ? n : 0u;
        const Row dy_row = row_of(a.dy, false, (size_t)row * a.lddy, n_in), h_row = row_of(a.h, a.h_f32, (size_t)row * a.ldh, n_in);
        const Row dh_row = row_of(a.dh, a.h_f32, (size_t)row * a.lddh, a.dh ? n_in : 0u);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            load8<PAST>(rdy[j], dy_row, false, col[j]);
            load8<PAST>(rh[j], h_row, a.h_f32, col[j]);
        }
        if (a.dh) {
#pragma unroll
            for (int j = 0; j < CH; ++j) load8<PAST>(rd[j], dh_row, a.h_f32, col[j]);
        }
        if ((n & 7u) != 0u) {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const uint32_t tail = in ? tail_of(col[j], n) : 0u;
                load_tail(rdy[j], dy_row, false, tail);
                load_tail(rh[j], h_row, a.h_f32, tail);
                if (a.dh) load_tail(rd[j], dh_row, a.h_f32, tail);
            }
        }
        rstd = in ? a.rstd[row] : 0.0f;
    };
    uint32_t turn = 0u;
    if (AHEAD) load_row(blockIdx.x * RPB + slot);
    for (uint32_t row0 = blockIdx.x * RPB; row0 < a.rows; row0 += gridDim.x * RPB, turn ^= 1u) {     // the same trips for every wave: they meet
        const uint32_t row = row0 + slot;
        const bool in = row < a.rows;
        const uint32_t n_in = in ? n : 0u;
        if (!AHEAD) load_row(row);
        const float r = rstd;
        float dy[CH][8], h[CH][8], add[CH][8];
        float part = 0.0f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            values8(rdy[j], false, dy[j]);
            values8(rh[j], a.h_f32, h[j]);
            if (a.dh) values8(rd[j], a.h_f32, add[j]);
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[j][i] = __builtin_fmaf(dy[j][i] * r, h[j][i], dw[j][i]);
                dy[j][i] *= w[j][i];
                t[i] = dy[j][i] * h[j][i];
            }
            part += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
        }
        if (AHEAD) load_row(row + gridDim.x * RPB);
        const float c = row_sum<WPR>(part, meet[turn], slot, sub, lane) / (float)n * r * r;
        if (a.dx) {
            const Row dx_row = row_of(a.dx, a.h_f32, (size_t)row * a.lddx, n_in), dx16_row = row_of(a.dx16, false, (size_t)row * a.lddx16, a.dx16 ? n_in : 0u);
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const uint32_t tail = in ? tail_of(col[j], n) : 0u;
                float d[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = r * (dy[j][i] - h[j][i] * c);
                if (a.dh) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] += add[j][i];
                }
                store8<PAST>(dx_row, a.h_f32, col[j], tail, d);
                if (a.dx16) store8<PAST>(dx16_row, false, col[j], tail, d);
            }
        }
    }
    if (!a.partial) return;
    const uint32_t pitch = (n + 7u) & ~7u;             // whole chunks
    const Row p_row = row_of(a.partial, true, (size_t)blockIdx.x * pitch, pitch);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        if (RPB > 1) {
            __syncthreads();
            float4* mine = &join[(slot * WPR + sub) * 128u + lane];
            mine[0] = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
            mine[64] = make_float4(dw[j][4], dw[j][5], dw[j][6], dw[j][7]);
            __syncthreads();
            if (slot == 0u) {
#pragma unroll
                for (uint32_t o = 1; o < RPB; ++o) {
                    const float4 p = join[(o * WPR + sub) * 128u + lane], q = join[(o * WPR + sub) * 128u + 64u + lane];
                    dw[j][0] += p.x; dw[j][1] += p.y; dw[j][2] += p.z; dw[j][3] += p.w;
                    dw[j][4] += q.x; dw[j][5] += q.y; dw[j][6] += q.z; dw[j][7] += q.w;
                }
            }
        }
        if (slot == 0u) store8<false>(p_row, true, col[j], 0u, dw[j]);
    }
}

}  // namespace

// out[j] = sum over the rows of `partial` [rows x pitch].  A block takes 32 columns (a cache line of a row); thread t adds the rows t / 32, t / 32 + 32, ... of
// column t % 32, and the sums meet in a fixed order.  Blocks of 64 columns leave compute units without work (63 rows x 5632: 0.5 us more in all), of 16
// read half lines (1024 rows x 11008: 8 us more).
__global__ void __launch_bounds__(1024)
column_sum_kernel(const float* __restrict__ partial, uint32_t rows, uint32_t pitch, uint32_t n, float* __restrict__ out) {
    __shared__ float meet[16][32];
    const uint32_t c = blockIdx.x * 32u + (threadIdx.x & 31u);
    float s = 0.0f;
    if (c < n) {
#pragma unroll 8
        for (uint32_t r = threadIdx.x >> 5; r < rows; r += 32u) s += partial[(size_t)r * pitch + c];
    }
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 63u) < 32u) meet[threadIdx.x >> 6][threadIdx.x & 31u] = s;
    __syncthreads();
    if (threadIdx.x < 32u && c < n) {
        s = meet[0][threadIdx.x];
#pragma unroll
        for (uint32_t i = 1; i < 16u; ++i) s += meet[i][threadIdx.x];
        out[c] = s;
    }
}

hipError_t launch_column_sum(const float* partial, uint32_t rows, uint32_t pitch, uint32_t n, float* out, hipStream_t st) {
    hipLaunchKernelGGL(column_sum_kernel, dim3((n + 31u) / 32u), dim3(1024), 0, st, partial, rows, pitch, n, out);
    return hipGetLastError();
}

namespace {

// Waves per row and chunks per lane: a chunk each up to sixteen waves (8192 columns), then more chunks.  Many waves with little each hide the loads of one another
// and of the reductions (us, four chunks a lane / two / one, forward: 16384 x 4096 into MXFP8 90 / 81 / 79, into bf16 98 / 93 / 88, 2336 x 1376 into MXFP8 9.8 /
// 8.1 / 7.8; 4096 x 2048 18.1 / 16.0 / 16.0).
struct NormShape {
    int wpr, ch;
};
NormShape norm_shape(int64_t n) {
    const int64_t units = (n + 511) / 512;
    int wpr = 1, ch = 1;
    while (wpr < 16 && wpr < units) wpr *= 2;
    while ((int64_t)wpr * ch < units) ch *= 2;
    return {wpr, ch};
}
uint32_t rows_per_block(int wpr) { return wpr < 4 ? 4u / (uint32_t)wpr : 1u; }

template <int WPR, int CH>
void launch_fwd(NormFwdArgs a, int format, hipStream_t st) {
    const uint32_t rpb = rows_per_block(WPR), tiles = (a.rows + 31u) / 32u;
    a.by_tile = format != kFmtNone && a.rows >= 1024u;
    // results that the next kernel reads (bytes) go past the memory-side cache where it cannot hold them, codes as those of the quantizers
    const double values = (double)a.rows * a.n;
    a.past = format == kFmtNone ? values * 2.0 >= 256.0 * 1024.0 * 1024.0 : values * (format == kFmtMx8 ? 1.0 : 0.5) >= 64.0 * 1024.0 * 1024.0;
    a.inv_n = 1.0 / a.n;
    const uint32_t blocks = a.by_tile ? (tiles + 7u) / 8u * 8u * (32u / rpb) : (a.rows + rpb - 1u) / rpb, wide = blocks < (1u << 20) ? blocks : 1u << 20;
    const dim3 grid(wide, (blocks + wide - 1u) / wide), block(WPR < 4 ? 256 : 64 * WPR);      // (a dimension has fewer than 2^32 threads)
    if (format == kFmtMx4) hipLaunchKernelGGL((rmsnorm_fwd_kernel<WPR, CH, kFmtMx4>), grid, block, 0, st, a);
    else if (format == kFmtMx8) hipLaunchKernelGGL((rmsnorm_fwd_kernel<WPR, CH, kFmtMx8>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rmsnorm_fwd_kernel<WPR, CH, kFmtNone>), grid, block, 0, st, a);
}

// Blocks of a backward pass, each a row of partial sums of the weight's gradient.  Two waves per SIMD unit are enough with the next row's loads ahead (us, 256 / 512 /
// 1024 / 2048 blocks of four waves: 8192 x 2048 fp32 55.1 / 56.0 / 58.6 / 61.8, 2048 x 2048 bf16 12.4 / 11.3 / 12.0 / 15.9; a compute unit each for wider ones:
// 4096 x 8192 40.4 with 256 blocks of sixteen waves, 57.9 with 128).
uint32_t bwd_blocks(int64_t rows, int64_t n) {
    const int wpr = norm_shape(n).wpr;
    const int64_t all = (rows + rows_per_block(wpr) - 1) / rows_per_block(wpr), most = wpr <= 4 ? 512 : 256;
    return (uint32_t)(all < most ? all : most);
}

}  // namespace

#define NORM_SHAPES(X) X(1, 1) X(2, 1) X(4, 1) X(8, 1) X(16, 1) X(16, 2) X(16, 4)

hipError_t launch_rmsnorm_fwd(const NormFwdArgs& a, int format, hipStream_t st) {
    if (a.rows == 0) return hipSuccess;
    const NormShape s = norm_shape(a.n);
#define NORM_CASE(W, C) if (s.wpr == W && s.ch == C) launch_fwd<W, C>(a, format, st);
    NORM_SHAPES(NORM_CASE)
#undef NORM_CASE
    return hipGetLastError();
}

size_t rmsnorm_bwd_workspace(int64_t rows, int64_t n) { return (size_t)bwd_blocks(rows, n) * (size_t)((n + 7) / 8 * 8) * sizeof(float); }

hipError_t launch_rmsnorm_bwd(const NormBwdArgs& args, float* dweight, float* workspace, hipStream_t st) {
    if (args.rows == 0) {
        if (!dweight) return hipSuccess;
        return launch_column_sum(nullptr, 0u, 0u, args.n, dweight, st);
    }
    NormBwdArgs a = args;
    a.partial = dweight ? workspace : nullptr;
    const NormShape s = norm_shape(a.n);
    const uint32_t blocks = bwd_blocks(a.rows, a.n);
    // Where the memory-side cache cannot hold what is read, loads and results go past it: 16384 x 4096 bf16 (402 MB read) 94 -> 88 us; below, the results wait
    // in it for the layer that takes them (8192 x 2048 fp32, 168 MB read: 56.0 us with results past it, 53.9 without).
    const bool past = (double)a.rows * a.n * (2.0 + (a.h_f32 ? 4.0 : 2.0) * (a.dh ? 2.0 : 1.0)) >= 256.0 * 1024.0 * 1024.0;
#define NORM_CASE(W, C)                                                                                                                     \
    if (s.wpr == W && s.ch == C) {                                                                                                          \
        if (past) hipLaunchKernelGGL((rmsnorm_bwd_kernel<W, C, true>), dim3(blocks), dim3(W < 4 ? 256 : 64 * W), 0, st, a);                  \
        else hipLaunchKernelGGL((rmsnorm_bwd_kernel<W, C, false>), dim3(blocks), dim3(W < 4 ? 256 : 64 * W), 0, st, a);                      \
    }
    NORM_SHAPES(NORM_CASE)
#undef NORM_CASE
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !dweight) return e;
    return launch_column_sum(workspace, blocks, (a.n + 7u) & ~7u, a.n, dweight, st);
}

}  // namespace quartet
