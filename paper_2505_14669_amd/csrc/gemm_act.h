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

// A matrix's part of a wave's tile: a buffer resource that ends with the matrix's last element in these rows, so rows past the matrix are neither read
// nor written without a predicate; a lane whose columns lie outside takes an offset that no resource reaches.
struct ActTile {
    __amdgpu_buffer_rsrc_t res;
    uint32_t row_bytes;
};
__device__ __forceinline__ ActTile act_tile(const void* p, uint32_t size, uint32_t ld, uint32_t row_base, uint32_t rows, uint32_t n) {
    const size_t row_bytes = (size_t)ld * size;
    return {make_rsrc(static_cast<const uint8_t*>(p) + row_base * row_bytes, p && rows ? (rows - 1u) * (uint32_t)row_bytes + n * size : 0u), (uint32_t)row_bytes};
}
enum ActExtra { kExtraNone, kExtraOne, kExtraFp32, kExtraBoth };
constexpr int kThroughL2 = 16;      // cache policy of a buffer store: sc1, as store_through16

// Epilogue of the streaming kernels for quartet_mxfp4_gemm_act: the wave's accumulator tile leaves in passes of eight rows through its scratch as in
// store_tile_rows8 (same image in LDS, same chunk of four columns of every 32-column slice in a lane), and every chunk takes its bias, goes through the
// activation and meets its gate and residual.  Those are loaded DEPTH passes ahead, in the order of the passes between their stores: the
// vector-memory counter retires in order, so what a pass waits for is older than the stores of the passes in between.  Loads and stores here are builtins:
// the compiler counts them and waits for the right ones (it would wait for every store of the preceding passes if it did not see them).  The ring's loads
// are older than all of it.
// Whether every store was issued: TM * 4 * TN of results, what the kernels' first barrier behind a tile counts on.
// EXTRA: what a chunk meets, so that no register is kept for what does not exist: nothing, one bf16 matrix (gate or residual), an fp32 residual, or a gate and a
// residual of either type.
template <int TM, int TN, int EXTRA, int DEPTH, bool OUT_BF16, typename ACC, int AM, int AN>
__device__ __forceinline__ bool store_tile_act(ACC (&acc)[AM][AN], float* wbuf, void* d, uint32_t ldd, float alpha, uint32_t row_base, uint32_t col_base,
                                               uint32_t m, uint32_t n, uint32_t lane, const GemmActArgs& e) {
    static_assert(TN == 2 || TN == 4, "the slice swap of odd rows pairs the slices up");
    constexpr bool A32 = sizeof(ACC) == sizeof(v16f);
    static_assert(AM == (A32 ? TM : 2 * TM) && AN == (A32 ? TN : 2 * TN), "the accumulators must make up the tile");
    constexpr uint32_t PASSES = TM * 4, W = TN * 32;
    const uint32_t sub = lane >> 3, c = lane & 7u;
    const uint32_t lhalf = lane >> 5, wq = lane >> 4;
    float* wr = wbuf + lhalf * 4u * W + (lane & 31u);
    float* wr_even = wbuf + 2u * wq * W + (lane & 15u) + (wq & 1u) * 16u;
    float* wr_odd = wbuf + 2u * wq * W + (lane & 15u) - (wq & 1u) * 16u;
    const uint32_t rswz = A32 ? (sub ^ (sub >> 2)) & 1u : sub & 1u;
    const float* rd = wbuf + sub * W + 4u * (A32 ? c : c ^ (((sub >> 1) & 1u) * 4u));
    const uint32_t row_in_tile = A32 ? sub : 4u * (sub >> 1) + (sub & 1u);
    auto row_step = [](uint32_t p) { return A32 ? p * 8u : (p >> 1) * 16u + (p & 1u) * 2u; };
    auto write_pass = [&](uint32_t p) __attribute__((always_inline)) {
        if constexpr (A32) {
#pragma unroll
            for (uint32_t j = 0; j < TN; ++j)
#pragma unroll
                for (uint32_t t = 0; t < 4; ++t) wr[t * W + ((j ^ ((t & 1u) ^ lhalf)) * 32u)] = acc[p >> 2][j][(p & 3u) * 4u + t];
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 2u * TN; ++j)
#pragma unroll
                for (uint32_t t = 0; t < 2; ++t) ((j & 1u) ? wr_odd : wr_even)[t * W + (j ^ (2u * t)) * 16u] = acc[p >> 1][j][(p & 1u) * 2u + t];
        }
    };
    const bool whole = (n & 3u) == 0u && act_wide(e, ldd);      // wave-uniform: every chunk lies inside or outside, at a multiple of its size
    if (!whole) {
        // one pass after the other, the code of one: only the accumulators have to be named
#pragma unroll 1
        for (uint32_t p = 0; p < PASSES; ++p) {
#pragma unroll
            for (uint32_t named = 0; named < PASSES; ++named)
                if (named == p) write_pass(named);
            float vv[TN][4];
#pragma unroll
            for (uint32_t j = 0; j < TN; ++j) {
                const float4 t = *reinterpret_cast<const float4*>(&rd[(j ^ rswz) * 32u]);
                vv[j][0] = t.x; vv[j][1] = t.y; vv[j][2] = t.z; vv[j][3] = t.w;
            }
            const uint32_t row = row_base + row_in_tile + row_step(p);
#pragma unroll
            for (uint32_t j = 0; j < TN; ++j) {
                const uint32_t col = col_base + j * 32u + 4u * c;
                ActChunk extra;
                float bias[4];
                load_act_chunk(extra, e, row, col, m, n, false);
                load_bias(bias, e, col, n);
#pragma unroll
                for (uint32_t t = 0; t < 4; ++t) vv[j][t] = vv[j][t] * alpha + bias[t];
                if (e.pre) store_act_chunk<true>(e.pre, e.ldpre, row, col, m, n, false, vv[j]);
                activate(vv[j], e.act);
                combine_act_chunk(vv[j], extra, e);
                store_act_chunk<OUT_BF16>(d, ldd, row, col, m, n, false, vv[j]);
            }
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0), said here: otherwise the compiler, not sure of every branch's loads, says it in the main loop
        return false;
    }
    constexpr uint32_t SD = OUT_BF16 ? 2u : 4u;
    const uint32_t rows = row_base < m ? (m - row_base < TM * 32u ? m - row_base : TM * 32u) : 0u;
    // EXTRA = one bf16 matrix: `one` of them, otherwise the residual and the gate
    const bool gates = EXTRA == kExtraOne && e.mul != nullptr;
    const uint32_t sr = e.res_kind == 2 ? 4u : 2u;
    const ActTile td = act_tile(d, SD, ldd, row_base, rows, n), tp = act_tile(e.pre, 2u, e.ldpre, row_base, rows, n);
    const ActTile tr = act_tile(gates ? e.mul : e.residual, gates ? 2u : sr, gates ? e.ldmul : e.ldres, row_base, rows, n);
    const ActTile tm = act_tile(EXTRA == kExtraBoth ? e.mul : nullptr, 2u, e.ldmul, row_base, rows, n);
    uint32_t at[TN];                                             // the lane's columns
    float bias[TN][4];
#pragma unroll
    for (uint32_t j = 0; j < TN; ++j) at[j] = col_base + j * 32u + 4u * c;
    // byte offset of chunk j in the lane's row of pass 0
    auto place = [&](uint32_t j, uint32_t size, uint32_t row_bytes) { return at[j] < n ? row_in_tile * row_bytes + at[j] * size : kOutOfRange; };
    if (e.bias_kind == 2) {
        const __amdgpu_buffer_rsrc_t b = make_rsrc(e.bias, n * 4u);
#pragma unroll
        for (uint32_t j = 0; j < TN; ++j) {
            const v4u_t t = __builtin_amdgcn_raw_buffer_load_b128(b, (int)(at[j] * 4u), 0, 0);
            bias[j][0] = u2f(t.x); bias[j][1] = u2f(t.y); bias[j][2] = u2f(t.z); bias[j][3] = u2f(t.w);
        }
    } else {
        const __amdgpu_buffer_rsrc_t b = make_rsrc(e.bias, e.bias_kind ? n * 2u : 0u);
#pragma unroll
        for (uint32_t j = 0; j < TN; ++j) {
            const v2u_t t = __builtin_amdgcn_raw_buffer_load_b64(b, (int)(at[j] * 2u), 0, 0);
            bias[j][0] = bf16_lo(t.x); bias[j][1] = bf16_hi(t.x); bias[j][2] = bf16_lo(t.y); bias[j][3] = bf16_hi(t.y);
        }
    }
    constexpr int D = EXTRA == kExtraNone ? 1 : DEPTH;
    v2u_t one[D][TN], gate[D][TN];
    v4u_t full[D][TN];
    auto load_pass = [&](uint32_t p) __attribute__((always_inline)) {
        const uint32_t s = p % D;
        const int soff = (int)(row_step(p) * tr.row_bytes);
#pragma unroll
        for (uint32_t j = 0; j < TN; ++j) {
            if (EXTRA == kExtraOne) one[s][j] = __builtin_amdgcn_raw_buffer_load_b64(tr.res, (int)place(j, 2u, tr.row_bytes), soff, 0);
            if (EXTRA == kExtraFp32) full[s][j] = __builtin_amdgcn_raw_buffer_load_b128(tr.res, (int)place(j, 4u, tr.row_bytes), soff, 0);
            if (EXTRA == kExtraBoth) {
                if (e.res_kind == 2) {
                    full[s][j] = __builtin_amdgcn_raw_buffer_load_b128(tr.res, (int)place(j, 4u, tr.row_bytes), soff, 0);
                } else {
                    const v2u_t t = __builtin_amdgcn_raw_buffer_load_b64(tr.res, (int)place(j, 2u, tr.row_bytes), soff, 0);
                    full[s][j].x = t.x; full[s][j].y = t.y;
                }
                gate[s][j] = __builtin_amdgcn_raw_buffer_load_b64(tm.res, (int)place(j, 2u, tm.row_bytes), (int)(row_step(p) * tm.row_bytes), 0);
            }
        }
    };
    auto combine = [&](uint32_t p, float* v) __attribute__((always_inline)) {      // v: the pass's 4 TN values
        const uint32_t s = p % D;
        if (EXTRA == kExtraOne) {
            if (gates) {
#pragma unroll
                for (uint32_t j = 0; j < TN; ++j, v += 4) {
                    v[0] *= bf16_lo(one[s][j].x); v[1] *= bf16_hi(one[s][j].x); v[2] *= bf16_lo(one[s][j].y); v[3] *= bf16_hi(one[s][j].y);
                }
            } else {
#pragma unroll
                for (uint32_t j = 0; j < TN; ++j, v += 4) {
                    v[0] += bf16_lo(one[s][j].x); v[1] += bf16_hi(one[s][j].x); v[2] += bf16_lo(one[s][j].y); v[3] += bf16_hi(one[s][j].y);
                }
            }
        }
        if (EXTRA == kExtraFp32) {
#pragma unroll
            for (uint32_t j = 0; j < TN; ++j, v += 4) {
                v[0] += u2f(full[s][j].x); v[1] += u2f(full[s][j].y); v[2] += u2f(full[s][j].z); v[3] += u2f(full[s][j].w);
            }
        }
        if (EXTRA == kExtraBoth) {
#pragma unroll
            for (uint32_t j = 0; j < TN; ++j, v += 4) combine_act_chunk(reinterpret_cast<float (&)[4]>(*v), ActChunk{full[s][j], gate[s][j]}, e);
        }
    };
#pragma unroll
    for (uint32_t p = 0; p < D && p < PASSES; ++p) load_pass(p);
    write_pass(0u);
#pragma unroll
    for (uint32_t p = 0; p < PASSES; ++p) {
        float vv[TN * 4];
#pragma unroll
        for (uint32_t j = 0; j < TN; ++j) {
            const float4 t = *reinterpret_cast<const float4*>(&rd[(j ^ rswz) * 32u]);
            vv[4 * j] = t.x; vv[4 * j + 1] = t.y; vv[4 * j + 2] = t.z; vv[4 * j + 3] = t.w;
        }
        if (p + 1u < PASSES) write_pass(p + 1u);      // behind the reads in the wave's LDS queue
#pragma unroll
        for (uint32_t t = 0; t < 4u * TN; ++t) vv[t] = vv[t] * alpha + bias[t >> 2][t & 3u];
        if (e.pre) {
#pragma unroll
            for (uint32_t j = 0; j < TN; ++j) {
                const v2u_t z = {bf16_pack2(vv[4 * j], vv[4 * j + 1]), bf16_pack2(vv[4 * j + 2], vv[4 * j + 3])};
                __builtin_amdgcn_raw_buffer_store_b64(z, tp.res, (int)place(j, 2u, tp.row_bytes), (int)(row_step(p) * tp.row_bytes), kThroughL2);
            }
        }
        activate(vv, e.act);
        combine(p, vv);
        if (p + D < PASSES) load_pass(p + D);
        if (EXTRA != kExtraNone && p + 1u == PASSES) {       // nothing is left of the loads: as above, and free (D passes' stores are younger than the last load)
            constexpr uint32_t younger = D * TN < 63 ? D * TN : 63;
            __builtin_amdgcn_s_waitcnt(0x0F70u | (younger & 15u) | ((younger >> 4) << 14));
        }
#pragma unroll
        for (uint32_t j = 0; j < TN; ++j) {
            const int voff = (int)place(j, SD, td.row_bytes), soff = (int)(row_step(p) * td.row_bytes);
            if (OUT_BF16) {
                const v2u_t o = {bf16_pack2(vv[4 * j], vv[4 * j + 1]), bf16_pack2(vv[4 * j + 2], vv[4 * j + 3])};
                __builtin_amdgcn_raw_buffer_store_b64(o, td.res, voff, soff, kThroughL2);
            } else {
                v4u_t o = {f2u(vv[4 * j]), f2u(vv[4 * j + 1]), f2u(vv[4 * j + 2]), f2u(vv[4 * j + 3])};
                __builtin_amdgcn_raw_buffer_store_b128(o, td.res, voff, soff, kThroughL2);
                asm volatile("s_nop 1" : "+v"(o));      // two wait states before the data's registers are written again, as behind every wide store here
            }
        }
    }
    return true;
}

}  // namespace quartet
