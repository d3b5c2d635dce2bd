// Few rows times FB4 weights: y[r][n] = sum_c x[r][c] W[n][c].
//
// 16x16x32 bf16 MFMAs with 16 weight rows as the first operand and up to 16 rows of x as the second.  A weight's magnitude is an
// integer 0 .. 15 and its block's scale a power of two, so the decoded weight is a bf16 number: eight nibbles become two registers of
// E4M3 bytes by a byte permutation of the dialect's eight magnitudes (LDS, 8 bytes a dialect), and the converter to bf16 takes the
// block's scale along.  The channels of a product may come in any order as long as both operands have the same: a lane holds 32
// successive channels of one row (16 bytes of codes, one block's scale and dialect, or two's), eight for each of four MFMAs, and of
// eight the even ones come before the odd ones, as the nibbles' extraction leaves them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fb4_tables.hpp"

namespace fb4 {

constexpr int kMatvecMaxRows = 64;

typedef __bf16 mv_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mv_bf16x8 __attribute__((ext_vector_type(8)));
typedef float mv_f32x4 __attribute__((ext_vector_type(4)));

struct MatvecShape {
    uint32_t n, chunks;            // rows of the weights; 32-channel pieces of a row
    uint32_t x_stride;             // in units of 8 elements
    uint32_t waves;
    long long out_stride;          // elements
    uint16_t rows;
    uint16_t f32;                  // float results
};

// Two registers of E4M3 bytes of eight codes (a word), even elements and odd ones.
__device__ __forceinline__ void e4m3_of_codes(uint32_t w, uint2 table, uint32_t& even, uint32_t& odd)
{
    even = __builtin_amdgcn_perm(table.y, table.x, w & 0x07070707u) | ((w << 4) & 0x80808080u);
    odd = __builtin_amdgcn_perm(table.y, table.x, (w >> 4) & 0x07070707u) | (w & 0x80808080u);
}

__device__ __forceinline__ mv_bf16x8 weights_of(uint32_t w, uint2 table, float scale)
{
    uint32_t even, odd;
    e4m3_of_codes(w, table, even, odd);
    const mv_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, scale, true);
    const mv_bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, scale, true);
    return mv_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight channels of x, the even ones first.
__device__ __forceinline__ mv_bf16x8 channels_of(uint4 v)
{
    const uint4 o = make_uint4(__builtin_amdgcn_perm(v.y, v.x, 0x05040100u), __builtin_amdgcn_perm(v.w, v.z, 0x05040100u),
                               __builtin_amdgcn_perm(v.y, v.x, 0x07060302u), __builtin_amdgcn_perm(v.w, v.z, 0x07060302u));
    return __builtin_bit_cast(mv_bf16x8, o);
}

// A workgroup takes 16 kTiles rows of the weights and all rows of x (16 kSets at most); its wavefronts share the channels, kSteps times
// 128 in turn, and meet in LDS.
template <int kTiles, int kSets, bool kHalf>
__global__ __launch_bounds__(512) void matvec_kernel(const uint8_t* codes, const uint16_t* meta, const uint16_t* x, const uint8_t* blob,
                                                     const float* bias, void* out, MatvecShape s)
{
    constexpr int kSteps = 2;                    // a row's whole lines of 128 bytes
    constexpr uint32_t kOut = 16 * kTiles;
    extern __shared__ __align__(16) uint8_t lds[];
    uint2* tables = reinterpret_cast<uint2*>(lds);                 // [32] dialects' magnitudes
    float* meet = reinterpret_cast<float*>(lds + 256);             // [waves][16 kSets][kOut]
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t r = lane & 15u, g = lane >> 4;
    if (threadIdx.x < 64) {                      // (an integer's bf16 exponent and upper mantissa bits, rebiased)
        const uint2 m = reinterpret_cast<const uint2*>(blob + kOffDecode)[threadIdx.x];
        uint32_t b = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = ((i < 2 ? m.x : m.y) >> (16 * (i & 1))) & 0xFFFFu;
            b |= (v ? (v >> 4) - (120u << 3) : 0u) << (8 * i);
        }
        reinterpret_cast<uint32_t*>(tables)[threadIdx.x] = b;
    }
    const uint32_t first = blockIdx.x * kOut;
    const uint8_t* code_row[kTiles];
    const uint8_t* meta_row[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {           // (behind the last row that one again)
        const size_t row = min(first + 16u * t + r, s.n - 1u);
        code_row[t] = codes + row * s.chunks * 16u;
        meta_row[t] = reinterpret_cast<const uint8_t*>(meta) + row * s.chunks * (kHalf ? 4u : 2u);
    }
    const uint16_t* x_row[kSets];
    bool has[kSets];
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        has[u] = 16u * u + r < s.rows;
        x_row[u] = x + (size_t)(16u * u + r) * s.x_stride * 8u;
    }
    mv_f32x4 acc[kTiles][kSets];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
#pragma unroll
        for (int u = 0; u < kSets; ++u) acc[t][u] = mv_f32x4{0, 0, 0, 0};
    }
    __syncthreads();
    for (uint32_t c0 = wave * 4u * kSteps; c0 < s.chunks; c0 += s.waves * 4u * kSteps) {
        uint4 cw[kSteps][kTiles], xw[kSteps][kSets][4];
        uint32_t mw[kSteps][kTiles];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const uint32_t c = c0 + 4u * i + g;
            const bool live = c < s.chunks;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {   // (codes of zeros are weights of zero)
                cw[i][t] = make_uint4(0, 0, 0, 0);
                mw[i][t] = 0;
                if (live) {
                    cw[i][t] = *reinterpret_cast<const uint4*>(code_row[t] + (size_t)c * 16u);
                    mw[i][t] = kHalf ? reinterpret_cast<const uint32_t*>(meta_row[t])[c] : reinterpret_cast<const uint16_t*>(meta_row[t])[c];
                }
            }
#pragma unroll
            for (int u = 0; u < kSets; ++u) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    xw[i][u][j] = make_uint4(0, 0, 0, 0);
                    if (live && has[u]) xw[i][u][j] = reinterpret_cast<const uint4*>(x_row[u] + (size_t)c * 32u)[j];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            uint2 table[kTiles][kHalf ? 2 : 1];
            float scale[kTiles][kHalf ? 2 : 1];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
#pragma unroll
                for (int k = 0; k < (kHalf ? 2 : 1); ++k) {
                    const uint32_t m = kHalf ? (mw[i][t] >> (16 * k)) & 0xFFFFu : mw[i][t], did = m & 0xFFu;
                    table[t][k] = tables[did & 31u];
                    if (did > 31u) table[t][k] = make_uint2(0, 0);
                    scale[t][k] = __builtin_bit_cast(float, (max(m >> 8, 4u) - 3u) << 23);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mv_bf16x8 b[kSets];
#pragma unroll
                for (int u = 0; u < kSets; ++u) b[u] = channels_of(xw[i][u][j]);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    const uint32_t w = j == 0 ? cw[i][t].x : j == 1 ? cw[i][t].y : j == 2 ? cw[i][t].z : cw[i][t].w;
                    const mv_bf16x8 a = weights_of(w, table[t][kHalf ? j / 2 : 0], scale[t][kHalf ? j / 2 : 0]);
#pragma unroll
                    for (int u = 0; u < kSets; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b[u], acc[t][u], 0, 0, 0);
                }
            }
        }
    }
    // accumulator i: weight row 4 (lane / 16) + i, row of x lane % 16
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) *reinterpret_cast<mv_f32x4*>(meet + ((wave * 16u * kSets + 16u * u + r) * kOut + 16u * t + 4u * g)) = acc[t][u];
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < s.rows * kOut; i += s.waves * 64u) {
        const uint32_t row = i / kOut, col = i - row * kOut;
        if (first + col >= s.n) continue;
        float sum = bias ? bias[first + col] : 0.0f;
        for (uint32_t w = 0; w < s.waves; ++w) sum += meet[(w * 16u * kSets + row) * kOut + col];
        const size_t at = (size_t)((long long)row * s.out_stride) + first + col;
        if (s.f32) reinterpret_cast<float*>(out)[at] = sum;
        else reinterpret_cast<__bf16*>(out)[at] = (__bf16)sum;
    }
}

}  // namespace fb4
