// Few rows times FB4 weights: y[r][n] = sum_c x[r][c] W[n][c].
//
// 16x16x32 bf16 MFMAs with 16 weight rows as the first operand and up to 16 rows of x as the second.  A weight's magnitude is an
// integer 0 .. 15 and its block's scale a power of two, so the decoded weight is a bf16 number: eight nibbles become two registers of
// E4M3 bytes by a byte permutation of the dialect's eight magnitudes (LDS, 8 bytes a dialect), and the converter to bf16 takes the
// block's scale along.  The channels of a product may come in any order as long as both operands have the same: a lane holds 32
// successive channels of one row (16 bytes of codes, one block's scale and dialect, or two's), eight for each of four MFMAs, and of
// eight the even ones come before the odd ones, as the nibbles' extraction leaves them.  The weights are exact and so is every product; the sums are fp32,
// and the result is rounded to its type once.
//
// What bounds it: the reads of the codes.  49152 x 8192, one row (227 MB): 52.6 us, 4.3 TB/s (46 where part of the weights is still in the last cache);
// 16384 x 4096, 16 rows: 14.5, of which x through the L2s -- 16 rows are read by each of 256 workgroups -- and the first reads' latency are half; 6912 x
// 1152, one row: 3.7 to 4.3, and 4610 x 1184 in blocks of 16, 37 rows: 8.2, a launch and that latency.
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

// Chunks whose scales and dialects a workgroup holds at a time: 32 KiB of all its rows, at most.
constexpr uint32_t matvec_chunks(int tiles, bool half) { return 1024u / tiles / (half ? 2 : 1); }

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

// A workgroup takes 16 kTiles rows of the weights and all rows of x (16 kSets at most); its wavefronts share the channels, 128 at a time in
// turn, and meet in LDS.  What a turn reads is asked for while the one before it is computed.  Scales and dialects come through LDS, up to 16
// KiB of a row's words side by side at a time: as a lane's own reads, two bytes to a chunk of 16, they are as many requests as the codes (49152 x
// 8192, one row: 61 us so, 52.7 through LDS).  kDirect: those reads all the same, where a wavefront has a turn or two and the way
// through LDS would be one more wait (6912 x 1152: 3.7 and 4.4 us).
template <int kTiles, int kSets, bool kHalf, bool kDirect>
__global__ __launch_bounds__(512) void matvec_kernel(const uint8_t* codes, const uint16_t* meta, const uint16_t* x, const uint8_t* blob,
                                                     const float* bias, void* out, MatvecShape s)
{
    constexpr uint32_t kOut = 16 * kTiles;
    constexpr int kScales = kHalf ? 2 : 1;
    constexpr uint32_t kWord = kHalf ? 4 : 2, kMost = matvec_chunks(kTiles, kHalf);   // bytes of a chunk's scales and dialects; chunks at a time
    extern __shared__ __align__(16) uint8_t lds[];
    uint2* tables = reinterpret_cast<uint2*>(lds);                 // [32] dialects' magnitudes
    uint8_t* words = lds + 256;                                    // [kOut] rows, 16 bytes further apart than they are long
    float* meet = reinterpret_cast<float*>(lds + 256);             // [waves][16 kSets][kOut], when the words are done with
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
    // Tile t's rows from `from` on: a tile that would pass the last row ends there, and one of fewer rows than 16 has the last one
    // several times.  One offset for all tiles and a base each, which stays in scalar registers.
    const uint32_t first = blockIdx.x * kOut;
    const uint8_t* code_base[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const size_t from = min(first + 16u * t, max(s.n, 16u) - 16u);
        code_base[t] = codes + from * s.chunks * 16u;
    }
    const uint32_t row = min(r, s.n - 1u);
    auto row_of = [&](uint32_t at) __attribute__((always_inline)) {   // of the workgroup's rows as they are computed
        return (size_t)min(first + (at & ~15u), max(s.n, 16u) - 16u) + min(at & 15u, s.n - 1u);
    };
    const uint16_t* x_row[kSets];
    bool has[kSets];
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        has[u] = 16u * u + r < s.rows;
        x_row[u] = x + (size_t)(16u * u + r) * s.x_stride * 8u;
    }
    struct Turn {
        uint4 codes[kTiles], x[kSets][4];
        uint32_t meta[kDirect ? kTiles : 1];
    };
    auto ask = [&](uint32_t c0, Turn& w) __attribute__((always_inline)) {
        const uint32_t c = c0 + g, code_at = (row * s.chunks + c) * 16u;
        const bool live = c < s.chunks;          // (codes of zeros are weights of zero)
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            w.codes[t] = make_uint4(0, 0, 0, 0);
            if (live) w.codes[t] = *reinterpret_cast<const uint4*>(code_base[t] + code_at);
            if (kDirect) {
                const size_t at = row_of(16u * t + r) * s.chunks + c;
                w.meta[t] = 0;
                if (live) w.meta[t] = kHalf ? reinterpret_cast<const uint32_t*>(meta)[at] : meta[at];
            }
        }
#pragma unroll
        for (int u = 0; u < kSets; ++u) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w.x[u][j] = make_uint4(0, 0, 0, 0);
                if (live && has[u]) w.x[u][j] = reinterpret_cast<const uint4*>(x_row[u] + (size_t)c * 32u)[j];
            }
        }
    };
    mv_f32x4 acc[kTiles][kSets];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
#pragma unroll
        for (int u = 0; u < kSets; ++u) acc[t][u] = mv_f32x4{0, 0, 0, 0};
    }
    const uint32_t pitch = min(s.chunks, kMost) * kWord + 16u & ~15u;
    auto compute = [&](const Turn& w, uint32_t c0) __attribute__((always_inline)) {   // c0: from the words' first chunk on
        uint32_t word[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const uint8_t* at = words + (16u * t + r) * pitch + min(c0 + g, kMost - 1u) * kWord;   // (behind the last chunk: any, its codes are zeros)
            if (kDirect) word[t] = w.meta[t];
            else word[t] = kHalf ? *reinterpret_cast<const uint32_t*>(at) : *reinterpret_cast<const uint16_t*>(at);
        }
        uint2 table[kTiles][kScales];
        float scale[kTiles][kScales];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
#pragma unroll
            for (int k = 0; k < kScales; ++k) {
                const uint32_t m = kHalf ? (word[t] >> (16 * k)) & 0xFFFFu : word[t], did = m & 0xFFu;
                table[t][k] = tables[did & 31u];
                if (did > 31u) table[t][k] = make_uint2(0, 0);
                scale[t][k] = __builtin_bit_cast(float, (max(m >> 8, 4u) - 3u) << 23);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            mv_bf16x8 b[kSets];
#pragma unroll
            for (int u = 0; u < kSets; ++u) b[u] = channels_of(w.x[u][j]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                const uint32_t y = j == 0 ? w.codes[t].x : j == 1 ? w.codes[t].y : j == 2 ? w.codes[t].z : w.codes[t].w;
                const mv_bf16x8 a = weights_of(y, table[t][kHalf ? j / 2 : 0], scale[t][kHalf ? j / 2 : 0]);
#pragma unroll
                for (int u = 0; u < kSets; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b[u], acc[t][u], 0, 0, 0);
            }
        }
    };
    // The words of chunks `from` .. of all rows: 16 bytes a thread where they lie so, else one by one.
    auto fetch_words = [&](uint32_t from, uint32_t n) __attribute__((always_inline)) {
        const uint8_t* base = reinterpret_cast<const uint8_t*>(meta);
        const size_t row_bytes = (size_t)s.chunks * kWord;
        const uint32_t per = 16u / kWord, pieces = (n + per - 1u) / per;
        if (n % per == 0 && row_bytes % 16u == 0 && (reinterpret_cast<uintptr_t>(meta) & 15u) == 0) {
            for (uint32_t i = threadIdx.x; i < kOut * pieces; i += s.waves * 64u) {
                const uint32_t at = i / pieces, p = i - at * pieces;
                *reinterpret_cast<uint4*>(words + at * pitch + 16u * p) = *reinterpret_cast<const uint4*>(base + row_of(at) * row_bytes + from * kWord + 16u * p);
            }
        } else {
            for (uint32_t i = threadIdx.x; i < kOut * n; i += s.waves * 64u) {
                const uint32_t at = i / n, p = i - at * n;
                const uint8_t* x0 = base + row_of(at) * row_bytes + (from + p) * kWord;
                if (kHalf) *reinterpret_cast<uint32_t*>(words + at * pitch + 4u * p) = *reinterpret_cast<const uint32_t*>(x0);
                else *reinterpret_cast<uint16_t*>(words + at * pitch + 2u * p) = *reinterpret_cast<const uint16_t*>(x0);
            }
        }
    };
    const uint32_t stride = s.waves * 4u;
    Turn a, b;
    for (uint32_t from = 0; from < s.chunks; from += kDirect ? s.chunks : kMost) {   // (kMost is whole rounds of the wavefronts' turns)
        const uint32_t n = kDirect ? s.chunks : min(s.chunks - from, kMost);
        uint32_t c = wave * 4u;
        ask(from + c, a);
        if (from) __syncthreads();
        if (!kDirect) fetch_words(from, n);
        __syncthreads();
        while (c < n) {
            if (c + stride < n) ask(from + c + stride, b);
            compute(a, c);
            c += stride;
            if (c >= n) break;
            if (c + stride < n) ask(from + c + stride, a);
            compute(b, c);
            c += stride;
        }
    }
    __syncthreads();
    // accumulator i: weight row 4 (lane / 16) + i, row of x lane % 16
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) *reinterpret_cast<mv_f32x4*>(meet + ((wave * 16u * kSets + 16u * u + r) * kOut + 16u * t + 4u * g)) = acc[t][u];
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < s.rows * kOut; i += s.waves * 64u) {
        const uint32_t at_row = i / kOut, col = i - at_row * kOut;
        if (first + col >= s.n) continue;
        // (its place in its tile, which may begin earlier)
        const uint32_t begin = first + (col & ~15u), place = col + (begin - min(begin, max(s.n, 16u) - 16u));
        float sum = bias ? bias[first + col] : 0.0f;
        for (uint32_t w = 0; w < s.waves; ++w) sum += meet[(w * 16u * kSets + at_row) * kOut + place];
        const size_t at = (size_t)((long long)at_row * s.out_stride) + first + col;
        if (s.f32) reinterpret_cast<float*>(out)[at] = sum;
        else reinterpret_cast<__bf16*>(out)[at] = (__bf16)sum;
    }
}

}  // namespace fb4
