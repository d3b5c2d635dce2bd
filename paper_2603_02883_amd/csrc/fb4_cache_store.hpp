// Keys and values into the pages of an 8-bit cache (fb4_cache_store).
//
// A page and head has one power-of-two scale for its keys and one for its values: the smallest 2^e with largest magnitude <= 448 * 2^e,
// read off the bits of the largest bf16, e = exponent - 8, one more where the mantissa is above 1.75.  E4M3 is a floating format, so a page
// whose scale grows loses nothing but what becomes subnormal, and tokens can come one by one.
//
// Keys lie [place][channel], values [channel][place]: what the attention's two products contract over is contiguous in both, so that its
// operands come straight from memory.
//
// A workgroup takes one head's keys or values of the runs (tokens of one page, side by side) that begin among `span` tokens: the run's
// last token for every place (`owner`, LDS), then its rows into registers -- a thread's item is 8 channels of four successive places --
// with the largest magnitude on the way, then 8 bytes per place of the keys, or four per channel of the values: the transposition
// is one of 4 x 4 bytes in registers.
//
// What bounds it: 16 sequences of up to 4096 tokens, 8 heads of 128 channels (352 MB): 87 to 90 us, 4.0 TB/s, the memory stream with the run's chain
// of waits (slots, rows, the maximum's meeting) in it -- five wavefronts per SIMD hide what they can, eight (by fewer registers) took 89 too.
// A token each of 64 sequences: 9 us, that chain, once; the page's other elements are read only where its scale grows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fb4 {

constexpr uint32_t kStoreThreads = 256, kStoreMaxPage = 128;
constexpr uint32_t kStoreLowest = 10, kStoreHighest = 247;   // scale bytes: every element is a normal bf16, or (256 with the highest) 2^128

typedef float store_f32x2 __attribute__((ext_vector_type(2)));

struct StoreStrides {
    uint32_t head, token;   // in units of 8 elements
};
struct StoreShape {
    uint32_t tokens, pages, span;
    uint16_t heads_k;
    uint8_t page_bits, pieces;   // pieces: 16-byte ones of a row, dim / 8
};

// 2^-e of scale byte e + 127, up to 253 (10 .. 247: a normal number either way), and 0 of 254
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// E4M3 of two bf16 in `w`, times `f`, in the low 16 bits; what is no number is NaN.
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t w, float f)
{
    const float a = __builtin_bit_cast(float, w << 16), b = __builtin_bit_cast(float, w & 0xFFFF0000u);
    uint32_t v = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a * f, b * f, 0, false) & 0xFFFFu;
    if ((w & 0x7FFFu) >= 0x7F80u) v = (v & 0xFF00u) | 0x7Fu;
    if ((w & 0x7FFF0000u) >= 0x7F800000u) v = (v & 0x00FFu) | 0x7F00u;
    return v;
}

// Four elements to a scale that is larger by the factor 1 / f.
__device__ __forceinline__ uint32_t e4m3_again(uint32_t w, float f)
{
    const store_f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * f, a[1] * f, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * f, b[1] * f, v, true);
}

// kRounds: items of a thread (page / 4 * pieces of them in all, at most 512).
template <int kRounds>
__global__ __launch_bounds__(kStoreThreads) void cache_store_kernel(const uint16_t* k, const uint16_t* v, const int32_t* slots, uint8_t* cache, uint8_t* scales,
                                                                    StoreStrides sk, StoreStrides sv, StoreShape s)
{
    __shared__ __align__(16) int32_t owner[kStoreMaxPage];
    __shared__ uint32_t largest[kStoreThreads / 64];
    const uint32_t tid = threadIdx.x;
    const uint32_t which = blockIdx.x & 1u, hb = blockIdx.x >> 1, chunk = hb / s.heads_k, head = hb - chunk * s.heads_k;
    const uint32_t page = 1u << s.page_bits, quads = page / 4u, items = quads * s.pieces;
    const uint32_t page_bytes = s.pieces * 8u << s.page_bits;
    const uint16_t* x = which ? v + (size_t)head * sv.head * 8u : k + (size_t)head * sk.head * 8u;
    const size_t token_stride = (size_t)(which ? sv.token : sk.token) * 8u;
    auto page_at = [&](uint32_t t) {   // of token t; 0xFFFFFFFF: none
        const uint32_t p = (uint32_t)slots[t] >> s.page_bits;   // (a negative slot's is past all pages)
        return p < s.pages ? p : 0xFFFFFFFFu;
    };
    // an item's channels and places: of keys the channels' pieces side by side in a wavefront, of values the places, as they are written
    uint32_t piece[kRounds], quad[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const uint32_t j = min(tid + i * kStoreThreads, items - 1u);   // (past the last: nothing is read or written)
        quad[i] = which ? j & (quads - 1u) : j / s.pieces;
        piece[i] = which ? j >> (s.page_bits - 2u) : j - quad[i] * s.pieces;
    }
    // ---- tokens of the span that begin a run: every wavefront finds them itself
    const uint32_t lane = tid & 63u, first = chunk * s.span, n = min(s.span, s.tokens - first);
    uint64_t begins[2] = {0, 0};
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        if (64u * i >= n) break;
        const uint32_t t = first + min(64u * i + lane, n - 1u), p = page_at(t);
        begins[i] = __ballot(64u * i + lane < n && p != 0xFFFFFFFFu && (t == 0 || page_at(t - 1u) != p));
    }
    while (begins[0] | begins[1]) {
        const uint32_t i = begins[0] ? 0u : 1u, bit = (uint32_t)__builtin_ctzll(begins[i]), t0 = first + 64u * i + bit;
        if (i) begins[1] &= begins[1] - 1u;
        else begins[0] &= begins[0] - 1u;
        const uint32_t p = (uint32_t)__builtin_amdgcn_readfirstlane((int)page_at(t0));
        const size_t at_scale = ((size_t)which * s.pages + p) * s.heads_k + head;
        const uint32_t before = min((uint32_t)scales[at_scale], kStoreHighest);
        // ---- the places' tokens, by the first wavefront; a token by itself is everyone's
        const bool alone = t0 + 1u >= s.tokens || page_at(t0 + 1u) != p;
        const uint32_t place = (uint32_t)slots[t0] & (page - 1u);
        if (!alone && tid < 64u) {
            owner[tid] = owner[64u + tid] = -1;
            for (uint32_t at = t0; at < s.tokens; at += 64u) {
                const uint32_t t = min(at + lane, s.tokens - 1u), slot = (uint32_t)slots[t];
                const uint64_t out = __ballot(at + lane >= s.tokens || slot >> s.page_bits != p);
                const uint32_t run = out ? (uint32_t)__builtin_ctzll(out) : 64u;
                if (lane < run) atomicMax(&owner[slot & (page - 1u)], (int32_t)t);
                if (run < 64u) break;
            }
        }
        if (!alone) __syncthreads();
        // ---- rows, and the largest magnitude
        uint4 w[kRounds][4];
        uint32_t have[kRounds], most = 0;
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            int4 from = make_int4(-1, -1, -1, -1);
            if (!alone) from = *reinterpret_cast<const int4*>(owner + 4u * quad[i]);
            int32_t t[4] = {from.x, from.y, from.z, from.w};
            if (alone && quad[i] == place / 4u) {
#pragma unroll
                for (uint32_t a = 0; a < 4; ++a) t[a] = (place & 3u) == a ? (int32_t)t0 : -1;
            }
            have[i] = 0;
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                w[i][a] = make_uint4(0, 0, 0, 0);
                if (t[a] >= 0 && tid + i * kStoreThreads < items) {
                    w[i][a] = *reinterpret_cast<const uint4*>(x + (size_t)t[a] * token_stride + 8u * piece[i]);
                    have[i] |= 1u << a;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const uint32_t q[4] = {w[i][a].x, w[i][a].y, w[i][a].z, w[i][a].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t lo = q[j] & 0x7FFFu, hi = (q[j] >> 16) & 0x7FFFu;
                    most = max(most, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
                }
            }
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, d));
        if ((tid & 63u) == 0) largest[tid >> 6] = most;
        const bool begun = alone ? place == 0u : owner[0] >= 0;
        __syncthreads();
        most = max(max(largest[0], largest[1]), max(largest[2], largest[3]));
        // (biased exponent, one more from 1.75 + 2^-7 on; less 8)
        uint32_t scale = max((most + 0x1Fu) >> 7, kStoreLowest + 8u) - 8u;
        const bool again = !begun && before < scale;   // what the page holds besides is rounded to the larger scale
        if (!begun) scale = max(scale, before);
        // (2^-126 times E4M3's largest is far below half of its least, as 0 times it is, where larger growths have no exponent left)
        const float f = inverse_scale(scale), f_old = again ? inverse_scale(min(scale - before, 127u) + 127u) : 1.0f;
        uint8_t* to = cache + at_scale * page_bytes;
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            if (tid + i * kStoreThreads >= items || (have[i] == 0 && !again)) continue;
            uint32_t y[4][2];   // of every place, eight channels
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                y[a][0] = e4m3_pair(w[i][a].x, f) | e4m3_pair(w[i][a].y, f) << 16;
                y[a][1] = e4m3_pair(w[i][a].z, f) | e4m3_pair(w[i][a].w, f) << 16;
            }
            if (which == 0) {
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    uint2* at = reinterpret_cast<uint2*>(to + ((4u * quad[i] + a) * s.pieces + piece[i]) * 8u);
                    if (have[i] >> a & 1u) {
                        *at = make_uint2(y[a][0], y[a][1]);
                    } else if (again) {
                        const uint2 o = *at;
                        *at = make_uint2(e4m3_again(o.x, f_old), e4m3_again(o.y, f_old));
                    }
                }
            } else {
                uint32_t z[8];   // of every channel, four places
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t lo01 = __builtin_amdgcn_perm(y[1][h], y[0][h], 0x05010400u), hi01 = __builtin_amdgcn_perm(y[1][h], y[0][h], 0x07030602u);
                    const uint32_t lo23 = __builtin_amdgcn_perm(y[3][h], y[2][h], 0x05010400u), hi23 = __builtin_amdgcn_perm(y[3][h], y[2][h], 0x07030602u);
                    z[4 * h] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
                    z[4 * h + 1] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
                    z[4 * h + 2] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
                    z[4 * h + 3] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
                }
                uint32_t* at = reinterpret_cast<uint32_t*>(to + ((8u * piece[i]) << s.page_bits) + 4u * quad[i]);
                const uint32_t row = page / 4u;
                if (have[i] == 15u) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) at[c * row] = z[c];
                } else if (again) {
                    const uint32_t mask = (have[i] & 1u ? 0xFFu : 0u) | (have[i] & 2u ? 0xFF00u : 0u) | (have[i] & 4u ? 0xFF0000u : 0u) | (have[i] & 8u ? 0xFF000000u : 0u);
                    uint32_t o[8];
#pragma unroll
                    for (int c = 0; c < 8; ++c) o[c] = at[c * row];
#pragma unroll
                    for (int c = 0; c < 8; ++c) at[c * row] = (z[c] & mask) | (e4m3_again(o[c], f_old) & ~mask);
                } else {
                    uint8_t* byte = reinterpret_cast<uint8_t*>(at);
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        if (have[i] >> a & 1u) {
#pragma unroll
                            for (int c = 0; c < 8; ++c) byte[(c << s.page_bits) + a] = (uint8_t)(z[c] >> (8 * a));
                        }
                    }
                }
            }
        }
        if (tid == 0) scales[at_scale] = (uint8_t)scale;
        __syncthreads();   // (the next run's owners)
    }
}

}  // namespace fb4
