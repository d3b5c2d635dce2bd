// Keys and values into the pages of an 8-bit cache (fb4_cache_store).
//
// A page and head has one power-of-two scale for its keys and one for its values: the smallest 2^e with largest magnitude <= 448 * 2^e,
// read off the bits of the largest bf16, e = exponent - 8, one more where the mantissa is above 1.75.  E4M3 is a floating format, so a page
// whose scale grows loses nothing but what becomes subnormal, and tokens can come one by one.
//
// Keys lie [place][channel], values [channel][place]: what the attention's two products contract over is contiguous in both, so that its
// operands come straight from memory.  The transposition is here, through LDS.
//
// A workgroup takes one head's keys or values of the runs (tokens of one page, side by side) that begin among `span` tokens: the run's
// last token for every place (`owner`), their rows into LDS with the largest magnitude on the way, then the page's
// pieces of 8 or 16 bytes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fb4 {

constexpr uint32_t kStoreThreads = 256, kStoreMaxPage = 128, kStoreMaxDim = 128;
constexpr uint32_t kStoreLowest = 10, kStoreHighest = 247;   // scale bytes: every element is a normal bf16; the largest bf16 fits

typedef float store_f32x2 __attribute__((ext_vector_type(2)));

struct StoreStrides {
    uint32_t head, token;   // in units of 8 elements
};
struct StoreShape {
    uint32_t tokens, pages, span;
    uint16_t heads_k;
    uint8_t page_bits, pieces;   // pieces: 16-byte ones of a row, dim / 8
};

// 2^-e of scale byte e + 127 (10 .. 247: a normal number either way)
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

__global__ __launch_bounds__(kStoreThreads) void cache_store_kernel(const uint16_t* k, const uint16_t* v, const int32_t* slots, uint8_t* cache, uint8_t* scales,
                                                                    StoreStrides sk, StoreStrides sv, StoreShape s)
{
    // rows of bf16: two channels a word, one word behind each (a value's 16 places of one channel are in 16 rows: without it in one bank)
    __shared__ uint32_t rows[kStoreMaxPage * (kStoreMaxDim / 2 + 1)];
    __shared__ int32_t owner[kStoreMaxPage];
    __shared__ uint32_t largest[kStoreThreads / 64];
    __shared__ uint32_t run_end;
    const uint32_t tid = threadIdx.x;
    const uint32_t which = blockIdx.x & 1u, hb = blockIdx.x >> 1, chunk = hb / s.heads_k, head = hb - chunk * s.heads_k;
    const uint32_t page = 1u << s.page_bits, words = s.pieces * 4u, pitch = words + 1u;
    const uint32_t page_bytes = s.pieces * 8u << s.page_bits;
    const uint16_t* x = which ? v + (size_t)head * sv.head * 8u : k + (size_t)head * sk.head * 8u;
    const size_t token_stride = (size_t)(which ? sv.token : sk.token) * 8u;
    auto page_at = [&](uint32_t t) {   // of token t; 0xFFFFFFFF: none
        const uint32_t p = (uint32_t)slots[t] >> s.page_bits;   // (a negative slot's is past all pages)
        return p < s.pages ? p : 0xFFFFFFFFu;
    };
    const uint32_t first = chunk * s.span, last = min(first + s.span, s.tokens);
    for (uint32_t t0 = first; t0 < last; ++t0) {
        const uint32_t p = page_at(t0);
        if (p == 0xFFFFFFFFu || (t0 > 0 && page_at(t0 - 1u) == p)) continue;   // (uniform: everyone reads the same)
        // ---- the run and its tokens' places
        for (uint32_t i = tid; i < page; i += kStoreThreads) owner[i] = -1;
        if (tid == 0) run_end = s.tokens;
        __syncthreads();
        for (uint32_t at = t0;; at += kStoreThreads) {
            const uint32_t t = at + tid;
            const bool in = t < s.tokens && page_at(t) == p;
            if (!in && t < s.tokens) atomicMin(&run_end, t);
            __syncthreads();
            const uint32_t end = run_end;
            if (t < end && in) atomicMax(&owner[(uint32_t)slots[t] & (page - 1u)], (int32_t)t);
            if (end <= at + kStoreThreads || at + kStoreThreads >= s.tokens) break;
            __syncthreads();   // (everyone has read run_end before it changes again)
        }
        __syncthreads();
        // ---- rows into LDS, and the largest magnitude
        uint32_t most = 0;
        for (uint32_t i = tid; i < page * s.pieces; i += kStoreThreads) {
            const uint32_t r = i / s.pieces, c = i - r * s.pieces;
            const int32_t t = owner[r];
            if (t < 0) continue;
            const uint4 w = *reinterpret_cast<const uint4*>(x + (size_t)t * token_stride + 8u * c);
            const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                rows[r * pitch + 4u * c + j] = q[j];
                const uint32_t lo = q[j] & 0x7FFFu, hi = (q[j] >> 16) & 0x7FFFu;
                most = max(most, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
            }
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, d));
        if ((tid & 63u) == 0) largest[tid >> 6] = most;
        const size_t at_scale = ((size_t)which * s.pages + p) * s.heads_k + head;
        const uint32_t before = min((uint32_t)scales[at_scale], kStoreHighest);
        __syncthreads();
        most = max(max(largest[0], largest[1]), max(largest[2], largest[3]));
        // (biased exponent, one more from 1.75 + 2^-7 on; less 8)
        uint32_t scale = max((most + 0x1Fu) >> 7, kStoreLowest + 8u) - 8u;
        const bool begun = owner[0] >= 0, again = !begun && before < scale;
        if (!begun) scale = max(scale, before);
        const float f = inverse_scale(scale), f_old = again ? inverse_scale(scale - before + 127u) : 1.0f;
        uint8_t* to = cache + at_scale * page_bytes;
        if (which == 0) {
            for (uint32_t i = tid; i < page * s.pieces; i += kStoreThreads) {
                const uint32_t r = i / s.pieces, c = i - r * s.pieces;
                uint2* at = reinterpret_cast<uint2*>(to + i * 8u);
                if (owner[r] >= 0) {
                    const uint32_t* w = rows + r * pitch + 4u * c;
                    *at = make_uint2(e4m3_pair(w[0], f) | e4m3_pair(w[1], f) << 16, e4m3_pair(w[2], f) | e4m3_pair(w[3], f) << 16);
                } else if (again) {
                    const uint2 w = *at;
                    *at = make_uint2(e4m3_again(w.x, f_old), e4m3_again(w.y, f_old));
                }
            }
        } else {
            // two channels' 16 places: words of the same rows
            const uint32_t sixteenths = page / 16u;
            for (uint32_t i = tid; i < words * sixteenths; i += kStoreThreads) {
                const uint32_t c2 = i / sixteenths, j = i - c2 * sixteenths;
                uint32_t lo[4], hi[4], set[4];
                uint32_t have = 0;
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    lo[a] = hi[a] = set[a] = 0;
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const uint32_t r = 16u * j + 4u * a + b;
                        if (owner[r] >= 0) {
                            const uint32_t y = e4m3_pair(rows[r * pitch + c2], f);
                            lo[a] |= (y & 0xFFu) << (8 * b);
                            hi[a] |= (y >> 8) << (8 * b);
                            set[a] |= 0xFFu << (8 * b);
                            ++have;
                        }
                    }
                }
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    uint8_t* at = to + ((2u * c2 + y) << s.page_bits) + 16u * j;
                    uint32_t* n = y ? hi : lo;
                    if (again && have < 16u) {
                        const uint4 w = *reinterpret_cast<const uint4*>(at);
                        const uint32_t o[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int a = 0; a < 4; ++a) n[a] |= e4m3_again(o[a], f_old) & ~set[a];
                    }
                    if (again || have == 16u) {
                        *reinterpret_cast<uint4*>(at) = make_uint4(n[0], n[1], n[2], n[3]);
                    } else if (have) {
#pragma unroll
                        for (int a = 0; a < 4; ++a) {
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                if (set[a] >> (8 * b) & 1u) at[4 * a + b] = (uint8_t)(n[a] >> (8 * b));
                            }
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
