// Attention over a cache of pages in 8 bits (fb4_cache_attention).
//
// S^T = K Q^T and O^T = V^T P^T as 16x16x32 bf16 MFMAs, one pass over the keys with the running maximum and sum of the softmax, 64 keys a
// step of a wavefront.  A first operand's lane holds eight successive values of one row of 16, so keys come [key][channel] and values
// [channel][key] out of the cache straight into registers; the converter from E4M3 to bf16 takes the page's scale along (a power of two:
// exact).  Which keys make up the 16 rows of a product is free, and so is the order of the channels as long as both operands agree: lane group g =
// lane / 16 of the accumulators holds rows 4 g .. 4 g + 3, and row r of tile t is key 16 (r / 4) + 4 t + r % 4 of the 64, so that after four
// tiles group g has the 16 successive keys 16 g .. of the lane's query -- as the second product's operands want them: P goes from
// accumulators to operand without leaving the lane, and a lane reads 16 bytes of V, the same 16 keys of one channel.  A page has at
// least 16 tokens, so each of these sixteenths lies in one page.
//
// Rows of a product's second operand are the queries of a key head: the n tokens of a sequence times the query heads that share it, token
// by token, cut into tiles of 16 (a workgroup's wavefronts take every fourth step of the keys) or of 128 (each wavefront 32 rows, all steps).
//
// Roundings to fewer bits than 32: the weights to bf16 as the second product's operand, half a bf16 step of each, beside which the output's own
// is as large; keys and values are bf16 numbers as they are held.  Products, maxima, sums (of the unrounded weights) and parts are fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fb4 {

constexpr uint32_t kCacheWaves = 4, kCacheStep = 64;   // keys
constexpr uint32_t kCacheMaxBatch = 4096;
constexpr uint32_t kTileRows = 128;   // of the kernel for many queries
constexpr float kCacheLog2E = 1.44269504088896340736f, kCacheLn2 = 0.69314718055994530942f;

typedef __bf16 cache_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 cache_bf16x8 __attribute__((ext_vector_type(8)));
typedef float cache_f32x2 __attribute__((ext_vector_type(2)));
typedef float cache_f32x4 __attribute__((ext_vector_type(4)));

struct CacheStrides {
    uint32_t head, token;   // in units of 8 elements
};
struct CacheShape {
    uint32_t tokens, max_pages, pages;
    uint16_t batch, heads, heads_k;
    uint8_t page_bits, row;   // row: dim / 8, and 128 if causal
    float scale;
    __host__ __device__ uint32_t dim8() const { return row & 127u; }
    __host__ __device__ bool causal() const { return row > 127u; }
};

#define FB4_INLINE __attribute__((always_inline))

// ------------------------------------------------------------------------------------------------ which part of the work
// Sequences lie in `starts` one behind the other; the tiles of sequence b are numbered from place(b) = starts[b] * group / rows + b on, which
// leaves each its whole tiles and a begun one, so that a workgroup finds its sequence from `starts` alone.
struct CacheRows {
    uint32_t first, n;      // first query token, query tokens
    uint32_t len;           // keys
};
__device__ __forceinline__ uint32_t start_of(const int32_t* starts, uint32_t b, uint32_t tokens) { return (uint32_t)min(max(starts[b], 0), (int32_t)tokens); }
// (group 0: the start itself, for the sequence of a token)
__device__ __forceinline__ uint32_t place_of(uint32_t start, uint32_t b, uint32_t group, uint32_t tile_rows) { return group ? start * group / tile_rows + b : start; }
__device__ __forceinline__ CacheRows rows_of(const int32_t* starts, const int32_t* lens, uint32_t b, const CacheShape& s)
{
    CacheRows r;
    r.first = start_of(starts, b, s.tokens);
    const uint32_t end = start_of(starts, b + 1u, s.tokens);
    r.n = end > r.first ? end - r.first : 0u;
    r.len = (uint32_t)min(max((int64_t)lens[b], (int64_t)0), (int64_t)s.max_pages << s.page_bits);
    return r;
}
__host__ __device__ __forceinline__ uint32_t tiles_of(uint32_t n, uint32_t group, uint32_t tile_rows) { return (n * group + tile_rows - 1u) / tile_rows; }
__host__ __device__ __forceinline__ uint32_t steps_of(uint32_t len) { return (len + kCacheStep - 1u) / kCacheStep; }

// The last sequence whose place is at most `slot`, by a wavefront: 64 candidates at a time.
__device__ __forceinline__ uint32_t sequence_of(const int32_t* starts, uint32_t slot, uint32_t group, uint32_t tile_rows, const CacheShape& s)
{
    const uint32_t lane = threadIdx.x & 63u, stride = (s.batch + 63u) / 64u;
    if (s.batch == 1u) return 0;
    uint32_t b = lane * stride;
    uint64_t yes = __ballot(b < s.batch && place_of(start_of(starts, b < s.batch ? b : 0u, s.tokens), b, group, tile_rows) <= slot);
    const uint32_t base = (uint32_t)(63 - __builtin_clzll(yes | 1ull)) * stride;
    if (stride == 1u) return base;
    b = base + lane;
    yes = __ballot(lane < stride && b < s.batch && place_of(start_of(starts, min(b, s.batch - 1u), s.tokens), b, group, tile_rows) <= slot);
    return base + (uint32_t)(63 - __builtin_clzll(yes | 1ull));
}

// Parts: where tiles are few, the keys of each are shared by several workgroups, of about `share` steps each -- the same for all, so that
// sequences of unlike lengths get parts by their lengths.  Tiles of few rows: all tiles' steps over kCacheTarget workgroups (512,
// 768 and 1024, a token each, us: 32 sequences of up to 8192 keys 99, 88, 96; 16: 52, 47, 48; one of 65536: 30.5, 38, 36).  Tiles of 128: the
// best number of parts by the times below.  A tile of one part writes its rows itself.
constexpr uint32_t kCacheLeastShare = 2 * kCacheWaves, kCacheTarget = 768, kTilesTarget = 1536;
// Parts of each of n tiles of `steps` sixteenths of a step.  512 tiles run at a time, two to a compute unit, and steps take 1.2 times as long then as one by one
// (1.65 and 2 us of 128 channels); a tile's beginning and end take as long as six; parts, their joining twelve and one more per 256 parts.
// (24 heads of 128 channels, 128 tokens over 1024 keys: one part 34.9, two 36.8; over 2048: 63.5, four 39.0.  16 heads of 72 channels, 1350 tokens
// over 2048: one 55, two 61; over 4096: 104, 85; 3500 tokens over 12000: one 373, two 408; 5000: 648, 552.)
// In integers (costs in 160ths of a step): the attention's launch and the joining one each compute it, in kernels compiled apart, and where parts lie in the
// workspace hangs on the same number in both.
__host__ __device__ inline uint32_t tile_parts(uint32_t n, uint32_t steps)
{
    uint64_t least = 0;
    uint32_t best = 1;
#pragma unroll
    for (uint32_t p = 1; p <= 16u; ++p) {
        if (p > 1u && (n * p > kTilesTarget || steps < 16u * p * kCacheLeastShare)) break;
        const uint64_t cost = (uint64_t)((n * p + 511u) / 512u) * (steps / p + 96u) * (n * p > 256u ? 12u : 10u) + (p > 1u ? 1920u + n * p * 5u / 8u : 0u);
        if (p == 1u || cost < least) {
            best = p;
            least = cost;
        }
    }
    return best;
}
// Steps to a part of `tiles` tiles with `sum` steps.
__host__ __device__ __forceinline__ uint32_t share_of_tiles(uint64_t sum, uint32_t tiles, uint32_t heads_k, uint32_t tile_rows)
{
    uint32_t share;
    if (tile_rows < kTileRows) {
        share = (uint32_t)((sum * heads_k + kCacheTarget - 1u) / kCacheTarget);
    } else {
        const uint32_t n = tiles ? tiles : 1u, steps = (uint32_t)((sum * 16u + n - 1u) / n), parts = 16u * tile_parts(n * heads_k, steps);
        share = (steps + parts - 1u) / parts;
    }
    return share > kCacheLeastShare ? share : kCacheLeastShare;
}
__device__ __forceinline__ uint32_t share_of(const int32_t* starts, const int32_t* lens, uint32_t group, uint32_t tile_rows, const CacheShape& s)
{
    uint64_t sum = 0;
    uint32_t tiles = 0;
    for (uint32_t b = threadIdx.x & 63u; b < s.batch; b += 64u) {
        const CacheRows r = rows_of(starts, lens, b, s);
        const uint32_t n = tiles_of(r.n, group, tile_rows);
        sum += (uint64_t)n * steps_of(r.len);
        tiles += n;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        sum += __shfl_xor(sum, d);
        tiles += __shfl_xor(tiles, d);
    }
    return share_of_tiles(sum, tiles, s.heads_k, tile_rows);
}
// (of 128 rows to the nearest number: one more than meant is a round more)
__host__ __device__ __forceinline__ uint32_t parts_of(uint32_t len, uint32_t share, uint32_t tile_rows)
{
    const uint32_t parts = (steps_of(len) + (tile_rows < kTileRows ? share - 1u : share / 2u)) / share;
    return parts ? parts : 1u;
}

// Walks the sequences' tiles times parts, by a wavefront: until position `at` (-> its sequence, and `at` from its first one on), or
// to sequence `stop` (-> the position of its first one in `at`).  Behind all: batch.
__device__ __forceinline__ uint32_t walk_parts(const int32_t* starts, const int32_t* lens, uint32_t group, uint32_t tile_rows, uint32_t share, uint32_t stop,
                                               uint32_t& at, const CacheShape& s)
{
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t before = 0;
    for (uint32_t b0 = 0; b0 < s.batch; b0 += 64u) {
        const uint32_t b = b0 + lane;
        uint32_t mine = 0;
        if (b < s.batch) {
            const CacheRows r = rows_of(starts, lens, b, s);
            mine = tiles_of(r.n, group, tile_rows) * parts_of(r.len, share, tile_rows);
        }
        uint32_t sum = mine;
#pragma unroll
        for (uint32_t d = 1; d < 64; d *= 2) {
            const uint32_t y = __shfl_up(sum, d);
            if (lane >= d) sum += y;
        }
        if (stop < b0 + 64u) {
            at = before + __shfl(sum - mine, stop - b0);
            return stop;
        }
        const uint64_t behind = __ballot(before + sum > at);
        if (stop == 0xFFFFFFFFu && behind) {
            const uint32_t l = (uint32_t)__builtin_ctzll(behind);
            at -= before + __shfl(sum - mine, l);
            return b0 + l;
        }
        before += __shfl(sum, 63);
    }
    return s.batch;
}

// ------------------------------------------------------------------------------------------------ a step's weights, and bytes
// What a query's weights are relative to: the largest product so far (-Inf: none), and its rounded product with the factor c = scale log2 e
// (0: none).  Weights are exp2(S c - off), by one fused multiply-add whose product is exact, so that the rounding of `off` is one factor in all
// weights and in their sum.  Beyond |off| = 2^20 that factor could itself be no small number, and the 16 queries go on with exp2((S - most) c).
struct CacheState {
    float most, off, sum;
    bool large;   // (of all 16)
};
// Moves it, and what is relative to it, when a weight would pass 2^8.
template <int kD16>
__device__ __forceinline__ void cache_reference(const cache_f32x4 (&sc)[4], CacheState& s, cache_f32x4 (&o)[kD16], float factor)
{
#pragma clang fp contract(off)   // (a rounded product is meant)
    float larger = -__builtin_inff();
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) larger = fmaxf(larger, sc[t][i]);
    }
    if (__any((larger - s.most) * factor > 8.0f)) {
        // (finite, so that a score of +Inf has an infinite weight and sum: no number in the output, +Inf in lse)
        larger = fmaxf(larger, s.most);
        larger = fmaxf(larger, __shfl_xor(larger, 16));
        larger = fminf(fmaxf(larger, __shfl_xor(larger, 32)), 0x1.fffffep127f);
        const float fresh = larger == -__builtin_inff() ? 0.0f : larger * factor;
        const bool was_large = s.large;
        s.large = s.large || __any(fabsf(fresh) > 0x1p20f);
        // from what the weights so far are relative to: the rounded product, or (large) the exact one
        const float moved = was_large ? (s.most - larger) * factor : s.large ? fmaf(-larger, factor, s.off) : s.off - fresh;
        const float shrink = s.most == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(moved);
        s.most = larger;
        s.off = fresh;
        s.sum *= shrink;
#pragma unroll
        for (int d = 0; d < kD16; ++d) o[d] *= shrink;
    }
}
// Weights of four tiles of products (16 keys of this lane's query) as the second product's operands.
__device__ __forceinline__ void cache_powers(const cache_f32x4 (&sc)[4], CacheState& s, cache_bf16x8 (&p)[2], float factor)
{
    float w[16];
    if (s.large) {
        const float base = s.most == -__builtin_inff() ? 0.0f : s.most;
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = (sc[i / 4][i % 4] - base) * factor;
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = fmaf(sc[i / 4][i % 4], factor, -s.off);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = __builtin_amdgcn_exp2f(w[i]);
    // (the sum from the unrounded weights, pairwise: one rounding of the row's a step)
    s.sum += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7])) + (((w[8] + w[9]) + (w[10] + w[11])) + ((w[12] + w[13]) + (w[14] + w[15])));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            y[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((cache_f32x2{w[8 * h + 2 * i], w[8 * h + 2 * i + 1]}), cache_bf16x2));
        p[h] = __builtin_bit_cast(cache_bf16x8, make_uint4(y[0], y[1], y[2], y[3]));
    }
}
// At the end: relative to the exact product of maximum and factor, whose difference from another wavefront's or part's is then one of maxima.
template <int kD16>
__device__ __forceinline__ void cache_exact(CacheState& s, cache_f32x4 (&o)[kD16], float factor)
{
    s.sum += __shfl_xor(s.sum, 16);
    s.sum += __shfl_xor(s.sum, 32);
    const float f = s.large || s.most == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(fmaf(-s.most, factor, s.off));
    s.sum *= f;
#pragma unroll
    for (int d = 0; d < kD16; ++d) o[d] *= f;
}

// Eight E4M3 bytes times a power of two, in bf16.
__device__ __forceinline__ cache_bf16x8 cache_decode(uint32_t lo, uint32_t hi, float f)
{
    const cache_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, true);
    const cache_bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, true);
    return cache_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The first n of 16 bytes, zeros behind.
__device__ __forceinline__ uint4 first_bytes(uint4 w, uint32_t n)
{
    auto mask = [&](uint32_t i) { return n >= 4u * i + 4u ? 0xFFFFFFFFu : n <= 4u * i ? 0u : (1u << (8u * (n - 4u * i))) - 1u; };
    return make_uint4(w.x & mask(0), w.y & mask(1), w.z & mask(2), w.w & mask(3));
}
// Bytes that are no finite bf16 with their page's scale, as 1 each: what is added to a magnitude for that to carry into the sign, and no further.
// 0x7F is E4M3's NaN; with the largest scale, 2^120 (byte 247), 0x78 is 2^128.
__device__ __forceinline__ uint32_t past_numbers(uint32_t scale_byte) { return scale_byte < 247u ? 0x01010101u : 0x08080808u; }
__device__ __forceinline__ uint4 nans_of(uint4 w, uint32_t past)
{
    auto some = [past](uint32_t x) { return (((x & 0x7F7F7F7Fu) + past) >> 7) & 0x01010101u; };
    return make_uint4(some(w.x), some(w.y), some(w.z), some(w.w));
}
__device__ __forceinline__ uint4 without(uint4 w, uint4 nans) { return make_uint4(w.x & ~(nans.x * 0xFFu), w.y & ~(nans.y * 0xFFu), w.z & ~(nans.z * 0xFFu), w.w & ~(nans.w * 0xFFu)); }
// Eight keys from `key` on as an operand: 1 for those before `limit`.
__device__ __forceinline__ cache_bf16x8 seen_keys(uint32_t key, uint32_t limit)
{
    uint32_t y[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) y[i] = (key + 2u * i < limit ? 0x3F80u : 0u) | (key + 2u * i + 1u < limit ? 0x3F800000u : 0u);
    return __builtin_bit_cast(cache_bf16x8, make_uint4(y[0], y[1], y[2], y[3]));
}
// What lies behind a query's last key has weight 0, but 0 times NaN or Inf is no number.  So the keys that some query does not see come into the products
// without them; where there was one, a walk over these keys at the end, with products of ones, says which accumulators become NaN.
template <int kD16, int kSets, typename Pieces>
__device__ __forceinline__ void mark_nans(cache_f32x4 (&o)[kSets][kD16], Pieces pieces, uint32_t key, const uint32_t (&limit)[kSets])
{
#pragma unroll
    for (int d = 0; d < kD16; ++d) {
        const uint4 n = pieces(d);
        const cache_bf16x8 a0 = cache_decode(n.x * 0x38u, n.y * 0x38u, 1.0f), a1 = cache_decode(n.z * 0x38u, n.w * 0x38u, 1.0f);   // (0x38: 1)
#pragma unroll
        for (int u = 0; u < kSets; ++u) {
            cache_f32x4 x = {0, 0, 0, 0};
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, seen_keys(key, limit[u]), x, 0, 0, 0);
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, seen_keys(key + 8u, limit[u]), x, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[u][d][i] = x[i] > 0.0f ? __builtin_nanf("") : o[u][d][i];
        }
    }
}
__device__ __forceinline__ uint2 rounded(cache_f32x4 x, float f)
{
    const cache_bf16x2 lo = __builtin_convertvector((cache_f32x2{x[0] * f, x[1] * f}), cache_bf16x2), hi = __builtin_convertvector((cache_f32x2{x[2] * f, x[3] * f}), cache_bf16x2);
    return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

// A position's rows in the workspace, and their {maximum, sum} behind them.
__device__ __forceinline__ float* part_rows(float* workspace, uint32_t position, uint32_t rows, uint32_t dim) { return workspace + (size_t)position * rows * (dim + 2u); }
__device__ __forceinline__ float2* part_states(float* workspace, uint32_t position, uint32_t rows, uint32_t dim)
{
    return reinterpret_cast<float2*>(part_rows(workspace, position, rows, dim) + rows * dim);
}

// ------------------------------------------------------------------------------------------------ attention
// kD32: channels / 32, rounded up; kWhole: a row is kD32 whole steps and 16-byte pieces.  kSplit: parts, into the workspace: by
// position floats [rows][dim], then {maximum, sum} of every row; position = (parts in front) * heads_k + key head.
//
// What bounds it: the reads of the cache.  A step's keys and values are asked for one step ahead into registers, so that two wavefronts per SIMD
// (which amdgpu_waves_per_eu holds: three registers more had halved them, 32 sequences in parts 115 and 88 us) keep 8 x 16 KiB of a compute unit
// on their way.  96 sequences of up to 8192 keys, a token each, 24 heads over 8 of 128 channels: 233 us, 5.1 TB/s; one of 333 keys: 8, its
// chain of lengths, table, keys and values.  Two sets of 16 rows to a wavefront took 141 to 140 us where one takes 98 to 140 (64 sequences, 3 to 30
// rows) and are not kept.
template <int kD32, bool kWhole, bool kSplit>
__global__ __launch_bounds__(64 * kCacheWaves) __attribute__((amdgpu_waves_per_eu(2))) void cache_attention_kernel(const uint16_t* q, const uint8_t* cache, const uint8_t* scales, const int32_t* tables,
                                                                          const int32_t* lens, const int32_t* starts, uint16_t* out, float* lse, float* workspace,
                                                                          CacheStrides sq, CacheStrides so, CacheShape s)
{
    constexpr int kSets = 1;   // (of 16 rows, as the shared functions take them)
    constexpr uint32_t kRows = 16, kPitch = 32 * kD32 + 4;
    __shared__ __align__(16) float meet[kCacheWaves][16][kPitch];
    __shared__ float2 states[kCacheWaves][16];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t r = lane & 15u, g = lane >> 4;
    auto scalar = [](uint32_t x) FB4_INLINE { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
    const uint32_t position = scalar(blockIdx.x / s.heads_k), hk = blockIdx.x - position * s.heads_k, group = scalar((uint32_t)s.heads / s.heads_k);
    // ---- sequence, tile, steps
    uint32_t b, tile, part = 0, parts = 1;
    CacheRows rows;
    if (kSplit) {
        const uint32_t share = scalar(share_of(starts, lens, group, kRows, s));
        uint32_t at = position;
        b = scalar(walk_parts(starts, lens, group, kRows, share, 0xFFFFFFFFu, at, s));
        if (b >= s.batch) return;
        rows = rows_of(starts, lens, b, s);
        parts = parts_of(rows.len, share, kRows);
        tile = scalar(at) / parts;
        part = scalar(at) - tile * parts;
    } else {
        b = scalar(sequence_of(starts, position, group, kRows, s));
        rows = rows_of(starts, lens, b, s);
        tile = position - place_of(rows.first, b, group, kRows);
        if (tile >= tiles_of(rows.n, group, kRows)) return;
    }
    const uint32_t n_rows = min(rows.n * group - tile * kRows, kRows);
    // ---- this lane's queries (behind the last that one again), and the keys before which each ends
    const uint32_t pieces = s.dim8(), dim = pieces * 8u;
    cache_bf16x8 qf[kSets][kD32];
    uint32_t limit[kSets];
    auto limit_of = [&](uint32_t row) FB4_INLINE {
        const uint32_t token = (tile * kRows + row) / group;
        return s.causal() ? (uint32_t)max((int64_t)rows.len - (int64_t)rows.n + (int64_t)token + 1, (int64_t)0) : rows.len;
    };
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        const uint32_t row = min(16u * u + r, n_rows - 1u), at = tile * kRows + row, token = at / group, head = hk * group + (at - token * group);
        limit[u] = limit_of(row);
        const uint16_t* x = q + ((size_t)head * sq.head + (size_t)(rows.first + token) * sq.token) * 8u;
#pragma unroll
        for (int i = 0; i < kD32; ++i) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if (kWhole || kD32 * g + i < pieces) w = reinterpret_cast<const uint4*>(x)[kD32 * g + i];
            qf[u][i] = __builtin_bit_cast(cache_bf16x8, w);
        }
    }
    const uint32_t least = scalar(limit_of(0)), steps = steps_of(scalar(limit_of(n_rows - 1u)));
    const uint32_t from = (uint32_t)((uint64_t)steps * part / parts), to = (uint32_t)((uint64_t)steps * (part + 1u) / parts);
    const uint32_t bits = s.page_bits, in_page = (1u << bits) - 1u, held = (rows.len + in_page) >> bits;   // pages with a key
    const int32_t* table = tables + (size_t)b * s.max_pages;
    const size_t page_bytes = (size_t)dim << bits;
    const uint8_t* values = cache + (size_t)s.pages * s.heads_k * page_bytes;

    // ---- a step's operands.  For the keys a lane is in the sixteenth r / 4, for the values in the sixteenth g.
    struct Where {
        int32_t k, v;   // pages, -1: none
    };
    auto page_of = [&](uint32_t key) FB4_INLINE {
        const uint32_t i = key >> bits;
        const int32_t p = s.max_pages ? table[min(i, s.max_pages - 1u)] : -1;   // (not after its length has come)
        return i < held && (uint32_t)p < s.pages ? p : -1;
    };
    auto find = [&](uint32_t step) FB4_INLINE { return Where{page_of(step * kCacheStep + 16u * (r >> 2)), page_of(step * kCacheStep + 16u * g)}; };
    uint4 kr[4][(kD32 + 1) / 2], vr[2 * kD32];   // four tiles of keys; 16 channels each
    float k_scale = 0.0f, v_scale = 0.0f;
    auto scale_of = [&](uint32_t byte) FB4_INLINE { return __builtin_bit_cast(float, byte << 23); };
    auto past_of = [&](float scale) FB4_INLINE { return past_numbers(__builtin_bit_cast(uint32_t, scale) >> 23); };
    auto fetch_k = [&](uint32_t step, int32_t p) FB4_INLINE {
        const size_t at = (size_t)max(p, 0) * s.heads_k + hk;   // (what no page has: another's, whose products are replaced)
        k_scale = scale_of(scales[at]);
        const uint8_t* base = cache + at * page_bytes + (size_t)((step * kCacheStep + 16u * (r >> 2) + (r & 3u)) & in_page) * dim + kD32 * 8u * g;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint8_t* x = base + 4u * t * dim;
            if (kWhole && kD32 % 2 == 0) {
#pragma unroll
                for (int i = 0; i < kD32 / 2; ++i) kr[t][i] = reinterpret_cast<const uint4*>(x)[i];
            } else {
#pragma unroll
                for (int i = 0; i < kD32; ++i) {
                    uint2 w = make_uint2(0, 0);
                    if (kWhole || kD32 * g + i < pieces) w = reinterpret_cast<const uint2*>(x)[i];
                    if (i % 2) kr[t][i / 2].z = w.x, kr[t][i / 2].w = w.y;
                    else kr[t][i / 2].x = w.x, kr[t][i / 2].y = w.y;
                }
            }
        }
    };
    auto fetch_v = [&](uint32_t step, int32_t p) FB4_INLINE {
        const size_t at = (size_t)max(p, 0) * s.heads_k + hk;
        v_scale = scale_of(scales[(size_t)s.pages * s.heads_k + at]);
        const uint8_t* base = values + at * page_bytes + ((size_t)r << bits) + ((step * kCacheStep + 16u * g) & in_page);
#pragma unroll
        for (int d = 0; d < 2 * kD32; ++d) {
            vr[d] = make_uint4(0, 0, 0, 0);
            if (p >= 0 && (kWhole || 16u * d + r < dim)) vr[d] = *reinterpret_cast<const uint4*>(base + ((size_t)(16u * d) << bits));
        }
    };

    const float factor = s.scale * kCacheLog2E;
    cache_f32x4 o[kSets][2 * kD32];
    CacheState state[kSets];
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        state[u] = CacheState{-__builtin_inff(), 0.0f, 0.0f, false};
#pragma unroll
        for (int d = 0; d < 2 * kD32; ++d) o[u][d] = cache_f32x4{0, 0, 0, 0};
    }
    uint32_t step = from + wave, nans = 0;
    Where here = {-1, -1}, next = {-1, -1};
    if (step < to) {
        here = find(step);
        fetch_k(step, here.k);
        fetch_v(step, here.v);
        next = find(step + kCacheWaves);
    }
    for (; step < to; step += kCacheWaves) {
        const bool more = step + kCacheWaves < to;
        // ---- S^T
        cache_f32x4 sc[kSets][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int u = 0; u < kSets; ++u) sc[u][t] = cache_f32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kD32; ++i) {
                const cache_bf16x8 a = i % 2 ? cache_decode(kr[t][i / 2].z, kr[t][i / 2].w, k_scale) : cache_decode(kr[t][i / 2].x, kr[t][i / 2].y, k_scale);
#pragma unroll
                for (int u = 0; u < kSets; ++u) sc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[u][i], sc[u][t], 0, 0, 0);
            }
        }
        const Where after = next;
        if (more) {
            fetch_k(step + kCacheWaves, after.k);
            next = find(step + 2u * kCacheWaves);
        }
        // ---- what a query does not see
        const uint32_t key = step * kCacheStep + 16u * g;   // the first of this lane's
        const bool cut = step * kCacheStep + kCacheStep > least || __any(here.v < 0);
        if (cut) {
#pragma unroll
            for (int u = 0; u < kSets; ++u) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[u][t][i] = here.v < 0 || key + 4u * t + i >= limit[u] ? -__builtin_inff() : sc[u][t][i];
                }
            }
        }
        // ---- weights
        cache_bf16x8 p[kSets][2];
#pragma unroll
        for (int u = 0; u < kSets; ++u) cache_reference(sc[u], state[u], o[u], factor);
#pragma unroll
        for (int u = 0; u < kSets; ++u) cache_powers(sc[u], state[u], p[u], factor);
        // ---- O^T
        if (step * kCacheStep + kCacheStep > least) {
            const uint32_t n = rows.len > key ? min(rows.len - key, 16u) : 0u;   // (behind a sequence's end a page may hold anything)
            const uint32_t past = past_of(v_scale);
#pragma unroll
            for (int d = 0; d < 2 * kD32; ++d) {
                vr[d] = first_bytes(vr[d], n);
                const uint4 bad = nans_of(vr[d], past);
                nans |= bad.x | bad.y | bad.z | bad.w;
                vr[d] = without(vr[d], bad);
            }
        }
#pragma unroll
        for (int d = 0; d < 2 * kD32; ++d) {
            const cache_bf16x8 a0 = cache_decode(vr[d].x, vr[d].y, v_scale), a1 = cache_decode(vr[d].z, vr[d].w, v_scale);
#pragma unroll
            for (int u = 0; u < kSets; ++u) {
                o[u][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, p[u][0], o[u][d], 0, 0, 0);
                o[u][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, p[u][1], o[u][d], 0, 0, 0);
            }
        }
        here = after;
        if (more) fetch_v(step + kCacheWaves, here.v);
    }
    if (__any(nans != 0u)) {
        const uint32_t first = max(from, least / kCacheStep);
        for (step = first + (wave + kCacheWaves - (first - from) % kCacheWaves) % kCacheWaves; step < to; step += kCacheWaves) {
            const uint32_t key = step * kCacheStep + 16u * g, n = rows.len > key ? min(rows.len - key, 16u) : 0u;
            fetch_v(step, page_of(key));
            const uint32_t past = past_of(v_scale);
            mark_nans(o, [&](int d) FB4_INLINE { return nans_of(first_bytes(vr[d], n), past); }, key, limit);
        }
    }
    // ---- the wavefronts meet
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        cache_exact(state[u], o[u], factor);
#pragma unroll
        for (int d = 0; d < 2 * kD32; ++d) *reinterpret_cast<cache_f32x4*>(&meet[wave][r][16 * d + 4 * g]) = o[u][d];
        if (g == 0) states[wave][r] = make_float2(state[u].most, state[u].sum);
        __syncthreads();
        const uint32_t row = threadIdx.x >> 4, at_row = 16u * u + row;
        if (at_row < n_rows) {
            float most = states[0][row].x, w[kCacheWaves], total = 0.0f;
#pragma unroll
            for (int i = 1; i < (int)kCacheWaves; ++i) most = fmaxf(most, states[i][row].x);
            const float base = most == -__builtin_inff() ? 0.0f : most;
#pragma unroll
            for (int i = 0; i < (int)kCacheWaves; ++i) {
                w[i] = __builtin_amdgcn_exp2f((states[i][row].x - base) * factor);
                total = fmaf(states[i][row].y, w[i], total);
            }
            const uint32_t at = tile * kRows + at_row, token = at / group, head = hk * group + (at - token * group);
            const float inverse = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;   // (a NaN stays; no key: zeros)
            for (uint32_t c = 4u * (threadIdx.x & 15u); c < dim; c += 64u) {
                cache_f32x4 x = *reinterpret_cast<const cache_f32x4*>(&meet[0][row][c]) * w[0];
#pragma unroll
                for (int i = 1; i < (int)kCacheWaves; ++i) {
                    const cache_f32x4 y = *reinterpret_cast<const cache_f32x4*>(&meet[i][row][c]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = fmaf(y[j], w[i], x[j]);
                }
                if (kSplit && parts > 1u) {
                    *reinterpret_cast<cache_f32x4*>(part_rows(workspace, blockIdx.x, kRows, dim) + at_row * dim + c) = x;
                } else {
                    uint16_t* place = out + ((size_t)head * so.head + (size_t)(rows.first + token) * so.token) * 8u + c;
                    *reinterpret_cast<uint2*>(place) = rounded(x, inverse);
                }
            }
            if ((threadIdx.x & 15u) == 0) {
                if (kSplit && parts > 1u) part_states(workspace, blockIdx.x, kRows, dim)[at_row] = make_float2(most, total);
                else if (lse) lse[(size_t)(rows.first + token) * s.heads + head] = total == 0.0f ? -__builtin_inff() : fmaf(base, s.scale, kCacheLn2 * __builtin_amdgcn_logf(total));
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------ attention of many queries
// Where a row's piece lies in LDS.  A read of 16 bytes a lane takes the 64 banks in four turns of 16 lanes: of lane group g the rows 0 .. 3 and 12 ..
// 15 with the rows 4 .. 11 of g + 1 (g even; and the other way round).  In each turn the pieces p of one half and p + slots / 4 of the other have
// to lie in different banks: slots are exchanged by row, so that either half's are closed under that step.  (Rows 16 bytes further apart than they
// are long instead, which does for 16 rows of one group: of 128 channels a prompt's LDS busy 49 % of the cycles against 35, 1755 us against 1742, 64 channels,
// 5 sequences of 900 queries 166 and 161.  Kept so, as 0 slots, for rows of 12 pieces, which would leave every fourth slot of 16 unused: frames of 72 channels, one
// clip 297 and 311, two 490 and 500, four 984 and 950, 3500 tokens over 12000 373 and 378.)
template <uint32_t kSlots>
__device__ __forceinline__ uint32_t slot_of_piece(uint32_t piece, uint32_t row)
{
    if (kSlots == 0) return piece;
    constexpr uint32_t kLow = kSlots ? kSlots / 4 : 1, kShift = kSlots == 16 ? 0 : kSlots == 8 ? 1 : 2;
    const uint32_t y = row >> kShift, x = y / kLow;   // x: row / 4
    return piece ^ ((((x ^ x >> 1) & 1u) * 2u + (x >> 1)) * kLow + y % kLow);
}
// As above, for 128 rows to a workgroup, 32 to a wavefront.  A step's keys and values come into LDS once for all four, decoded: wavefront w asks
// for the w-th sixteenth of each two steps ahead and puts it down as bf16 one step ahead, so that the converter's half rate (7 cycles for two
// elements) is paid once for 128 rows.  Rows of keys lie by tile and operand row, rows of values by channel, in pieces of 16 bytes that slot_of_piece
// places.
//
// What bounds it: no one unit -- vector instructions 45 % of the cycles, matrix cores 38 %, LDS 35 % (a prompt of 16384 tokens, 24 heads over 8 of
// 128 channels, 1649 GFLOP: 1750 to 1800 us, 0.92 to 0.94 PFLOP/s), and a wavefront's phases one after the other: without staging it takes 0.71 of the
// time, without the exponentials 0.88, without the reads of keys 0.89, without the barrier 0.90.  Two clips' frame of 1350 queries over 22950 keys, 16
// heads of 72 channels, 262 GFLOP: 484 to 502 us, 26 to 28 of it joining (72 channels take the products of 96, and of 11 tiles the last is 70 rows).
// Two wavefronts per SIMD with 200 to 243 of their 256 registers are what the sizes allow; 64 rows to a wavefront at one per SIMD took 3379 us, eight
// wavefronts to a workgroup 1767 and 597 for the frame, E4M3 in LDS decoded by every wavefront 2275, the next keys' products beside the weights 2500.
template <int kD32, bool kWhole, bool kSplit>
__global__ __launch_bounds__(64 * kCacheWaves) __attribute__((amdgpu_waves_per_eu(2)))
void cache_tiles_kernel(const uint16_t* q, const uint8_t* cache, const uint8_t* scales, const int32_t* tables, const int32_t* lens, const int32_t* starts, uint16_t* out,
                        float* lse, float* workspace, CacheStrides sq, CacheStrides so, CacheShape s)
{
    constexpr int kSets = 2;
    constexpr bool kApart = kD32 == 3;   // rows 16 bytes apart instead of exchanged pieces
    constexpr uint32_t kSlotsK = kApart ? 0 : 4 * kD32, kSlotsV = kApart ? 0 : kCacheStep / 8;
    constexpr uint32_t kPitchK = 64 * kD32 + 16 * kApart, kPitchV = 2 * kCacheStep + 16 * kApart;
    constexpr uint32_t kKeys = kCacheStep * kPitchK, kBuffer = kKeys + 32 * kD32 * kPitchV;
    constexpr int kAsksK = kD32, kAsksV = (kD32 + 1) / 2;   // of 64 lanes: 8 bytes of a key each, 16 of a channel
    __shared__ __align__(256) uint8_t lds[2 * kBuffer];
    __shared__ uint32_t notes[2][4];                        // of a buffer's sixteenths: kNone, kNan
    constexpr uint32_t kNone = 1, kNan = 2;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t r = lane & 15u, g = lane >> 4;
    auto scalar = [](uint32_t x) FB4_INLINE { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
    const uint32_t position = scalar(blockIdx.x / s.heads_k), hk = blockIdx.x - position * s.heads_k, group = scalar((uint32_t)s.heads / s.heads_k);
    uint32_t b, tile, part = 0, parts = 1;
    CacheRows rows;
    if (kSplit) {
        const uint32_t share = scalar(share_of(starts, lens, group, kTileRows, s));
        uint32_t at = position;
        b = scalar(walk_parts(starts, lens, group, kTileRows, share, 0xFFFFFFFFu, at, s));
        if (b >= s.batch) return;
        rows = rows_of(starts, lens, b, s);
        parts = parts_of(rows.len, share, kTileRows);
        tile = scalar(at) / parts;
        part = scalar(at) - tile * parts;
    } else {
        const uint32_t slot = s.tokens * group / kTileRows + s.batch - 1u - position;   // (of a causal prompt the longest first)
        b = scalar(sequence_of(starts, slot, group, kTileRows, s));
        rows = rows_of(starts, lens, b, s);
        tile = slot - place_of(rows.first, b, group, kTileRows);
        if (tile >= tiles_of(rows.n, group, kTileRows)) return;
    }
    rows.first = scalar(rows.first), rows.n = scalar(rows.n), rows.len = scalar(rows.len), tile = scalar(tile), part = scalar(part), parts = scalar(parts);
    const uint32_t n_rows = min(rows.n * group - tile * kTileRows, kTileRows), first_row = wave * 32u;
    const uint32_t pieces = s.dim8(), dim = pieces * 8u;
    cache_bf16x8 qf[kSets][kD32];
    uint32_t limit[kSets];
    auto limit_of = [&](uint32_t row) FB4_INLINE {
        const uint32_t token = (tile * kTileRows + row) / group;
        return s.causal() ? (uint32_t)max((int64_t)rows.len - (int64_t)rows.n + (int64_t)token + 1, (int64_t)0) : rows.len;
    };
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        const uint32_t row = min(first_row + 16u * u + r, n_rows - 1u), at = tile * kTileRows + row, token = at / group, head = hk * group + (at - token * group);
        limit[u] = limit_of(row);
        const uint16_t* x = q + ((size_t)head * sq.head + (size_t)(rows.first + token) * sq.token) * 8u;
#pragma unroll
        for (int i = 0; i < kD32; ++i) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if (kWhole || kD32 * g + i < pieces) w = reinterpret_cast<const uint4*>(x)[kD32 * g + i];
            qf[u][i] = __builtin_bit_cast(cache_bf16x8, w);
        }
    }
    // the keys that all rows of this wavefront see, of the workgroup; the keys that any sees
    const uint32_t least = scalar(limit_of(min(first_row, n_rows - 1u))), least_of_all = scalar(limit_of(0)), steps = steps_of(scalar(limit_of(n_rows - 1u)));
    const uint32_t from = scalar((uint32_t)((uint64_t)steps * part / parts)), to = scalar((uint32_t)((uint64_t)steps * (part + 1u) / parts));
    const uint32_t bits = s.page_bits, in_page = (1u << bits) - 1u, held = (rows.len + in_page) >> bits;
    const int32_t* table = tables + (size_t)b * s.max_pages;
    const size_t page_bytes = (size_t)dim << bits;
    const uint8_t* values = cache + (size_t)s.pages * s.heads_k * page_bytes;
    auto page_of = [&](uint32_t key) FB4_INLINE {   // -1: none
        const uint32_t i = key >> bits;
        const int32_t p = s.max_pages ? table[min(i, s.max_pages - 1u)] : -1;   // (not after its length has come)
        return i < held && (uint32_t)p < s.pages ? p : -1;
    };
    // ---- this wavefront's sixteenth of a step, into registers and from there into LDS
    const uint32_t mine = 16u * wave;
    struct Asked {   // two steps' are on their way
        uint2 k[kAsksK];
        uint4 v[kAsksV];
        uint32_t k_byte, v_byte;
        bool there;
    };
    Asked even, odd;
    auto ask = [&](Asked& w, uint32_t step, int32_t page) FB4_INLINE {
        const uint32_t p = scalar((uint32_t)max(page, 0)), place = (step * kCacheStep + mine) & in_page;
        w.there = (int32_t)scalar((uint32_t)page) >= 0;
        const size_t at = (size_t)p * s.heads_k + hk;
        const uint8_t* k = cache + at * page_bytes + place * dim;
        const uint8_t* v = values + at * page_bytes + place;
        w.k_byte = scales[at];
        w.v_byte = scales[(size_t)s.pages * s.heads_k + at];
#pragma unroll
        for (int i = 0; i < kAsksK; ++i) {
            const uint32_t j = 64u * i + lane;
            w.k[i] = make_uint2(0, 0);
            if (kWhole || j < 16u * pieces) w.k[i] = reinterpret_cast<const uint2*>(k)[j];
        }
#pragma unroll
        for (int i = 0; i < kAsksV; ++i) {
            const uint32_t c = 64u * i + lane;
            w.v[i] = make_uint4(0, 0, 0, 0);
            if (c < dim) w.v[i] = *reinterpret_cast<const uint4*>(v + ((size_t)c << bits));
        }
    };
    auto put = [&](Asked& w, uint32_t step, uint32_t buffer) FB4_INLINE {
        const float fk = __builtin_bit_cast(float, w.k_byte << 23), fv = __builtin_bit_cast(float, w.v_byte << 23);
        uint8_t* to_k = lds + buffer;
        uint8_t* to_v = lds + buffer + kKeys;
#pragma unroll
        for (int i = 0; i < kAsksK; ++i) {
            const uint32_t j = 64u * i + lane, key = kWhole ? j / (4u * kD32) : j / pieces, c = j - key * (kWhole ? 4u * kD32 : pieces);
            // key 4 t + x of sixteenth w: row 4 w + x of tile t
            const uint32_t row = 4u * wave + (key & 3u);
            if (kWhole || j < 16u * pieces)
                *reinterpret_cast<cache_bf16x8*>(to_k + ((key & ~3u) * 4u + row) * kPitchK + 16u * slot_of_piece<kSlotsK>(c, row)) = cache_decode(w.k[i].x, w.k[i].y, fk);
        }
        // a page that is not there, what lies behind the end: zeros; and no NaN or Inf that a query does not see
        const uint32_t key = step * kCacheStep + mine;
        uint32_t note = w.there ? 0u : kNone;
        if (!w.there || key + 16u > least_of_all) {
            const uint32_t n = w.there && rows.len > key ? min(rows.len - key, 16u) : 0u;
            const uint32_t past = past_numbers(w.v_byte);
            uint32_t some = 0;
#pragma unroll
            for (int i = 0; i < kAsksV; ++i) {
                w.v[i] = first_bytes(w.v[i], n);
                const uint4 bad = nans_of(w.v[i], past);
                some |= bad.x | bad.y | bad.z | bad.w;
                w.v[i] = without(w.v[i], bad);
            }
            if (__any(some != 0u)) note |= kNan;
        }
#pragma unroll
        for (int i = 0; i < kAsksV; ++i) {
            const uint32_t c = 64u * i + lane;
            if (c < 32u * kD32) {   // (channels past the row: zeros)
                uint8_t* at = to_v + c * kPitchV;
                *reinterpret_cast<cache_bf16x8*>(at + 16u * slot_of_piece<kSlotsV>(2u * wave, c & 15u)) = cache_decode(w.v[i].x, w.v[i].y, fv);
                *reinterpret_cast<cache_bf16x8*>(at + 16u * slot_of_piece<kSlotsV>(2u * wave + 1u, c & 15u)) = cache_decode(w.v[i].z, w.v[i].w, fv);
            }
        }
        if (lane == 0) notes[buffer != 0u][wave] = note;
    };
    const float factor = s.scale * kCacheLog2E;
    cache_f32x4 o[kSets][2 * kD32];
    CacheState state[kSets];
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        state[u] = CacheState{-__builtin_inff(), 0.0f, 0.0f, false};
#pragma unroll
        for (int d = 0; d < 2 * kD32; ++d) o[u][d] = cache_f32x4{0, 0, 0, 0};
    }
    uint32_t k_at[kD32], v_at[2];
#pragma unroll
    for (uint32_t i = 0; i < kD32; ++i) k_at[i] = r * kPitchK + 16u * slot_of_piece<kSlotsK>(kD32 * g + i, r);
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) v_at[h] = kKeys + r * kPitchV + 16u * slot_of_piece<kSlotsV>(2u * g + h, r);
    const bool idle = first_row >= n_rows;
    int32_t page = -1;
    if (!kWhole) {   // channels past the row, of keys: zeros for good (the queries' are too, but 0 times what was here need not be)
        for (uint32_t i = threadIdx.x; i < 2u * kBuffer / 16u; i += 64u * kCacheWaves) reinterpret_cast<uint4*>(lds)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
    }
    if (from < to) {
        auto at = [&](uint32_t step) FB4_INLINE { return page_of(step * kCacheStep + mine); };
        ask(even, from, at(from));
        ask(odd, from + 1u, at(from + 1u));
        page = at(from + 2u);
        put(even, from, 0);
        ask(even, from + 2u, page);
        page = at(from + 3u);
    }
    uint32_t seen_notes = 0;
    // step: its operands are in `buffer`; those of the next, in w, go to the other, and those of the one two behind that are asked for
    auto run_step = [&](uint32_t step, uint32_t buffer, Asked& w) FB4_INLINE {
        __syncthreads();   // this step's operands are there; everyone is done with the other buffer
        const uint8_t* keys = lds + buffer + (kApart ? k_at[0] : 0u);
        const uint8_t* vals = lds + buffer + (kApart ? v_at[0] : 0u);
        if (!idle) {
            const uint32_t note = notes[buffer != 0u][g];
            cache_f32x4 sc[kSets][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int u = 0; u < kSets; ++u) sc[u][t] = cache_f32x4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < kD32; ++i) {
                    const cache_bf16x8 a = *reinterpret_cast<const cache_bf16x8*>(keys + 16u * t * kPitchK + (kApart ? 16u * i : k_at[i]));
#pragma unroll
                    for (int u = 0; u < kSets; ++u) sc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[u][i], sc[u][t], 0, 0, 0);
                }
            }
            const uint32_t key = step * kCacheStep + 16u * g;
            if (step * kCacheStep + kCacheStep > least || __any(note & kNone)) {
#pragma unroll
                for (int u = 0; u < kSets; ++u) {
                    const uint32_t seen = note & kNone ? 0u : limit[u];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) sc[u][t][i] = key + 4u * t + i >= seen ? -__builtin_inff() : sc[u][t][i];
                    }
                }
            }
            cache_bf16x8 p[kSets][2];
#pragma unroll
            for (int u = 0; u < kSets; ++u) cache_reference(sc[u], state[u], o[u], factor);
#pragma unroll
            for (int u = 0; u < kSets; ++u) cache_powers(sc[u], state[u], p[u], factor);
#pragma unroll
            for (int d = 0; d < 2 * kD32; ++d) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const cache_bf16x8 a = *reinterpret_cast<const cache_bf16x8*>(vals + 16u * d * kPitchV + (kApart ? 16u * h : v_at[h]));
#pragma unroll
                    for (int u = 0; u < kSets; ++u) o[u][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[u][h], o[u][d], 0, 0, 0);
                }
            }
            seen_notes |= note;
        }
        if (step + 1u < to) {
            put(w, step + 1u, kBuffer - buffer);
            ask(w, step + 3u, page);
            page = page_of((step + 4u) * kCacheStep + mine);
        }
    };
    for (uint32_t step = from; step < to;) {
        run_step(step, 0, odd);
        if (++step >= to) break;
        run_step(step, kBuffer, even);
        ++step;
    }
    if (__any(seen_notes & kNan)) {
        for (uint32_t step = max(from, least_of_all / kCacheStep); step < to; ++step) {
            const uint32_t key = step * kCacheStep + 16u * g;
            const int32_t at = page_of(key);
            const size_t place = (size_t)max(at, 0) * s.heads_k + hk;
            const uint8_t* v = values + place * page_bytes + (key & in_page);
            const uint32_t n = at >= 0 && rows.len > key ? min(rows.len - key, 16u) : 0u, past = past_numbers(scales[(size_t)s.pages * s.heads_k + place]);
            mark_nans(o, [&](int d) FB4_INLINE {
                const uint32_t c = 16u * d + r;
                return nans_of(c < dim ? first_bytes(*reinterpret_cast<const uint4*>(v + ((size_t)c << bits)), n) : make_uint4(0, 0, 0, 0), past);
            }, key, limit);
        }
    }
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
        cache_exact(state[u], o[u], factor);
        const uint32_t row = first_row + 16u * u + r;
        if (row >= n_rows) continue;
        const uint32_t at = tile * kTileRows + row, token = at / group, head = hk * group + (at - token * group);
        const float total = state[u].sum, inverse = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
#pragma unroll
        for (int d = 0; d < 2 * kD32; ++d) {
            const uint32_t c = 16u * d + 4u * g;
            if (!kWhole && c >= dim) continue;
            if (kSplit && parts > 1u) {
                *reinterpret_cast<cache_f32x4*>(part_rows(workspace, blockIdx.x, kTileRows, dim) + row * dim + c) = o[u][d];
            } else {
                uint16_t* place = out + ((size_t)head * so.head + (size_t)(rows.first + token) * so.token) * 8u + c;
                *reinterpret_cast<uint2*>(place) = rounded(o[u][d], inverse);
            }
        }
        if (g == 0) {
            const float base = state[u].most == -__builtin_inff() ? 0.0f : state[u].most;
            if (kSplit && parts > 1u) part_states(workspace, blockIdx.x, kTileRows, dim)[row] = make_float2(state[u].most, total);
            else if (lse) lse[(size_t)(rows.first + token) * s.heads + head] = total == 0.0f ? -__builtin_inff() : fmaf(base, s.scale, kCacheLn2 * __builtin_amdgcn_logf(total));
        }
    }
}

// The parts of a row meet: sum of parts' sums and rows times exp2((their maximum - the largest) c), both in fp32.  kWaves = 4: four wavefronts to a row,
// where rows are few and parts many; 1: kJoinRows rows to a wavefront, one after the other, so that finding their parts, a chain of reads, comes once for
// them.  Half a wavefront takes a part, four channels a lane.  (The whole call, one row to a wavefront's turn and four wavefronts to a row, us: 24 rows over
// 65536 keys 61, 37; 192 over 8192: 43, 34; 768: 91, 89; 4080: 49, 59; 32400: 175, 273.  Sixteen wavefronts to a row: 24 rows 15.9, four 15.0.)
// What bounds it is that chain, about 10 us, then the parts' rows: 43200 rows of three parts of 72 channels 28 us.
constexpr uint32_t kJoinRows = 4, kJoinWaves = 4, kJoinFew = 1024;
template <int kWaves>
__global__ __launch_bounds__(256) void cache_join_kernel(float* workspace, const int32_t* lens, const int32_t* starts, uint16_t* out,
                                                         float* lse, uint32_t n_positions, uint32_t tile_rows, CacheStrides so, CacheShape s)
{
    __shared__ cache_f32x4 meet[kWaves][32];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    auto scalar = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
    const uint32_t group = scalar((uint32_t)s.heads / s.heads_k), dim = s.dim8() * 8u, n_rows = s.tokens * s.heads;
    const uint32_t first_row = kWaves > 1 ? blockIdx.x : (blockIdx.x * 4u + wave) * kJoinRows;
    const uint32_t share = scalar(share_of(starts, lens, group, tile_rows, s));
    const float factor = s.scale * kCacheLog2E;
    const uint32_t c = 4u * (lane & 31u);
    CacheRows rows = {0, 0, 0};
    uint32_t base = 0, parts = 1;
    for (uint32_t row = first_row; row < min(first_row + (kWaves > 1 ? 1u : kJoinRows), n_rows); ++row) {
        const uint32_t token = scalar(row / s.heads), head = row - token * s.heads, hk = scalar(head / group);
        if (token < rows.first || token - rows.first >= rows.n) {   // (the first row's sequence, and another one's later)
            const uint32_t b = scalar(sequence_of(starts, token, 0u, 1u, s));
            rows = rows_of(starts, lens, b, s);
            if (token < rows.first || token - rows.first >= rows.n) {   // (of none; with several wavefronts the whole workgroup)
                rows.n = 0;   // (the sequence found may be the next row's, whose parts are not known yet)
                continue;
            }
            base = 0;
            walk_parts(starts, lens, group, tile_rows, share, b, base, s);
            base = scalar(base);
            parts = scalar(parts_of(rows.len, share, tile_rows));
        }
        if (parts == 1u) continue;   // (written already)
        const uint32_t at = (token - rows.first) * group + (head - hk * group), tile = at / tile_rows;
        const uint32_t first = (base + tile * parts) * s.heads_k + hk;   // of the parts' positions
        const uint32_t n = min(parts, first < n_positions ? (n_positions - first + s.heads_k - 1u) / s.heads_k : 0u);
        const uint32_t in_tile = at - tile * tile_rows;
        const size_t step = (size_t)s.heads_k * tile_rows * (dim + 2u);   // floats from part to part
        const float* from = part_rows(workspace, first, tile_rows, dim) + in_tile * dim + c;
        const float* state = reinterpret_cast<const float*>(part_states(workspace, first, tile_rows, dim) + in_tile);
        auto state_of = [&](uint32_t p) { return *reinterpret_cast<const float2*>(state + p * step); };
        // (the first parts' rows are asked for before their maxima are known)
        const uint32_t p0 = (kWaves > 1 ? 2u * wave : 0u) + (lane >> 5);
        auto part = [&](uint32_t p) { return *reinterpret_cast<const cache_f32x4*>(from + p * step); };
        cache_f32x4 x[4], o = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            x[i] = cache_f32x4{0, 0, 0, 0};
            if (c < dim && p0 + 2u * kWaves * i < n) x[i] = part(p0 + 2u * kWaves * i);
        }
        float most = -__builtin_inff(), sum = 0.0f;
        float2 mine = make_float2(-__builtin_inff(), 0.0f);
        if (lane < n) mine = state_of(lane);
        for (uint32_t p = lane; p < n; p += 64u) most = fmaxf(most, p < 64u ? mine.x : state_of(p).x);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        const float reference = most == -__builtin_inff() ? 0.0f : most;
        for (uint32_t p = lane; p < n; p += 64u) {
            const float2 st = p < 64u ? mine : state_of(p);
            sum = fmaf(st.y, __builtin_amdgcn_exp2f((st.x - reference) * factor), sum);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        const float weight = __builtin_amdgcn_exp2f((mine.x - reference) * factor);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {   // (rows of zeros where there is none)
            const float w = __shfl(weight, p0 + 2u * kWaves * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = fmaf(x[i][j], w, o[j]);
        }
        if (c < dim) {
#pragma unroll 4
            for (uint32_t p = p0 + 8u * kWaves; p < n; p += 2u * kWaves) {
                const float w = __builtin_amdgcn_exp2f((state_of(p).x - reference) * factor);
                const cache_f32x4 y = part(p);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = fmaf(y[j], w, o[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], 32);
        if (kWaves > 1) {
            if (lane < 32u) meet[wave][lane] = o;
            __syncthreads();
            if (wave > 0) return;
            for (int i = 1; i < kWaves; ++i) o += meet[i][lane & 31u];
        }
        const float inverse = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
        if (c < dim && lane < 32u) {
            uint16_t* place = out + ((size_t)head * so.head + (size_t)token * so.token) * 8u + c;
            *reinterpret_cast<uint2*>(place) = rounded(o, inverse);
        }
        if (lse && lane == 0) lse[(size_t)token * s.heads + head] = sum == 0.0f ? -__builtin_inff() : fmaf(reference, s.scale, kCacheLn2 * __builtin_amdgcn_logf(sum));
    }
}

#undef FB4_INLINE

}  // namespace fb4
