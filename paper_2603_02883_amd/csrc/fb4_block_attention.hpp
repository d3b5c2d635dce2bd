// Attention over blocks of keys, and the choice of the blocks.
//
// Choice: for every block of queries and of keys the mean of its rows (block_means_kernel), then per block of queries the
// products with the keys' means and the largest `top` of them (select_blocks_kernel).  All of it in double: the result is a
// list of numbers, which two nearly equal scores would make depend on the order of their sums.
//
// Attention: S^T = K Q^T and O^T = V^T P^T as 32x32x16 MFMAs, one pass over the keys with the running maximum and sum of the
// softmax.  Transposed so that a lane's 16 accumulators are 16 keys of ONE query: maximum and sum stay inside the lane, and
// the two half-wavefronts, which hold different keys, meet once per tile.  The accumulators of a block of 32 keys are keys
// 8 (i / 4) + 4 (lane / 32) + i % 4, i = 0 .. 15; a B operand of the second product wants eight keys per lane and any order of
// the keys will do as long as V^T has the same one, so P goes from accumulator to operand without leaving the lane: step s
// takes the accumulators 8 s .. 8 s + 7, and V^T's operand is read as the rows 16 s + 4 (lane / 32) + {0..3} and 8 further, by
// the LDS read that transposes 4 rows x 16 columns.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fb4_mfma.hpp"

namespace fb4 {

constexpr int kMeanThreads = 256;
constexpr uint32_t kSelectMaxBlocks = 2048;   // of keys: a row of scores and its order stay in LDS

// ------------------------------------------------------------------------------------------------ choice of the blocks
struct BlockShape {
    uint32_t tokens_q, tokens_k;
    uint16_t heads, heads_k;      // heads_k divides heads
    uint16_t block_q, block_k;
    uint32_t blocks_q, blocks_k;
};

// lens: [batch][2], clamped to what is there.
__device__ __forceinline__ uint32_t length_of(const int32_t* lens, uint32_t b, uint32_t which, uint32_t tokens)
{
    return lens ? (uint32_t)min(max(lens[2u * b + which], 0), (int32_t)tokens) : tokens;
}

// One workgroup per block of rows; means: double [batch * heads][blocks_q][dim], then [batch * heads_k][blocks_k][dim].
template <int kLanes>
__global__ __launch_bounds__(kMeanThreads) void block_means_kernel(const uint16_t* q, const uint16_t* k, const int32_t* lens, double* means,
                                                                   uint32_t n_q, uint32_t pieces, BlockShape s)
{
    constexpr uint32_t kRows = kMeanThreads / kLanes;   // rows per step
    __shared__ double part[kRows][kLanes * 8];
    const bool is_k = blockIdx.x >= n_q;
    const uint32_t at = is_k ? blockIdx.x - n_q : blockIdx.x, blocks = is_k ? s.blocks_k : s.blocks_q;
    const uint32_t g = at / blocks, block = at - g * blocks;   // g = batch * heads + head
    const uint32_t tokens = is_k ? s.tokens_k : s.tokens_q, size = is_k ? s.block_k : s.block_q;
    const uint32_t len = length_of(lens, g / (is_k ? s.heads_k : s.heads), is_k, tokens);
    const uint32_t first = block * size, n = len > first ? min(len - first, size) : 0u;
    const uint32_t l = threadIdx.x % kLanes, sub = threadIdx.x / kLanes;
    double sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const uint16_t* base = (is_k ? k : q) + ((size_t)g * tokens + first) * (pieces * 8u) + 8u * l;
    for (uint32_t r0 = 0; r0 < n; r0 += 4u * kRows) {
        uint4 v[4];   // (a thread's reads before its sums)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t r = r0 + i * kRows + sub;
            v[i] = make_uint4(0, 0, 0, 0);
            if (l < pieces && r < n) v[i] = *reinterpret_cast<const uint4*>(base + (size_t)r * (pieces * 8u));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum[2 * j] += (double)__builtin_bit_cast(float, w[j] << 16);
                sum[2 * j + 1] += (double)__builtin_bit_cast(float, w[j] & 0xFFFF0000u);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) part[sub][8u * l + j] = sum[j];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < pieces * 8u; c += kMeanThreads) {
        double total = 0.0;
        for (uint32_t r = 0; r < kRows; ++r) total += part[r][c];
        means[(size_t)blockIdx.x * (pieces * 8u) + c] = n ? total / (double)n : 0.0;
    }
}

// A number's place in the order: larger is better, a NaN below every number (and above 0, which is no block), -0 is 0.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    return x != x ? 1u : x == 0.0f ? 0x80000000u : u >> 31 ? ~u : u | 0x80000000u;   // (-Inf comes to 0x007FFFFF)
}
__device__ __forceinline__ float number_of(uint32_t order)
{
    return order == 1u ? __builtin_nanf("") : __builtin_bit_cast(float, order >> 31 ? order & 0x7FFFFFFFu : ~order);
}
__device__ __forceinline__ uint64_t order_of(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return x != x ? 1ull : x == 0.0 ? 0x8000000000000000ull : u >> 63 ? ~u : u | 0x8000000000000000ull;
}

typedef double select_f64x2 __attribute__((ext_vector_type(2)));
typedef double select_f64x4 __attribute__((ext_vector_type(4)));
constexpr int kSelectThreads = 512;
constexpr uint32_t kSelectRows = 16;   // blocks of queries to a workgroup

// A workgroup takes 16 blocks of queries of one head: their scores with all the head's blocks of keys by 16x16x4 MFMAs in double,
// then the largest `top` of every row.  The channels of a product may come in any order as long as both operands have the same:
// lane group k of 16 holds channels 16 c + 4 k .. + 3 for the four steps of chunk c, which are 32 bytes of its row.
// LDS keeps the scores rounded to fp32, half of what the doubles would take, so that one workgroup's search runs beside another's
// products.  Rounding keeps the order but for what becomes equal, so the fp32 values decide unless the border falls between
// equal ones; those blocks' scores are then formed again in double.
// D16: channels / 16, rounded up; kValues: scores of a row per lane.
// Measured: 24 heads x 1024 x 1024 blocks x 128 channels 424 us with doubles in LDS and a search bit by bit on four wavefronts.
template <int D16, int kValues>
__global__ __launch_bounds__(kSelectThreads) __attribute__((amdgpu_waves_per_eu(kValues > 16 ? 2 : 4)))
void select_blocks_kernel(const double* means, const int32_t* lens, int32_t* chosen, float* scores, uint32_t top, uint32_t n_q, uint32_t dim,
                          uint32_t row_tiles, uint32_t n_workgroups, BlockShape s)
{
    constexpr uint32_t kWaves = kSelectThreads / 64, kRowDoubles = 16 * D16, kPieces = kRowDoubles / 2;
    __shared__ __align__(16) uint32_t order[kSelectRows][64 * kValues];
    __shared__ __align__(16) double queries[kSelectRows * kRowDoubles];   // 16-byte piece p of row r at p ^ (r % 8)
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t pos = xcd_local_position(blockIdx.x, n_workgroups);
    const uint32_t g = pos / row_tiles, block0 = (pos - g * row_tiles) * kSelectRows;
    const uint32_t b = g / s.heads, h = g - b * s.heads, gk = b * s.heads_k + h / (s.heads / s.heads_k);
    const uint32_t len_q = length_of(lens, b, 0, s.tokens_q), len_k = length_of(lens, b, 1, s.tokens_k);
    const uint32_t n = (len_k + s.block_k - 1) / s.block_k;   // blocks with a key
    const uint32_t rows = min(s.blocks_q - block0, kSelectRows);
    const double* mq = means + ((size_t)g * s.blocks_q + block0) * dim;
    const double* mk = means + ((size_t)n_q + (size_t)gk * s.blocks_k) * dim;
    for (uint32_t i = threadIdx.x; i < kSelectRows * kPieces; i += kSelectThreads) {
        const uint32_t r = i / kPieces, p = i - r * kPieces;
        select_f64x2 w = {0.0, 0.0};
        if (r < rows && 2u * p < dim) w = *reinterpret_cast<const select_f64x2*>(mq + (size_t)r * dim + 2u * p);
        *reinterpret_cast<select_f64x2*>(queries + r * kRowDoubles + 2u * (p ^ (r & 7u))) = w;
    }
    __syncthreads();
    // ---- scores
    const uint32_t r = lane & 15u, k4 = 4u * (lane >> 4);
    for (uint32_t t = wave; 16u * t < n; t += kWaves) {
        const double* row = mk + (size_t)(16u * t + r) * dim;
        const bool there = 16u * t + r < n;
        select_f64x4 acc = {0, 0, 0, 0};
        constexpr int kChunks = D16 > 6 ? (D16 + 1) / 2 : D16;   // read at a time (128 registers hold no 8)
#pragma unroll 1
        for (int c0 = 0; c0 < D16; c0 += kChunks) {
            select_f64x2 keys[2 * kChunks];
#pragma unroll
            for (int i = 0; i < 2 * kChunks; ++i) {
                const uint32_t c = 16u * (c0 + i / 2) + k4 + 2u * (i % 2);
                keys[i] = select_f64x2{0.0, 0.0};
                if (there && c < dim) keys[i] = *reinterpret_cast<const select_f64x2*>(row + c);
            }
#pragma unroll
            for (int i = 0; i < 2 * kChunks; ++i) {
                if (D16 % kChunks && c0 + i / 2 >= D16) break;
                const uint32_t p = 8u * (c0 + i / 2) + k4 / 2u + i % 2;
                const select_f64x2 a = *reinterpret_cast<const select_f64x2*>(queries + r * kRowDoubles + 2u * (p ^ (r & 7u)));
                acc = __builtin_amdgcn_mfma_f64_16x16x4f64(a[0], keys[i][0], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f64_16x16x4f64(a[1], keys[i][1], acc, 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)   // accumulator i: row lane / 16 + 4 i, column lane % 16
            order[(lane >> 4) + 4u * i][16u * t + r] = there ? order_of((float)acc[i]) : 0;
    }
    __syncthreads();
    // ---- the largest of every row
    const uint64_t before = (1ull << lane) - 1;
    for (uint32_t row = wave; row < rows; row += kWaves) {
        const uint32_t have = (block0 + row) * s.block_q < len_q ? n : 0u;   // (no query: no blocks)
        const uint32_t want = min(top, have);
        uint32_t mine[kValues];   // (0: no block)
#pragma unroll
        for (int i = 0; i < kValues; ++i) mine[i] = 64u * i + lane < have ? order[row][64u * i + lane] : 0;
        auto at_least = [&](uint32_t bound) {
            uint32_t count = 0;
#pragma unroll
            for (int i = 0; i < kValues; ++i) count += (uint32_t)__popcll(__ballot(mine[i] >= bound));
            return count;
        };
        // Where the want-th largest lies: at_least(low) >= want > at_least(high).  By halves of the numbers' range (ten steps for
        // 1024 scores) until exactly `want` are at least `low`, or two numbers are left with none between them; then by halves of their
        // places in the order.
        uint32_t low = 1, high = 0, count = have;
        if (want > 0 && want < have) {
#pragma unroll
            for (int i = 0; i < kValues; ++i) {
                high = max(high, mine[i]);
                low = max(low, mine[i] ? ~mine[i] : 0u);
            }
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                high = max(high, (uint32_t)__shfl_xor(high, d));
                low = max(low, (uint32_t)__shfl_xor(low, d));
            }
            low = ~__builtin_amdgcn_readfirstlane(low);
            high = __builtin_amdgcn_readfirstlane(high) + 1u;   // (a NaN's or number's place: no overflow)
            bool numbers = true;
            while (count != want && high - low > 1u) {
                uint32_t trial = low + (high - low) / 2u;
                if (numbers) {
                    const uint32_t half = __builtin_amdgcn_readfirstlane(order_of(0.5f * number_of(low) + 0.5f * number_of(high - 1u)));
                    numbers = half > low && half < high;   // (not for a NaN, nor between neighbours)
                    if (numbers) trial = half;
                }
                const uint32_t c = at_least(trial);
                if (c >= want) {
                    low = trial;
                    count = c;
                } else {
                    high = trial;
                }
            }
        }
        // Those above `low` are in; of those equal to it all, or -- more than there is room for -- the best in double, ties to the
        // lower block.
        uint32_t ties = want - (want > 0 && count != want ? at_least(low + 1u) : 0u), out = 0;
        const bool all_equal = count == want;
        uint64_t bound = 0;
        uint64_t exact[kValues];
        if (!all_equal && want > 0) {
            const double* x = mq + (size_t)row * dim;
#pragma unroll
            for (int i = 0; i < kValues; ++i) {
                exact[i] = 0;
                if (mine[i] != low) continue;
                const double* y = mk + (size_t)(64u * i + lane) * dim;
                double sum = 0.0;
                for (uint32_t c = 0; c < dim; ++c) sum = fma(x[c], y[c], sum);
                exact[i] = order_of(sum);
            }
            for (int bit = 63; bit >= 0; --bit) {
                const uint64_t trial = bound | 1ull << bit;
                uint32_t c = 0;
#pragma unroll
                for (int i = 0; i < kValues; ++i) c += (uint32_t)__popcll(__ballot(exact[i] >= trial));
                if (c >= ties) bound = trial;
            }
#pragma unroll
            for (int i = 0; i < kValues; ++i) ties -= (uint32_t)__popcll(__ballot(exact[i] > bound));
        }
        const size_t at_row = ((size_t)g * s.blocks_q + block0 + row) * top;
        int32_t* to = chosen + at_row;
        float* to_score = scores ? scores + at_row : nullptr;
#pragma unroll
        for (int i = 0; i < kValues; ++i) {
            if (64u * i >= have || out >= want) break;
            bool taken = mine[i] >= low && mine[i];
            if (!all_equal) {
                const bool here = mine[i] == low;
                const uint64_t equal = __ballot(here && exact[i] == bound);
                taken = (taken && !here) || (here && (exact[i] > bound || (exact[i] == bound && (uint32_t)__popcll(equal & before) < ties)));
                ties -= min(ties, (uint32_t)__popcll(equal));
            }
            const uint64_t all = __ballot(taken);
            if (taken) {
                const uint32_t at = out + (uint32_t)__popcll(all & before);
                to[at] = (int32_t)(64u * i + lane);
                if (to_score) to_score[at] = number_of(mine[i]);
            }
            out += (uint32_t)__popcll(all);
        }
        for (uint32_t at = want + lane; at < top; at += 64) {
            to[at] = -1;
            if (to_score) to_score[at] = __builtin_nanf("");
        }
    }
}

// ------------------------------------------------------------------------------------------------ attention
constexpr uint32_t kTileKeys = 64;
constexpr uint32_t kAllBlocks = 0xFFFFFFFFu;   // no list (FB4_ALL_BLOCKS in 32 bits)

typedef float attn_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 attn_bf16x2 __attribute__((ext_vector_type(2)));
typedef short attn_s16x4 __attribute__((ext_vector_type(4)));

struct AttentionShape {
    uint32_t tokens_q, tokens_k, top;
    uint16_t heads, heads_k;
    uint8_t block_q, block_k, pieces;   // (block sizes in units of 64 tokens; dim / 8)
    uint8_t spare;
    uint32_t blocks_q, n_workgroups;
    float scale;
};
// Strides in units of 8 elements.
struct TensorStrides {
    uint32_t batch, head, token;
};

// A workgroup of kWaves wavefronts takes one block of 32 * kWaves queries of one head; every wavefront holds 32 of them as B
// operands and walks the listed blocks' tiles of 64 keys, which the workgroup stages in LDS.
// D32: channels / 32, rounded up (channels beyond dim are zero).
template <int D32, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void block_attention_kernel(const uint16_t* q, const uint16_t* k, const uint16_t* v, uint16_t* out, float* lse,
                                                                      const int32_t* blocks, const int32_t* lens, TensorStrides sv, TensorStrides so,
                                                                      AttentionShape s)
{
    constexpr int kSteps = D32 * 2;
    constexpr uint32_t kPitch = D32 * 64 + 16;   // bytes of a row in LDS
    __shared__ __align__(16) uint8_t lds_k[kTileKeys * kPitch], lds_v[kTileKeys * kPitch];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t half = lane >> 5, col = lane & 31u;
    const uint32_t pos = xcd_local_position(blockIdx.x, s.n_workgroups);
    const uint32_t g = pos / s.blocks_q, block = pos - g * s.blocks_q;   // g = batch * heads + head
    const uint32_t b = g / s.heads, h = g - b * s.heads, hk = h / (s.heads / s.heads_k);
    const uint32_t len_q = length_of(lens, b, 0, s.tokens_q), len_k = length_of(lens, b, 1, s.tokens_k);
    const uint32_t dim = s.pieces * 8u, first_q = block * s.block_q * 64u;
    if (first_q >= len_q) return;
    const uint32_t block_keys = s.block_k * 64u, blocks_k = (len_k + block_keys - 1) / block_keys;   // blocks with a key
    const uint16_t* kg = k + (size_t)(b * s.heads_k + hk) * s.tokens_k * dim;
    const uint16_t* vg = v + ((size_t)b * sv.batch + (size_t)hk * sv.head) * 8u;
    const uint32_t row = first_q + wave * 32u + col;   // this lane's query
    mfma_bf16x8 qf[kSteps];
    {
        const uint16_t* from = q + ((size_t)g * s.tokens_q + min(row, s.tokens_q - 1u)) * dim;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const uint32_t c = 16u * i + 8u * half;
            uint4 w = make_uint4(0, 0, 0, 0);
            if (c < dim) w = *reinterpret_cast<const uint4*>(from + c);
            qf[i] = __builtin_bit_cast(mfma_bf16x8, w);
        }
    }
    const float factor = s.scale * 1.44269504088896340736f;   // to powers of two
    mfma_f32x16 o[D32];
#pragma unroll
    for (int d = 0; d < D32; ++d) o[d] = mfma_f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    float most = -__builtin_inff(), sum = 0.0f;   // of this lane's query: largest product so far, sum over this lane's keys
    const int32_t* list = blocks + (size_t)pos * s.top;
    const bool all = s.top == kAllBlocks;
    const uint32_t entries = all ? blocks_k : s.top;
    for (uint32_t e = 0; e < entries; ++e) {
        const uint32_t which = all ? e : (uint32_t)list[e];
        if (which >= blocks_k) continue;   // (a negative one too)
        const uint32_t end = min((which + 1) * block_keys, len_k);
        for (uint32_t key0 = which * block_keys; key0 < end; key0 += kTileKeys) {
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < kTileKeys * D32 * 4; i += 64 * kWaves) {
                const uint32_t r = i / (D32 * 4), p = i - r * (D32 * 4);
                uint4 kw = make_uint4(0, 0, 0, 0), vw = make_uint4(0, 0, 0, 0);
                if (key0 + r < end && p < s.pieces) {
                    kw = *reinterpret_cast<const uint4*>(kg + (size_t)(key0 + r) * dim + 8u * p);
                    vw = *reinterpret_cast<const uint4*>(vg + ((size_t)(key0 + r) * sv.token + p) * 8u);
                }
                *reinterpret_cast<uint4*>(lds_k + r * kPitch + 16u * p) = kw;
                *reinterpret_cast<uint4*>(lds_v + r * kPitch + 16u * p) = vw;
            }
            __syncthreads();
            mfma_f32x16 sc[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                sc[j] = mfma_f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const uint4 a = *reinterpret_cast<const uint4*>(lds_k + (32u * j + col) * kPitch + 32u * i + 16u * half);
                    sc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(mfma_bf16x8, a), qf[i], sc[j], 0, 0, 0);
                }
            }
            if (key0 + kTileKeys > end) {   // (the sequence's last tile)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (key0 + 32u * j + 8u * (i / 4) + 4u * half + i % 4 >= end) sc[j][i] = -__builtin_inff();
                    }
                }
            }
            float larger = most;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int i = 0; i < 16; ++i) larger = fmaxf(larger, sc[j][i]);
            }
            larger = fmaxf(larger, __shfl_xor(larger, 32));
            // (nothing but -Inf so far: 0 in the place of the maximum, so that the powers are 0.  The powers are of differences: a
            // product with the maximum taken off by a fused multiply-add keeps the product's rounding, which is no small
            // number for large scores)
            const float base = larger == -__builtin_inff() ? 0.0f : larger;
            const float shrink = most == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((most - larger) * factor);
            most = larger;
            float tile_sum = 0.0f;   // (added to the row's at the end: one rounding per tile and not per key)
#pragma unroll
            for (int d = 0; d < D32; ++d) {
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= shrink;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[j][i] = __builtin_amdgcn_exp2f((sc[j][i] - base) * factor);
                    tile_sum += sc[j][i];
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    // P in bf16 for the matrix cores, the sum from the unrounded values: a rounding is half a bf16 step of a
                    // weight, as the output's own is of the result
                    uint32_t w[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        w[c] = __builtin_bit_cast(uint32_t, __builtin_convertvector((attn_f32x2{sc[j][8 * i + 2 * c], sc[j][8 * i + 2 * c + 1]}), attn_bf16x2));
                    const mfma_bf16x8 p = __builtin_bit_cast(mfma_bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
                    for (int d = 0; d < D32; ++d) {
                        // lane t of 16 reads 8 bytes of row t / 4 and gets column t of the four rows
                        const uint32_t r = 32u * j + 16u * i + 4u * half + (lane & 15u) / 4u, c = 32u * d + 16u * ((lane >> 4) & 1u) + 4u * (lane & 3u);
                        typedef __attribute__((address_space(3))) attn_s16x4* lds_s16x4;
                        const attn_s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(lds_v + r * kPitch + 2u * c));
                        const attn_s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(lds_v + (r + 8u) * kPitch + 2u * c));
                        const uint4 a = make_uint4(__builtin_bit_cast(uint2, v0).x, __builtin_bit_cast(uint2, v0).y, __builtin_bit_cast(uint2, v1).x,
                                                   __builtin_bit_cast(uint2, v1).y);
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(mfma_bf16x8, a), p, o[d], 0, 0, 0);
                    }
                }
            }
            sum = fmaf(sum, shrink, tile_sum);
        }
    }
    sum += __shfl_xor(sum, 32);
    if (row >= min(len_q, first_q + s.block_q * 64u)) return;
    const float inverse = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;   // (a NaN stays; no key: zeros)
    uint16_t* to = out + ((size_t)b * so.batch + (size_t)h * so.head + (size_t)row * so.token) * 8u;
#pragma unroll
    for (int d = 0; d < D32; ++d) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t c = 32u * d + 8u * i + 4u * half;
            uint32_t w[2];
#pragma unroll
            for (int x = 0; x < 2; ++x)
                w[x] = __builtin_bit_cast(uint32_t, __builtin_convertvector((attn_f32x2{o[d][4 * i + 2 * x] * inverse, o[d][4 * i + 2 * x + 1] * inverse}), attn_bf16x2));
            if (c < dim) *reinterpret_cast<uint2*>(to + c) = make_uint2(w[0], w[1]);
        }
    }
    if (lse && half == 0)
        lse[(size_t)g * s.tokens_q + row] = sum == 0.0f ? -__builtin_inff() : most * s.scale + 0.69314718055994530942f * __builtin_amdgcn_logf(sum);
}

}  // namespace fb4
