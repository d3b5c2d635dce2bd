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
// Blocks of queries to a workgroup, in sixteens (the rows of an MFMA): two where their scores fill LDS, which halves what is read of
// the keys' means -- from L2, at 9 TB/s, which one each was bound by.
constexpr int select_sets(int values) { return values == 16 ? 2 : 1; }
constexpr int select_threads(int values) { return 512 * select_sets(values); }

// A workgroup takes 16 blocks of queries of one head (32 with 513 to 1024 blocks of keys): their scores with all the head's blocks of
// keys by 16x16x4 MFMAs in double, then the largest `top` of every row.  The channels of a product may come in any order as long as both
// operands have the same: lane group k of 16 holds channels 16 c + 4 k .. + 3 for the four steps of chunk c, which are 32 bytes of its row.
// LDS keeps the scores rounded to fp32, half of what the doubles would take: up to 512 blocks of keys three workgroups and more share a
// compute unit and one's search runs beside another's products; beyond, one fills it (144 to 160 KiB) and products and search take turns.
// Rounding keeps the order but for what becomes equal, so the fp32 values decide unless the border falls between
// equal ones; those blocks' scores are then formed again in double.
// D16: channels / 16, rounded up; kValues: scores of a row per lane.
// Measured, means included (24 heads x 1024 x 1024 blocks x 128 channels): 346-356 us, of which the means' kernel 148 at 5.5 TB/s; 424
// with doubles in LDS and a search bit by bit on four wavefronts.  The MFMAs alone are 82 us; the rest is reads of the keys' means from
// L2 and the search.
template <int D16, int kValues>
__global__ __launch_bounds__(select_threads(kValues)) __attribute__((amdgpu_waves_per_eu(kValues > 16 ? 2 : 4)))
void select_blocks_kernel(const double* means, const int32_t* lens, int32_t* chosen, float* scores, uint32_t top, uint32_t n_q, uint32_t dim,
                          uint32_t row_tiles, uint32_t n_workgroups, BlockShape s)
{
    constexpr int kSets = select_sets(kValues);
    constexpr uint32_t kThreads = select_threads(kValues), kWaves = kThreads / 64, kSelectRows = 16 * kSets, kRowDoubles = 16 * D16, kPieces = kRowDoubles / 2;
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
    for (uint32_t i = threadIdx.x; i < kSelectRows * kPieces; i += kThreads) {
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
        select_f64x4 acc[kSets] = {};
        constexpr int kChunks = D16 > 4 ? (D16 + 1) / 2 : D16;   // read at a time (128 registers hold no 8)
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
#pragma unroll
                for (int u = 0; u < kSets; ++u) {
                    const select_f64x2 a = *reinterpret_cast<const select_f64x2*>(queries + (16u * u + r) * kRowDoubles + 2u * (p ^ (r & 7u)));
                    acc[u] = __builtin_amdgcn_mfma_f64_16x16x4f64(a[0], keys[i][0], acc[u], 0, 0, 0);
                    acc[u] = __builtin_amdgcn_mfma_f64_16x16x4f64(a[1], keys[i][1], acc[u], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // accumulator i: row lane / 16 + 4 i, column lane % 16
#pragma unroll
            for (int u = 0; u < kSets; ++u) order[16u * u + (lane >> 4) + 4u * i][16u * t + r] = there ? order_of((float)acc[u][i]) : 0;
        }
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
constexpr uint32_t kAllBlocks = 0xFFFFFFFFu;   // no list (FB4_ALL_BLOCKS in 32 bits)
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

typedef float attn_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 attn_bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t attn_u32x4 __attribute__((ext_vector_type(4)));
typedef short attn_s16x4 __attribute__((ext_vector_type(4)));

struct AttentionShape {
    uint32_t tokens_q, tokens_k, top;
    uint16_t heads, heads_k;
    uint8_t block_q, block_k;     // in units of 64 tokens
    uint16_t parts;               // workgroups that share a block of queries, each with a run of its list
    uint32_t blocks_q, n_workgroups;
    float scale;
};
// Strides in units of 8 elements.
struct TensorStrides {
    uint32_t batch, head, token;
};

#define FB4_INLINE __attribute__((always_inline))   // (a lambda that is not inlined keeps what it captures in memory)

// Keys between two barriers.  Two buffers of keys and of values: a workgroup of two wavefronts with long rows would keep others off
// its compute unit with 64.
constexpr int attention_keys(int pieces, int waves) { return waves == 2 && pieces > 9 ? 32 : 64; }

// A workgroup of kWaves wavefronts takes one block of 32 * kWaves queries of one head; every wavefront holds 32 of them as B
// operands and walks the listed blocks' keys in groups of 32.
//
// The walk overlaps: while the vector ALU turns group i's products into weights, the matrix cores form P V of group i - 1 and then
// Q K of group i + 1, so that a wavefront alone keeps both busy (16 MFMAs of 32 cycles per group with 128 channels, about 70
// instructions of 4).  Keys are therefore wanted a group early and values a group late, and their buffers change over at
// different times: between the barriers before the last groups of tile t and of t + 1, the keys of t + 2 and the values of t + 1
// (tiles of one group: of t) come in.
//
// kP: 16-byte pieces per row (dim / 8).  Keys and values go from memory straight into LDS (1 KiB per wavefront and load, lane i's 16
// bytes at place i).  Those places are contiguous, so rows cannot be padded; instead piece p of a row lies at p ^ f(row): for the
// keys f as in attention_scores_dma_kernel, which spreads the 16 rows that one pass of an operand read takes over all 64 banks; for
// the values, of whose rows a pass takes four pieces of four successive ones, so that these fall into different banks (16 pieces:
// 4 (r % 4), 8: 4 (r / 2 % 2); other lengths spread by themselves, or nearly).  With an odd kP the upper half of the last step of 16
// channels lies past the row: its lanes read a zeroed piece.
//
// Weights are exp2(S c - m), c = scale log2 e, m a reference that moves only when a power would pass 2^8: until then the accumulators need
// not be scaled, and the two half-wavefronts, which hold different keys of the same query, need not meet.  A fused multiply-add
// takes m off the exact product, so m's own rounding is one factor in all weights and in their sum, and when m moves they are scaled by the
// power of the rounded values' difference; beyond |m| = 2^20 that factor could itself be no small number, and the wavefront goes on with
// exp2((S - max) c).
// kSplit: a part of the list; the accumulators, maximum and sum go to `out` as floats (see join_parts_kernel).
// Measured (channels; listed keys): 24 heads x 16384 queries x 2048 of 128: 434-463 us by card, 0.89-0.95 PFLOP/s, held by the power limit (on zeros
// 340) and the loads into LDS (a fifth); 65536 queries, random lists: 1870 us, 11 GB from beyond the L2s; 272 x 1350 queries x 448 of 72:
// 97 us, a third of it first reads and output; 48 single queries x 8192 of 128: 42 us, 4.7 TB/s.
template <int kP, int kWaves, bool kSplit>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2)))
void block_attention_kernel(const uint16_t* q, const uint16_t* k, const uint16_t* v, uint16_t* out, float* lse, const int32_t* blocks,
                            const int32_t* lens, TensorStrides sv, TensorStrides so, AttentionShape s)
{
    constexpr int kSteps = (kP + 1) / 2, kTiles = (kP + 3) / 4;   // of 16 channels; of 32
    constexpr int kKeys = attention_keys(kP, kWaves), kGroups = kKeys / 32;
    constexpr uint32_t kRowBytes = kP * 16, kBytes = kKeys * kRowBytes, kPositions = kKeys * kP, kLoads = (kPositions + 63) / 64;
    constexpr int kMine = (kLoads + kWaves - 1) / kWaves;         // of a wavefront, at most
    constexpr uint32_t kG = kP % 16 == 0 ? 16 : kP % 8 == 0 ? 8 : kP % 4 == 0 ? 4 : kP % 2 == 0 ? 2 : 1;
    // Each buffer an array of its own: the compiler then sees that the loads into one do not touch the reads from another.  (64 bytes
    // more: zeros for the keys, what reads of unused channels may touch for the values)
    constexpr uint32_t kPadK = kP % 2 ? 64 : 0, kPadV = kP % 4 ? 64 : 0;
    __shared__ __align__(1024) uint8_t lds_k0[kBytes + kPadK], lds_k1[kBytes + kPadK], lds_v0[kBytes + kPadV], lds_v1[kBytes + kPadV];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t half = lane >> 5, col = lane & 31u;
    const uint32_t pos = xcd_local_position(blockIdx.x, s.n_workgroups);
    // (divisions run in the vector ALU: the addresses made of their results stay in scalar registers so)
    auto scalar = [](uint32_t x) FB4_INLINE { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
    const uint32_t item = kSplit ? scalar(pos / s.parts) : pos, part = kSplit ? pos - item * s.parts : 0u;
    const uint32_t g = scalar(item / s.blocks_q), block = item - g * s.blocks_q;   // g = batch * heads + head
    const uint32_t b = scalar(g / s.heads), h = g - b * s.heads, hk = scalar(h / (s.heads / s.heads_k));
    const uint32_t len_q = scalar(length_of(lens, b, 0, s.tokens_q)), len_k = scalar(length_of(lens, b, 1, s.tokens_k));
    const uint32_t first_q = block * s.block_q * 64u;
    if (first_q >= len_q) return;
    const uint32_t block_keys = s.block_k * 64u, blocks_k = (len_k + block_keys - 1) / block_keys;   // blocks with a key
    const uint8_t* kg = reinterpret_cast<const uint8_t*>(k) + (size_t)(b * s.heads_k + hk) * s.tokens_k * kRowBytes;
    const uint8_t* vg = reinterpret_cast<const uint8_t*>(v) + ((size_t)b * sv.batch + (size_t)hk * sv.head) * 16u;
    const uint32_t end_q = min(len_q, first_q + s.block_q * 64u);
    const uint32_t row = first_q + wave * 32u + col;                 // this lane's query

    // ---- the tiles: entries of the list, and of each the tiles with a key
    const bool all = s.top == kAllBlocks;
    const int32_t* list = blocks + (size_t)item * s.top;
    const uint32_t n_entries = all ? blocks_k : s.top;
    uint32_t entry = kSplit ? (uint32_t)((uint64_t)n_entries * part / s.parts) : 0u;
    const uint32_t last_entry = kSplit ? (uint32_t)((uint64_t)n_entries * (part + 1) / s.parts) : n_entries;
    struct Tile { uint32_t key, n; };   // first key, keys (0: no tile)
    uint32_t cursor = 0, block_end = 0, held_from = entry;
    int32_t held = 0;                   // a lane's entry of 64 (a read per entry would wait for the tiles' reads before it)
    if (!all && entry < last_entry) held = list[min(entry + lane, last_entry - 1)];
    auto next_tile = [&]() FB4_INLINE {
        while (cursor >= block_end) {
            if (entry >= last_entry) return Tile{0, 0};
            if (!all && entry - held_from == 64) {
                held_from = entry;
                held = list[min(entry + lane, last_entry - 1)];
            }
            const uint32_t which = all ? entry : (uint32_t)__builtin_amdgcn_readlane(held, entry - held_from);
            ++entry;
            if (which < blocks_k) {     // (a negative one is not either)
                cursor = which * block_keys;
                block_end = min(cursor + block_keys, len_k);
            }
        }
        const Tile t = {cursor, (uint32_t)min(block_end - cursor, (uint32_t)kKeys)};
        cursor += kKeys;
        return t;
    };

    // ---- tiles from memory: this wavefront's loads wave, wave + kWaves, ..
    auto key_place = [](uint32_t r) FB4_INLINE { return (r / (16u / kG)) & (kG - 1u); };                                    // f(row)
    auto value_place = [](uint32_t r) FB4_INLINE { return kP == 16 ? 4u * (r & 3u) : kP == 8 ? 4u * ((r >> 1) & 1u) : 0u; };
    // a lane's place in a tile, in bytes, for every load; for one, where the next is whole runs of 16 rows further (f is the same there)
    constexpr bool kRegular = (64 * kWaves) % (16 * kP) == 0;
    constexpr int kPlaces = kRegular ? 1 : kMine;
    uint32_t from_k[kPlaces], from_v[kPlaces];
#pragma unroll
    for (int i = 0; i < kPlaces; ++i) {
        const uint32_t j = 64u * (i * kWaves + wave) + lane, r = j / kP, p = j - r * kP;
        from_k[i] = r * kRowBytes + ((p ^ key_place(r)) << 4);
        from_v[i] = r * sv.token * 16u + ((p ^ value_place(r)) << 4);
    }
    auto copy = [&](const uint8_t* from, uint8_t* to) FB4_INLINE {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
    };
    auto fetch = [&](const Tile& t, const uint8_t* base, const uint32_t* from, uint32_t row_bytes, uint8_t* buffer, bool values) FB4_INLINE {
        if (t.n == (uint32_t)kKeys) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const uint32_t load = i * kWaves + wave;
                const uint8_t* at = kRegular ? base + (size_t)(i * (64 * kWaves / kP)) * row_bytes + from[0] : base + from[i % kPlaces];
                if ((i + 1) * kWaves * 64 <= (int)kPositions || 64u * load + lane < kPositions) copy(at, buffer + __builtin_amdgcn_readfirstlane(load * 1024u));
            }
        } else if (t.n) {
#pragma unroll 1
            for (uint32_t load = wave; load < kLoads; load += kWaves) {
                const uint32_t j = 64u * load + lane, r = j / kP, p = j - r * kP;
                if (r < t.n) {   // (a lane that takes no part leaves its 16 bytes alone)
                    copy(base + r * row_bytes + ((p ^ (values ? value_place(r) : key_place(r))) << 4), buffer + __builtin_amdgcn_readfirstlane(load * 1024u));
                } else if (values && j < kPositions) {
                    // values behind the last key: zeros, which their weights of 0 leave zeros (the keys' products are replaced)
                    *reinterpret_cast<uint4*>(buffer + j * 16u) = make_uint4(0, 0, 0, 0);
                }
            }
        }
    };
    auto fetch_k = [&](const Tile& t, uint8_t* buffer) FB4_INLINE { fetch(t, kg + (size_t)t.key * kRowBytes, from_k, kRowBytes, buffer, false); };
    auto fetch_v = [&](const Tile& t, uint8_t* buffer) FB4_INLINE { fetch(t, vg + (size_t)t.key * sv.token * 16u, from_v, sv.token * 16u, buffer, true); };

    // (what the buffers hold is asked for at once: a short list's walk is little more than its first reads' wait)
    Tile now = next_tile();
    fetch_k(now, lds_k0);
    Tile then = now.n ? next_tile() : Tile{0, 0};
    fetch_k(then, lds_k1);
    if (kGroups == 2) fetch_v(now, lds_v0);
    // ---- this wavefront's queries as B operands (past the last one that one: a padded row's values touch no other's rounding)
    mfma_bf16x8 qf[kSteps];
    {
        const uint16_t* from = q + ((size_t)g * s.tokens_q + min(row, end_q - 1u)) * (kP * 8);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if (!(kP % 2 && i == kSteps - 1) || half == 0) w = *reinterpret_cast<const uint4*>(from + 16 * i + 8 * half);
            qf[i] = __builtin_bit_cast(mfma_bf16x8, w);
        }
    }
    const float factor = s.scale * kLog2E;   // c
    mfma_f32x16 o[kTiles], sc = {}, sd = {};   // accumulators; products of the groups at hand, in turn
    mfma_bf16x8 p[2] = {};               // weights of the group before it, as operands
#pragma unroll
    for (int d = 0; d < kTiles; ++d) o[d] = mfma_f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    // of this lane's query: the largest product that the reference is made of, the reference (-Inf: no product yet), what is taken off
    // (the rounded product; 0 where there is none), the sum over this lane's keys
    float most = -__builtin_inff(), reference = -__builtin_inff(), off = 0.0f, sum = 0.0f;
    bool large = false;                                  // (of the wavefront)

    // LDS offsets: the keys' operand, row lane % 32 of 32, piece 2 step + lane / 32; the values', 8 bytes of row (lane % 16) / 4
    const uint32_t k_row = col * kRowBytes, k_swz = key_place(col);
    const uint32_t v_r = 4u * half + (lane & 15u) / 4u;
    const uint32_t v_swz = value_place(v_r);   // (8 and 16 rows further the same)
    const uint32_t v_piece = 2u * ((lane >> 4) & 1u) + ((lane & 3u) >> 1), v_at = v_r * kRowBytes + 8u * (lane & 1u);
    uint32_t k_at[kSteps], v_place[kTiles];   // (whole, so that a buffer and a group are constants in the reads)
#pragma unroll
    for (int i = 0; i < kSteps; ++i) k_at[i] = k_row + (((2u * i + half) ^ k_swz) << 4);
#pragma unroll
    for (int d = 0; d < kTiles; ++d) v_place[d] = v_at + (((4u * d + v_piece) ^ v_swz) << 4);
    auto key_operand = [&](const uint8_t* keys, int group, int i) FB4_INLINE {
        const uint32_t at = k_at[i] + 32u * group * kRowBytes;
        return __builtin_bit_cast(mfma_bf16x8, *reinterpret_cast<const uint4*>(keys + ((kP % 2 && i == kSteps - 1 && half) ? kBytes : at)));
    };
    auto value_operand = [&](const uint8_t* values, int group, int i, int d) FB4_INLINE {
        // lane t of 16 reads 8 bytes of row t / 4 and gets column t of the four rows.  (Channels past the row: what lies behind, in
        // accumulators that nobody reads)
        typedef __attribute__((address_space(3))) attn_s16x4* lds_s16x4;
        const uint8_t* from = values + v_place[d] + (32u * group + 16u * i) * kRowBytes;
        const uint2 v0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(from)));
        const uint2 v1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(from + 8u * kRowBytes)));
        return __builtin_bit_cast(mfma_bf16x8, make_uint4(v0.x, v0.y, v1.x, v1.y));
    };
    // The instructions' order is the source's: a scheduling barrier behind every MFMA's slot, which holds what runs beside it.
    constexpr int kProducts = 2 * kTiles;          // of P V per group
    constexpr int kAhead = 4;                      // operands read ahead of their MFMA
    constexpr int kReady = kProducts < kAhead ? kProducts : kAhead;
    mfma_bf16x8 ready[kReady];                     // the first operands of the next P V, read before its step
    auto get_ready = [&](const uint8_t* values, int group, int x) FB4_INLINE { ready[x] = value_operand(values, group, x / kTiles, x % kTiles); };
    // P V of the group whose weights are in p; `beside(x)`: what goes with product x
    auto add_values = [&](const uint8_t* values, int group, auto beside) FB4_INLINE {
        mfma_bf16x8 a[kProducts];
#pragma unroll
        for (int x = 0; x < kReady; ++x) a[x] = ready[x];
#pragma unroll
        for (int x = 0; x < kProducts; ++x) {
            o[x % kTiles] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[x], p[x / kTiles], o[x % kTiles], 0, 0, 0);
            if (x + kAhead < kProducts) a[x + kAhead] = value_operand(values, group, (x + kAhead) / kTiles, (x + kAhead) % kTiles);
            beside(x);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // One step: weights of the group in `sc`, which are keys `first` .. of a tile of n; P V of the group before it, Q K of the one
    // behind into `next`.
    auto step = [&](mfma_f32x16& sc, mfma_f32x16& next, uint32_t first, uint32_t n, const uint8_t* values, int v_group, const uint8_t* keys,
                    int k_group, auto later) FB4_INLINE {
        if (first + 32u > n) {   // (a sequence's last tile)
            uint32_t key = first + 4u * half;
            asm volatile("" : "+v"(key));   // (opaque: else sixteen sums are kept for it all the time)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = key + 8u * (i / 4) + i % 4 >= n ? -__builtin_inff() : sc[i];
        }
        mfma_bf16x8 a[kSteps];
        float larger = -__builtin_inff();
        add_values(values, v_group, [&](int x) FB4_INLINE {
            // the first operands of Q K; the maximum, not before the products it is of are done
            constexpr int kFirst = kProducts > 4 ? 2 : 0, kShare = 16 / (kProducts - kFirst), kEarly = kSteps < kAhead ? kSteps : kAhead;
#pragma unroll
            for (int i = 0; i < kEarly; ++i) {
                if (x == (kProducts > kEarly + 1 - i ? kProducts - kEarly - 1 + i : 0)) a[i] = key_operand(keys, k_group, i);
            }
            if (x >= kFirst) {
#pragma unroll
                for (int i = (x - kFirst) * kShare; i < (x == kProducts - 1 ? 16 : (x - kFirst + 1) * kShare); ++i) larger = fmaxf(larger, sc[i]);
            }
        });
        if (__any(fmaf(larger, factor, -reference) > 8.0f)) {
#pragma clang fp contract(off)   // (a rounded product is meant)
            larger = fmaxf(larger, most);
            // (finite, so that a score of +Inf has an infinite weight and sum: no number in the output, +Inf in lse)
            larger = fminf(fmaxf(larger, __shfl_xor(larger, 32)), 0x1.fffffep127f);
            const float product = larger * factor, fresh = larger == -__builtin_inff() ? 0.0f : product;
            const bool was_large = large;
            large = large || __any(fabsf(fresh) > 0x1p20f);
            // from what the weights so far are relative to: the rounded product, or (large) the exact one
            const float moved = was_large ? (most - larger) * factor : large ? fmaf(-larger, factor, off) : off - fresh;
            const float shrink = most == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(moved);
            most = larger;
            // (large: the rounding is no small part of 8, so the next move comes that much sooner, or, past fp32, with every group)
            reference = !large ? product : fabsf(product) < __builtin_inff() ? fmaf(-fabsf(product), 0x1p-22f, product) : -__builtin_inff();
            off = fresh;
            sum *= shrink;
#pragma unroll
            for (int d = 0; d < kTiles; ++d) {
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= shrink;
            }
        }
        // In bf16 for the matrix cores, the sum from the unrounded weights: a rounding is half a bf16 step of a weight, as the output's
        // own is of the result.  (The sum: one rounding of the row's per group and not per key)
        float x = 0.0f, y = 0.0f;
        uint32_t w[8];
        auto products = [&](auto power) FB4_INLINE {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if (i == 0) next = mfma_f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
                next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], qf[i], next, 0, 0, 0);
                if (i + kAhead < kSteps) a[i + kAhead] = key_operand(keys, k_group, i + kAhead);
#pragma unroll
                for (int c = 8 * i / kSteps; c < 8 * (i + 1) / kSteps; ++c) {
                    const float w0 = power(sc[2 * c]), w1 = power(sc[2 * c + 1]);
                    x += w0;
                    y += w1;
                    w[c] = __builtin_bit_cast(uint32_t, __builtin_convertvector((attn_f32x2{w0, w1}), attn_bf16x2));
                }
#pragma unroll
                for (int r = 0; r < kReady; ++r) {   // in the last slots, whose operands are read
                    if (i == (kSteps > kReady ? kSteps - kReady + r : kSteps - 1)) later(r);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        if (large) {
            const float base = most == -__builtin_inff() ? 0.0f : most;
            products([&](float z) FB4_INLINE { return __builtin_amdgcn_exp2f((z - base) * factor); });
        } else {
            products([&](float z) FB4_INLINE { return __builtin_amdgcn_exp2f(fmaf(z, factor, -off)); });
        }
        sum += x + y;
#pragma unroll
        for (int i = 0; i < 2; ++i) p[i] = __builtin_bit_cast(mfma_bf16x8, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
    };
    auto landed = [&]() FB4_INLINE {
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wavefront's loads are in LDS
        __syncthreads();                      // ... and everyone's; everyone is done with the buffers that come next
    };
    if (now.n) {
        // the zeroed pieces; values for the step before the first group, whose weights are 0
        if (kP % 2 && threadIdx.x < 8) reinterpret_cast<uint32_t*>((threadIdx.x & 4u ? lds_k1 : lds_k0) + kBytes)[threadIdx.x & 3u] = 0;
        for (uint32_t i = threadIdx.x; i < (kBytes + kPadV) / 16; i += 64 * kWaves) *reinterpret_cast<uint4*>(lds_v1 + 16u * i) = make_uint4(0, 0, 0, 0);
        landed();
#pragma unroll
        for (int i = 0; i < kSteps; ++i) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_operand(lds_k0, 0, i), qf[i], sc, 0, 0, 0);
        // A tile from its last group on, and the next one's first; its keys and values in k_now and v_now, the next one's keys in k_then,
        // the previous one's values in v_then, whose place the next one's take.  False: it was the last.  (From a wait on, so that
        // nothing is in flight where the loop comes round: the compiler knows less there and would wait at the first read)
        auto tile = [&](mfma_f32x16& s_now, mfma_f32x16& s_then, uint8_t* k_now, uint8_t* k_then, uint8_t* v_now, uint8_t* v_then) FB4_INLINE {
            landed();
#pragma unroll
            for (int r = 0; r < kReady; ++r) get_ready(kGroups == 2 ? v_now : v_then, 0, r);
            const Tile after = then.n ? next_tile() : Tile{0, 0};
            fetch_k(after, k_now);
            if (kGroups == 2) {
                fetch_v(then, v_then);
                step(s_then, s_now, 32, now.n, v_now, 0, k_then, 0, [&](int r) FB4_INLINE { get_ready(v_now, 1, r); });
            } else {
                fetch_v(now, v_now);
                step(s_now, s_then, 0, now.n, v_then, 0, k_then, 0, [](int) {});
            }
            now = then;
            then = after;
            if (now.n == 0) return false;
            if (kGroups == 2) step(s_now, s_then, 0, now.n, v_now, 1, k_then, 1, [](int) {});
            return true;
        };
        const uint8_t* last_values;
#pragma unroll
        for (int r = 0; r < kReady; ++r) get_ready(lds_v1, kGroups - 1, r);
        if (kGroups == 2) step(sc, sd, 0, now.n, lds_v1, 1, lds_k0, 1, [](int) {});
        for (;;) {
            last_values = lds_v0;
            if (!tile(sc, sd, lds_k0, lds_k1, lds_v0, lds_v1)) break;
            last_values = lds_v1;
            if (!tile(kGroups == 2 ? sc : sd, kGroups == 2 ? sd : sc, lds_k1, lds_k0, lds_v1, lds_v0)) break;
        }
        if (kGroups == 1) {
            landed();
#pragma unroll
            for (int r = 0; r < kReady; ++r) get_ready(last_values, 0, r);
        }
        add_values(last_values, kGroups - 1, [](int) {});   // of the last group
    }
    sum += __shfl_xor(sum, 32);
    const size_t at_row = (size_t)g * s.tokens_q + row;
    if (kSplit) {
        // relative to the exact product of maximum and factor, whose difference from another part's is then one of maxima
        const float exact = large || most == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(fmaf(-most, factor, off));
        sum *= exact;
#pragma unroll
        for (int d = 0; d < kTiles; ++d) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= exact;
        }
        if (row >= end_q) return;
        const size_t n_rows = (size_t)(s.n_workgroups / s.parts / s.blocks_q) * s.tokens_q;
        float* to = reinterpret_cast<float*>(out) + (part * n_rows + at_row) * (kP * 8);
#pragma unroll
        for (int d = 0; d < kTiles; ++d) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c = 32u * d + 8u * i + 4u * half;
                if (c < kP * 8u) *reinterpret_cast<float4*>(to + c) = make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
            }
        }
        if (half == 0) *reinterpret_cast<float2*>(reinterpret_cast<float*>(out) + s.parts * n_rows * (kP * 8) + 2 * (part * n_rows + at_row)) = make_float2(most, sum);
        return;
    }
    const float inverse = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;   // (a NaN stays; no key: zeros)
    if (lse && half == 0 && row < end_q) {
        const float log_sum = __builtin_amdgcn_logf(sum);
        lse[at_row] = sum == 0.0f ? -__builtin_inff() : large ? fmaf(most, s.scale, kLn2 * log_sum) : kLn2 * (off + log_sum);
    }
    // Rows through LDS, 16 bytes to a lane: from the accumulators a store is 32 rows' 16 bytes each (17 x 16 x 1350 x 72: 11 of 100 us).
    // Every wavefront has a buffer of its own, once all are done with the tiles.
    __syncthreads();
    uint8_t* mine = wave == 0 ? lds_k0 : wave == 1 ? lds_k1 : wave == 2 ? lds_v0 : lds_v1;
#pragma unroll
    for (int d = 0; d < kTiles; ++d) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w[2];
#pragma unroll
            for (int x = 0; x < 2; ++x)
                w[x] = __builtin_bit_cast(uint32_t, __builtin_convertvector((attn_f32x2{o[d][4 * i + 2 * x] * inverse, o[d][4 * i + 2 * x + 1] * inverse}), attn_bf16x2));
            // channels 32 d + 8 i + 4 half ..: half of piece 4 d + i
            if (4 * d + i < kP) *reinterpret_cast<uint2*>(mine + col * kRowBytes + (((4u * d + i) ^ k_swz) << 4) + 8u * half) = make_uint2(w[0], w[1]);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");   // (other lanes read them)
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    uint16_t* to = out + ((size_t)b * so.batch + (size_t)h * so.head) * 8u;
#pragma unroll
    for (int i = 0; i < (kP + 1) / 2; ++i) {
        const uint32_t j = 64u * i + lane, r = j / kP, p16 = j - r * kP, at = first_q + wave * 32u + r;
        if (r >= 32u || at >= end_q) break;
        const attn_u32x4 w = *reinterpret_cast<const attn_u32x4*>(mine + r * kRowBytes + ((p16 ^ key_place(r)) << 4));
        attn_u32x4* place = reinterpret_cast<attn_u32x4*>(to + ((size_t)at * so.token + p16) * 8u);
        if (kP % 8 == 0) __builtin_nontemporal_store(w, place);   // (whole lines; 72 channels' parts of lines are better kept: 99.6 / 102.8 us)
        else *place = w;
    }
}

#undef FB4_INLINE

// The parts of a row's list meet: accumulators and sums relative to the parts' own maxima (-Inf: no key), a part's weight
// exp2((its maximum - the largest) c): of a difference, which is small where the weight is not, however large both are.
// Workspace: float [parts][rows][dim], then {maximum, sum} [parts][rows].  32 lanes, four channels each, take a row's parts one after
// the other, four reads ahead, eight rows to a workgroup; of many parts (kMany) a workgroup's eight sets of lanes take every eighth
// and meet in LDS, so that a row waits for few reads one behind the other (48 rows x 21 parts x 128 channels 20.8 us with one walk
// over the parts, 4.1 so; 25600 rows x 2 parts x 72 channels 27 us so).
template <bool kMany>
__global__ __launch_bounds__(256) void join_parts_kernel(const float* workspace, const int32_t* lens, uint16_t* out, float* lse, TensorStrides so,
                                                         uint32_t parts, uint32_t n_rows, uint32_t tokens_q, uint32_t heads, uint32_t dim, float scale)
{
    __shared__ float4 meet[kMany ? 8 : 1][32];
    const uint32_t l = threadIdx.x & 31u, set = threadIdx.x >> 5, c = 4u * l;
    const uint32_t at = kMany ? blockIdx.x : min(blockIdx.x * 8u + set, n_rows - 1u);   // (a set past the last row does its work again)
    const uint32_t first = kMany ? set : 0u, step = kMany ? 8u : 1u;
    const uint32_t g = at / tokens_q, row = at - g * tokens_q, b = g / heads, h = g - b * heads;
    const bool live = row < length_of(lens, b, 0, tokens_q);
    const float2* state = reinterpret_cast<const float2*>(workspace + (size_t)parts * n_rows * dim) + at;
    float most = -__builtin_inff(), sum = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (live) {   // (a row that no part wrote is not read)
        for (uint32_t p = l; p < parts; p += 32) most = fmaxf(most, state[(size_t)p * n_rows].x);
    }
#pragma unroll
    for (int d = 1; d < 32; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    const float base = most == -__builtin_inff() ? 0.0f : most, factor = scale * kLog2E;
    if (live) {
        for (uint32_t p = l; p < parts; p += 32) {
            const float2 st = state[(size_t)p * n_rows];
            sum = fmaf(st.y, __builtin_amdgcn_exp2f((st.x - base) * factor), sum);
        }
    }
#pragma unroll
    for (int d = 1; d < 32; d *= 2) sum += __shfl_xor(sum, d);
    if (live && c < dim) {
#pragma unroll 4
        for (uint32_t p = first; p < parts; p += step) {
            const float w = __builtin_amdgcn_exp2f((state[(size_t)p * n_rows].x - base) * factor);
            const float4 x = *reinterpret_cast<const float4*>(workspace + ((size_t)p * n_rows + at) * dim + c);
            o = make_float4(fmaf(x.x, w, o.x), fmaf(x.y, w, o.y), fmaf(x.z, w, o.z), fmaf(x.w, w, o.w));
        }
    }
    if (kMany) {
        meet[set][l] = o;
        __syncthreads();
        if (set > 0) return;
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            const float4 x = meet[i][l];
            o = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
        }
    }
    if (!live) return;
    const float inverse = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
    uint16_t* to = out + ((size_t)b * so.batch + (size_t)h * so.head + (size_t)row * so.token) * 8u;
    const attn_bf16x2 lo = __builtin_convertvector((attn_f32x2{o.x * inverse, o.y * inverse}), attn_bf16x2);
    const attn_bf16x2 hi = __builtin_convertvector((attn_f32x2{o.z * inverse, o.w * inverse}), attn_bf16x2);
    if (c < dim) *reinterpret_cast<uint2*>(to + c) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
    if (lse && l == 0) lse[at] = sum == 0.0f ? -__builtin_inff() : fmaf(base, scale, kLn2 * __builtin_amdgcn_logf(sum));
}

}  // namespace fb4
