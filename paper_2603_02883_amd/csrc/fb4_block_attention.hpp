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
constexpr uint32_t kAllBlocks = 0xFFFFFFFFu;   // no list (FB4_ALL_BLOCKS in 32 bits)

typedef float attn_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 attn_bf16x2 __attribute__((ext_vector_type(2)));
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

// Keys between two barriers.  Two buffers of keys and values: with 128 channels a workgroup of two wavefronts would keep others off
// its compute unit with 64.
constexpr int attention_keys(int pieces, int waves) { return waves == 2 && pieces > 8 ? 32 : 64; }

// A workgroup of kWaves wavefronts takes one block of 32 * kWaves queries of one head; every wavefront holds 32 of them as B
// operands and walks the listed blocks kKeys keys at a time.
// kP: 16-byte pieces per row (dim / 8).  Keys and values go from memory straight into LDS (1 KiB per wavefront and load, lane i's 16
// bytes at place i), the next tile's while this one's are used.  Those places are contiguous, so rows cannot be padded; instead
// piece p of a row lies at p ^ f(row): for the keys f as in attention_scores_dma_kernel, which spreads the 16 rows that one pass of
// an operand read takes over all 64 banks; for the values, of whose rows a pass takes four pieces of four successive ones, so
// that these fall into different banks (16 pieces: 4 (r % 4), 8: 4 (r / 2 % 2); other lengths spread by themselves, or nearly).
// With an odd kP the upper half of the last step of 16 channels lies past the row: its lanes read a zeroed piece.
// The running maximum moves only when a power would pass 2^8: until then the accumulators need not be scaled, and the two
// half-wavefronts, which hold different keys of the same query, need not meet.
// kSplit: a part of the list; the accumulators, maximum and sum go to `out` as floats (see join_parts_kernel).
template <int kP, int kWaves, bool kSplit>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2)))
void block_attention_kernel(const uint16_t* q, const uint16_t* k, const uint16_t* v, uint16_t* out, float* lse, const int32_t* blocks,
                            const int32_t* lens, TensorStrides sv, TensorStrides so, AttentionShape s)
{
    constexpr int kSteps = (kP + 1) / 2, kTiles = (kP + 3) / 4;   // of 16 channels; of 32
    constexpr int kKeys = attention_keys(kP, kWaves), kGroups = kKeys / 32;
    constexpr uint32_t kRowBytes = kP * 16, kBytes = kKeys * kRowBytes, kPositions = kKeys * kP, kLoads = (kPositions + 63) / 64;
    constexpr uint32_t kG = kP % 16 == 0 ? 16 : kP % 8 == 0 ? 8 : kP % 4 == 0 ? 4 : kP % 2 == 0 ? 2 : 1;
    // Two buffers, as two arrays: the compiler then sees that the loads into one do not touch the reads from the other.  Keys,
    // values, 64 bytes that reads of unused channels may touch (zeros at their start).
    __shared__ __align__(1024) uint8_t lds_a[2 * kBytes + 64];
    __shared__ __align__(1024) uint8_t lds_b[2 * kBytes + 64];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t half = lane >> 5, col = lane & 31u;
    const uint32_t pos = xcd_local_position(blockIdx.x, s.n_workgroups);
    const uint32_t item = kSplit ? pos / s.parts : pos, part = kSplit ? pos - item * s.parts : 0u;
    const uint32_t g = item / s.blocks_q, block = item - g * s.blocks_q;   // g = batch * heads + head
    const uint32_t b = g / s.heads, h = g - b * s.heads, hk = h / (s.heads / s.heads_k);
    const uint32_t len_q = length_of(lens, b, 0, s.tokens_q), len_k = length_of(lens, b, 1, s.tokens_k);
    const uint32_t first_q = block * s.block_q * 64u;
    if (first_q >= len_q) return;
    const uint32_t block_keys = s.block_k * 64u, blocks_k = (len_k + block_keys - 1) / block_keys;   // blocks with a key
    const uint8_t* kg = reinterpret_cast<const uint8_t*>(k) + (size_t)(b * s.heads_k + hk) * s.tokens_k * kRowBytes;
    const uint8_t* vg = reinterpret_cast<const uint8_t*>(v) + ((size_t)b * sv.batch + (size_t)hk * sv.head) * 16u;
    const uint32_t end_q = min(len_q, first_q + s.block_q * 64u);
    const uint32_t row = first_q + wave * 32u + col;                 // this lane's query
    const bool works = first_q + wave * 32u < end_q;                 // (a wavefront without a query helps to load)

    // ---- the tiles: entries of the list, and of each the tiles with a key
    const bool all = s.top == kAllBlocks;
    const int32_t* list = blocks + (size_t)item * s.top;
    const uint32_t n_entries = all ? blocks_k : s.top;
    uint32_t entry = kSplit ? (uint32_t)((uint64_t)n_entries * part / s.parts) : 0u;
    const uint32_t last_entry = kSplit ? (uint32_t)((uint64_t)n_entries * (part + 1) / s.parts) : n_entries;
    uint32_t key0 = 0, end = 0;   // the next tile's first key, the end of its block's keys
    auto seek = [&]() {           // to the next entry with a key; false: there is none
        for (; entry < last_entry; ++entry) {
            const uint32_t which = all ? entry : (uint32_t)list[entry];
            if (which < blocks_k) {   // (a negative one is not either)
                key0 = __builtin_amdgcn_readfirstlane(which * block_keys);
                end = min(key0 + block_keys, len_k);
                ++entry;
                return true;
            }
        }
        return false;
    };
    bool more = seek();

    auto fetch = [&](uint8_t* buffer) {   // the tile at key0, and on to the next
        const uint8_t* kt = kg + (size_t)key0 * kRowBytes;
        const uint8_t* vt = vg + (size_t)key0 * sv.token * 16u;
        const uint32_t valid = min(end - key0, (uint32_t)kKeys);
        uint32_t l = lane;
        asm volatile("" : "+v"(l));   // (opaque: else every load's offset is kept in a register of its own)
#pragma unroll
        for (uint32_t i0 = 0; i0 < kLoads; i0 += kWaves) {
            const uint32_t i = i0 + wave;
            if (i0 + kWaves > kLoads && i >= kLoads) break;
            const uint32_t j = 64u * i + l, r = j / kP, p = j - r * kP;
            const uint32_t pk = p ^ ((r / (16u / kG)) & (kG - 1u)), pv = p ^ (kP == 16 ? 4u * (r & 3u) : kP == 8 ? 4u * ((r >> 1) & 1u) : 0u);
            const uint32_t at = __builtin_amdgcn_readfirstlane(i * 1024u);
            if (r < valid) {   // (a lane that takes no part leaves its 16 bytes alone)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(kt + r * kRowBytes + pk * 16u),
                                                 (__attribute__((address_space(3))) void*)(buffer + at), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(vt + (size_t)r * sv.token * 16u + pv * 16u),
                                                 (__attribute__((address_space(3))) void*)(buffer + kBytes + at), 16, 0, 0);
            } else if (j < kPositions) {
                // values behind the last key: zeros, which their weights of 0 leave zeros (the keys' scores are replaced)
                *reinterpret_cast<uint4*>(buffer + kBytes + j * 16u) = make_uint4(0, 0, 0, 0);
            }
        }
        key0 += kKeys;
        if (key0 >= end) more = seek();
    };

    // ---- this wavefront's queries as B operands
    mfma_bf16x8 qf[kSteps];
    {
        const uint16_t* from = q + ((size_t)g * s.tokens_q + min(row, s.tokens_q - 1u)) * (kP * 8);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if (!(kP % 2 && i == kSteps - 1) || half == 0) w = *reinterpret_cast<const uint4*>(from + 16 * i + 8 * half);
            qf[i] = __builtin_bit_cast(mfma_bf16x8, w);
        }
    }
    const float factor = s.scale * 1.44269504088896340736f;   // to powers of two
    mfma_f32x16 o[kTiles];
#pragma unroll
    for (int d = 0; d < kTiles; ++d) o[d] = mfma_f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    float most = -__builtin_inff(), sum = 0.0f;   // of this lane's query: what is taken off its products; sum over this lane's keys

    // LDS offsets: the keys' operand, row lane % 32 of 32, piece 2 step + lane / 32; the values', 8 bytes of row (lane % 16) / 4
    const uint32_t k_row = col * kRowBytes, k_swz = (col / (16u / kG)) & (kG - 1u);
    const uint32_t v_r = 4u * half + (lane & 15u) / 4u;
    const uint32_t v_swz = kP == 16 ? 4u * (v_r & 3u) : kP == 8 ? 4u * ((v_r >> 1) & 1u) : 0u;   // (8 and 16 rows further the same)
    const uint32_t v_piece = 2u * ((lane >> 4) & 1u) + ((lane & 3u) >> 1), v_at = v_r * kRowBytes + 8u * (lane & 1u);

    auto compute = [&](const uint8_t* buffer, uint32_t n) {   // n: keys of the tile
        if (!works) return;
        mfma_f32x16 sc[kGroups];
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            sc[j] = mfma_f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const uint32_t at = 32u * j * kRowBytes + k_row + (((2u * i + half) ^ k_swz) << 4);
                const uint4 a = *reinterpret_cast<const uint4*>(buffer + ((kP % 2 && i == kSteps - 1 && half) ? 2u * kBytes : at));
                sc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(mfma_bf16x8, a), qf[i], sc[j], 0, 0, 0);
            }
        }
        if (n < (uint32_t)kKeys) {   // (a sequence's last tile)
#pragma unroll
            for (int j = 0; j < kGroups; ++j) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (32u * j + 8u * (i / 4) + 4u * half + i % 4 >= n) sc[j][i] = -__builtin_inff();
                }
            }
        }
        float larger = sc[0][0];
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
#pragma unroll
            for (int i = 0; i < 16; ++i) larger = fmaxf(larger, sc[j][i]);
        }
        if (__any((larger - most) * factor > 8.0f)) {
            larger = fmaxf(larger, most);
            larger = fmaxf(larger, __shfl_xor(larger, 32));
            // (of the difference: 1 where the maximum stays)
            const float shrink = most == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((most - larger) * factor);
            most = larger;
            sum *= shrink;
#pragma unroll
            for (int d = 0; d < kTiles; ++d) {
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= shrink;
            }
        }
        const float base = most == -__builtin_inff() ? 0.0f : most;   // (nothing but -Inf so far: the powers are to be 0)
        float tile_sum = 0.0f;   // (one rounding of the row's sum per tile and not per key)
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                // (of a difference: a fused product less the maximum's would keep that product's rounding, large for large scores)
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
                for (int d = 0; d < kTiles; ++d) {
                    // lane t of 16 reads 8 bytes of row t / 4 and gets column t of the four rows.  (Channels past the row: what lies
                    // behind, in accumulators that nobody reads)
                    typedef __attribute__((address_space(3))) attn_s16x4* lds_s16x4;
                    const uint8_t* from = buffer + kBytes + (32u * j + 16u * i) * kRowBytes + v_at + (((4u * d + v_piece) ^ v_swz) << 4);
                    const uint2 v0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(from)));
                    const uint2 v1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(from + 8u * kRowBytes)));
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(mfma_bf16x8, make_uint4(v0.x, v0.y, v1.x, v1.y)), p, o[d], 0, 0, 0);
                }
            }
        }
        sum += tile_sum;
    };

    if (kP % 2 && threadIdx.x < 8) reinterpret_cast<uint32_t*>((threadIdx.x & 4u ? lds_b : lds_a) + 2 * kBytes)[threadIdx.x & 3u] = 0;   // the zeroed pieces
    uint32_t n_a = 0, n_b = 0;   // keys of the tiles in the buffers, 0: none
    if (more) {
        n_a = min(end - key0, (uint32_t)kKeys);
        fetch(lds_a);
    }
    while (n_a) {
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wavefront's part of the tile is in LDS
        __syncthreads();                      // ... and everyone's; the other buffer is free
        n_b = more ? min(end - key0, (uint32_t)kKeys) : 0u;
        if (more) fetch(lds_b);
        compute(lds_a, n_a);
        if (!n_b) break;
        __builtin_amdgcn_s_waitcnt(0x0F70);
        __syncthreads();
        n_a = more ? min(end - key0, (uint32_t)kKeys) : 0u;
        if (more) fetch(lds_a);
        compute(lds_b, n_b);
    }
    sum += __shfl_xor(sum, 32);
    if (row >= end_q) return;
    const size_t at_row = (size_t)g * s.tokens_q + row;
    if (kSplit) {
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
    uint16_t* to = out + ((size_t)b * so.batch + (size_t)h * so.head + (size_t)row * so.token) * 8u;
#pragma unroll
    for (int d = 0; d < kTiles; ++d) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t c = 32u * d + 8u * i + 4u * half;
            uint32_t w[2];
#pragma unroll
            for (int x = 0; x < 2; ++x)
                w[x] = __builtin_bit_cast(uint32_t, __builtin_convertvector((attn_f32x2{o[d][4 * i + 2 * x] * inverse, o[d][4 * i + 2 * x + 1] * inverse}), attn_bf16x2));
            if (c < kP * 8u) *reinterpret_cast<uint2*>(to + c) = make_uint2(w[0], w[1]);
        }
    }
    if (lse && half == 0) lse[at_row] = sum == 0.0f ? -__builtin_inff() : most * s.scale + 0.69314718055994530942f * __builtin_amdgcn_logf(sum);
}

// The parts of a row's list meet: accumulators and sums relative to the parts' own maxima.  Workspace: float [parts][rows][dim], then
// {maximum, sum} [parts][rows].  A workgroup per row: eight parts at a time, four channels to a thread, so that a row waits for few
// reads one behind the other (48 rows x 21 parts x 128 channels 20.8 us with a wavefront that walks over the parts).
__global__ __launch_bounds__(256) void join_parts_kernel(const float* workspace, const int32_t* lens, uint16_t* out, float* lse, TensorStrides so,
                                                         uint32_t parts, uint32_t n_rows, uint32_t tokens_q, uint32_t heads, uint32_t dim, float scale)
{
    __shared__ float4 meet[8][32];
    const uint32_t lane = threadIdx.x & 63, at = blockIdx.x, c = 4u * (threadIdx.x & 31u), sub = threadIdx.x >> 5;
    const uint32_t g = at / tokens_q, row = at - g * tokens_q, b = g / heads, h = g - b * heads;
    if (row >= length_of(lens, b, 0, tokens_q)) return;
    const float2* state = reinterpret_cast<const float2*>(workspace + (size_t)parts * n_rows * dim) + at;
    const float factor = scale * 1.44269504088896340736f;
    float most = -__builtin_inff(), sum = 0.0f;
    for (uint32_t p = lane; p < parts; p += 64) most = fmaxf(most, state[(size_t)p * n_rows].x);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    const float base = most == -__builtin_inff() ? 0.0f : most;
    for (uint32_t p = lane; p < parts; p += 64) {
        const float2 st = state[(size_t)p * n_rows];
        sum = fmaf(st.y, __builtin_amdgcn_exp2f((st.x - base) * factor), sum);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c < dim) {
#pragma unroll 4
        for (uint32_t p = sub; p < parts; p += 8) {
            const float w = __builtin_amdgcn_exp2f((state[(size_t)p * n_rows].x - base) * factor);
            const float4 x = *reinterpret_cast<const float4*>(workspace + ((size_t)p * n_rows + at) * dim + c);
            o = make_float4(fmaf(x.x, w, o.x), fmaf(x.y, w, o.y), fmaf(x.z, w, o.z), fmaf(x.w, w, o.w));
        }
    }
    meet[sub][threadIdx.x & 31u] = o;
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        const float4 x = meet[i][threadIdx.x];
        o = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
    }
    const float inverse = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
    uint16_t* to = out + ((size_t)b * so.batch + (size_t)h * so.head + (size_t)row * so.token) * 8u;
    const attn_bf16x2 lo = __builtin_convertvector((attn_f32x2{o.x * inverse, o.y * inverse}), attn_bf16x2);
    const attn_bf16x2 hi = __builtin_convertvector((attn_f32x2{o.z * inverse, o.w * inverse}), attn_bf16x2);
    if (c < dim) *reinterpret_cast<uint2*>(to + c) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
    if (lse && threadIdx.x == 0) lse[at] = sum == 0.0f ? -__builtin_inff() : most * scale + 0.69314718055994530942f * __builtin_amdgcn_logf(sum);
}

}  // namespace fb4
