// Pages and slots of new tokens (fb4_cache_plan): integers only, and few of them, so what counts is the number of launches and of
// steps that wait for each other.  One workgroup: sums over the sequences before each one of what they give back and want, then every
// page that moves and every new token finds its sequence by halves of those sums (LDS) and is handled by a thread of its own.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fb4 {

constexpr uint32_t kPlanThreads = 1024, kPlanEach = 4, kPlanMaxBatch = kPlanThreads * kPlanEach;
constexpr uint32_t kPlanOwnTokens = 16384;   // as many tokens' slots the one workgroup writes itself

struct PlanShape {
    uint32_t batch, max_pages, n_free, tokens;
    uint32_t page_bits;
};

__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, uint32_t bits) { return (tokens >> bits) + ((tokens & ((1u << bits) - 1u)) != 0u); }

// The last i in 0 .. n - 1 with from[i] <= x (from[0] = 0, ascending): of equal ones the last, which is the one that has something.
__device__ __forceinline__ uint32_t owner_of(const int32_t* from, uint32_t n, uint32_t x)
{
    uint32_t low = 0, high = n;   // from[low] <= x < from[high]
    while (high - low > 1u) {
        const uint32_t mid = (low + high) / 2u;
        if ((uint32_t)from[mid] <= x) low = mid;
        else high = mid;
    }
    return low;
}

__device__ __forceinline__ void place_token(uint32_t t, uint32_t total, const int32_t* starts, const int32_t* lens, const int32_t* tables, int32_t* slots,
                                            int32_t* positions, PlanShape s)
{
    int32_t slot = -1, position = 0;
    if (t < total) {
        const uint32_t b = owner_of(starts, s.batch, t);
        position = lens[b] - (starts[b + 1] - (int32_t)t);
        const int32_t page = tables[(size_t)b * s.max_pages + ((uint32_t)position >> s.page_bits)];
        if (page >= 0 && page < (int32_t)(0x80000000u >> s.page_bits)) slot = (page << s.page_bits) + (position & (int32_t)((1u << s.page_bits) - 1u));
    }
    slots[t] = slot;
    if (positions) positions[t] = position;
}

__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(const int32_t* lens, const int32_t* adds, const int32_t* free_count, int32_t* tables,
                                                                  int32_t* free_pages, int32_t* lens_out, int32_t* free_count_out, int32_t* starts_out,
                                                                  int32_t* slots, int32_t* positions, PlanShape s)
{
    // before each sequence: pages given back, pages taken, tokens granted; and their sums
    __shared__ int32_t back[kPlanMaxBatch + 1], take[kPlanMaxBatch + 1], starts[kPlanMaxBatch + 1];
    __shared__ int32_t held[kPlanMaxBatch], now[kPlanMaxBatch];   // tokens before and after
    __shared__ int64_t wave_sums[kPlanThreads / 64][3];
    __shared__ int32_t totals[2];                                 // pages taken, tokens granted
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const int64_t capacity = (int64_t)s.max_pages << s.page_bits;
    const int32_t count = min(max(free_count[0], 0), (int32_t)s.n_free);
    // (b * kPlanEach + i: so that a thread's sequences are neighbours)
    uint32_t old[kPlanEach], cut[kPlanEach], need[kPlanEach];
    int64_t want[kPlanEach], sums[3] = {0, 0, 0};
    uint32_t gives[kPlanEach];
#pragma unroll
    for (uint32_t i = 0; i < kPlanEach; ++i) {
        const uint32_t b = tid * kPlanEach + i;
        old[i] = cut[i] = need[i] = gives[i] = 0;
        want[i] = 0;
        if (b < s.batch) {
            old[i] = (uint32_t)min(max((int64_t)lens[b], (int64_t)0), capacity);
            const int64_t add = adds[b], after = (int64_t)old[i] + add;
            cut[i] = add < 0 ? (uint32_t)max(after, (int64_t)0) : old[i];
            gives[i] = pages_of(old[i], s.page_bits) - pages_of(cut[i], s.page_bits);
            if (add > 0 && after <= capacity) {
                want[i] = add;
                need[i] = pages_of((uint32_t)after, s.page_bits) - pages_of(old[i], s.page_bits);
            }
        }
        sums[0] += gives[i];
        sums[1] += need[i];
        sums[2] += want[i];
    }
    // sums over the threads before this one
    int64_t before[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        int64_t x = sums[k];
#pragma unroll
        for (uint32_t d = 1; d < 64; d *= 2) {
            const int64_t y = __shfl_up(x, d);
            if (lane >= d) x += y;
        }
        if (lane == 63u) wave_sums[wave][k] = x;
        before[k] = x - sums[k];
    }
    if (tid < 2u) totals[tid] = 0;
    __syncthreads();
    int64_t given = 0;
    for (uint32_t w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) {
#pragma unroll
            for (int k = 0; k < 3; ++k) before[k] += wave_sums[w][k];
        }
        given += wave_sums[w][0];
    }
    const int64_t there = min((int64_t)count + given, (int64_t)s.n_free);
    // The sequences that grow and are served are the first ones that do: sums only grow.  Those behind want nothing; their places in
    // `take` and `starts` are the totals.
#pragma unroll
    for (uint32_t i = 0; i < kPlanEach; ++i) {
        const uint32_t b = tid * kPlanEach + i;
        const bool fits = before[1] + need[i] <= there && before[2] + want[i] <= (int64_t)s.tokens;
        if (b < s.batch) {
            back[b] = (int32_t)before[0];
            held[b] = (int32_t)old[i];
            now[b] = (int32_t)(want[i] && fits ? old[i] + (uint32_t)want[i] : cut[i]);
            // (beyond the border neither sum fits 31 bits for sure: the totals replace them below)
            take[b] = fits ? (int32_t)before[1] : -1;
            starts[b] = fits ? (int32_t)before[2] : -1;
            if (fits && want[i]) {
                atomicMax(&totals[0], (int32_t)(before[1] + need[i]));
                atomicMax(&totals[1], (int32_t)(before[2] + want[i]));
            }
        }
        before[0] += gives[i];
        before[1] += need[i];
        before[2] += want[i];
    }
    __syncthreads();
    const int32_t taken = totals[0], granted = totals[1];
#pragma unroll
    for (uint32_t i = 0; i < kPlanEach; ++i) {
        const uint32_t b = tid * kPlanEach + i;
        if (b < s.batch) {
            if (take[b] < 0 || take[b] > taken) take[b] = taken;
            if (starts[b] < 0 || starts[b] > granted) starts[b] = granted;
        }
    }
    if (tid == 0) {
        back[s.batch] = (int32_t)given;
        take[s.batch] = taken;
        starts[s.batch] = granted;
    }
    __syncthreads();
    // ---- pages back onto the free list
    for (uint32_t p = tid; p < (uint32_t)given; p += kPlanThreads) {
        const int64_t place = (int64_t)count + p;
        if (place >= (int64_t)s.n_free) break;
        const uint32_t b = owner_of(back, s.batch, p);
        free_pages[place] = tables[(size_t)b * s.max_pages + pages_of((uint32_t)now[b], s.page_bits) + (p - (uint32_t)back[b])];
    }
    __syncthreads();
    // ---- pages off its end
    for (uint32_t p = tid; p < (uint32_t)taken; p += kPlanThreads) {
        const uint32_t b = owner_of(take, s.batch, p);
        tables[(size_t)b * s.max_pages + pages_of((uint32_t)held[b], s.page_bits) + (p - (uint32_t)take[b])] = free_pages[there - 1 - p];
    }
    for (uint32_t b = tid; b < s.batch; b += kPlanThreads) lens_out[b] = now[b];
    for (uint32_t b = tid; b <= s.batch; b += kPlanThreads) starts_out[b] = starts[b];
    if (tid == 0) free_count_out[0] = (int32_t)(there - taken);
    if (s.tokens > kPlanOwnTokens) return;
    __syncthreads();
    for (uint32_t t = tid; t < s.tokens; t += kPlanThreads) place_token(t, (uint32_t)granted, starts, now, tables, slots, positions, s);
}

// The slots of many tokens, from what the kernel above wrote.
__global__ __launch_bounds__(256) void cache_slots_kernel(const int32_t* starts_in, const int32_t* lens, const int32_t* tables, int32_t* slots,
                                                          int32_t* positions, PlanShape s)
{
    __shared__ int32_t starts[kPlanMaxBatch + 1];
    for (uint32_t b = threadIdx.x; b <= s.batch; b += 256) starts[b] = starts_in[b];
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t t = (blockIdx.x * 4u + i) * 256u + threadIdx.x;
        if (t < s.tokens) place_token(t, (uint32_t)starts[s.batch], starts, lens, tables, slots, positions, s);
    }
}

}  // namespace fb4
