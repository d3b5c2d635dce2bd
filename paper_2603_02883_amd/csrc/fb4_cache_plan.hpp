// Pages and slots of new tokens (fb4_cache_plan): integers only, and few of them, so what counts is the number of launches and of
// steps that wait for each other.  One workgroup, a thread per sequence (four beyond 1024): sums over the sequences before each one of what
// they give back and want, by wavefronts in registers.  A sequence that grows by up to 16 tokens, which take one new page at most, is its
// thread's own; the pages and tokens of the others find their sequence by halves of the sums (LDS) and have a thread each.
// What bounds it is that chain: 256 sequences a token further 2.6 us on the card (4.5 to 5.1 per call, the launch), 48 with prompts of up to 4096 tokens 7.2 and
// 3.5 to 5 for the slots.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fb4 {

constexpr uint32_t kPlanMost = 1024, kPlanMaxBatch = 4096;
constexpr uint32_t kPlanFew = 16;            // tokens of a sequence that its thread places itself: at most one new page
// As many tokens' slots the one workgroup writes itself (4 sequences that grow by up to 4096: 5.6 us so, 7.1 with a second launch; 8: 11.9, 7.6; 16: 30.5, 8.5).
constexpr uint32_t kPlanOwnTokens = 8192;

struct PlanShape {
    uint32_t batch, max_pages, n_free, tokens;
    uint32_t page_bits, threads;
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

__device__ __forceinline__ int32_t slot_of(int32_t page, uint32_t position, uint32_t bits)
{
    return page >= 0 && page < (int32_t)(0x80000000u >> bits) ? (page << bits) + (int32_t)(position & ((1u << bits) - 1u)) : -1;
}

// Sum over the lanes up to this one, held at 2^32 - 1 (sums beyond are no one's any more).
__device__ __forceinline__ uint32_t lanes_before(uint32_t x)
{
#define FB4_PLAN_ADD(ctrl, rows) x = __builtin_elementwise_add_sat(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xF, false))
    FB4_PLAN_ADD(0x111, 0xF);   // one lane to the right in a row of 16, two, four, eight
    FB4_PLAN_ADD(0x112, 0xF);
    FB4_PLAN_ADD(0x114, 0xF);
    FB4_PLAN_ADD(0x118, 0xF);
    FB4_PLAN_ADD(0x142, 0xA);   // a row's last lane to the next row; the second row's to the upper half
    FB4_PLAN_ADD(0x143, 0xC);
#undef FB4_PLAN_ADD
    return x;
}

template <uint32_t kEach>
__global__ __launch_bounds__(kPlanMost) void cache_plan_kernel(const int32_t* lens, const int32_t* adds, const int32_t* free_count, int32_t* tables,
                                                               int32_t* free_pages, int32_t* lens_out, int32_t* free_count_out, int32_t* starts_out,
                                                               int32_t* slots, int32_t* positions, PlanShape s)
{
    // before each sequence: pages given back, pages taken, tokens granted; tokens before and after
    constexpr uint32_t kBatch = kEach * kPlanMost;
    __shared__ int32_t back[kBatch + 1], take[kBatch + 1], starts[kBatch + 1], held[kBatch], now[kBatch];
    __shared__ uint32_t wave_sums[3][kPlanMost / 64];
    __shared__ uint32_t totals[3];   // pages taken, tokens granted, whether a sequence grows by many
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), bits = s.page_bits;
    const uint32_t capacity = s.max_pages << bits;   // (below 2^31)
    const uint32_t count = (uint32_t)min(max(free_count[0], 0), (int32_t)s.n_free);
    uint32_t old[kEach], cut[kEach], gives[kEach], need[kEach], want[kEach], sums[3] = {0, 0, 0};
    int32_t page0[kEach];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {   // (b: a thread's sequences are neighbours)
        const uint32_t b = tid * kEach + i;
        old[i] = cut[i] = gives[i] = need[i] = want[i] = 0;
        page0[i] = -1;
        if (b < s.batch) {
            const int32_t len = lens[b], add = adds[b];
            old[i] = (uint32_t)min(max(len, 0), (int32_t)capacity);
            const int64_t after = (int64_t)old[i] + add;
            cut[i] = add < 0 ? (uint32_t)max(after, (int64_t)0) : old[i];
            gives[i] = pages_of(old[i], bits) - pages_of(cut[i], bits);
            if (add > 0 && after <= (int64_t)capacity) {
                want[i] = (uint32_t)add;
                need[i] = pages_of((uint32_t)after, bits) - pages_of(old[i], bits);
                if (want[i] <= kPlanFew && (old[i] & ((1u << bits) - 1u))) page0[i] = tables[(size_t)b * s.max_pages + (old[i] >> bits)];
            }
        }
        sums[0] += gives[i];
        sums[1] += need[i];
        sums[2] = __builtin_elementwise_add_sat(sums[2], want[i]);
    }
    uint32_t before[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const uint32_t x = lanes_before(sums[k]);
        if (lane == 63u) wave_sums[k][wave] = x;
        before[k] = __shfl_up(x, 1);
        if (lane == 0) before[k] = 0;
    }
    if (tid < 3u) totals[tid] = 0;
    __syncthreads();
    const uint32_t waves = s.threads / 64u;
    uint32_t given = 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const uint32_t x = lanes_before(lane < waves ? wave_sums[k][lane] : 0u);
        if (wave) before[k] = __builtin_elementwise_add_sat(before[k], (uint32_t)__builtin_amdgcn_readlane((int)x, wave - 1u));
        if (k == 0) given = (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
    }
    const uint32_t there = min(count + given, s.n_free);   // (both below 2^31)
    // The sequences that grow and are served are the first ones that do: sums only grow.
    uint32_t take_from[kEach], start[kEach];
    bool served[kEach];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t b = tid * kEach + i, pages = __builtin_elementwise_add_sat(before[1], need[i]), tokens = __builtin_elementwise_add_sat(before[2], want[i]);
        served[i] = want[i] && pages <= there && tokens <= s.tokens;
        take_from[i] = before[1];
        start[i] = before[2];
        const uint64_t yes = __ballot(served[i]), many = __ballot(served[i] && want[i] > kPlanFew);
        if (yes) {
            const uint32_t l = (uint32_t)(63 - __builtin_clzll(yes));
            const uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)pages, l), t = (uint32_t)__builtin_amdgcn_readlane((int)tokens, l);
            if (lane == 0) {
                atomicMax(&totals[0], p);
                atomicMax(&totals[1], t);
                if (many) atomicMax(&totals[2], 1u);
            }
        }
        if (b < s.batch) {
            back[b] = (int32_t)before[0];
            held[b] = (int32_t)old[i];
            now[b] = (int32_t)(served[i] ? old[i] + want[i] : cut[i]);
        }
        before[0] += gives[i];
        before[1] = pages;
        before[2] = tokens;
    }
    __syncthreads();
    // (behind the border, where the sums still count what was not served, the totals)
    const uint32_t taken = totals[0], granted = totals[1];
    const bool many = totals[2] != 0u;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t b = tid * kEach + i;
        if (b < s.batch) {
            take[b] = (int32_t)min(take_from[i], taken);
            starts[b] = (int32_t)min(start[i], granted);
            starts_out[b] = starts[b];
            lens_out[b] = now[b];
        }
    }
    if (tid == 0) {
        back[s.batch] = (int32_t)given;
        take[s.batch] = (int32_t)taken;
        starts[s.batch] = starts_out[s.batch] = (int32_t)granted;
        free_count_out[0] = (int32_t)(there - taken);
    }
    if (given || many) __syncthreads();
    // ---- pages back onto the free list
    if (given) {
        for (uint32_t p = tid; p < given; p += s.threads) {
            const uint64_t place = (uint64_t)count + p;
            if (place >= s.n_free) break;
            const uint32_t b = owner_of(back, s.batch, p);
            free_pages[place] = tables[(size_t)b * s.max_pages + pages_of((uint32_t)now[b], bits) + (p - (uint32_t)back[b])];
        }
        __syncthreads();
    }
    // ---- a page off its end, and a few tokens: the sequence's own thread
    const bool place_here = s.tokens <= kPlanOwnTokens;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        if (!served[i] || want[i] > kPlanFew) continue;
        const uint32_t b = tid * kEach + i;
        int32_t page1 = -1;
        if (need[i]) {
            page1 = free_pages[there - 1u - take_from[i]];
            tables[(size_t)b * s.max_pages + pages_of(old[i], bits)] = page1;
        }
        if (!place_here) continue;
        for (uint32_t j = 0; j < want[i]; ++j) {
            const uint32_t position = old[i] + j;
            const bool first = (old[i] & ((1u << bits) - 1u)) && position >> bits == old[i] >> bits;
            slots[start[i] + j] = slot_of(first ? page0[i] : page1, position, bits);
            if (positions) positions[start[i] + j] = (int32_t)position;
        }
    }
    // ---- pages and tokens of the others
    if (many) {
        for (uint32_t p = tid; p < taken; p += s.threads) {
            const uint32_t b = owner_of(take, s.batch, p);
            if ((uint32_t)(now[b] - held[b]) > kPlanFew)
                tables[(size_t)b * s.max_pages + pages_of((uint32_t)held[b], bits) + (p - (uint32_t)take[b])] = free_pages[there - 1u - p];
        }
        if (place_here) {
            for (uint32_t t = tid; t < granted; t += s.threads) {
                const uint32_t b = owner_of(starts, s.batch, t);
                if ((uint32_t)(now[b] - held[b]) <= kPlanFew) continue;
                // (a new page from the list itself: the table's entry is on its way)
                const uint32_t position = (uint32_t)held[b] + (t - (uint32_t)starts[b]), at = position >> bits, fresh = pages_of((uint32_t)held[b], bits);
                const int32_t page = at < fresh ? tables[(size_t)b * s.max_pages + at] : free_pages[there - 1u - ((uint32_t)take[b] + at - fresh)];
                slots[t] = slot_of(page, position, bits);
                if (positions) positions[t] = (int32_t)position;
            }
        }
    }
    if (place_here) {
        for (uint32_t t = granted + tid; t < s.tokens; t += s.threads) {
            slots[t] = -1;
            if (positions) positions[t] = 0;
        }
    }
}

// The slots of many tokens, from what the kernel above wrote.
__global__ __launch_bounds__(256) void cache_slots_kernel(const int32_t* starts_in, const int32_t* lens, const int32_t* tables, int32_t* slots,
                                                          int32_t* positions, PlanShape s)
{
    __shared__ int32_t starts[kPlanMaxBatch + 1];
    for (uint32_t b = threadIdx.x; b <= s.batch; b += 256) starts[b] = starts_in[b];
    __syncthreads();
    const uint32_t total = (uint32_t)starts[s.batch];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t t = (blockIdx.x * 4u + i) * 256u + threadIdx.x;
        if (t >= s.tokens) break;
        int32_t slot = -1;
        uint32_t position = 0;
        if (t < total) {
            const uint32_t b = owner_of(starts, s.batch, t);
            position = (uint32_t)lens[b] - ((uint32_t)starts[b + 1] - t);
            slot = slot_of(tables[(size_t)b * s.max_pages + (position >> s.page_bits)], position, s.page_bits);
        }
        slots[t] = slot;
        if (positions) positions[t] = (int32_t)position;
    }
}

}  // namespace fb4
