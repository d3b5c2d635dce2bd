// Norms of queries and keys per head with the position rotation in the same pass.
//
// A row is one head of one token: `dim` channels, 16 bytes of which a lane holds; rows stay in registers from the read to
// the write, so every element is read once and written once.  A wavefront takes as many successive tokens as rows fit its 64
// lanes (7 of 72 channels, 4 of 128), forms every lane's angles once and goes through the heads with them, eight heads' reads
// ahead of their use; a workgroup's wavefronts take successive runs of tokens, and an XCD's workgroups too.  Tokens side by side, not
// heads: a head's successive tokens lie side by side in the output, and lines that two wavefronts write in part cost more than
// lines that they read in part (16 heads of 72 channels of 17 frames, permuted input: 87 us with a token's heads side by side on 9 of
// 16 lanes).
// Bound by the memory stream.  Measured, queries and keys of 128 channels: 16 x 1024 tokens, 24 + 24 heads of a packed projection
// 83.5 us (4.8 TB/s; why not more was not found); 65536 tokens, 24 + 8 heads 191 us (5.6 TB/s; 229 with neighbouring workgroups on different
// XCDs and four heads ahead); the permuted input above 61.5 us (3.4 TB/s: a row of 144 bytes lies in two lines or three, in channels 36
// apart, of which others read the rest).
//   t = positions[a] * freqs[p] in double, brought to (-1/2, 1/2] revolutions there (a far position times a frequency
//   needs more than fp32's 24 bits), then the hardware's sine and cosine of revolutions (1.2e-7 off at most, measured over
//   2^18 arguments: a thirtieth of a percent of a bf16 step).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fb4_mfma.hpp"

namespace fb4 {

constexpr int kRopeThreads = 256;
enum { kRopeAdjacent = 0, kRopeHalves = 1 };

// Strides in units of 8 elements (16 bytes).
struct RopeStrides {
    uint32_t batch, head, token;
};

// What does not fit kernel arguments of their own: 24 bytes.
struct RopeShape {
    uint32_t tokens, n_tokens;   // per sequence; in all
    uint16_t heads_q, heads_k;
    float eps;
    uint8_t pieces;              // dim / 8
    uint8_t axis_end[3];         // pairs of the first axis, of the first two, of the first three
    uint8_t n_axes, pairs;       // pairs rotated in all
    uint8_t flags;               // kRopeNorm, kRopeShared
    uint8_t chunks;              // wavefronts that share the heads of a run of tokens
};
enum { kRopeNorm = 1, kRopeShared = 2 };   // positions are the same for all sequences

typedef __bf16 rope_bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t rope_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t rope_u32x2 __attribute__((ext_vector_type(2)));
typedef float rope_f32x2 __attribute__((ext_vector_type(2)));

constexpr int kRopeAhead = 8;   // heads whose rows are read before the first of them is used

template <int kPairing>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(const uint16_t* q, const uint16_t* k, uint16_t* q_out, uint16_t* k_out,
                                                                    const float* gamma_q, const float* gamma_k, const double* freqs,
                                                                    const int32_t* positions, RopeStrides sq, RopeStrides sk, RopeShape s)
{
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t pieces = s.pieces, rows = 64u / pieces, sub = lane / pieces, l = lane - sub * pieces;
    constexpr uint32_t kTeam = kRopeThreads / 64;   // successive runs of tokens to a workgroup
    const uint32_t teams = ((s.n_tokens + rows - 1u) / rows + kTeam - 1u) / kTeam;
    const uint32_t pos = xcd_local_position(blockIdx.x, teams * s.chunks);
    const uint32_t team = __builtin_amdgcn_readfirstlane(pos / s.chunks), chunk = pos - team * s.chunks, run = team * kTeam + wave;
    const uint32_t t = run * rows + sub;
    if (run * rows >= s.n_tokens) return;
    const bool live = sub < rows && t < s.n_tokens;
    const uint32_t b = live ? t / s.tokens : 0u, n = live ? t - b * s.tokens : 0u;
    // ---- this lane's channels: two runs of four, which make four pairs
    const uint32_t turned = s.pairs / 4u;   // (halves: lanes that hold pairs; pairs is a multiple of 4 there)
    const uint32_t ca = kPairing == kRopeAdjacent ? 8u * l : l < turned ? 4u * l : 2u * s.pairs + 8u * (l - turned);
    const uint32_t cb = kPairing == kRopeAdjacent || l >= turned ? ca + 4u : s.pairs + 4u * l;
    const uint16_t* from_q = q + ((size_t)b * sq.batch + (size_t)n * sq.token) * 8u;
    const uint16_t* from_k = k + ((size_t)b * sk.batch + (size_t)n * sk.token) * 8u;
    const uint32_t heads = s.heads_q + s.heads_k, each = (heads + s.chunks - 1u) / s.chunks;
    const uint32_t first = chunk * each, last = min(heads, first + each);
    uint4 ahead[kRopeAhead];
    auto read = [&](uint32_t i) {
        const bool is_k = i >= s.heads_q;
        const uint16_t* row = (is_k ? from_k : from_q) + (size_t)(is_k ? (i - s.heads_q) * (uint64_t)sk.head : i * (uint64_t)sq.head) * 8u;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (live && i < last) {
            if (kPairing == kRopeAdjacent) {
                v = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const rope_u32x4*>(row + ca)));
            } else {
                const uint2 va = *reinterpret_cast<const uint2*>(row + ca), vb = *reinterpret_cast<const uint2*>(row + cb);
                v = make_uint4(va.x, va.y, vb.x, vb.y);
            }
        }
        return v;
    };
#pragma unroll
    for (int i = 0; i < kRopeAhead; ++i) ahead[i] = read(first + i);
    // ---- the token's angles
    float cosine[4], sine[4];
    bool rotates[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t p = 4u * l + j;
        rotates[j] = p < s.pairs;
        const uint32_t axis = p < s.axis_end[0] ? 0u : p < s.axis_end[1] ? 1u : p < s.axis_end[2] ? 2u : 3u;
        double revolutions = 0.0;
        if (live && rotates[j]) revolutions = (double)positions[(size_t)(s.flags & kRopeShared ? n : t) * s.n_axes + axis] * freqs[p] * 0.15915494309189533577;
        const float f = (float)(revolutions - rint(revolutions));
        cosine[j] = __builtin_amdgcn_cosf(f);
        sine[j] = __builtin_amdgcn_sinf(f);
    }
    const bool norm = s.flags & kRopeNorm, passes = 2u * s.pairs < 8u * pieces;   // some channels keep their values
    float gq[8], gk[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t c = (j < 4 ? ca : cb) + j % 4;
        gq[j] = norm && gamma_q && live ? gamma_q[c] : 1.0f;
        gk[j] = norm && gamma_k && live ? gamma_k[c] : 1.0f;
    }
    const size_t out_q = ((size_t)b * s.heads_q * s.tokens + n) * (8u * pieces), out_k = ((size_t)b * s.heads_k * s.tokens + n) * (8u * pieces);
    for (uint32_t i0 = first; i0 < last; i0 += kRopeAhead) {
#pragma unroll
        for (int a = 0; a < kRopeAhead; ++a) {
            const uint32_t i = i0 + a;
            if (i >= last) break;
            const uint32_t w[4] = {ahead[a].x, ahead[a].y, ahead[a].z, ahead[a].w};
            ahead[a] = read(i + kRopeAhead);
            const bool is_k = i >= s.heads_q;
            auto element = [&](int j) { return __builtin_bit_cast(float, j % 2 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16); };
            float x[8];   // the two runs
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = element(j);
            if (norm) {
                // over a row's lanes: lane l adds what lies d further, so that its first has all
                auto row_sum = [&](auto sum) {
                    for (uint32_t d = 1; d < pieces; d *= 2) {
                        const auto other = __shfl(sum, (int)(lane + d));
                        sum += l + d < pieces ? other : 0;
                    }
                    return __shfl(sum, (int)(lane - l));
                };
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = fmaf(x[j], x[j], sum);
                const float v = row_sum(sum) / (8.0f * pieces) + s.eps;
                const bool ordinary = v >= 0x1p-100f && v <= 0x1p100f;
                const float r = rsqrtf(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= r;
                if (__any(!ordinary && live)) {
                    // squares that leave fp32, an Inf or NaN, a zero row without eps: that row in double, as the formula says
                    double sum_d = 0.0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum_d += (double)element(j) * (double)element(j);
                    const double r_d = 1.0 / sqrt(row_sum(sum_d) / (8.0 * pieces) + (double)s.eps);
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = ordinary ? x[j] : (float)((double)element(j) * r_d);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= is_k ? gk[j] : gq[j];
            }
            float y[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int u = kPairing == kRopeAdjacent ? 2 * j : j, v = kPairing == kRopeAdjacent ? 2 * j + 1 : 4 + j;
                y[u] = fmaf(x[u], cosine[j], -(x[v] * sine[j]));
                y[v] = fmaf(x[u], sine[j], x[v] * cosine[j]);
                if (passes && !rotates[j]) {   // (0 times an Inf of the other channel would be a NaN)
                    y[u] = x[u];
                    y[v] = x[v];
                }
            }
            if (live) {
                uint16_t* row = (is_k ? k_out + out_k : q_out + out_q) + (size_t)(is_k ? i - s.heads_q : i) * s.tokens * (8u * pieces);
                uint32_t o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector((rope_f32x2{y[2 * j], y[2 * j + 1]}), rope_bf16x2));
                if (kPairing == kRopeAdjacent) {
                    __builtin_nontemporal_store((rope_u32x4{o[0], o[1], o[2], o[3]}), reinterpret_cast<rope_u32x4*>(row + ca));
                } else {
                    __builtin_nontemporal_store((rope_u32x2{o[0], o[1]}), reinterpret_cast<rope_u32x2*>(row + ca));
                    __builtin_nontemporal_store((rope_u32x2{o[2], o[3]}), reinterpret_cast<rope_u32x2*>(row + cb));
                }
            }
        }
    }
}

}  // namespace fb4
