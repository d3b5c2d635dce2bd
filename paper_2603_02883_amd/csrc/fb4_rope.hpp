// Norms of queries and keys per head with the position rotation in the same pass.
//
// A row is one head of one token: `dim` channels, 16 bytes of which a lane holds; rows stay in registers from the read to
// the write, so every element is read once and written once.  The angles belong to the token: the wavefront that takes a
// token forms them once and goes through the token's heads with them.
//   t = positions[a] * freqs[p] in double, brought to (-1/2, 1/2] revolutions there (a far position times a frequency
//   needs more than fp32's 24 bits), then the hardware's sine and cosine of revolutions (1.2e-7 off at most, measured over
//   2^18 arguments: a thirtieth of a percent of a bf16 step).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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
    uint8_t chunks;              // wavefronts that share a token's heads
};
enum { kRopeNorm = 1, kRopeShared = 2 };   // positions are the same for all sequences

typedef __bf16 rope_bf16x2 __attribute__((ext_vector_type(2)));
typedef float rope_f32x2 __attribute__((ext_vector_type(2)));

// kLanes: lanes per row, the power of two from dim / 8 on.
template <int kPairing, int kLanes>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(const uint16_t* q, const uint16_t* k, uint16_t* q_out, uint16_t* k_out,
                                                                    const float* gamma_q, const float* gamma_k, const double* freqs,
                                                                    const int32_t* positions, RopeStrides sq, RopeStrides sk, RopeShape s)
{
    constexpr uint32_t kRows = 64 / kLanes;   // heads per step of a wavefront
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t unit = blockIdx.x * (kRopeThreads / 64) + wave;
    const uint32_t t = unit / s.chunks, chunk = unit - t * s.chunks;
    if (t >= s.n_tokens) return;
    const uint32_t b = t / s.tokens, n = t - b * s.tokens;
    const uint32_t l = lane % kLanes, sub = lane / kLanes;
    const bool in_row = l < s.pieces;
    // ---- this lane's channels: two runs of four, which make four pairs
    const uint32_t turned = s.pairs / 4u;   // (halves: lanes that hold pairs; pairs is a multiple of 4 there)
    const uint32_t ca = kPairing == kRopeAdjacent ? 8u * l : l < turned ? 4u * l : 2u * s.pairs + 8u * (l - turned);
    const uint32_t cb = kPairing == kRopeAdjacent || l >= turned ? ca + 4u : s.pairs + 4u * l;
    // ---- the token's angles
    float cosine[4], sine[4];
    bool rotates[4];
    {
        const int32_t* at = positions + (size_t)(s.flags & kRopeShared ? n : t) * s.n_axes;
        int32_t where[4] = {0, 0, 0, 0};
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            if (a < s.n_axes) where[a] = at[a];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t p = 4u * l + j;
            rotates[j] = p < s.pairs;
            const int32_t pos = p < s.axis_end[0] ? where[0] : p < s.axis_end[1] ? where[1] : p < s.axis_end[2] ? where[2] : where[3];
            const double revolutions = rotates[j] ? (double)pos * freqs[p] * 0.15915494309189533577 : 0.0;
            const float f = (float)(revolutions - rint(revolutions));
            cosine[j] = __builtin_amdgcn_cosf(f);
            sine[j] = __builtin_amdgcn_sinf(f);
        }
    }
    const bool passes = 2u * s.pairs < 8u * s.pieces;   // some channels keep their values
    const uint32_t steps_q = (s.heads_q + kRows - 1) / kRows, steps = steps_q + (s.heads_k + kRows - 1) / kRows;
    const uint32_t each = (steps + s.chunks - 1) / s.chunks;
    for (uint32_t i = chunk * each; i < min(steps, (chunk + 1) * each); ++i) {
        const bool is_k = i >= steps_q;
        const uint32_t heads = is_k ? s.heads_k : s.heads_q, head = (is_k ? i - steps_q : i) * kRows + sub;
        const RopeStrides& st = is_k ? sk : sq;
        const bool live = in_row && head < heads;
        uint2 va = make_uint2(0, 0), vb = make_uint2(0, 0);
        if (live) {
            const uint16_t* row = (is_k ? k : q) + ((size_t)b * st.batch + (size_t)n * st.token + (size_t)head * st.head) * 8u;
            va = *reinterpret_cast<const uint2*>(row + ca);
            vb = *reinterpret_cast<const uint2*>(row + cb);
        }
        float x[8];   // the two runs
        const uint32_t w[4] = {va.x, va.y, vb.x, vb.y};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __builtin_bit_cast(float, w[j] << 16);
            x[2 * j + 1] = __builtin_bit_cast(float, w[j] & 0xFFFF0000u);
        }
        if (s.flags & kRopeNorm) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(x[j], x[j], sum);
#pragma unroll
            for (int d = 1; d < kLanes; d *= 2) sum += __shfl_xor(sum, d);
            const float v = sum / (8.0f * s.pieces) + s.eps;
            if (v >= 0x1p-100f && v <= 0x1p100f) {
                const float r = rsqrtf(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= r;
            }
            if (__any(!(v >= 0x1p-100f && v <= 0x1p100f))) {
                // squares that leave fp32, an Inf or NaN, a zero row without eps: that row in double, as the formula says
                double sum_d = 0.0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const double e = (double)__builtin_bit_cast(float, j % 2 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
                    sum_d += e * e;
                }
#pragma unroll
                for (int d = 1; d < kLanes; d *= 2) sum_d += __shfl_xor(sum_d, d);
                const double r = 1.0 / sqrt(sum_d / (8.0 * s.pieces) + (double)s.eps);
                if (!(v >= 0x1p-100f && v <= 0x1p100f)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = (float)((double)__builtin_bit_cast(float, j % 2 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16) * r);
                }
            }
            const float* gamma = is_k ? gamma_k : gamma_q;
            if (gamma && live) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] *= gamma[ca + j];
                    x[4 + j] *= gamma[cb + j];
                }
            }
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
            uint16_t* row = (is_k ? k_out : q_out) + (((size_t)b * heads + head) * s.tokens + n) * (8u * s.pieces);
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector((rope_f32x2{y[2 * j], y[2 * j + 1]}), rope_bf16x2));
            *reinterpret_cast<uint2*>(row + ca) = make_uint2(o[0], o[1]);
            *reinterpret_cast<uint2*>(row + cb) = make_uint2(o[2], o[3]);
        }
    }
}

}  // namespace fb4
