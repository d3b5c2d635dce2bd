// What the kernels on the matrix cores share: operand and accumulator types of the 32x32x16 bf16 MFMA, and which workgroup takes
// which place of the work.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fb4 {

typedef __bf16 mfma_bf16x8 __attribute__((ext_vector_type(8)));
typedef float mfma_f32x16 __attribute__((ext_vector_type(16)));

// Workgroups are dealt to the eight XCDs in turn, and each XCD has its own L2.  The workgroups of one attention
// group read the same keys, so they should share an L2: workgroup b works on position (b % 8) * (n / 8) + b / 8
// of the launch, which puts consecutive positions on one XCD (the last n % 8 workgroups keep their own number).
__device__ __forceinline__ uint32_t xcd_local_position(uint32_t b, uint32_t n)
{
    const uint32_t chunk = n / 8u;
    return b < chunk * 8u ? (b % 8u) * chunk + b / 8u : b;
}

}  // namespace fb4
