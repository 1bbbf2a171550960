// Codes of activation checkpoints (act8.hip, norm.hip).
#ifndef MGWFBP_ACT_CODE_H
#define MGWFBP_ACT_CODE_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ops {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Four whole numbers of -127 .. 127 to bytes: added to 1.5 * 2^23 a number's last eight bits are those of the sum, which rounds to
// nearest even on the way.
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
    auto bits = [](float x) { return __builtin_bit_cast(uint32_t, x + 12582912.f); };
    const uint32_t low = __builtin_amdgcn_perm(bits(b), bits(a), 0x0c0c0400), high = __builtin_amdgcn_perm(bits(d), bits(c), 0x04000c0c);
    return low | high;
}

// Code i of eight that lie side by side.
__device__ __forceinline__ float code_of(const u32x2& q, int i) { return static_cast<float>(static_cast<int32_t>(q[i / 4]) << (24 - 8 * (i % 4)) >> 24); }

}  // namespace ops

#endif
