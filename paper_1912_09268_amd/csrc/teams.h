// Lanes that work on a row together: sums over 16 or 64 lanes of a wavefront, or over a workgroup of whole wavefronts.
#ifndef MGWFBP_TEAMS_H
#define MGWFBP_TEAMS_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ops {

// x of another lane of the same sixteen, by the data path between lanes (a few cycles, where a shuffle through LDS takes a hundred).
template <int CTRL> __device__ __forceinline__ float lane_of(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ double lane_of(double x) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t low = __builtin_amdgcn_update_dpp(0, static_cast<int>(bits), CTRL, 0xf, 0xf, true);
    const uint32_t high = __builtin_amdgcn_update_dpp(0, static_cast<int>(bits >> 32), CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, static_cast<uint64_t>(high) << 32 | low);
}
__device__ __forceinline__ float from_lane(float x, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); }
__device__ __forceinline__ double from_lane(double x, int lane) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t low = __builtin_amdgcn_readlane(static_cast<int>(bits), lane), high = __builtin_amdgcn_readlane(static_cast<int>(bits >> 32), lane);
    return __builtin_bit_cast(double, static_cast<uint64_t>(high) << 32 | low);
}

// join of x over the wavefront's aligned pieces of LANES lanes, in every lane, in one order: neighbours, pairs, mirrored halves of eight, of
// sixteen, and the four sixteens.
template <int LANES, typename F, typename J> __device__ __forceinline__ F lanes_all(F x, J&& join) {
    static_assert(LANES == 1 || LANES == 2 || LANES == 4 || LANES == 8 || LANES == 16 || LANES == 64);
    if constexpr (LANES > 1) x = join(x, lane_of<0xb1>(x));  // 1 0 3 2
    if constexpr (LANES > 2) x = join(x, lane_of<0x4e>(x));  // 2 3 0 1
    if constexpr (LANES > 4) x = join(x, lane_of<0x141>(x)); // eight lanes mirrored
    if constexpr (LANES > 8) x = join(x, lane_of<0x140>(x)); // sixteen lanes mirrored
    if constexpr (LANES == 64) x = join(join(from_lane(x, 0), from_lane(x, 16)), join(from_lane(x, 32), from_lane(x, 48)));
    return x;
}
template <int LANES, typename F> __device__ __forceinline__ F lanes_sum(F x) {
    return lanes_all<LANES>(x, [](F a, F b) { return a + b; });
}

// The sum of x over the THREADS lanes of a workgroup, in every lane; `room` holds a number for each wavefront and may be used
// again after the next barrier.
template <int THREADS, typename F> __device__ __forceinline__ F workgroup_sum(F x, F* room) {
    x = lanes_sum<64>(x);
    if (threadIdx.x % 64 == 0) room[threadIdx.x / 64] = x;
    __syncthreads();
    F sum = room[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) sum += room[w];
    return sum;
}

}  // namespace ops

#endif
