// Lanes that work on a row together: sums over 16 or 64 lanes of a wavefront, or over a workgroup of whole wavefronts.
#ifndef MGWFBP_TEAMS_H
#define MGWFBP_TEAMS_H

#include <hip/hip_runtime.h>

namespace ops {

// The sum of x over the wavefront's aligned pieces of LANES lanes, in every lane, in one order.
template <int LANES, typename F> __device__ __forceinline__ F lanes_sum(F x) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d /= 2) x += __shfl_xor(x, d);
    return x;
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
