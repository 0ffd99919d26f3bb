// Sums over many partial results of a block of kSumThreads threads, 32 of them side by side: a lane has one, a warp takes every 32nd part, and the
// warps' sums are added in order, so that the same parts give the same bits.
#pragma once
#include "common.cuh"

namespace esc {

constexpr int kSumThreads = 1024;

// Of the `parts` values at[0], at[stride], ...: the sum, to warp 0.  By the whole block; a lane that is not `in` reads nothing.
__device__ __forceinline__ float sum_rows(const float* at, bool in, int parts, size_t stride) {
    __shared__ float acc[kSumThreads / 32][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    float s = 0.f;
    if (in) {
        at += warp * stride;
        const size_t step = kSumThreads / 32 * stride;             // added, not multiplied: 64 bits
#pragma unroll 8
        for (int i = warp; i < parts; i += kSumThreads / 32, at += step) s += __ldcg(at);
    }
    acc[warp][lane] = s;
    __syncthreads();
    if (warp == 0)
#pragma unroll
        for (int v = 1; v < kSumThreads / 32; ++v) s += acc[v][lane];
    return s;
}

}  // namespace esc
