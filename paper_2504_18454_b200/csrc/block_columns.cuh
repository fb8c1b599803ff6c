// Sums over tokens of the block operators' weight gradients: CTAs leave binary32 rows in the workspace, joined here.
#pragma once
#include "block_common.cuh"

namespace palsgd {
namespace block {

// Rows of binary32 sums [K][parts][cols], joined in a fixed order: the columns of up to two results lie behind one another.
struct ColumnSumArgs {
    const float* part;
    void*    out[2];              // columns 0 .. split-1, and the rest; may be NULL
    int64_t  ow[2];               // worker strides
    uint32_t parts, cols, split;
};
template <typename T>
__global__ void __launch_bounds__(256) column_sum_kernel(const __grid_constant__ ColumnSumArgs a)
{
    __shared__ float run[8][32];
    let_next_start();
    wait_for_previous();
    const uint32_t k = blockIdx.y, lane = threadIdx.x & 31, r = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    const float* p = a.part + (uint64_t)k * a.parts * a.cols;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i < a.cols) {
        uint32_t b = r;
        for (; b + 24 < a.parts; b += 32)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[j] += p[(uint64_t)(b + 8 * j) * a.cols + i];
        for (; b < a.parts; b += 8) v[0] += p[(uint64_t)b * a.cols + i];
    }
    run[r][lane] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    if (r == 0 && i < a.cols) {
        float t = 0.0f;
#pragma unroll
        for (int b = 0; b < 8; ++b) t += run[b][lane];
        const uint32_t which = i >= a.split;
        if (a.out[which]) static_cast<T*>(a.out[which])[(int64_t)k * a.ow[which] + i - (which ? a.split : 0)] = from_f<T>(t);
    }
}

}  // namespace block
}  // namespace palsgd
