// Sums over tokens of the block operators' weight gradients: CTAs leave binary32 rows in the workspace, joined here; zeros where there
// are no tokens.
#pragma once
#include "block_common.cuh"

namespace palsgd {
namespace block {

// Rows of binary32 sums [K][parts][ld], ld a multiple of four, joined in a fixed order: a thread has four columns and every
// eighth row.  The columns of two results lie behind one another, or those of one are the rows of a matrix.
struct ColumnSumArgs {
    const float* part;
    void*    out[2];              // columns 0 .. split-1, and the rest
    int64_t  ow[2];               // worker strides
    uint32_t parts, cols, ld, split;
    uint32_t wrap, inside;        // columns of a row of out[0] in `part`, and in out[0]
    int64_t  row;                 // out[0]'s row stride
};
template <typename T>
__global__ void __launch_bounds__(256) column_sum_kernel(const __grid_constant__ ColumnSumArgs a)
{
    __shared__ float4 run[8][32];
    let_next_start();
    wait_for_previous();
    const uint32_t k = blockIdx.y, lane = threadIdx.x & 31, r = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * 4;
    const float* p = a.part + (uint64_t)k * a.parts * a.ld + c;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c < a.cols) {
#pragma unroll 4
        for (uint32_t b = r; b < a.parts; b += 8) {
            const float4 t = __ldg(reinterpret_cast<const float4*>(p + (uint64_t)b * a.ld));
            v.x += t.x; v.y += t.y; v.z += t.z; v.w += t.w;
        }
    }
    run[r][lane] = v;
    __syncthreads();
    if (threadIdx.x >= 128) return;
    const uint32_t i = blockIdx.x * 128 + threadIdx.x;
    if (i >= a.cols) return;
    float t = 0.0f;
#pragma unroll
    for (int b = 0; b < 8; ++b) t += reinterpret_cast<const float*>(run[b])[threadIdx.x];
    if (i >= a.split) {
        static_cast<T*>(a.out[1])[(int64_t)k * a.ow[1] + i - a.split] = from_f<T>(t);
    } else {
        const uint32_t m = i / a.wrap, c = i - m * a.wrap;
        if (c < a.inside) static_cast<T*>(a.out[0])[(int64_t)k * a.ow[0] + m * a.row + c] = from_f<T>(t);
    }
}

// Weight gradients of no tokens: up to three matrices of zeros.
struct ZeroArgs { void* p[3]; int64_t w[3], r[3]; uint32_t rows[3], cols[3]; };

template <typename T>
__global__ void __launch_bounds__(256) zero_kernel(const __grid_constant__ ZeroArgs a)
{
    let_next_start();
    wait_for_previous();
    const uint32_t i = blockIdx.y;
    T* p = static_cast<T*>(a.p[i]) + (int64_t)blockIdx.z * a.w[i];
    for (uint32_t r = blockIdx.x; r < a.rows[i]; r += gridDim.x)
        for (uint32_t c = threadIdx.x; c < a.cols[i]; c += 256) p[(int64_t)r * a.r[i] + c] = from_f<T>(0.0f);
}

}  // namespace block
}  // namespace palsgd
