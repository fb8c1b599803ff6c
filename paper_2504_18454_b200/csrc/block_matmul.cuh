// Matrix kernels of the gated feed-forward block.
#pragma once
#include "block_common.cuh"

namespace palsgd {
namespace block {

// An operand of worker k: element (i, kk) at data + k*w + (mn ? kk*r + i : i*r + kk).
struct Operand {
    const void* p;
    int64_t w, r;
    int mn;
};

struct MatArgs {
    Operand A[2], B[2];           // up to two products into one sum; the gate/up pass: B[0], B[1] into two sums
    int      n_seg;
    uint32_t M, N, Kd;
    int      act, save;
    void*    out[3];              // forward: h; hidden gradient: dg, du, h; plain: the product
    int64_t  ow, orow;
    void*    gate; void* up; uint8_t* gate_e; uint8_t* up_e;
    int64_t  gw, gr, uw, ur, gew, ger, uew, uer;
};

enum { MAT_PLAIN = 0, MAT_GATED = 1, MAT_HIDDEN = 2 };

template <bool SLOPE, bool FAST>
__device__ __forceinline__ float act_by(int kind, float g, float& slope)
{
    switch (kind) {
        case PALSGD_ACT_SILU: return act<PALSGD_ACT_SILU, SLOPE, FAST>(g, slope);
        case PALSGD_ACT_GELU: return act<PALSGD_ACT_GELU, SLOPE, FAST>(g, slope);
        case PALSGD_ACT_GELU_TANH: return act<PALSGD_ACT_GELU_TANH, SLOPE, FAST>(g, slope);
        default: return act<PALSGD_ACT_RELU, SLOPE, FAST>(g, slope);
    }
}

// 64 x 64 outputs of one worker by 256 threads, 16 steps of the inner axis at a time through shared memory.
template <typename T, int MODE>
__global__ void __launch_bounds__(256) mat_kernel(const __grid_constant__ MatArgs a)
{
    constexpr int NB = MODE == MAT_GATED ? 2 : 1;
    __shared__ float As[16][65], Bs[NB][16][65], Ct[NB][64][65];
    const uint32_t w = blockIdx.z, m0 = blockIdx.x * 64, n0 = blockIdx.y * 64;
    const uint32_t tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float c[NB][4][4] = {};
    for (int seg = 0; seg < a.n_seg; ++seg)
        for (uint32_t k0 = 0; k0 < a.Kd; k0 += 16) {
            for (uint32_t i = threadIdx.x; i < 16 * 64; i += 256) {
                const Operand& A = a.A[seg];
                uint32_t r = A.mn ? i & 63 : i >> 4, kk = A.mn ? i >> 6 : i & 15;
                As[kk][r] = m0 + r < a.M && k0 + kk < a.Kd
                    ? to_f(static_cast<const T*>(A.p)[(int64_t)w * A.w + (A.mn ? (int64_t)(k0 + kk) * A.r + (m0 + r) : (int64_t)(m0 + r) * A.r + (k0 + kk))]) : 0.0f;
                for (int b = 0; b < NB; ++b) {
                    const Operand& B = a.B[MODE == MAT_GATED ? b : seg];
                    r = B.mn ? i & 63 : i >> 4; kk = B.mn ? i >> 6 : i & 15;
                    Bs[b][kk][r] = n0 + r < a.N && k0 + kk < a.Kd
                        ? to_f(static_cast<const T*>(B.p)[(int64_t)w * B.w + (B.mn ? (int64_t)(k0 + kk) * B.r + (n0 + r) : (int64_t)(n0 + r) * B.r + (k0 + kk))]) : 0.0f;
                }
            }
            __syncthreads();
            for (int kk = 0; kk < 16; ++kk)
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) c[b][i][j] = fmaf(As[kk][ty + 16 * i], Bs[b][kk][tx + 16 * j], c[b][i][j]);
            __syncthreads();
        }
    for (int b = 0; b < NB; ++b)
        for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 4; ++j) Ct[b][ty + 16 * i][tx + 16 * j] = c[b][i][j];
    __syncthreads();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint32_t it = warp; it < 128; it += 8) {        // a warp takes 32 columns of a row: a group of a checkpoint
        const uint32_t m = m0 + it / 2, nb = n0 + (it & 1) * 32, n = nb + lane;
        if (m >= a.M || nb >= a.N) continue;
        const bool on = n < a.N;
        const float v = Ct[0][it / 2][(it & 1) * 32 + lane];
        const int64_t oo = (int64_t)w * a.ow + (int64_t)m * a.orow + n;
        const int64_t go = (int64_t)w * a.gw + (int64_t)m * a.gr + n, uo = (int64_t)w * a.uw + (int64_t)m * a.ur + n;
        const int64_t geo = (int64_t)w * a.gew + (int64_t)m * a.ger + nb / 32, ueo = (int64_t)w * a.uew + (int64_t)m * a.uer + nb / 32;
        float slope = 0.0f;
        if constexpr (MODE == MAT_PLAIN) {
            if (on) static_cast<T*>(a.out[0])[oo] = from_f<T>(v);
        } else if constexpr (MODE == MAT_GATED) {
            const float u = Ct[NB - 1][it / 2][(it & 1) * 32 + lane];
            if (on) static_cast<T*>(a.out[0])[oo] = from_f<T>(act_by<false, false>(a.act, v, slope) * u);
            if (a.save == PALSGD_SAVE_FULL && on) {
                static_cast<T*>(a.gate)[go] = from_f<T>(v);
                static_cast<T*>(a.up)[uo] = from_f<T>(u);
            } else if (a.save == PALSGD_SAVE_8BIT) {
                for (int b = 0; b < 2; ++b) {
                    const float x = on ? (b ? u : v) : 0.0f;
                    uint32_t mx = __float_as_uint(x) & 0x7FFFFFFFu;
                    mx = __reduce_max_sync(0xFFFFFFFFu, mx);
                    const uint32_t E = act8_exponent(mx);
                    if (on) static_cast<int8_t*>(b ? a.up : a.gate)[b ? uo : go] = (int8_t)act8_quant(x, act8_inverse(E));
                    if (lane == 0) (b ? a.up_e : a.gate_e)[b ? ueo : geo] = (uint8_t)E;
                }
            }
        } else if (on) {
            float g, u;
            if (a.save == PALSGD_SAVE_8BIT) {
                g = (float)static_cast<const int8_t*>(a.gate)[go] * act8_step(a.gate_e[geo]);
                u = (float)static_cast<const int8_t*>(a.up)[uo] * act8_step(a.up_e[ueo]);
            } else {
                g = to_f(static_cast<const T*>(a.gate)[go]);
                u = to_f(static_cast<const T*>(a.up)[uo]);
            }
            const float ag = act_by<true, false>(a.act, g, slope);
            static_cast<T*>(a.out[0])[oo] = from_f<T>(v * u * slope);
            static_cast<T*>(a.out[1])[oo] = from_f<T>(v * ag);
            static_cast<T*>(a.out[2])[oo] = from_f<T>(ag * u);
        }
    }
}

}  // namespace block
}  // namespace palsgd
