// Row kernels of the block operators: 8-bit checkpoints, and the norm of queries and keys with the position rotation.
// Both move every byte once and compute little: memory bandwidth bounds them.
#pragma once
#include "block_common.cuh"

namespace palsgd {
namespace block {

// ------------------------------------------------------------------------------------------------ 8-bit checkpoints

struct Act8Args {
    void*    x;                   // pack: read; unpack: written
    int8_t*  q;
    uint8_t* e;
    int64_t  xw, xr, qw, qr, ew, er;
    uint64_t rows, cols;
    uint32_t units_per_row;       // pieces of V values, padded to whole groups
    uint64_t units;               // rows * units_per_row
};

// A unit is V consecutive values, 32/V lanes share a group, and a thread takes one unit: 16 (bf16) or 32 (fp32) bytes
// of x and 8 of q a lane where the layout allows (V = 8), else one value (V = 1, a warp is a group).
template <typename T, int V, bool PACK>
__global__ void __launch_bounds__(256) act8_kernel(const __grid_constant__ Act8Args a)
{
    constexpr int kLanes = 32 / V;
    T* const x = static_cast<T*>(a.x) + (int64_t)blockIdx.y * a.xw;
    int8_t* const q = a.q + (int64_t)blockIdx.y * a.qw;
    uint8_t* const e = a.e + (int64_t)blockIdx.y * a.ew;
    const uint64_t step = (uint64_t)gridDim.x * blockDim.x;
    const uint64_t end = (a.units + 31) / 32 * 32;       // whole warps take part in the exchange below
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < end; i += step) {
        uint64_t row = a.units < 0x80000000ull ? (uint32_t)i / a.units_per_row : i / a.units_per_row;
        const uint64_t c = (i - row * a.units_per_row) * V;
        const bool on = row < a.rows && c < a.cols;
        if (!on) row = 0;
        const int64_t xo = (int64_t)row * a.xr + (int64_t)c, qo = (int64_t)row * a.qr + (int64_t)c;
        const int64_t eo = (int64_t)row * a.er + (int64_t)(c / 32);
        float v[V];
        if constexpr (PACK) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = 0.0f;
            if (on) Vec<T, V>::load(x + xo, v);
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
#pragma unroll
            for (int s = kLanes / 2; s; s >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, s));
            const uint32_t E = act8_exponent(m);
            const float inv = act8_inverse(E);
            if (on) {
                if constexpr (V == 8) {
                    uint32_t w[2] = {0, 0};
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j / 4] |= ((uint32_t)act8_quant(v[j], inv) & 0xFFu) << (8 * (j & 3));
                    *reinterpret_cast<uint2*>(q + qo) = make_uint2(w[0], w[1]);
                } else {
                    q[qo] = (int8_t)act8_quant(v[0], inv);
                }
                if (threadIdx.x % kLanes == 0) e[eo] = (uint8_t)E;
            }
        } else if (on) {
            const float s = act8_step(e[eo]);
            if constexpr (V == 8) {
                const uint2 w = __ldg(reinterpret_cast<const uint2*>(q + qo));
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3))) * s;
            } else {
                v[0] = (float)q[qo] * s;
            }
            Vec<T, V>::store(x + xo, v);
        }
    }
}

// ------------------------------------------------------------------------------------------------ q/k norm + rotation

struct HeadsArg {
    const void* x;                // input heads
    const void* d;                // backward: gradient of the output heads
    void*       out;              // forward: output heads; backward: gradient of the input heads
    const void* w;                // norm weights, one row per worker
    int64_t xw, xt, xh, dw, dt, dh, ow, ot, oh, ww;
    uint32_t heads;
    float*   part;                // backward: [K][CTAs of this side][head_dim] partial sums of the weight gradient
};

struct QkArgs {
    HeadsArg side[2];             // q, k
    uint32_t ctas[2];             // of one worker, by their shares of the heads: q's first
    const float* cos_t;
    const float* sin_t;
    const int32_t* pos;
    int64_t  pos_w;
    uint64_t tokens, table_rows;
    uint32_t head_dim, rot, pair_slots, slots;   // slots: two vectors of V values each; the first pair_slots hold pairs
    uint32_t lanes;               // lanes of a warp that share one head: a power of two, NS * lanes >= slots
    int      interleaved;
    int      table_wide;          // the rows of the angle tables start on 16-byte boundaries
    float    eps;
};

// What a lane holds of one head under way: the two vectors of each of its NS slots, as they lie in memory.
template <typename T, int V, int NS, bool BACK>
struct QkItem {
    Raw<T, V> x[NS][2], d[BACK ? NS : 1][2];
    int64_t out;
    int32_t pos;
    bool live;
};

template <bool SECOND, typename A, typename B>
__device__ __forceinline__ auto& either(A& a, B& b)
{
    if constexpr (SECOND) return b;
    else return a;
}

// A warp takes a few tokens at a time and walks their heads; `lanes` lanes share a head, and a slot of a lane holds both
// halves of its rotation pairs, so the rotation needs no exchange: for split halves vectors s and s + rot/(2V), for
// interleaved pairs two neighbouring vectors (V > 1: the pairs lie inside a vector; V = 1: the slot is the pair).  The
// only exchanges are the sums over a head.  The next items are under way while one is worked on: two of them forward, one
// backward (it is twice the size).  Angles are read when their item is due -- all heads of a token read the same ones, so
// they come from L1 -- and the norm weights stay in registers throughout.
template <typename T, int V, int NS, bool BACK>
__global__ void __launch_bounds__(256, NS == 1 ? 2 : 1) qk_kernel(const __grid_constant__ QkArgs a)
{
    const uint32_t side = blockIdx.x >= a.ctas[0], cta = blockIdx.x - (side ? a.ctas[0] : 0), ctas = a.ctas[side];
    const HeadsArg& h = a.side[side];
    const uint32_t k = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t sub = lane & (a.lanes - 1), group = lane / a.lanes, groups = 32 / a.lanes;
    const uint32_t n_vec = a.head_dim / V;
    uint32_t at[NS][2];           // first element of each vector, or ~0
    T w[NS][2][V];
    float acc[NS][2][V];
    const T* wp = static_cast<const T*>(h.w) + (int64_t)k * h.ww;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const uint32_t slot = s * a.lanes + sub;
        const uint32_t split = a.interleaved ? 0 : a.pair_slots;
        uint32_t v0, v1;
        if (slot < split) { v0 = slot; v1 = slot + split; }
        else { v0 = 2 * split + 2 * (slot - split); v1 = v0 + 1; }
        at[s][0] = slot < a.slots && v0 < n_vec ? v0 * V : ~0u;
        at[s][1] = slot < a.slots && v1 < n_vec ? v1 * V : ~0u;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                w[s][p][j] = at[s][p] != ~0u ? wp[at[s][p] + j] : from_f<T>(0.0f);
                acc[s][p][j] = 0.0f;
            }
        }
    }
    const float inv_n = 1.0f / (float)a.head_dim;
    const uint32_t half = a.rot / 2;
    // the warp's groups: `abreast` heads of each of `tokens` tokens
    uint32_t abreast = 1;
    while (abreast < groups && abreast < h.heads) abreast *= 2;
    const uint32_t tokens = groups / abreast, first = group % abreast, rounds = (h.heads + abreast - 1) / abreast;
    const uint64_t step = (uint64_t)ctas * 8 * tokens;

    uint64_t t = ((uint64_t)cta * 8 + warp) * tokens;                  // of the item to be fetched
    uint32_t round = 0;
    using Item = QkItem<T, V, NS, BACK>;
    constexpr int kAhead = BACK ? 1 : 2;
    auto fetch = [&](Item& it) {
        const uint64_t tk = t + group / abreast;
        const uint32_t hd = round * abreast + first;
        it.live = tk < a.tokens && hd < h.heads;
        it.pos = a.rot && it.live ? __ldg(a.pos + (int64_t)k * a.pos_w + (int64_t)tk) : 0;
        const int64_t hx = (int64_t)k * h.xw + (int64_t)tk * h.xt + (int64_t)hd * h.xh;
        const int64_t hg = (int64_t)k * h.dw + (int64_t)tk * h.dt + (int64_t)hd * h.dh;
        it.out = (int64_t)k * h.ow + (int64_t)tk * h.ot + (int64_t)hd * h.oh;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const bool on = it.live && at[s][p] != ~0u;
                raw_zero(it.x[s][p]);
                if (on) raw_load(it.x[s][p], static_cast<const T*>(h.x) + hx + at[s][p]);
                if constexpr (BACK) {
                    raw_zero(it.d[s][p]);
                    if (on) raw_load(it.d[s][p], static_cast<const T*>(h.d) + hg + at[s][p]);
                }
            }
        if (++round == rounds) { round = 0; t += step; }
    };
    auto work = [&](const Item& it) {
        const bool ok = !a.rot || (it.pos >= 0 && (uint64_t)it.pos < a.table_rows);
        const float* ct = a.cos_t + (ok ? (uint64_t)it.pos * half : 0);
        const float* st = a.sin_t + (ok ? (uint64_t)it.pos * half : 0);
        float c[NS][V], sn[NS][V];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint32_t i = (s * a.lanes + sub) * V;                       // first pair of the slot
            if (V > 1 && a.table_wide && i + V <= half && ok && it.live) {
                if constexpr (V > 1) {
#pragma unroll
                    for (int j = 0; j < V; j += 4) { Vec<float, 4>::load(ct + i + j, c[s] + j); Vec<float, 4>::load(st + i + j, sn[s] + j); }
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const bool on = i + j < half && ok && it.live;
                    c[s][j] = on ? __ldg(ct + i + j) : 1.0f;
                    sn[s][j] = on ? __ldg(st + i + j) : 0.0f;
                }
            }
        }
        float x[NS][2][V], d[BACK ? NS : 1][2][V];
        float sq = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                raw_get(it.x[s][p], x[s][p]);
                if constexpr (BACK) raw_get(it.d[s][p], d[s][p]);
#pragma unroll
                for (int j = 0; j < V; ++j) sq = fmaf(x[s][p][j], x[s][p][j], sq);
            }
        for (uint32_t m = a.lanes / 2; m; m >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, m);
        const float r = 1.0f / sqrtf(fmaf(sq, inv_n, a.eps)) + (ok ? 0.0f : __uint_as_float(0x7FFFFFFFu));   // outside the table: NaN
        auto& y = either<BACK>(x, d);
        if constexpr (!BACK) {
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int j = 0; j < V; ++j) x[s][p][j] = x[s][p][j] * r * to_f(w[s][p][j]);
        }
        // forward: (a, b) -> (a c - b s, b c + a s); backward: by the opposite angle
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if (V == 1 || !a.interleaved) {
                if (s * a.lanes + sub < a.pair_slots) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float si = BACK ? -sn[s][j] : sn[s][j], co = c[s][j];
                        const float p0 = y[s][0][j], p1 = y[s][1][j];
                        y[s][0][j] = fmaf(p0, co, -(p1 * si));
                        y[s][1][j] = fmaf(p1, co, p0 * si);
                    }
                }
            } else if constexpr (V > 1) {
#pragma unroll
                for (int j = 0; j < V; ++j) {                                // pair j of the slot: element 2j of its 2V values
                    const float si = BACK ? -sn[s][j] : sn[s][j], co = c[s][j];
                    const float p0 = y[s][2 * j / V][2 * j % V], p1 = y[s][2 * j / V][2 * j % V + 1];
                    y[s][2 * j / V][2 * j % V] = fmaf(p0, co, -(p1 * si));
                    y[s][2 * j / V][2 * j % V + 1] = fmaf(p1, co, p0 * si);
                }
            }
        }
        if constexpr (BACK) {
            float dot = 0.0f;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        x[s][p][j] *= r;                                      // xh
                        acc[s][p][j] = fmaf(d[s][p][j], x[s][p][j], acc[s][p][j]);
                        d[s][p][j] *= to_f(w[s][p][j]);
                        dot = fmaf(d[s][p][j], x[s][p][j], dot);
                    }
            for (uint32_t m = a.lanes / 2; m; m >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, m);
            dot *= inv_n;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int j = 0; j < V; ++j) d[s][p][j] = r * fmaf(-x[s][p][j], dot, d[s][p][j]);
        }
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int p = 0; p < 2; ++p)
                if (it.live && at[s][p] != ~0u) Vec<T, V>::store(static_cast<T*>(h.out) + it.out + at[s][p], y[s][p]);
    };

    // items of this warp: (token groups) * rounds; all lanes walk the same ones
    const uint64_t mine = t < a.tokens ? ((a.tokens - 1 - t) / step + 1) * rounds : 0;
    Item ahead[kAhead];
    uint64_t fetched = 0;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (fetched < mine) { fetch(ahead[i]); ++fetched; }
    for (uint64_t i = 0; i < mine; ++i) {
        const Item cur = ahead[0];
#pragma unroll
        for (int j = 0; j + 1 < kAhead; ++j) ahead[j] = ahead[j + 1];
        if (fetched < mine) { fetch(ahead[kAhead - 1]); ++fetched; }
        work(cur);
    }
    if constexpr (BACK) {
        // the CTA's sum in a fixed order: groups of a warp by a butterfly, then the eight warps one after another
        extern __shared__ float sum[];                                    // [8][head_dim]
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float v = acc[s][p][j];
                    for (uint32_t m = 16; m >= a.lanes; m >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, m);
                    if (group == 0 && at[s][p] != ~0u) sum[warp * a.head_dim + at[s][p] + j] = v;
                }
        __syncthreads();
        float* const part = h.part + ((uint64_t)k * ctas + cta) * a.head_dim;
        for (uint32_t i = threadIdx.x; i < a.head_dim; i += 256) {
            float v = 0.0f;
#pragma unroll
            for (int wi = 0; wi < 8; ++wi) v += sum[wi * a.head_dim + i];
            part[i] = v;
        }
    }
}

struct QkSumArgs {
    const float* part[2];
    void*    dw[2];
    int64_t  dww[2];
    uint32_t parts[2], head_dim;
    uint32_t heads[2];
};

// The CTAs' partial sums of the weight gradients, joined in a fixed order: eight interleaved runs, then those.
template <typename T>
__global__ void __launch_bounds__(256) qk_sum_kernel(const __grid_constant__ QkSumArgs a)
{
    __shared__ float run[8][32];
    const uint32_t side = blockIdx.y, k = blockIdx.z;
    if (a.heads[side] == 0) return;
    const uint32_t i = blockIdx.x * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
    const uint32_t parts = a.parts[side];
    const float* p = a.part[side] + (uint64_t)k * parts * a.head_dim;
    float v = 0.0f;
    if (i < a.head_dim)
        for (uint32_t b = r; b < parts; b += 8) v += p[(uint64_t)b * a.head_dim + i];
    run[r][threadIdx.x & 31] = v;
    __syncthreads();
    if (r == 0 && i < a.head_dim) {
        float t = 0.0f;
#pragma unroll
        for (int b = 0; b < 8; ++b) t += run[b][threadIdx.x & 31];
        static_cast<T*>(a.dw[side])[(int64_t)k * a.dww[side] + i] = from_f<T>(t);
    }
}

}  // namespace block
}  // namespace palsgd
