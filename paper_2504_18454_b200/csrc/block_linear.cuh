// Kernels of the matrix product with bias, activation and residual beside the matrix kernel: calls of few tokens, the
// epilogue of products whose inner axis was cut into shares, and the gradient before the activation with its column sums.
#pragma once
#include "block_matmul.cuh"

namespace palsgd {
namespace block {

struct LinearEnd {                // what follows the sums
    MatOut bias, residual, y, pre, pre_e;                               // p may be NULL but for y's
    int save;
};

// ---------------------------------------------------------------------------------------------- few tokens
//
// Up to eight tokens at a time: bound by reading the weights once (for more tokens, by the multiplications: small calls).  A warp takes four rows of w over its slice of the inner axis, in
// pieces of 16 bytes a lane, and multiplies each with all of the tokens in binary32 (the tokens come from the caches).  A CTA's
// eight warps are `groups` row groups by slices; slices are joined in shared memory in order, and one thread finishes each
// value.  (bfloat16, 8 workers of one token, 2048 -> 5632: 36 us for 185 MB, 28 at the rate of a copy.  The matrix kernel's tile of one token multiplies 255 rows of zeros, and a few outputs give it too few tiles.)
constexpr uint32_t kFewTokens = 8, kFewRows = 4;

struct FewArgs {
    const void *x, *w;
    int64_t  xw, xr, ww, wr;
    uint32_t M, N, D;
    uint32_t groups;              // row groups of a CTA: 8 / groups slices of the inner axis
    uint32_t slice;               // values of a slice: a multiple of a warp's step
    int      act;
    LinearEnd end;
};

template <typename T>
__device__ __forceinline__ float few_act(int kind, float z)             // one value a thread: no copies of the kernel by activation
{
    float slope;
    switch (kind) {
        case PALSGD_ACT_SILU: return act<PALSGD_ACT_SILU, false, sizeof(T) == 2>(z, slope);
        case PALSGD_ACT_GELU: return act<PALSGD_ACT_GELU, false, sizeof(T) == 2>(z, slope);
        case PALSGD_ACT_GELU_TANH: return act<PALSGD_ACT_GELU_TANH, false, sizeof(T) == 2>(z, slope);
        case PALSGD_ACT_RELU: return act<PALSGD_ACT_RELU, false, sizeof(T) == 2>(z, slope);
        default: return z;
    }
}

template <typename T, int MT, bool WIDE>
__global__ void __launch_bounds__(256, MT >= 4 ? 2 : 3) few_kernel(const __grid_constant__ FewArgs a)
{
    constexpr int V = 16 / (int)sizeof(T), H = V / 2, C = kFewRows * MT;
    constexpr uint32_t kStep = 32 * V;
    __shared__ float sums[8][C];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = warp % a.groups, slice = warp / a.groups;
    const int64_t k = blockIdx.y;
    const uint32_t n0 = blockIdx.x * a.groups * kFewRows, m0 = blockIdx.z * MT, M = min(a.M - m0, (uint32_t)MT);
    let_next_start();
    wait_for_previous();
    const T *x = static_cast<const T*>(a.x) + k * a.xw + (int64_t)m0 * a.xr, *w[kFewRows];
#pragma unroll
    for (uint32_t r = 0; r < kFewRows; ++r)               // (rows past the end: the last one, and their sums are not used)
        w[r] = static_cast<const T*>(a.w) + k * a.ww + (int64_t)min(n0 + group * kFewRows + r, a.N - 1) * a.wr;
    f2 acc[kFewRows][MT];
#pragma unroll
    for (uint32_t r = 0; r < kFewRows; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[r][m] = 0;
    auto piece = [&](const T* row, uint32_t c) {
        if constexpr (WIDE) return c < a.D ? __ldg(reinterpret_cast<const uint4*>(row + c)) : make_uint4(0, 0, 0, 0);
        else return get16(reinterpret_cast<const unsigned char*>(row + c), c < a.D ? min(a.D - c, (uint32_t)V) * (uint32_t)sizeof(T) : 0);
    };
    auto widen = [](const uint4& q, f2 (&v)[H]) {
        if constexpr (sizeof(T) == 2) {
            v[0] = f2_wide(q.x); v[1] = f2_wide(q.y); v[2] = f2_wide(q.z); v[3] = f2_wide(q.w);
        } else {
            v[0] = f2_of(__uint_as_float(q.x), __uint_as_float(q.y)); v[1] = f2_of(__uint_as_float(q.z), __uint_as_float(q.w));
        }
    };
    const uint32_t last = min(a.D, (slice + 1) * a.slice);
    constexpr int U = MT == 8 ? 1 : 2;                    // steps whose weights are under way together
    for (uint32_t c0 = slice * a.slice; c0 < last; c0 += U * kStep) {
        uint4 q[U][kFewRows];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (uint32_t r = 0; r < kFewRows; ++r) q[u][r] = c0 + u * kStep < last ? piece(w[r], c0 + u * kStep + lane * V) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t c = c0 + u * kStep + lane * V;
            f2 wv[kFewRows][H];
#pragma unroll
            for (uint32_t r = 0; r < kFewRows; ++r) widen(q[u][r], wv[r]);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                f2 xv[H];
                widen((uint32_t)m < M && c0 + u * kStep < last ? piece(x + (int64_t)m * a.xr, c) : make_uint4(0, 0, 0, 0), xv);
#pragma unroll
                for (uint32_t r = 0; r < kFewRows; ++r)
#pragma unroll
                    for (int i = 0; i < H; ++i) acc[r][m] = f2_fma(wv[r][i], xv[i], acc[r][m]);
            }
        }
    }
    // the lanes' sums: every step halves the values that a lane keeps, until it has one; then the rest of the lanes are added
    float v[C];
#pragma unroll
    for (uint32_t r = 0; r < kFewRows; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float p, q;
            f2_get(acc[r][m], p, q);
            v[r * MT + m] = p + q;
        }
    int d = 16;
#pragma unroll
    for (int h = C / 2; h >= 1; h /= 2, d /= 2)
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const bool upper = lane & d;
            const float send = upper ? v[i] : v[i + h], keep = upper ? v[i + h] : v[i];
            v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, d);
        }
    for (; d; d /= 2) v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], d);
    if (lane % (32 / C) == 0) sums[warp][lane / (32 / C)] = v[0];
    __syncthreads();
    // one thread for each value: column of the CTA's, token
    const uint32_t cols = a.groups * kFewRows, col = threadIdx.x % cols, t = threadIdx.x / cols, m = m0 + t, n = n0 + col;
    const bool on = t < M && n < a.N;
    const LinearEnd& e = a.end;
    float z = 0.0f;
    if (on) {
        const uint32_t at = (col % kFewRows) * MT + t;
        z = sums[col / kFewRows][at];
        for (uint32_t s = 1; s < 8 / a.groups; ++s) z += sums[s * a.groups + col / kFewRows][at];
        if (e.bias.p) z += to_f(static_cast<const T*>(e.bias.p)[k * e.bias.w + n]);
    }
    if (e.save == PALSGD_SAVE_8BIT) {                     // 32 columns a CTA: a warp holds a group of one token
        float top = fabsf(z);
#pragma unroll
        for (int s = 16; s; s >>= 1) top = act8_max(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
        const uint32_t E = act8_exponent(top);
        if (on) {
            static_cast<int8_t*>(e.pre.p)[k * e.pre.w + (int64_t)m * e.pre.r + n] = (int8_t)act8_quant4(z, z, z, z, act8_inverse(E));
            if (lane == 0) static_cast<uint8_t*>(e.pre_e.p)[k * e.pre_e.w + (int64_t)m * e.pre_e.r + n / 32] = (uint8_t)E;
        }
    } else if (e.save == PALSGD_SAVE_FULL && on) {
        static_cast<T*>(e.pre.p)[k * e.pre.w + (int64_t)m * e.pre.r + n] = from_f<T>(z);
    }
    if (!on) return;
    float y = few_act<T>(a.act, z);
    if (e.residual.p) y += to_f(static_cast<const T*>(e.residual.p)[k * e.residual.w + (int64_t)m * e.residual.r + n]);
    static_cast<T*>(e.y.p)[k * e.y.w + (int64_t)m * e.y.r + n] = from_f<T>(y);
}

// ---------------------------------------------------------------------------------------------- shares

// The shares' sums of a product joined in a fixed order, and what follows them.  A thread has eight columns; four threads of
// a warp, 32 (the rows' units are whole groups).
struct LinearJoinArgs {
    const float* part;            // [splits][K][M][ld]
    int64_t  w, share;            // strides of a worker and of a share
    uint32_t splits, ld, M, N;
    uint64_t units;               // of one worker
    Divisor  per_row;             // 4 ceil(N / 32)
    LinearEnd end;
};

template <typename T, int ACT>
__global__ void __launch_bounds__(256) linear_join_kernel(const __grid_constant__ LinearJoinArgs a)
{
    let_next_start();
    wait_for_previous();
    const int64_t k = blockIdx.y;
    const LinearEnd& e = a.end;
    const uint64_t last = (a.units + 255) / 256 * 256;    // (whole warps: a group's threads look at one another)
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < last; i += (uint64_t)gridDim.x * 256) {
        const bool on = i < a.units;
        const uint64_t row = !on ? 0 : a.units < 0x80000000ull ? a.per_row.of((uint32_t)i) : i / a.per_row.d;
        const uint32_t c = on ? (uint32_t)(i - row * a.per_row.d) * 8 : 0, n = on && c < a.N ? min(a.N - c, 8u) : 0;
        f2 z[4] = {0, 0, 0, 0};
        if (n) {                                          // (the shares' rows hold a multiple of eight columns)
            const float* p = a.part + k * a.w + (int64_t)row * a.ld + c;
            row8_load(p, 8, true, z);
            for (uint32_t s = 1; s < a.splits; s += 4) {  // (four loads under way; the order of the sums is fixed)
                f2 v[4][4];
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u) if (s + u < a.splits) row8_load(p + (s + u) * a.share, 8, true, v[u]);
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u)
                    if (s + u < a.splits)
#pragma unroll
                        for (int j = 0; j < 4; ++j) z[j] = f2_add(z[j], v[u][j]);
            }
            if (e.bias.p) {
                f2 b[4];
                row8_load(static_cast<const T*>(e.bias.p) + k * e.bias.w + c, n, e.bias.wide, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) z[j] = f2_add(z[j], b[j]);
            }
        }
        if (e.save == PALSGD_SAVE_8BIT) {
            float v[8], top = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f2_get(z[j], v[2 * j], v[2 * j + 1]);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) if (j < n) top = act8_max(top, v[j]);
            top = act8_max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = act8_max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const uint32_t E = act8_exponent(top);
            const float inv = act8_inverse(E);
            if (n) {
                unsigned char* q = static_cast<unsigned char*>(e.pre.p) + k * e.pre.w + (int64_t)row * e.pre.r + c;
                const uint2 t = make_uint2(act8_quant4(v[0], v[1], v[2], v[3], inv), act8_quant4(v[4], v[5], v[6], v[7], inv));
                if (e.pre.wide && n == 8) *reinterpret_cast<uint2*>(q) = t;
                else put16<1>(q, n, make_uint4(t.x, t.y, 0, 0));
                if (c % 32 == 0) static_cast<uint8_t*>(e.pre_e.p)[k * e.pre_e.w + (int64_t)row * e.pre_e.r + c / 32] = (uint8_t)E;
            }
        } else if (e.save == PALSGD_SAVE_FULL && n) {
            row8_store(static_cast<T*>(e.pre.p) + k * e.pre.w + (int64_t)row * e.pre.r + c, n, e.pre.wide, z);
        }
        if (n == 0) continue;
        f2 unused;
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = linear_act<T, ACT, false>(z[j], unused);
        if (e.residual.p) {
            f2 r[4];
            row8_load(static_cast<const T*>(e.residual.p) + k * e.residual.w + (int64_t)row * e.residual.r + c, n, e.residual.wide, r);
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = f2_add(z[j], r[j]);
        }
        row8_store(static_cast<T*>(e.y.p) + k * e.y.w + (int64_t)row * e.y.r + c, n, e.y.wide, z);
    }
}

// ---------------------------------------------------------------------------------------------- gradient before the activation

// dz = dy act'(z) as the products' operand (bfloat16, or fp32 in three parts; dst NULL: dy itself is the operand), and its
// sums over a CTA's rows, unrounded, to the CTA's row of `part` -- or, where one CTA has all rows, the gradient of the bias
// itself.  `lanes` lanes have a row side by side, eight columns each, and a warp 32 / lanes rows.  Bound by memory; a lane has
// as many rows under way as it has registers for (bfloat16, tanh GELU, 2 x 4096 tokens, 5632 columns: 50 us for 277 MB, 42 at the
// rate of a copy).  The copies of other operands ride along in CTAs of their own.
struct SlopeArgs {
    const void *dy, *pre;         // pre: NULL without an activation
    const uint8_t* pre_e;         // 8 bits
    int64_t  dw, dr, pw, pr, ew, er;
    bf16*    dst;
    int64_t  dstw, ld, dst_part;  // worker, row and part strides
    float*   part;                // [K][row CTAs][part_ld]; NULL: none wanted, or `db` is written
    void*    db;
    int64_t  dbw;
    uint32_t M, N, rows;          // rows of a CTA
    uint32_t lanes, strips, ctas, part_ld;               // CTAs across, CTAs of a worker
    int      dy_wide, pre_wide;
    uint32_t first_copy[kMaxStaged + 1];                  // CTAs of the copies, behind those
};

// Eight values of a row as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<bf16> {
    uint4 q;
    __device__ __forceinline__ void load(const bf16* p, uint32_t n, bool wide) { q = wide && n == 8 ? __ldg(reinterpret_cast<const uint4*>(p)) : get16(reinterpret_cast<const unsigned char*>(p), 2 * n); }
    __device__ __forceinline__ void get(f2 (&v)[4]) const { v[0] = f2_wide(q.x); v[1] = f2_wide(q.y); v[2] = f2_wide(q.z); v[3] = f2_wide(q.w); }
};
template <> struct Raw8<float> {
    f2 r[4];
    __device__ __forceinline__ void load(const float* p, uint32_t n, bool wide) { row8_load(p, n, wide, r); }
    __device__ __forceinline__ void get(f2 (&v)[4]) const { v[0] = r[0]; v[1] = r[1]; v[2] = r[2]; v[3] = r[3]; }
};
struct RawAct8 {
    uint2    q;
    uint32_t e;
    __device__ __forceinline__ void load(const unsigned char* p, const uint8_t* exponent, uint32_t n, bool wide)
    {
        if (wide && n == 8) { q = __ldg(reinterpret_cast<const uint2*>(p)); }
        else { const uint4 t = get16(p, n); q = make_uint2(t.x, t.y); }
        e = n ? *exponent : 127u;
    }
    __device__ __forceinline__ void get(f2 (&v)[4]) const
    {
        const float s = act8_step(e);
        float f[8];
        act8_value4(q.x, s, f);
        act8_value4(q.y, s, f + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = f2_of(f[2 * i], f[2 * i + 1]);
    }
};

template <typename T, int ACT, bool EIGHT>
__global__ void __launch_bounds__(256, 3) slope_kernel(const __grid_constant__ SlopeArgs a, const __grid_constant__ StageArgs copies)
{
    constexpr int U = sizeof(T) == 2 ? 4 : 2;             // rows of a lane under way
    __shared__ float sums[8][256];
    const int64_t k = blockIdx.y;
    let_next_start();
    wait_for_previous();
    if (blockIdx.x >= a.ctas) {
        uint32_t i = 0;
        while (blockIdx.x >= a.first_copy[i + 1]) ++i;
        const uint32_t block = blockIdx.x - a.first_copy[i], blocks = a.first_copy[i + 1] - a.first_copy[i];
        if (copies.item[i].kind == STAGE_BF16) stage_item<2>(copies.item[i], k, block, blocks);   // (rows off the boundaries: two reads a unit)
        else stage_item<4>(copies.item[i], k, block, blocks);
        return;
    }
    const uint32_t chunk = blockIdx.x / a.strips, strip = blockIdx.x - chunk * a.strips;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, abreast = 32 / a.lanes;
    const uint32_t local = (lane % a.lanes) * 8, c = strip * a.lanes * 8 + local;
    const uint32_t n = c < a.N ? min(a.N - c, 8u) : 0;
    const bool room = a.dst && c < a.ld;                  // (the operand's rows hold a multiple of eight columns)
    const uint32_t first = chunk * a.rows, last = min(a.M, first + a.rows), step = 8 * abreast;
    f2 sum[4] = {0, 0, 0, 0};
#pragma unroll 1
    for (uint32_t r0 = first + warp * abreast + lane / a.lanes; r0 < last; r0 += U * step) {
        Raw8<T> dr[U];
        Raw8<T> zr[U];
        RawAct8 qr[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t r = r0 + u * step;
            const uint32_t m = r0 + u * step < last ? n : 0;
            dr[u].load(static_cast<const T*>(a.dy) + k * a.dw + r * a.dr + c, m, a.dy_wide);
            if constexpr (ACT != PALSGD_ACT_NONE) {
                if constexpr (EIGHT) qr[u].load(static_cast<const unsigned char*>(a.pre) + k * a.pw + r * a.pr + c, a.pre_e + k * a.ew + r * a.er + c / 32, m, a.pre_wide);
                else zr[u].load(static_cast<const T*>(a.pre) + k * a.pw + r * a.pr + c, m, a.pre_wide);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r0 + u * step >= last) break;
            f2 d[4], z[4];
            dr[u].get(d);
            if constexpr (ACT != PALSGD_ACT_NONE) {
                if constexpr (EIGHT) qr[u].get(z);
                else zr[u].get(z);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f2 slope;
                    linear_act<T, ACT, true>(z[i], slope);
                    d[i] = f2_mul(d[i], slope);           // (what lies behind the row's end is used nowhere)
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = f2_add(sum[i], d[i]);
            if (room) {
                bf16* to = a.dst + k * a.dstw + (int64_t)(r0 + u * step) * a.ld + c;
                if constexpr (sizeof(T) == 2) {
                    *reinterpret_cast<uint4*>(to) = make_uint4(f2_narrow(d[0]), f2_narrow(d[1]), f2_narrow(d[2]), f2_narrow(d[3]));
                } else {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) f2_get(d[i], v[2 * i], v[2 * i + 1]);
                    three_parts<8>(v, [&](int part, const uint32_t (&w)[4]) { *reinterpret_cast<uint4*>(to + part * a.dst_part) = make_uint4(w[0], w[1], w[2], w[3]); });
                }
            }
        }
    }
    if (!a.part && !a.db) return;
    for (uint32_t d = a.lanes; d < 32; d *= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = f2_add(sum[i], __shfl_xor_sync(0xFFFFFFFFu, sum[i], d));
    if (lane < a.lanes) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x, y;
            f2_get(sum[i], x, y);
            sums[warp][local + 2 * i] = x;
            sums[warp][local + 2 * i + 1] = y;
        }
    }
    __syncthreads();
    const uint32_t at = strip * a.lanes * 8 + threadIdx.x;
    if (threadIdx.x >= a.lanes * 8 || at >= a.N) return;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += sums[i][threadIdx.x];
    if (a.part) a.part[((uint64_t)k * (a.ctas / a.strips) + chunk) * a.part_ld + at] = t;
    else static_cast<T*>(a.db)[k * a.dbw + at] = from_f<T>(t);
}

// ---------------------------------------------------------------------------------------------- few tokens, backward
//
// Up to eight tokens: bound by reading w and writing dw once.  A lane has four columns; it keeps them of every token's x and of
// its sums of dx in registers and walks rows of w: dw's row is a sum over the tokens, dx's sums grow by the row.  Lanes that the
// columns leave over take rows side by side.  A CTA has `rows` rows, whose dz it forms once, in shared memory; the CTAs' sums of
// dx are joined in a fixed order.  All in binary32.
struct FewBackArgs {
    const void *dy, *pre, *x, *w;
    const uint8_t *pre_e, *x_e;   // 8 bits: of pre, of x
    int64_t  dyw, dyr, pw, pr, pew, per, xw, xr, xew, xer, ww, wr;
    MatOut   dx, dw;              // dx: p may be NULL; binary32 sums where there is more than one row CTA
    void*    db;
    int64_t  dbw;
    uint32_t M, N, D, rows, lanes;                       // lanes side by side in a row: 1 .. 256
    int      act, eight, x_wide, w_wide;                  // wide: four values start on a boundary of four
};

// Four values of a row, the first n of them inside it
__device__ __forceinline__ void load4(const float* p, uint32_t n, bool wide, float (&v)[4])
{
    if (wide && n >= 4) {
        const float4 q = __ldg(reinterpret_cast<const float4*>(p));
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = i < n ? __ldg(p + i) : 0.0f;
    }
}
__device__ __forceinline__ void load4(const bf16* p, uint32_t n, bool wide, float (&v)[4])
{
    if (wide && n >= 4) {
        const uint2 q = __ldg(reinterpret_cast<const uint2*>(p));
        v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
        v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = i < n ? to_f(__ldg(p + i)) : 0.0f;
    }
}
// ... of an 8-bit checkpoint (they lie in one group)
__device__ __forceinline__ void load4(const int8_t* p, const uint8_t* e, uint32_t n, bool wide, float (&v)[4])
{
    if (n == 0) {
        v[0] = v[1] = v[2] = v[3] = 0.0f;
        return;
    }
    const float s = act8_step(*e);
    if (wide && n >= 4) {
        act8_value4(__ldg(reinterpret_cast<const uint32_t*>(p)), s, v);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = i < n ? (float)__ldg(p + i) * s : 0.0f;
    }
}
__device__ __forceinline__ void store4(float* p, uint32_t n, bool wide, const float (&v)[4])
{
    if (wide && n >= 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) if (i < n) p[i] = v[i];
}
__device__ __forceinline__ void store4(bf16* p, uint32_t n, bool wide, const float (&v)[4])
{
    if (wide && n >= 4) *reinterpret_cast<uint2*>(p) = make_uint2(f2_narrow(f2_of(v[0], v[1])), f2_narrow(f2_of(v[2], v[3])));
    else
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) if (i < n) p[i] = from_f<bf16>(v[i]);
}

template <typename T>
__device__ __forceinline__ float few_slope(int kind, float z)
{
    float slope = 1.0f;
    switch (kind) {
        case PALSGD_ACT_SILU: act<PALSGD_ACT_SILU, true, sizeof(T) == 2>(z, slope); break;
        case PALSGD_ACT_GELU: act<PALSGD_ACT_GELU, true, sizeof(T) == 2>(z, slope); break;
        case PALSGD_ACT_GELU_TANH: act<PALSGD_ACT_GELU_TANH, true, sizeof(T) == 2>(z, slope); break;
        case PALSGD_ACT_RELU: act<PALSGD_ACT_RELU, true, sizeof(T) == 2>(z, slope); break;
        default: break;
    }
    return slope;
}

// Four values as they lie in memory
template <typename T> struct Raw4;
template <> struct Raw4<bf16> {
    uint2 q;
    __device__ __forceinline__ void load(const bf16* p, uint32_t n, bool wide)
    {
        if (wide && n >= 4) { q = __ldg(reinterpret_cast<const uint2*>(p)); return; }
        uint32_t h[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) h[i] = i < n ? __ldg(reinterpret_cast<const unsigned short*>(p) + i) : 0;
        q = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    }
    __device__ __forceinline__ void get(f2& a, f2& b) const { a = f2_wide(q.x); b = f2_wide(q.y); }
};
template <> struct Raw4<float> {
    float v[4];
    __device__ __forceinline__ void load(const float* p, uint32_t n, bool wide) { load4(p, n, wide, v); }
    __device__ __forceinline__ void get(f2& a, f2& b) const { a = f2_of(v[0], v[1]); b = f2_of(v[2], v[3]); }
};

constexpr uint32_t kFewBackRows = 256;                    // of a CTA, at most

template <typename T, int MT>
__global__ void __launch_bounds__(256, MT == 8 ? 2 : 3) few_backward_kernel(const __grid_constant__ FewBackArgs a)
{
    constexpr int U = sizeof(T) == 2 && MT < 8 ? 4 : 2;   // rows of w at a time; as many more under way
    __shared__ __align__(16) float dz[kFewBackRows][MT];
    __shared__ float joined[256][4 * MT + 1];
    const uint32_t tid = threadIdx.x, side = 256 / a.lanes, group = tid / a.lanes, d = (blockIdx.x * a.lanes + tid % a.lanes) * 4;
    const uint32_t n0 = blockIdx.y * a.rows, rows = min(a.rows, a.N - n0), in = d < a.D ? min(a.D - d, 4u) : 0;
    const int64_t k = blockIdx.z;
    let_next_start();
    wait_for_previous();
    const T* w = static_cast<const T*>(a.w) + k * a.ww + (int64_t)n0 * a.wr + d;
    T* dw = static_cast<T*>(a.dw.p) + k * a.dw.w + (int64_t)n0 * a.dw.r + d;
    Raw4<T> raw[U], next[U];
    auto fetch = [&](uint32_t r0, Raw4<T> (&to)[U]) {
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) to[u].load(w + (int64_t)(r0 + u * side) * a.wr, a.dx.p && r0 + u * side < rows ? in : 0, a.w_wide);
    };
    fetch(group, raw);
    f2 x[MT][2], acc[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        float v[4];
        const uint32_t there = (uint32_t)m < a.M ? in : 0;
        if (a.x_e) load4(static_cast<const int8_t*>(a.x) + k * a.xw + m * a.xr + d, a.x_e + k * a.xew + m * a.xer + d / 32, there, a.x_wide, v);
        else load4(static_cast<const T*>(a.x) + k * a.xw + m * a.xr + d, there, a.x_wide, v);
        x[m][0] = f2_of(v[0], v[1]); x[m][1] = f2_of(v[2], v[3]);
        acc[m][0] = acc[m][1] = 0;
    }
    for (uint32_t i = tid; i < rows * MT; i += 256) {
        const uint32_t m = i / rows, r = i - m * rows, n = n0 + r;       // (lanes side by side: columns)
        float v = 0.0f;
        if (m < a.M) {
            v = to_f(static_cast<const T*>(a.dy)[k * a.dyw + m * a.dyr + n]);
            if (a.act != PALSGD_ACT_NONE) {
                float z;
                if (a.eight) z = (float)static_cast<const int8_t*>(a.pre)[k * a.pw + m * a.pr + n] * act8_step(a.pre_e[k * a.pew + m * a.per + n / 32]);
                else z = to_f(static_cast<const T*>(a.pre)[k * a.pw + m * a.pr + n]);
                v *= few_slope<T>(a.act, z);
            }
        }
        dz[r][m] = v;
    }
    __syncthreads();
    if (a.db && blockIdx.x == 0 && tid < rows) {
        float t = 0.0f;
#pragma unroll
        for (int m = 0; m < MT; ++m) t += dz[tid][m];
        static_cast<T*>(a.db)[k * a.dbw + n0 + tid] = from_f<T>(t);
    }
    for (uint32_t r0 = group; r0 < rows; r0 += U * side) {
        fetch(r0 + U * side, next);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint32_t r = r0 + u * side;
            if (r >= rows) break;
            f2 w0, w1, s0 = 0, s1 = 0;
            raw[u].get(w0, w1);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const f2 g = f2_same(dz[r][m]);
                s0 = f2_fma(g, x[m][0], s0); s1 = f2_fma(g, x[m][1], s1);
                acc[m][0] = f2_fma(g, w0, acc[m][0]); acc[m][1] = f2_fma(g, w1, acc[m][1]);
            }
            float o[4];
            f2_get(s0, o[0], o[1]); f2_get(s1, o[2], o[3]);
            store4(dw + (int64_t)r * a.dw.r, in, a.dw.wide, o);
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) raw[u] = next[u];
    }
    if (!a.dx.p) return;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        f2_get(acc[m][0], joined[tid][4 * m], joined[tid][4 * m + 1]);
        f2_get(acc[m][1], joined[tid][4 * m + 2], joined[tid][4 * m + 3]);
    }
    __syncthreads();
    // the side-by-side rows' sums, in order: a thread for each token and column
    for (uint32_t i = tid; i < a.lanes * 4 * a.M; i += 256) {
        const uint32_t m = i / (a.lanes * 4), c = i - m * a.lanes * 4, at = blockIdx.x * a.lanes * 4 + c;
        float t = 0.0f;
        for (uint32_t g = 0; g < side; ++g) t += joined[g * a.lanes + c / 4][4 * m + c % 4];
        if (at >= a.D) continue;
        const int64_t to = k * a.dx.w + m * a.dx.r + at;
        if (gridDim.y > 1) static_cast<float*>(a.dx.p)[blockIdx.y * a.dx.part + to] = t;
        else static_cast<T*>(a.dx.p)[to] = from_f<T>(t);
    }
}

}  // namespace block
}  // namespace palsgd
