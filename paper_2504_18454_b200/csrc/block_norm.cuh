// Row kernels of the block operators: layer norm forward and backward.
//
// A team of lanes -- 4 to 32 of a warp, or up to 32 warps -- has a row at a time in its registers: mean, then the mean square
// around it (two passes over registers: a row whose mean is large against its spread loses what the mean is rounded by, not
// the digits that a difference of squares would), then the result, in one pass over memory.  A team walks rows with the next
// ones under way; its columns of w (and b), and in the backward pass its sums of dw and db, stay in registers over all of its
// rows.  The sums go to one row of the workspace for each CTA and are joined in a fixed order; where one CTA has all of a
// worker's rows it writes the gradients itself.
// Bound by memory: every byte is moved once.  (bfloat16, 2 x 16384 rows of 2048, with an addend: forward 100 us, backward 92 and
// 8 for the join of its sums; 537 MB each, 82 us at the rate of a copy.  fp32: forward 196, backward with the join 163, 164 at that
// rate.  bfloat16, rows of 2001: 192 and 215, bound by the instructions that shift pieces into place.)
#pragma once
#include "block_common.cuh"

namespace palsgd {
namespace block {

struct NormArgs {
    const void *x, *r;            // forward: input and what is added to it (may be NULL); backward: the sum, and the gradient past the norm
    const void *w, *b, *dy;
    void *y, *total;              // backward: y is dx
    float *mean, *rstd;           // forward: may be NULL
    float* part;                  // backward: [K][CTAs][part_ld >= 2 width]; NULL: the gradients themselves are written
    void  *dw_out, *db_out;
    int64_t dwo, dbo;
    int64_t xw, xr, rw, rr, dw, dr, yw, yr, tw, tr, ww, bw, mw, sw;      // worker and row strides, elements
    uint64_t rows;
    uint32_t width, lanes;        // lanes of a team: 4 .. 1024
    uint32_t part_ld;             // a row of `part`
    float    eps;
};

// A piece is 16 bytes of a row, V values.
template <typename T> constexpr int kPieceValues = 16 / (int)sizeof(T);

template <typename T, bool WIDE>
__device__ __forceinline__ uint4 piece_load(const T* row, uint32_t c, uint32_t width)
{
    if constexpr (WIDE) {
        return c < width ? __ldg(reinterpret_cast<const uint4*>(row + c)) : make_uint4(0, 0, 0, 0);
    } else {
        const uint32_t n = c < width ? min(width - c, (uint32_t)kPieceValues<T>) : 0;
        return get16(reinterpret_cast<const unsigned char*>(row + c), n * (uint32_t)sizeof(T));
    }
}

// Pieces on their way: every lane copies its own pieces of the rows to come into places of its own in shared memory,
// asynchronously, and reads them there: no barrier, and registers for one row only.  (The next row in registers took 200 of
// them a lane in the backward pass, which left eight warps an SM and 24 KB under way.)  Rows at any address come as the
// aligned 16-byte blocks that hold a byte of them: a lane's piece lies in its block and the next lane's (the team's last lane
// of a warp fetches one more).
template <typename T, bool WIDE, int N>
struct Ring {
    static constexpr uint32_t kPlaces = WIDE ? 32 : N == 1 ? 40 : 33;    // of 16 bytes: a warp's for one piece a lane
    uint32_t base, step;
    bool     last;                // the team's last lane of the warp
    __device__ __forceinline__ Ring(const void* raw, uint32_t lanes)
    {
        const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, of_warp = min(lanes, 32u);
        last = lane % of_warp == of_warp - 1;
        base = (uint32_t)__cvta_generic_to_shared(raw) + (warp * kPlaces + lane + (WIDE ? 0 : lane / of_warp)) * 16;
        step = (blockDim.x >> 5) * kPlaces * 16;
    }
    static __device__ __forceinline__ void copy(uint32_t to, const void* from, bool on)
    {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(on ? 16u : 0u) : "memory");
    }
    // piece c of a row into place i
    __device__ __forceinline__ void fetch(uint32_t i, const T* row, uint32_t c, uint32_t width) const
    {
        const uint32_t to = base + i * step;
        if constexpr (WIDE) {
            copy(to, row + (c < width ? c : 0), c < width);
        } else {
            const uintptr_t start = reinterpret_cast<uintptr_t>(row) & ~(uintptr_t)15, end = reinterpret_cast<uintptr_t>(row + width);
            const uintptr_t block = reinterpret_cast<uintptr_t>(row + c) & ~(uintptr_t)15;
            copy(to, reinterpret_cast<const void*>(block < end ? block : start), block < end);
            if (last) copy(to + 16, reinterpret_cast<const void*>(block + 16 < end ? block + 16 : start), block + 16 < end);
        }
    }
    __device__ __forceinline__ uint4 get(uint32_t i, const T* row, uint32_t c, uint32_t width) const
    {
        uint4 v;
        lds(base + i * step, v);
        if constexpr (!WIDE) {
            uint4 u;
            lds(base + i * step + 16, u);
            const uint32_t n = c < width ? min(width - c, (uint32_t)kPieceValues<T>) * (uint32_t)sizeof(T) : 0;
            v = shift16(v, u, (uint32_t)reinterpret_cast<uintptr_t>(row + c) & 15, n);
        }
        return v;
    }
    static __device__ __forceinline__ void lds(uint32_t at, uint4& v)
    {
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    }
    static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    // All but the last AHEAD rows are there.  (A lane's copies are complete for it alone: the others look behind the barrier.)
    template <int AHEAD>
    static __device__ __forceinline__ void wait()
    {
        asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
        if constexpr (!WIDE) __syncwarp();
    }
    // Every lane has read what the next copies write over.
    static __device__ __forceinline__ void left() { if constexpr (!WIDE) __syncwarp(); }
};
// Rows under way: as many as find room beside the SM's other CTAs, four at most.
template <typename T, bool WIDE, int N>
constexpr __host__ __device__ uint32_t norm_stage_bytes(int arrays, int warps) { return (uint32_t)(arrays * N) * warps * Ring<T, WIDE, N>::kPlaces * 16; }
template <typename T, bool WIDE, int N>
constexpr __host__ __device__ uint32_t norm_stages(int arrays, int warps, int ctas)
{
    const uint32_t n = (227 * 1024 / ctas - 2048) / norm_stage_bytes<T, WIDE, N>(arrays, warps);
    return n > 4 ? 4 : n;
}

template <typename T, bool WIDE>
__device__ __forceinline__ void piece_store(T* row, uint32_t c, uint32_t width, const uint4& v)
{
    if (c >= width) return;
    if constexpr (WIDE) *reinterpret_cast<uint4*>(row + c) = v;
    else put16<(int)sizeof(T)>(reinterpret_cast<unsigned char*>(row + c), min(width - c, (uint32_t)kPieceValues<T>) * (uint32_t)sizeof(T), v);
}
// A piece as V / 2 pairs of floats, and back
template <typename T>
__device__ __forceinline__ void piece_wide(const uint4& p, f2 (&v)[kPieceValues<T> / 2])
{
    if constexpr (sizeof(T) == 2) {
        v[0] = f2_wide(p.x); v[1] = f2_wide(p.y); v[2] = f2_wide(p.z); v[3] = f2_wide(p.w);
    } else {
        v[0] = f2_of(__uint_as_float(p.x), __uint_as_float(p.y)); v[1] = f2_of(__uint_as_float(p.z), __uint_as_float(p.w));
    }
}
template <typename T>
__device__ __forceinline__ uint4 piece_narrow(const f2 (&v)[kPieceValues<T> / 2])
{
    if constexpr (sizeof(T) == 2) {
        return make_uint4(f2_narrow(v[0]), f2_narrow(v[1]), f2_narrow(v[2]), f2_narrow(v[3]));
    } else {
        float a, b, c, d;
        f2_get(v[0], a, b); f2_get(v[1], c, d);
        return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
    }
}
// The pair at column c with what lies behind the row's end as zero
template <bool WIDE>
__device__ __forceinline__ f2 inside(f2 v, uint32_t c, uint32_t width)
{
    if (c + 1 < width) return v;
    if (WIDE || c >= width) return 0;
    float a, b;
    f2_get(v, a, b);
    return f2_of(a, 0.0f);
}

constexpr uint32_t kNormMostWarps = 32;                                 // of a team

// Sums of N values over a team, the same bits in all of its lanes.  `turn` alternates between calls: the places of one call
// are read while the next one's are written.
template <int N>
__device__ __forceinline__ void team_sum(float (&v)[N], uint32_t lanes, uint32_t team, float* places, uint32_t& turn)
{
    if (lanes >= 32) {
#pragma unroll
        for (int d = 16; d; d >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], d);
    } else {
        for (uint32_t d = lanes / 2; d; d >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], d);
    }
    if (lanes <= 32) return;
    const uint32_t warps = lanes / 32, warp = threadIdx.x >> 5, first = team * warps;
    float* p = places + turn * (2 * kNormMostWarps);
    turn ^= 1;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) p[i * kNormMostWarps + warp] = v[i];
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(lanes) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float* q = p + i * kNormMostWarps + first;
        if (warps == 2) {
            const float2 t = *reinterpret_cast<const float2*>(q);
            v[i] = t.x + t.y;
        } else {                                          // (a team's first warp is a multiple of its warps)
            float s = 0.0f;
            for (uint32_t j = 0; j < warps; j += 4) {
                const float4 t = *reinterpret_cast<const float4*>(q + j);
                s += (t.x + t.y) + (t.z + t.w);
            }
            v[i] = s;
        }
    }
}

// 1 / sqrt(v) to about a unit in the last place: the unit's approximation and one step of Newton's method.  (0 and infinity
// stay what they are: the step would make a NaN of them.)
__device__ __forceinline__ float inverse_root(float v)
{
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    const float e = fmaf(-v * r, r, 1.0f);
    const float better = fmaf(0.5f * r, e, r);
    return v > 1e-37f && v < 1e37f ? better : 1.0f / sqrtf(v);
}

// WARPS: of a CTA, 8 or as many as one team needs beyond that.  N: pieces a lane.  ADD: there is an addend (forward), a
// gradient that comes past the norm (backward).
template <typename T, int N, bool WIDE, bool ADD, int WARPS, int CTAS>
__global__ void __launch_bounds__(32 * WARPS, CTAS) norm_forward_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int V = kPieceValues<T>, H = V / 2, Q = ADD ? 2 * N : N, S = norm_stages<T, WIDE, N>(Q / N, WARPS, CTAS);    // Q: pieces of a lane for a row
    __shared__ __align__(16) float places[4 * kNormMostWarps];
    extern __shared__ __align__(16) unsigned char ring_raw[];
    const uint32_t team = threadIdx.x / a.lanes, teams = blockDim.x / a.lanes;
    const uint32_t first = (threadIdx.x - team * a.lanes) * V, step = a.lanes * V, width = a.width;
    const uint32_t beside = N == 1 && a.lanes < 32 ? team % (32 / a.lanes) : 0;    // teams of the warp before this one: a warp's teams go on together
    const Ring<T, WIDE, N> ring(ring_raw, a.lanes);
    const int64_t k = blockIdx.y;
    const T *w = static_cast<const T*>(a.w) + k * a.ww, *b = static_cast<const T*>(a.b) + k * a.bw;
    const uint64_t rows_step = (uint64_t)gridDim.x * teams;
    uint64_t row = (uint64_t)blockIdx.x * teams + team, ahead = row;
    uint32_t turn = 0, put = 0, got = 0;
    // the rows that a team is at, and comes to next
    const T *x = static_cast<const T*>(a.x) + k * a.xw + (int64_t)row * a.xr, *r = static_cast<const T*>(a.r) + (ADD ? k * a.rw + (int64_t)row * a.rr : 0);
    const T *x_next = x, *r_next = r;
    T* y = static_cast<T*>(a.y) + k * a.yw + (int64_t)row * a.yr;
    T* total = static_cast<T*>(a.total) + (ADD ? k * a.tw + (int64_t)row * a.tr : 0);
    const int64_t x_step = (int64_t)rows_step * a.xr, r_step = (int64_t)rows_step * a.rr, y_step = (int64_t)rows_step * a.yr, t_step = (int64_t)rows_step * a.tr;
    const float inv_width = 1.0f / (float)width;

    let_next_start();
    wait_for_previous();
    auto fetch = [&]() {
        if (ahead < a.rows) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ring.fetch(put * Q + i, x_next, first + i * step, width);
                if constexpr (ADD) ring.fetch(put * Q + N + i, r_next, first + i * step, width);
            }
            ahead += rows_step;
            x_next += x_step;
            if constexpr (ADD) r_next += r_step;
        }
        ring.commit();
        put = put + 1 == S ? 0 : put + 1;
    };
#pragma unroll 1
    for (int i = 0; i < S - 1; ++i) fetch();
    uint4 wp[N], bp[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        wp[i] = piece_load<T, WIDE>(w, first + i * step, width);
        bp[i] = piece_load<T, WIDE>(b, first + i * step, width);
    }
    for (; row - beside < a.rows; row += rows_step) {
        const bool on = N > 1 || row < a.rows;            // (narrow rows: one piece a lane)
        ring.left();
        fetch();                                          // into the place that the row before this one has left
        ring.template wait<S - 1>();
        f2 h[N][H], sum = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            piece_wide<T>(ring.get(got * Q + i, x, first + i * step, width), h[i]);
            if constexpr (ADD) {
                f2 t[H];
                piece_wide<T>(ring.get(got * Q + N + i, r, first + i * step, width), t);
#pragma unroll
                for (int j = 0; j < H; ++j) h[i][j] = f2_add(h[i][j], t[j]);
            }
#pragma unroll
            for (int j = 0; j < H; ++j) sum = f2_add(sum, h[i][j]);      // (behind the row's end: zeros)
        }
        got = got + 1 == S ? 0 : got + 1;
        if constexpr (ADD) {
#pragma unroll
            for (int i = 0; i < N; ++i) piece_store<T, WIDE>(total, first + i * step, on ? width : 0, piece_narrow<T>(h[i]));
            total += t_step;
        }
        float s[1] = {f2_total(sum)};
        team_sum<1>(s, a.lanes, team, places, turn);
        const float mean = s[0] * inv_width;
        sum = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t c = first + i * step;
            const f2 shift = f2_same(c < width ? -mean : 0.0f);          // (a piece behind the row's end stays zero)
#pragma unroll
            for (int j = 0; j < H; ++j) h[i][j] = f2_add(h[i][j], shift);
            if (!WIDE && c + V > width)
#pragma unroll
                for (int j = 0; j < H; ++j) h[i][j] = inside<WIDE>(h[i][j], c + 2 * j, width);
#pragma unroll
            for (int j = 0; j < H; ++j) sum = f2_fma(h[i][j], h[i][j], sum);
        }
        s[0] = f2_total(sum);
        team_sum<1>(s, a.lanes, team, places, turn);
        const float rstd = inverse_root(fmaf(s[0], inv_width, a.eps));
#pragma unroll
        for (int i = 0; i < N; ++i) {
            f2 wv[H], bv[H];
            piece_wide<T>(wp[i], wv);
            piece_wide<T>(bp[i], bv);
#pragma unroll
            for (int j = 0; j < H; ++j) bv[j] = f2_fma(f2_mul(h[i][j], f2_same(rstd)), wv[j], bv[j]);
            piece_store<T, WIDE>(y, first + i * step, on ? width : 0, piece_narrow<T>(bv));
        }
        if (first == 0 && on) {
            if (a.mean) a.mean[k * a.mw + (int64_t)row] = mean;
            if (a.rstd) a.rstd[k * a.sw + (int64_t)row] = rstd;
        }
        if constexpr (!WIDE) x += x_step;                 // (of an aligned row nothing but its place in shared memory counts)
        if constexpr (!WIDE && ADD) r += r_step;
        y += y_step;
    }
}

// dx = rstd (g - mean g - xh mean(g xh)) (+ what comes past the norm), g = dy w, xh = (x - mean) rstd; the CTA's sums of
// dy xh and dy go to its row of `part`.
template <typename T, int N, bool WIDE, bool ADD, int WARPS, int CTAS>
__global__ void __launch_bounds__(32 * WARPS, CTAS) norm_backward_kernel(const __grid_constant__ NormArgs a)
{
    constexpr bool kKeep = WARPS < 32;                    // the widest kernel forms xh and g twice: they would not fit its registers
    constexpr int V = kPieceValues<T>, H = V / 2, Q = ADD ? 3 * N : 2 * N, S = norm_stages<T, WIDE, N>(Q / N, WARPS, CTAS);
    __shared__ __align__(16) float places[4 * kNormMostWarps];
    extern __shared__ __align__(16) unsigned char ring_raw[];            // the ring; at the end [2][width] floats, where a CTA has more than one team
    const uint32_t team = threadIdx.x / a.lanes, teams = blockDim.x / a.lanes;
    const uint32_t first = (threadIdx.x - team * a.lanes) * V, step = a.lanes * V, width = a.width;
    const uint32_t beside = N == 1 && a.lanes < 32 ? team % (32 / a.lanes) : 0;    // teams of the warp before this one: a warp's teams go on together
    const Ring<T, WIDE, N> ring(ring_raw, a.lanes);
    const int64_t k = blockIdx.y;
    const T* w = static_cast<const T*>(a.w) + k * a.ww;
    const uint64_t rows_step = (uint64_t)gridDim.x * teams;
    uint64_t row = (uint64_t)blockIdx.x * teams + team, ahead = row;
    uint32_t turn = 0, put = 0, got = 0;
    const T* x = static_cast<const T*>(a.x) + k * a.xw + (int64_t)row * a.xr;
    const T* dy = static_cast<const T*>(a.dy) + k * a.dw + (int64_t)row * a.dr;
    const T* r = static_cast<const T*>(a.r) + (ADD ? k * a.rw + (int64_t)row * a.rr : 0);
    const T *x_next = x, *dy_next = dy, *r_next = r;
    T* dx = static_cast<T*>(a.y) + k * a.yw + (int64_t)row * a.yr;
    const int64_t x_step = (int64_t)rows_step * a.xr, d_step = (int64_t)rows_step * a.dr, r_step = (int64_t)rows_step * a.rr, y_step = (int64_t)rows_step * a.yr;
    const float inv_width = 1.0f / (float)width;

    let_next_start();
    wait_for_previous();
    auto fetch = [&]() {
        const bool more = ahead < a.rows;
        if (more || N == 1) {                             // (narrow rows, behind the last one: zeros, for the sums of a warp's other teams)
            const uint32_t some = N > 1 || more ? width : 0;
            if (N == 1 && !more) { x_next = static_cast<const T*>(a.x); dy_next = static_cast<const T*>(a.dy); r_next = static_cast<const T*>(a.r); }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ring.fetch(put * Q + i, x_next, first + i * step, some);
                ring.fetch(put * Q + N + i, dy_next, first + i * step, some);
                if constexpr (ADD) ring.fetch(put * Q + 2 * N + i, r_next, first + i * step, some);
            }
            ahead += rows_step;
            x_next += x_step;
            dy_next += d_step;
            if constexpr (ADD) r_next += r_step;
        }
        ring.commit();
        put = put + 1 == S ? 0 : put + 1;
    };
#pragma unroll 1
    for (int i = 0; i < S - 1; ++i) fetch();
    uint4 wp[N];
    f2 dw[N][H], db[N][H];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        wp[i] = piece_load<T, WIDE>(w, first + i * step, width);
#pragma unroll
        for (int j = 0; j < H; ++j) dw[i][j] = db[i][j] = 0;
    }
    float mean = 0.0f, rstd = 0.0f;
    const float *means = a.mean + k * a.mw, *rstds = a.rstd + k * a.sw;
    auto stats = [&](uint64_t at) {
        if (at >= a.rows) return;
        mean = __ldg(means + at);
        rstd = __ldg(rstds + at);
    };
    stats(row);
    for (; row - beside < a.rows; row += rows_step) {
        const bool on = N > 1 || row < a.rows;            // (narrow rows: one piece a lane)
        const float rs = rstd, mean_now = mean;
        stats(row + rows_step);
        ring.left();
        fetch();
        ring.template wait<S - 1>();
        const uint32_t some = on ? width : 0;
        // a piece's xh, d and g = d w.  (Behind the row's end d is zero, and xh has to be finite where it goes into the sums
        // of columns that are there: a piece cut by the end, and a team without a row.)
        auto load = [&](int i, f2 (&xh)[H], f2 (&d)[H], f2 (&g)[H]) {
            f2 wv[H];
            piece_wide<T>(ring.get(got * Q + i, x, first + i * step, some), xh);
            piece_wide<T>(ring.get(got * Q + N + i, dy, first + i * step, some), d);
            piece_wide<T>(wp[i], wv);
#pragma unroll
            for (int j = 0; j < H; ++j) {
                xh[j] = f2_mul(f2_add(xh[j], f2_same(-mean_now)), f2_same(rs));
                if ((!WIDE || N == 1) && first + i * step + V > some) xh[j] = inside<WIDE>(xh[j], first + i * step + 2 * j, some);
                g[j] = f2_mul(d[j], wv[j]);
            }
        };
        f2 xh[kKeep ? N : 1][H], g[kKeep ? N : 1][H], sg = 0, sx = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            f2 (&xi)[H] = xh[kKeep ? i : 0], (&gi)[H] = g[kKeep ? i : 0], d[H];
            load(i, xi, d, gi);
#pragma unroll
            for (int j = 0; j < H; ++j) {
                dw[i][j] = f2_fma(d[j], xi[j], dw[i][j]);
                db[i][j] = f2_add(db[i][j], d[j]);
                sg = f2_add(sg, gi[j]);
                sx = f2_fma(gi[j], xi[j], sx);
            }
        }
        float s[2] = {f2_total(sg), f2_total(sx)};
        team_sum<2>(s, a.lanes, team, places, turn);
        const f2 mg = f2_same(-s[0] * inv_width), mx = f2_same(-s[1] * inv_width);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            f2 t[H], (&xi)[H] = xh[kKeep ? i : 0], (&gi)[H] = g[kKeep ? i : 0];
            if constexpr (!kKeep) load(i, xi, t, gi);
            if constexpr (ADD) piece_wide<T>(ring.get(got * Q + 2 * N + i, r, first + i * step, some), t);
#pragma unroll
            for (int j = 0; j < H; ++j) {
                const f2 v = f2_add(f2_fma(xi[j], mx, gi[j]), mg);
                t[j] = ADD ? f2_fma(v, f2_same(rs), t[j]) : f2_mul(v, f2_same(rs));
            }
            piece_store<T, WIDE>(dx, first + i * step, some, piece_narrow<T>(t));
        }
        got = got + 1 == S ? 0 : got + 1;
        if constexpr (!WIDE) { x += x_step; dy += d_step; }
        if constexpr (!WIDE && ADD) r += r_step;
        dx += y_step;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();                                      // the ring's place is free
    float* const joined = reinterpret_cast<float*>(ring_raw);
    float* const part = a.part ? a.part + ((uint64_t)k * gridDim.x + blockIdx.x) * a.part_ld : nullptr;
    auto put_sum = [&](uint32_t which, uint32_t c, float v) {
        if (part) part[which * width + c] = v;
        else if (which) static_cast<T*>(a.db_out)[k * a.dbo + c] = from_f<T>(v);
        else static_cast<T*>(a.dw_out)[k * a.dwo + c] = from_f<T>(v);
    };
    auto each = [&](auto&& f) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < H; ++j) {
                const uint32_t c = first + i * step + 2 * j;
                float u, v, p, q;
                f2_get(dw[i][j], u, v);
                f2_get(db[i][j], p, q);
                if (c < width) f(c, u, p);
                if (c + 1 < width) f(c + 1, v, q);
            }
    };
    // the teams of a warp, then those of the CTA, one after another
    for (uint32_t d = a.lanes; d < 32; d *= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < H; ++j) {
                dw[i][j] = f2_add(dw[i][j], __shfl_xor_sync(0xFFFFFFFFu, dw[i][j], d));
                db[i][j] = f2_add(db[i][j], __shfl_xor_sync(0xFFFFFFFFu, db[i][j], d));
            }
    if (teams == 1) {
        each([&](uint32_t c, float u, float p) { put_sum(0, c, u); put_sum(1, c, p); });
        return;
    }
    const uint32_t turns = a.lanes <= 32 ? WARPS : teams, mine = a.lanes <= 32 ? threadIdx.x >> 5 : team;
    for (uint32_t t = 0; t < turns; ++t) {
        if (t == mine && beside == 0) {
            if (t == 0) each([&](uint32_t c, float u, float p) { joined[c] = u; joined[width + c] = p; });
            else each([&](uint32_t c, float u, float p) { joined[c] += u; joined[width + c] += p; });
        }
        __syncthreads();
    }
    for (uint32_t c = threadIdx.x; c < width; c += blockDim.x) { put_sum(0, c, joined[c]); put_sum(1, c, joined[width + c]); }
}

}  // namespace block
}  // namespace palsgd
