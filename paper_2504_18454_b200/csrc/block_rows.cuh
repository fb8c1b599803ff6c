// Row kernels of the block operators: 8-bit checkpoints, and the norm of queries and keys with the position rotation.
// Both move every byte once.  Checkpoints run at the copy rate (pack and unpack of 32768 x 5632 bfloat16: 168-173 us, 6.5-6.7
// TB/s); norm and rotation at 70-85 % of it, held by the latencies and instructions of a reduction for each head (8 workers,
// 2048 tokens, 12 + 12 heads of 64: forward 20.4-21.6 us, backward 33; 2 of 32768, 16 + 4 of 128: backward 190-199, 5.1-5.3 TB/s).
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
    uint64_t units;               // rows * (pieces of eight values of a row, padded to whole groups)
    Divisor  per_row;             // those pieces (units < 2^31)
};

// Eight int8 at any address, `n` of them inside the row: as get16 and put16.
__device__ __forceinline__ uint2 loose_load(const int8_t* p, uint32_t n)
{
    const uint32_t o = (uint32_t)reinterpret_cast<uintptr_t>(p) & 7;
    const uint2* base = reinterpret_cast<const uint2*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)7);
    const uint2 a = n ? __ldg(base) : make_uint2(0, 0), b = n && o + n > 8 ? __ldg(base + 1) : make_uint2(0, 0);
    const uint32_t s = 8 * (o & 3);
    const uint32_t w0 = o & 4 ? a.y : a.x, w1 = o & 4 ? b.x : a.y, w2 = o & 4 ? b.y : b.x;
    return make_uint2(__funnelshift_r(w0, w1, s), __funnelshift_r(w1, w2, s));
}
__device__ __forceinline__ void loose_store(int8_t* p, uint32_t n, uint2 w)
{
    const uint32_t o = (uint32_t)reinterpret_cast<uintptr_t>(p) & 7;
    if (n == 8 && o == 0) {
        *reinterpret_cast<uint2*>(p) = w;
    } else if (n == 8 && (o & 3) == 0) {
        reinterpret_cast<uint32_t*>(p)[0] = w.x; reinterpret_cast<uint32_t*>(p)[1] = w.y;
    } else if (n == 8 && (o & 1) == 0) {
        uint16_t* h = reinterpret_cast<uint16_t*>(p);
        h[0] = (uint16_t)w.x; h[1] = (uint16_t)(w.x >> 16); h[2] = (uint16_t)w.y; h[3] = (uint16_t)(w.y >> 16);
    } else if (n == 8) {
        uint16_t* h = reinterpret_cast<uint16_t*>(p + 1);
        p[0] = (int8_t)w.x; h[0] = (uint16_t)(w.x >> 8); h[1] = (uint16_t)__byte_perm(w.x, w.y, 0x0043); h[2] = (uint16_t)(w.y >> 8); p[7] = (int8_t)(w.y >> 24);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) if (j < n) p[j] = (int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    }
}
// A unit is eight consecutive values (four lanes share a group) and a thread takes U units 256 apart.  All of a thread's
// reads are under way before it works on the first; a CTA does this once and makes room for the next.
// FLAT: one long row; WIDE: rows on 16-byte (q: 8-byte) boundaries and of whole units; LOOSE: any.  One value a lane in
// place of LOOSE took 667 us to pack 32768 rows of 5633 bfloat16 where this takes 200 (5632: FLAT, 81 us, 6.9 TB/s).
enum { ACT8_FLAT = 0, ACT8_WIDE = 1, ACT8_LOOSE = 2 };
template <typename T, bool PACK, int LAYOUT>
__global__ void __launch_bounds__(256, LAYOUT == ACT8_LOOSE ? 4 : 6) act8_kernel(const __grid_constant__ Act8Args a)
{
    let_next_start();
    wait_for_previous();
    constexpr int U = sizeof(T) == 4 ? 2 : 4, kWords = sizeof(T) / 2;
    T* const x = static_cast<T*>(a.x) + (int64_t)blockIdx.y * a.xw;
    int8_t* const q = a.q + (int64_t)blockIdx.y * a.qw;
    uint8_t* const e = a.e + (int64_t)blockIdx.y * a.ew;
    // where unit u lies; how many values it has
    auto place = [&](int u, int64_t& xo, int64_t& qo, int64_t& eo) -> uint32_t {
        const uint64_t i = (uint64_t)blockIdx.x * (256 * U) + u * 256 + threadIdx.x;
        if constexpr (LAYOUT == ACT8_FLAT) {
            xo = qo = (int64_t)i * 8;
            eo = (int64_t)(i / 4);
            return i < a.units ? 8 : 0;
        } else {
            const uint64_t row = a.units < 0x80000000ull ? a.per_row.of((uint32_t)i) : i / a.per_row.d;
            const uint64_t c = (i - row * a.per_row.d) * 8;
            xo = (int64_t)row * a.xr + (int64_t)c;
            qo = (int64_t)row * a.qr + (int64_t)c;
            eo = (int64_t)row * a.er + (int64_t)(c / 32);
            return i < a.units && c < a.cols ? (uint32_t)(a.cols - c < 8 ? a.cols - c : 8) : 0;
        }
    };
    if constexpr (PACK) {
        uint4 r[U][kWords];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            int64_t xo, qo, eo;
            const uint32_t n = place(u, xo, qo, eo);
            if constexpr (LAYOUT == ACT8_LOOSE) {
#pragma unroll
                for (uint32_t j = 0; j < kWords; ++j) {
                    constexpr uint32_t per = 16 / sizeof(T);
                    r[u][j] = get16(reinterpret_cast<const unsigned char*>(x + xo + j * per), n > j * per ? min(n - j * per, per) * (uint32_t)sizeof(T) : 0);
                }
            } else {
#pragma unroll
                for (int j = 0; j < kWords; ++j) r[u][j] = n ? __ldg(reinterpret_cast<const uint4*>(x + xo) + j) : make_uint4(0, 0, 0, 0);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[8], m = 0.0f;
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
                const uint32_t w[4] = {r[u][j].x, r[u][j].y, r[u][j].z, r[u][j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (sizeof(T) == 4) v[4 * j + i] = __uint_as_float(w[i]);
                    else { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) m = act8_max(m, v[j]);
            m = act8_max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            m = act8_max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
            const uint32_t ex = act8_exponent(m);
            const float inv = act8_inverse(ex);
            int64_t xo, qo, eo;
            const uint32_t n = place(u, xo, qo, eo);
            if (n) {
                const uint2 w = make_uint2(act8_quant4(v[0], v[1], v[2], v[3], inv), act8_quant4(v[4], v[5], v[6], v[7], inv));
                if constexpr (LAYOUT == ACT8_LOOSE) loose_store(q + qo, n, w);
                else *reinterpret_cast<uint2*>(q + qo) = w;
                if (threadIdx.x % 4 == 0) e[eo] = (uint8_t)ex;
            }
        }
    } else {
        uint2 w[U];
        uint32_t ex[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            int64_t xo, qo, eo;
            const uint32_t n = place(u, xo, qo, eo);
            ex[u] = n ? __ldg(e + eo) : 0;
            if constexpr (LAYOUT == ACT8_LOOSE) w[u] = loose_load(q + qo, n);
            else w[u] = n ? __ldg(reinterpret_cast<const uint2*>(q + qo)) : make_uint2(0, 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[8];
            const float s = act8_step(ex[u]);
            act8_value4(w[u].x, s, v);
            act8_value4(w[u].y, s, v + 4);
            int64_t xo, qo, eo;
            const uint32_t n = place(u, xo, qo, eo);
            if (n) {
                if constexpr (LAYOUT != ACT8_LOOSE) {
                    Vec<T, 8>::store(x + xo, v);
                } else if constexpr (sizeof(T) == 2) {
                    put16<2>(reinterpret_cast<unsigned char*>(x + xo), 2 * n, make_uint4(f2_narrow(f2_of(v[0], v[1])), f2_narrow(f2_of(v[2], v[3])), f2_narrow(f2_of(v[4], v[5])), f2_narrow(f2_of(v[6], v[7]))));
                } else if (n == 8 && (reinterpret_cast<uintptr_t>(x + xo) & 7)) {
                    T* p = x + xo;
                    p[0] = v[0];
#pragma unroll
                    for (int i = 0; i < 3; ++i) reinterpret_cast<float2*>(p + 1)[i] = make_float2(v[2 * i + 1], v[2 * i + 2]);
                    p[7] = v[7];
                } else {
#pragma unroll
                    for (uint32_t j = 0; j < 2; ++j)
                        if (n > 4 * j)
                            put16<4>(reinterpret_cast<unsigned char*>(x + xo + 4 * j), 4 * min(n - 4 * j, 4u), make_uint4(__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3])));
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ q/k norm + rotation

constexpr uint32_t kQkThreads = 128;
// CTAs of an SM: four forward (five spill and are 6 % slower, three 19 %); three backward, whose registers four do not hold
// (8 workers, 2048 tokens, 12 + 12 heads of 64: 40.2 us with four, 32.9 with three; 2 of 32768, 16 + 4 of 128: 221 and 219)
__host__ __device__ constexpr int qk_ctas_per_sm(bool back) { return back ? 3 : 4; }
// items of a warp under way at a time, and a CTA's shared memory: the ring, or the warps' sums of the weight gradient
__host__ __device__ constexpr int qk_ring(int V, int NS) { return V == 1 ? 1 : NS == 1 ? 4 : 2; }
__host__ __device__ constexpr uint32_t qk_smem(int V, int NS, bool back, uint32_t head_dim)
{
    const uint32_t ring = V == 1 ? 0 : qk_ring(V, NS) * NS * 2 * (back ? 2 : 1) * 16 * kQkThreads, sums = back ? kQkThreads / 32 * head_dim * 4 : 0;
    return ring > sums ? ring : sums;
}

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
    uint32_t abreast[2];          // heads of a token that a warp works on at a time: a power of two
    const float* cos_t;
    const float* sin_t;
    const int32_t* pos;
    int64_t  pos_w;
    uint64_t tokens, table_rows;
    uint32_t head_dim, rot, pair_slots, slots;   // slots: two vectors of V values each; the first pair_slots hold pairs
    uint32_t lanes;               // lanes of a warp that share one head: a power of two, NS * lanes >= slots
    int      table_wide;          // the rows of the angle tables start on 16-byte boundaries
    float    eps;
};

// The 2V values of a slot as V pairs of floats, from the two vectors as they lie in memory.
template <typename T, int V>
__device__ __forceinline__ void slot_get(const uint4 (&r)[2], f2 (&v)[V])
{
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const uint32_t w[4] = {r[p].x, r[p].y, r[p].z, r[p].w};
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if constexpr (sizeof(T) == 2) v[p * (V / 2) + i] = f2_wide(w[i]);
            else v[p * (V / 2) + i] = f2_of(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ void slot_put(T* base, const uint32_t (&at)[2], const f2 (&v)[V])
{
    if constexpr (V == 1) {
        float a, b;
        f2_get(v[0], a, b);
        if (at[0] != ~0u) base[at[0]] = from_f<T>(a);
        if (at[1] != ~0u) base[at[1]] = from_f<T>(b);
    } else {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                if constexpr (sizeof(T) == 2) w[i] = f2_narrow(v[p * (V / 2) + i]);
                else {
                    float a, b;
                    f2_get(v[p * (V / 2) + i], a, b);
                    w[2 * i] = __float_as_uint(a); w[2 * i + 1] = __float_as_uint(b);
                }
            }
            if (at[p] != ~0u) *reinterpret_cast<uint4*>(base + at[p]) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// Where a value's partner of the rotation is: SPLIT the same place of another vector of the lane (halves of whole vectors);
// INTER the next value; CROSS (halves of other sizes) any place of the head, read from the ring's other lanes.
enum { QK_SPLIT = 0, QK_INTER = 1, QK_CROSS = 2 };

// A warp takes a few tokens at a time and walks their heads; `lanes` lanes share a head, and a slot of a lane holds both
// halves of its rotation pairs, so the rotation needs no exchange: for split halves vectors s and s + rot/(2V), for
// interleaved pairs two neighbouring vectors (V > 1: the pairs lie inside a vector; V = 1: the slot is the pair).  Values
// that are not rotated are pairs of angle zero.  The only exchanges are the sums over a head.
// It moves 4 bytes a value forward (bfloat16), and instructions weigh as much as memory: the arithmetic is in pairs of
// floats, and what depends on the token and not on the head is formed once per token (forward the products of weights and
// angles), so a warp's groups are spread over heads only as far as leaves four heads or so in a row to each.  Each lane
// brings what it will work on into shared memory by asynchronous copies, kRing items ahead (held in registers, one item
// ahead was all there was room for).  V = 1, for layouts without 16-byte boundaries, reads directly.
template <typename T, int V, int NS, bool BACK, int PAIRS, int LANES, int SIDE>
__device__ __forceinline__ void qk_walk(const QkArgs& a, const uint32_t cta, unsigned char* smem)
{
    constexpr bool kCross = PAIRS == QK_CROSS;
    constexpr bool kInside = PAIRS == QK_INTER || V == 1;                     // a rotation pair is one f2 (else: f2 i and V/2 + i)
    constexpr int H = V / 2;
    constexpr uint32_t kWarps = kQkThreads / 32;
    const uint32_t lanes = LANES ? LANES : a.lanes;
    const uint32_t ctas = a.ctas[SIDE];
    const HeadsArg& h = a.side[SIDE];
    const uint32_t k = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t sub = lane & (lanes - 1), group = lane / lanes, groups = 32 / lanes;
    const uint32_t n_vec = a.head_dim / V, half = a.rot / 2;
    uint32_t at[NS][2];           // first element of each vector, or ~0
    T w[NS][2 * V];               // two to a register where they are bfloat16
    f2 acc[BACK ? NS : 1][V];
    const T* wp = static_cast<const T*>(h.w) + (int64_t)k * h.ww;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const uint32_t slot = s * lanes + sub, split = PAIRS == QK_SPLIT ? a.pair_slots : 0;
        uint32_t v0, v1;
        if (PAIRS == QK_SPLIT && slot < split) { v0 = slot; v1 = slot + split; }
        // (the vectors of neighbouring lanes follow one another: interleaved in pairs, the two of a lane side by side, every
        // access took half-filled sectors -- fp32 backward of 2 x 16384 tokens, 16 + 4 heads of 128: 303 us, so 150)
        else if (PAIRS != QK_INTER || V > 1) { v0 = split + slot; v1 = v0 + a.slots - split; }
        else { v0 = 2 * slot; v1 = v0 + 1; }
        at[s][0] = slot < a.slots && v0 < n_vec ? v0 * V : ~0u;
        at[s][1] = slot < a.slots && v1 < n_vec ? v1 * V : ~0u;
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) {
            const uint32_t e = at[s][j / V];
            w[s][j] = e != ~0u ? wp[e + j % V] : from_f<T>(0.0f);
        }
        if constexpr (BACK) {
#pragma unroll
            for (int j = 0; j < V; ++j) acc[s][j] = 0;
        }
    }
    // CROSS: the partner of each value -- its weight, and where it lies in an item of the ring
    T w_of[kCross ? NS : 1][2 * V];
    uint32_t lies[kCross ? NS : 1][2 * V];
    if constexpr (kCross) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) {
                const uint32_t e = at[s][j / V] == ~0u ? 0 : at[s][j / V] + j % V;
                const uint32_t q = e < half ? e + half : e < a.rot ? e - half : e, v = q / V, p = v >= a.slots, sl = v - p * a.slots;
                w_of[s][j] = wp[q];
                lies[s][j] = ((sl / lanes) * 2 + p) * 512 + (sl % lanes) * 16 + q % V * (uint32_t)sizeof(T) - sub * 16;
            }
    }
    const float inv_n = 1.0f / (float)a.head_dim;
    // the warp's groups: `abreast` heads of each of `tokens` tokens
    const uint32_t abreast = a.abreast[SIDE], tokens = groups / abreast, first = group % abreast, my_token = group / abreast;
    const uint32_t rounds = (h.heads + abreast - 1) / abreast;
    const uint64_t step = (uint64_t)ctas * kWarps * tokens, start = ((uint64_t)cta * kWarps + warp) * tokens;
    const uint64_t turns = start < a.tokens ? (a.tokens - 1 - start) / step + 1 : 0;      // token groups of this warp

    // where the next item to be fetched lies
    constexpr int kRing = qk_ring(V, NS), kVecs = NS * 2 * (BACK ? 2 : 1);    // items under way; 16-byte pieces of one a lane
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(smem) + (warp * (kRing * kVecs) * 32 + lane) * 16;
    const T* const xb = static_cast<const T*>(h.x) + (int64_t)k * h.xw;
    const T* const db = static_cast<const T*>(h.d) + (int64_t)k * h.dw;
    T* const ob = static_cast<T*>(h.out) + (int64_t)k * h.ow;
    uint64_t ft = start + my_token;
    uint32_t fh = first;
    int64_t fx = (int64_t)ft * h.xt + (int64_t)fh * h.xh, fd = (int64_t)ft * h.dt + (int64_t)fh * h.dh;
    uint64_t left = turns * rounds;
    auto fetch = [&](uint32_t slot) {
        if constexpr (V > 1) {
            if (left) {
                if (ft < a.tokens && fh < h.heads) {
#pragma unroll
                    for (int s = 0; s < NS; ++s)
#pragma unroll
                        for (int p = 0; p < 2; ++p)
                            if (at[s][p] != ~0u) {
                                const uint32_t to = mine + (slot * kVecs + s * 2 + p) * 512;
                                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(xb + fx + at[s][p]) : "memory");
                                if constexpr (BACK)
                                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + NS * 2 * 512), "l"(db + fd + at[s][p]) : "memory");
                            }
                } else if constexpr (BACK) {                                 // not a head: zeros, which add nothing to the weight gradient
#pragma unroll
                    for (int i = 0; i < kVecs; ++i)                           // (an infinity of the item before it would: times 0 it is NaN)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(mine + (slot * kVecs + i) * 512), "r"(0) : "memory");
                }
                --left;
                fh += abreast;
                if (fh - first == rounds * abreast) {
                    ft += step;
                    fh = first;
                    fx = (int64_t)ft * h.xt + (int64_t)fh * h.xh;
                    if constexpr (BACK) fd = (int64_t)ft * h.dt + (int64_t)fh * h.dh;
                } else {
                    fx += abreast * h.xh;
                    if constexpr (BACK) fd += abreast * h.dh;
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    // an item's values: from its place in the ring, or (V = 1) from memory
    auto values = [&](uint32_t slot, bool second, int s, const T* from, f2 (&v)[V]) {
        if constexpr (V > 1) {
            uint4 r[2];
#pragma unroll
            for (int p = 0; p < 2; ++p)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[p].x), "=r"(r[p].y), "=r"(r[p].z), "=r"(r[p].w)
                             : "r"(mine + (slot * kVecs + (second ? NS * 2 : 0) + s * 2 + p) * 512));
            slot_get<T, V>(r, v);
        } else {
            v[0] = f2_of(from && at[s][0] != ~0u ? to_f(from[at[s][0]]) : 0.0f, from && at[s][1] != ~0u ? to_f(from[at[s][1]]) : 0.0f);
        }
    };
    // CROSS: the partners of a slot's values in an item
    auto partners = [&](uint32_t slot, bool second, int s, f2 (&v)[V]) {
        if constexpr (kCross) {
            const uint32_t from = mine + (slot * kVecs + (second ? NS * 2 : 0)) * 512;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float f[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (sizeof(T) == 4) {
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f[i]) : "r"(from + lies[s][2 * j + i]));
                    } else {
                        uint32_t h;
                        asm volatile("{\n .reg .b16 t;\n ld.shared.b16 t, [%1];\n cvt.u32.u16 %0, t;\n}" : "=r"(h) : "r"(from + lies[s][2 * j + i]));
                        f[i] = __uint_as_float(h << 16);
                    }
                }
                v[j] = f2_of(f[0], f[1]);
            }
        }
    };
    auto over_head = [&](f2 v2) {
        float v, u;
        f2_get(v2, v, u);
        v += u;
#pragma unroll
        for (uint32_t m = 1; m < 32; m *= 2)
            if (m < lanes) v += __shfl_xor_sync(0xFFFFFFFFu, v, m);         // (the same branch for the whole grid)
        return v;
    };
    auto position = [&](uint64_t turn) -> int32_t {
        const uint64_t tk = start + turn * step + my_token;
        return a.rot && tk < a.tokens ? __ldg(a.pos + (int64_t)k * a.pos_w + (int64_t)tk) : 0;
    };
    auto weight = [&](int s, int i) { return f2_of(to_f(w[s][2 * i]), to_f(w[s][2 * i + 1])); };

    // of the pairs of each f2 of the token: cosines and, with the signs of the rotation, sines; forward: times the weights
    f2 mc[NS][V], ms[NS][V];
    float bad = 0.0f;
    auto token = [&](int32_t pos) {
        const bool ok = !a.rot || (pos >= 0 && (uint64_t)pos < a.table_rows);
        const float* ct = a.cos_t + (ok ? (uint64_t)pos * half : 0);
        const float* st = a.sin_t + (ok ? (uint64_t)pos * half : 0);
        bad = ok ? 0.0f : __uint_as_float(0x7FFFFFFFu);                       // outside the table: NaN
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if constexpr (kCross) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float c[2], sn[2], w0[2], w1[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int k2 = 2 * j + i;
                        const uint32_t e = at[s][k2 / V] == ~0u ? a.rot : at[s][k2 / V] + k2 % V, n = e < half ? e : e - half;
                        const bool on = e < a.rot && ok;
                        c[i] = on ? __ldg(ct + n) : 1.0f;
                        sn[i] = on ? __ldg(st + n) : 0.0f;
                        if ((e < half) != BACK) sn[i] = -sn[i];               // (a, b) -> (a c - b s, b c + a s), or back
                        w0[i] = to_f(w[s][k2]);
                        w1[i] = to_f(w_of[s][k2]);
                    }
                    mc[s][j] = BACK ? f2_of(c[0], c[1]) : f2_of(c[0] * w0[0], c[1] * w0[1]);
                    ms[s][j] = BACK ? f2_of(sn[0], sn[1]) : f2_of(sn[0] * w1[0], sn[1] * w1[1]);
                }
                continue;
            }
            float c[V], sn[V];
            if constexpr (kInside && V > 1) {                                // pairs of two vectors, each of its own place
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const uint32_t i = at[s][p] == ~0u ? half : at[s][p] / 2;
                    if (a.table_wide && i + H <= half && ok) {
                        if constexpr (H == 4) {
                            Vec<float, 4>::load(ct + i, c + p * H); Vec<float, 4>::load(st + i, sn + p * H);
                        } else {
                            const float2 c2 = __ldg(reinterpret_cast<const float2*>(ct + i)), s2 = __ldg(reinterpret_cast<const float2*>(st + i));
                            c[p * H] = c2.x; c[p * H + 1] = c2.y; sn[p * H] = s2.x; sn[p * H + 1] = s2.y;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < H; ++j) {
                            const bool on = i + j < half && ok;
                            c[p * H + j] = on ? __ldg(ct + i + j) : 1.0f;
                            sn[p * H + j] = on ? __ldg(st + i + j) : 0.0f;
                        }
                    }
                }
            } else {
                const uint32_t i = (s * lanes + sub) * V;                   // first pair of the slot
                if (V > 1 && a.table_wide && i + V <= half && ok) {
                    if constexpr (V > 1) {
#pragma unroll
                        for (int j = 0; j < V; j += 4) { Vec<float, 4>::load(ct + i + j, c + j); Vec<float, 4>::load(st + i + j, sn + j); }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const bool on = i + j < half && ok;
                        c[j] = on ? __ldg(ct + i + j) : 1.0f;
                        sn[j] = on ? __ldg(st + i + j) : 0.0f;
                    }
                }
            }
            if constexpr (kInside) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    mc[s][j] = f2_of(c[j], c[j]);
                    ms[s][j] = BACK ? f2_of(sn[j], -sn[j]) : f2_of(-sn[j], sn[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < H; ++j) {
                    mc[s][j] = mc[s][H + j] = f2_of(c[2 * j], c[2 * j + 1]);
                    const f2 q = f2_of(sn[2 * j], sn[2 * j + 1]);
                    ms[s][j] = BACK ? q : f2_neg(q);
                    ms[s][H + j] = BACK ? f2_neg(q) : q;
                }
            }
            if constexpr (!BACK) {                                            // value times its own weight, partner times the partner's
                f2 wf[V];
#pragma unroll
                for (int j = 0; j < V; ++j) wf[j] = weight(s, j);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    mc[s][j] = f2_mul(mc[s][j], wf[j]);
                    ms[s][j] = f2_mul(ms[s][j], kInside ? f2_swap(wf[j]) : wf[(j + H) % V]);
                }
            }
        }
    };
    auto work = [&](uint32_t slot, bool live, int64_t xo, int64_t go, int64_t oo) {
        f2 x[NS][V], sq = 0;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            values(slot, false, s, live ? xb + xo : nullptr, x[s]);
#pragma unroll
            for (int j = 0; j < V; ++j) sq = f2_fma(x[s][j], x[s][j], sq);
        }
        // (a head that is not there reads zeros backward, and 0 for r: eps may be 0 and its position outside the table)
        const float mean = fmaf(over_head(sq), inv_n, a.eps), r = live ? rsqrtf(mean) + bad : 0.0f;
        const f2 rr = f2_of(r, r);
        f2 y[NS][V];
        if constexpr (!BACK) {
#pragma unroll
            for (int s = 0; s < NS; ++s) {
#pragma unroll
                for (int j = 0; j < V; ++j) x[s][j] = f2_mul(x[s][j], rr);
                f2 q[V];
                partners(slot, false, s, q);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    y[s][j] = f2_fma(x[s][j], mc[s][j], f2_mul(kCross ? f2_mul(q[j], rr) : kInside ? f2_swap(x[s][j]) : x[s][(j + H) % V], ms[s][j]));
            }
        } else {
            f2 dot = 0;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                f2 d[V], q[V];
                values(slot, true, s, live ? db + go : nullptr, d);
                partners(slot, true, s, q);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    y[s][j] = f2_fma(d[j], mc[s][j], f2_mul(kCross ? q[j] : kInside ? f2_swap(d[j]) : d[(j + H) % V], ms[s][j]));
                    x[s][j] = f2_mul(x[s][j], rr);                            // xh
                    acc[s][j] = f2_fma(y[s][j], x[s][j], acc[s][j]);
                    y[s][j] = f2_mul(y[s][j], weight(s, j));
                    dot = f2_fma(y[s][j], x[s][j], dot);
                }
            }
            const float m = over_head(dot) * -inv_n;
            const f2 mm = f2_of(m, m);
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int j = 0; j < V; ++j) y[s][j] = f2_mul(rr, f2_fma(x[s][j], mm, y[s][j]));
        }
        if (live) {
#pragma unroll
            for (int s = 0; s < NS; ++s) slot_put<T, V>(ob + oo, at[s], y[s]);
        }
    };

    if constexpr (V > 1) {                                                    // a lane without a vector reads zeros
#pragma unroll
        for (int i = 0; i < kRing * kVecs; ++i)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(mine + i * 512), "r"(0) : "memory");
    }
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) fetch(i);
    int32_t pos_next = position(0);
    uint32_t slot = 0;
    for (uint64_t turn = 0; turn < turns; ++turn) {
        const int32_t pos = pos_next;
        if (turn + 1 < turns) pos_next = position(turn + 1);
        token(pos);
        const uint64_t tk = start + turn * step + my_token;
        const bool in = tk < a.tokens;
        int64_t xo = (int64_t)tk * h.xt + (int64_t)first * h.xh, go = (int64_t)tk * h.dt + (int64_t)first * h.dh, oo = (int64_t)tk * h.ot + (int64_t)first * h.oh;
        for (uint32_t hd = first; hd - first < rounds * abreast; hd += abreast) {
            if constexpr (kCross) __syncwarp();                               // (all lanes have done with that item)
            fetch(slot == 0 ? kRing - 1 : slot - 1);                          // into the place of the item before this one
            if constexpr (V > 1) asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
            if constexpr (kCross) __syncwarp();                               // (and what the other lanes brought is there)
            work(slot, in && hd < h.heads, xo, go, oo);
            slot = slot + 1 == kRing ? 0 : slot + 1;
            if constexpr (V == 1) { xo += abreast * h.xh; go += abreast * h.dh; }
            oo += abreast * h.oh;
        }
    }
    if constexpr (BACK) {
        // the CTA's sum in a fixed order: groups of a warp by a butterfly, then the warps one after another
        __syncthreads();                                                      // (the ring is done with)
        float* const sum = reinterpret_cast<float*>(smem);                    // [kWarps][head_dim]
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) {
                float v, u;
                f2_get(acc[s][j / 2], v, u);
                if (j & 1) v = u;
                for (uint32_t m = 16; m >= lanes; m >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, m);
                if (group == 0 && at[s][j / V] != ~0u) sum[warp * a.head_dim + at[s][j / V] + j % V] = v;
            }
        __syncthreads();
        float* const part = h.part + ((uint64_t)k * ctas + cta) * a.head_dim;
        for (uint32_t i = threadIdx.x; i < a.head_dim; i += kQkThreads) {
            float v = 0.0f;
#pragma unroll
            for (uint32_t wi = 0; wi < kWarps; ++wi) v += sum[wi * a.head_dim + i];
            part[i] = v;
        }
    }
}

// (Two copies of the walk: with the side a constant its strides are constants of the instruction, not loads by index.)
// LANES: the lanes that share a head where the host picks a copy made for them (0: any; the sum over a head is then a
// chain of branches, which take a tenth of the time).
template <typename T, int V, int NS, bool BACK, int PAIRS, int LANES>
__global__ void __launch_bounds__(kQkThreads, NS == 1 ? qk_ctas_per_sm(BACK) : 1) qk_kernel(const __grid_constant__ QkArgs a)
{
    let_next_start();
    wait_for_previous();
    extern __shared__ __align__(16) unsigned char smem[];
    if (blockIdx.x < a.ctas[0]) qk_walk<T, V, NS, BACK, PAIRS, LANES, 0>(a, blockIdx.x, smem);
    else qk_walk<T, V, NS, BACK, PAIRS, LANES, 1>(a, blockIdx.x - a.ctas[0], smem);
}

struct QkSumArgs {
    const float* part[2];
    void*    dw[2];               // may be NULL where the side has no heads
    int64_t  dww[2];
    uint32_t parts[2], head_dim;
};

// The CTAs' partial sums of the weight gradients, joined in a fixed order: eight interleaved runs, then those.
template <typename T>
__global__ void __launch_bounds__(256) qk_sum_kernel(const __grid_constant__ QkSumArgs a)
{
    __shared__ float run[8][32];
    let_next_start();
    wait_for_previous();
    const uint32_t side = blockIdx.y, k = blockIdx.z;
    if (!a.dw[side]) return;
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
