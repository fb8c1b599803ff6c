// Row kernels of the block operators: cross entropy over a vocabulary, forward and backward.
//
// Forward: one pass over the logits.  A lane keeps the largest value that it has seen and the sum of e^(z - largest), four pieces of
// 16 bytes at a time with the next four -- of the next row, at a row's end -- under way; lanes, then warps, join theirs.  Rows are
// read by the aligned 16-byte pieces that hold their values (a vocabulary of odd size starts every row at another offset), what
// is outside set to -infinity.
// Backward: e^(z - lse) from what the forward call left, one read and one write a value (rows of a large lse are read twice).
// Backward bound by memory (bfloat16, 8 x 512 rows of 50257: 128 us, 823 MB at 98 % of the rate of a copy), forward in fp32 too (8 x 512 rows
// of 32768: 82 us, as a copy), in bfloat16 by its instructions and exponentials (8 x 512 rows of 50257: 88 us, 63 at the rate of a
// copy; with one largest value a piece instead of four pieces 91).
#pragma once
#include "block_common.cuh"

namespace palsgd {
namespace block {

struct LossArgs {
    const void*    z;
    const int32_t* target;
    const float*   dloss;         // backward
    float *loss, *lse;            // lse: written (forward), read (backward)
    void*          dz;            // backward; may be z
    int64_t  zw, zr, tw, lw, sw, gw, dw, dr;         // worker and row strides, elements
    uint64_t rows;
    uint32_t vocab, warps;        // of a team that has a row
};

constexpr float kLog2e = 1.4426950408889634f;

// A largest value and the sum of e^(z - largest).  No value yet, or none above -infinity: the sum is zero or NaN.
struct Soft { float top, sum; };
__device__ __forceinline__ float soft_scale(float from, float to)       // e^(from - to); 0 for from = -infinity, whatever to is
{
    return from == -INFINITY ? 0.0f : fast_exp2((from - to) * kLog2e);
}
__device__ __forceinline__ Soft soft_join(Soft a, Soft b)
{
    const float top = fmaxf(a.top, b.top);
    // (a side without a value counts for nothing; one that holds a NaN keeps it)
    return Soft{top, fmaf(a.sum, soft_scale(a.top, top), b.sum * soft_scale(b.top, top))};
}

// 16 bytes as floats
template <typename T>
__device__ __forceinline__ void floats_of(const uint4& p, float (&v)[16 / sizeof(T)])
{
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
        else v[i] = __uint_as_float(w[i]);
    }
}

__device__ __forceinline__ __nv_bfloat162 word_pair(uint32_t w)
{
    __nv_bfloat162 v;
    asm("mov.b32 %0, %1;" : "=r"(*reinterpret_cast<uint32_t*>(&v)) : "r"(w));
    return v;
}
// The largest of a lane's values (of numbers beside NaN, the numbers'); bfloat16 in pairs
template <typename T, int P>
__device__ __forceinline__ float largest(const uint4 (&q)[P])
{
    if constexpr (sizeof(T) == 2) {
        __nv_bfloat162 top = word_pair(q[0].x);
#pragma unroll
        for (int j = 0; j < P; ++j) top = __hmax2(top, __hmax2(__hmax2(word_pair(q[j].x), word_pair(q[j].y)), __hmax2(word_pair(q[j].z), word_pair(q[j].w))));
        return fmaxf(__low2float(top), __high2float(top));
    } else {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < P; ++j) top = fmaxf(top, fmaxf(fmaxf(__uint_as_float(q[j].x), __uint_as_float(q[j].y)), fmaxf(__uint_as_float(q[j].z), __uint_as_float(q[j].w))));
        return top;
    }
}

template <typename T>
__global__ void __launch_bounds__(1024) loss_forward_kernel(const __grid_constant__ LossArgs a)
{
    constexpr int V = 16 / (int)sizeof(T), P = 4;         // pieces of a lane at a time; as many more under way
    constexpr uint32_t kNothing = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;     // -infinity
    __shared__ Soft places[2][32];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, team = warp / a.warps, teams = (blockDim.x >> 5) / a.warps;
    const uint32_t size = a.warps * 32, me = threadIdx.x - team * size;
    const int64_t k = blockIdx.y;
    const uint64_t rows_step = (uint64_t)gridDim.x * teams;
    let_next_start();
    wait_for_previous();
    // a row, and what a team has come to in it
    struct Place {
        const uint4* p;
        const T*     z;
        uint64_t     row;
        uint32_t     off, end, pieces, i;                 // values of the first piece that are not the row's; the last one's end
    } now, next;
    auto enter = [&](uint64_t row) {
        Place at;
        at.row = row;
        at.z = static_cast<const T*>(a.z) + k * a.zw + (int64_t)row * a.zr;
        at.off = (uint32_t)(reinterpret_cast<uintptr_t>(at.z) & 15) / (uint32_t)sizeof(T);
        at.p = reinterpret_cast<const uint4*>(at.z - at.off);
        at.end = at.off + a.vocab;
        at.pieces = (at.end + V - 1) / V;
        at.i = me;
        return at;
    };
    auto fetch = [&](const Place& at, uint4 (&q)[P]) {
#pragma unroll
        for (int j = 0; j < P; ++j) q[j] = at.row < a.rows && at.i + j * size < at.pieces ? __ldg(at.p + at.i + j * size) : make_uint4(kNothing, kNothing, kNothing, kNothing);
    };
    now = enter((uint64_t)blockIdx.x * teams + team);
    uint4 q[P], ahead[P];
    fetch(now, q);
    Soft s{-INFINITY, 0.0f};
    for (uint32_t turn = 0; now.row < a.rows;) {
        // (the row ends at the same time for all lanes of the team)
        const bool ends = now.i - me + size * P >= now.pieces;
        if (ends) next = enter(now.row + rows_step);
        else { next = now; next.i += size * P; }
        fetch(next, ahead);
        auto rise = [&](float top) {                      // to a larger value (or only NaN so far)
            if (!(top <= s.top)) {
                s.sum *= soft_scale(s.top, top);
                s.top = top;
            }
        };
        auto add = [&](const float (&v)[V], f2 shift, f2& sum) {
            const f2 scale = f2_same(kLog2e);
#pragma unroll
            for (int e = 0; e < V; e += 2) {
                float x, y;
                f2_get(f2_mul(f2_add(f2_of(v[e], v[e + 1]), shift), scale), x, y);
                sum = f2_add(sum, f2_of(fast_exp2(x), fast_exp2(y)));
            }
        };
        // what lies outside the row, in its first and its last piece, is -infinity, as are pieces behind it
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const uint32_t at = now.i + j * size;
            if (at - lane >= now.pieces) break;            // (the same for the whole warp)
            if (at < now.pieces && (at == 0 || (at + 1) * V > now.end)) {
                uint32_t w[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (at * V + e >= now.off && at * V + e < now.end) continue;
                    if constexpr (sizeof(T) == 2) w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | 0xFF800000u : (w[e / 2] & 0xFFFF0000u) | 0xFF80u;
                    else w[e] = 0xFF800000u;
                }
                q[j] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        rise(largest<T, P>(q));
        const f2 shift = f2_same(s.top == -INFINITY ? -0.0f : -s.top);
        f2 sum = 0;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            if (now.i - lane + j * size >= now.pieces) break;
            float v[V];
            floats_of<T>(q[j], v);
            add(v, shift, sum);
        }
        s.sum += f2_total(sum);
        if (ends) {
#pragma unroll
            for (int d = 16; d; d >>= 1)
                s = soft_join(s, Soft{__shfl_xor_sync(0xFFFFFFFFu, s.top, d), __shfl_xor_sync(0xFFFFFFFFu, s.sum, d)});
            if (a.warps > 1) {                            // (the places of one row are read while the next one's are written)
                if (lane == 0) places[turn][warp] = s;
                asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(size) : "memory");
                if (me == 0) {
                    s = places[turn][warp];
                    for (uint32_t j = 1; j < a.warps; ++j) s = soft_join(s, places[turn][warp + j]);
                }
                turn ^= 1;
            }
            if (me == 0) {
                const float log_sum = logf(s.sum);
                const int32_t t = a.target[k * a.tw + (int64_t)now.row];
                a.lse[k * a.sw + (int64_t)now.row] = s.top == -INFINITY && s.sum == 0.0f ? -INFINITY : s.top + log_sum;
                float loss = 0.0f;
                if (t >= 0) loss = (uint32_t)t < a.vocab ? (s.top - to_f(now.z[t])) + log_sum : __uint_as_float(0x7FFFFFFFu);
                a.loss[k * a.lw + (int64_t)now.row] = loss;
            }
            s = Soft{-INFINITY, 0.0f};
        }
        now = next;
#pragma unroll
        for (int j = 0; j < P; ++j) q[j] = ahead[j];
    }
}

// dz = (e^(z - lse) - [target]) dloss of a part of a row: `pieces` of 16 bytes a lane, from where the row's copy in memory
// lets it.  Rows of z and dz that start alike are walked by aligned pieces, the ragged ends one value at a time; others at
// any address.
constexpr uint32_t kLossPieces = 8;                       // of a lane

// From here on binary32 holds lse to 2^-14 at best, and nothing of the sum where a row has nothing but the type's lowest value.  An
// lse that is the row's own, to its rounding, then gives way to the row's largest value and sum, formed again; any other is taken as
// it is.  One warp has the row: all of it is read before its gradient is written over it.  (By the whole team, its barriers left room
// for fewer CTAs: bfloat16, 8 x 512 x 50257, near rows 149 us, so 128, without far rows in the kernel 126.5; all rows far 833.)
constexpr float kFarLse = 1024.0f;
template <typename T>
__device__ __noinline__ void loss_far_row(const T* z, T* dz, uint32_t vocab, int32_t t, float d, float lse, uint32_t lane)
{
    Soft s{-INFINITY, 0.0f};
    for (uint32_t c = lane; c < vocab; c += 32) s = soft_join(s, Soft{to_f(z[c]), 1.0f});
#pragma unroll
    for (int b = 16; b; b >>= 1)
        s = soft_join(s, Soft{__shfl_xor_sync(0xFFFFFFFFu, s.top, b), __shfl_xor_sync(0xFFFFFFFFu, s.sum, b)});
    float rest = logf(s.sum);
    if (fabsf((s.top + rest) - lse) <= 0x1p-22f * fabsf(lse)) lse = s.top;
    else rest = 0.0f;
    for (uint32_t c = lane; c < vocab; c += 32) {
        float p = expf((to_f(z[c]) - lse) - rest);
        if (c == (uint32_t)t) p -= 1.0f;
        dz[c] = from_f<T>(p * d);
    }
}

struct LossGrid { Divisor parts; uint32_t units; };       // parts of a row; parts of all rows of a worker

template <typename T>
__global__ void __launch_bounds__(256, 6) loss_backward_kernel(const __grid_constant__ LossArgs a, const __grid_constant__ LossGrid g)
{
    constexpr int V = 16 / (int)sizeof(T), P = 4;
    const uint32_t warp = threadIdx.x >> 5, team = warp / a.warps, teams = (blockDim.x >> 5) / a.warps;
    const uint32_t size = a.warps * 32, me = threadIdx.x - team * size;
    const int64_t k = blockIdx.y;
    let_next_start();
    wait_for_previous();
    const uint32_t unit = blockIdx.x * teams + team;
    if (unit >= g.units) return;
    const uint32_t row = g.parts.of(unit), part = unit - row * g.parts.d;
    const T* z = static_cast<const T*>(a.z) + k * a.zw + (int64_t)row * a.zr;
    T* dz = static_cast<T*>(a.dz) + k * a.dw + (int64_t)row * a.dr;
    const int32_t t = a.target[k * a.tw + row];
    const bool bad = t >= 0 && (uint32_t)t >= a.vocab;
    const float d = bad ? __uint_as_float(0x7FFFFFFFu) : t < 0 ? 0.0f : a.dloss[k * a.gw + row];
    const float lse = a.lse[k * a.sw + row];
    if (fabsf(lse) >= kFarLse && fabsf(lse) < INFINITY && t >= 0) {
        if (part == 0 && me < 32) loss_far_row(z, dz, a.vocab, t, d, lse, me);
        return;
    }
    auto gradient = [&](uint4& q, int64_t c) {            // the piece whose first value is the row's c-th
        float v[V];
        floats_of<T>(q, v);
        if (t < 0) {
            q = make_uint4(0, 0, 0, 0);
            return;
        }
        if constexpr (sizeof(T) == 2) {
            // (first the difference, exact or rounded once, then its scale: as multiply-add with lse log2(e), that product's rounding,
            // and its overflow, does not cancel where z is near lse)
            const f2 shift = f2_same(-lse), scale = f2_same(kLog2e), dd = f2_same(d);
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x, y;
                f2_get(f2_mul(f2_add(f2_of(v[2 * i], v[2 * i + 1]), shift), scale), x, y);
                x = fast_exp2(x); y = fast_exp2(y);
                if (c + 2 * i == t) x -= 1.0f;
                if (c + 2 * i + 1 == t) y -= 1.0f;
                w[i] = f2_narrow(f2_mul(f2_of(x, y), dd));
            }
            q = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = expf(v[i] - lse);
                if (c + i == t) v[i] -= 1.0f;
                v[i] *= d;
            }
            q = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        }
    };
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(z) & 15) / (uint32_t)sizeof(T);
    const bool alike = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
    const uint32_t begin = part * size * kLossPieces;
    if (alike) {
        const uint32_t end = off + a.vocab, pieces = (end + V - 1) / V, last = min(pieces, begin + size * kLossPieces);
        const uint4* from = reinterpret_cast<const uint4*>(z - off);
        uint4* to = reinterpret_cast<uint4*>(dz - off);
        for (uint32_t i = begin + me; i < last; i += size * P) {
            uint4 q[P];
#pragma unroll
            for (int j = 0; j < P; ++j) if (i + j * size < last) q[j] = from[i + j * size];
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const uint32_t at = i + j * size;
                if (at >= last) break;
                gradient(q[j], (int64_t)at * V - off);
                if (at * V >= off && (at + 1) * V <= end) {
                    to[at] = q[j];
                } else {                                  // the neighbours' values in the piece stay
                    const uint32_t w[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const uint32_t c = at * V + e;
                        if (c < off || c >= end) continue;
                        if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t*>(to)[c] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
                        else reinterpret_cast<uint32_t*>(to)[c] = w[e];
                    }
                }
            }
        }
    } else {
        const uint32_t pieces = (a.vocab + V - 1) / V, last = min(pieces, begin + size * kLossPieces);
        for (uint32_t i = begin + me; i < last; i += size) {
            const uint32_t n = min(a.vocab - i * V, (uint32_t)V) * (uint32_t)sizeof(T);
            uint4 q = get16(reinterpret_cast<const unsigned char*>(z + (uint64_t)i * V), n);
            gradient(q, (int64_t)i * V);
            put16<(int)sizeof(T)>(reinterpret_cast<unsigned char*>(dz + (uint64_t)i * V), n, q);
        }
    }
}

}  // namespace block
}  // namespace palsgd
