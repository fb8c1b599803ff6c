// Pieces that the block operators' kernels share: storage types, 16-byte vectors, the gated activations.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/palsgd_block.h"

namespace palsgd {
namespace block {

using bf16 = __nv_bfloat16;

// Kernels of this library are launched so that one may start up while the kernel before it in the stream is still
// running (launch() in the host file): each lets the next one start at once, and touches no memory of others' before
// that kernel is complete.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f<bf16>(float v) { return __float2bfloat16_rn(v); }

// V consecutive values of T at p as floats: one 16-byte (or 32-byte, as two) access where V fills it, else one by one.
template <typename T, int V> struct Vec;
template <> struct Vec<float, 4> {
    static __device__ __forceinline__ void load(const float* p, float* v)
    {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p));
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    }
    static __device__ __forceinline__ void store(float* p, const float* v)
    {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <> struct Vec<float, 8> {
    static __device__ __forceinline__ void load(const float* p, float* v) { Vec<float, 4>::load(p, v); Vec<float, 4>::load(p + 4, v + 4); }
    static __device__ __forceinline__ void store(float* p, const float* v) { Vec<float, 4>::store(p, v); Vec<float, 4>::store(p + 4, v + 4); }
};
template <> struct Vec<bf16, 8> {
    static __device__ __forceinline__ void store(bf16* p, const float* v)
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// Division of t < 2^31 by a divisor d known on the host: with s = ceil(log2 d) and m = ceil(2^(31+s) / d) < 2^32, the
// quotient is t m >> (31 + s) (m d exceeds 2^(31+s) by less than 2^s, and t times that stays below 2^(31+s)).
struct Divisor {
    uint32_t d, m, s;
    __device__ __forceinline__ uint32_t of(uint32_t t) const { return (uint32_t)(((uint64_t)t * m) >> (31 + s)); }
};

// ---- two binary32 values in one 64-bit register: multiply and multiply-add of both in one instruction
using f2 = unsigned long long;
__device__ __forceinline__ f2 f2_of(float a, float b) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void f2_get(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 f2_mul(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 f2_fma(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f2 f2_swap(f2 v) { float a, b; f2_get(v, a, b); return f2_of(b, a); }
__device__ __forceinline__ f2 f2_neg(f2 v) { return v ^ 0x8000000080000000ull; }
// two bfloat16 in a word -> two floats, and back
__device__ __forceinline__ f2 f2_wide(uint32_t w) { return f2_of(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ uint32_t f2_narrow(f2 v)
{
    float a, b;
    f2_get(v, a, b);
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}

// ---- 16 bytes at any address, the first `bytes` of them inside a row (the others read as 0 and are not written).
// Reads are of whole aligned 16-byte blocks that hold a byte of the row, shifted into place; such a block lies inside the
// row's allocation, which starts and ends on a multiple of 16 bytes.  Writes are as wide as the address allows; ELEM: the
// size of the elements, on a multiple of which the address lies.
__device__ __forceinline__ uint4 shift16(const uint4& a, const uint4& b, uint32_t o, uint32_t bytes)    // from byte o of a on
{
    const uint32_t s = 8 * (o & 3);
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = o & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = o & 4 ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], s);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)                      // what lies behind the row's end is not of it
        if (4 * i + 4 > bytes) w[i] = 4 * i >= bytes ? 0u : w[i] & ((1u << (8 * (bytes & 3))) - 1u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 get16(const unsigned char* p, uint32_t bytes)
{
    const uint32_t o = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15;
    const uint4* base = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
    const uint4 a = bytes ? __ldg(base) : make_uint4(0, 0, 0, 0), b = bytes && o + bytes > 16 ? __ldg(base + 1) : make_uint4(0, 0, 0, 0);
    return shift16(a, b, o, bytes);
}
template <int ELEM>
__device__ __forceinline__ void put16(unsigned char* p, uint32_t bytes, const uint4& v)
{
    const uint32_t o = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if (bytes == 16 && o == 0) {
        *reinterpret_cast<uint4*>(p) = v;
    } else if (bytes == 16 && (o & 7) == 0) {
        reinterpret_cast<uint2*>(p)[0] = make_uint2(w[0], w[1]);
        reinterpret_cast<uint2*>(p)[1] = make_uint2(w[2], w[3]);
    } else if (bytes == 16 && (ELEM == 4 || (o & 3) == 0)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
    } else if (bytes == 16 && ELEM < 4) {                 // up to the next word, three words, the rest
        const uint32_t head = 4 - (o & 3), rest = w[3] >> (8 * head);
        if (ELEM == 1 && (head & 1)) *p = (unsigned char)w[0];
        if (head >= 2) *reinterpret_cast<uint16_t*>(p + (head & 1)) = (uint16_t)(w[0] >> (8 * (head & 1)));
#pragma unroll
        for (int i = 0; i < 3; ++i) reinterpret_cast<uint32_t*>(p + head)[i] = __funnelshift_r(w[i], w[i + 1], 8 * head);
        unsigned char* q = p + head + 12;
        if (head <= 2) *reinterpret_cast<uint16_t*>(q) = (uint16_t)rest;
        if (ELEM == 1 && (head & 1)) q[head == 1 ? 2 : 0] = (unsigned char)(head == 1 ? rest >> 16 : rest);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 16 / ELEM; ++j)
            if (j * ELEM < bytes) {
                if constexpr (ELEM == 4) reinterpret_cast<uint32_t*>(p)[j] = w[j];
                else if constexpr (ELEM == 2) reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
                else p[j] = (unsigned char)(w[j / 4] >> (8 * (j & 3)));
            }
    }
}

// ---- 8-bit checkpoints: the step 2^(E-127) of a group from the largest magnitude in it (as bits: NaN > Inf > finite).
// Adding 2^16 to the bits carries into the exponent exactly when the mantissa is >= 1.9921875 = 127.5/64, the values
// that would round to 128 steps; ties (127.5) go to the even 128 and are among them.  A carry out of the largest finite
// exponent is a value that rounds to 2^128: not representable, like an infinity.
__device__ __forceinline__ uint32_t act8_exponent(uint32_t amax_bits)
{
    const uint32_t b = amax_bits + 0x10000u;
    const int e = (int)(b >> 23) - 6;
    return b >= 0x7F800000u ? 255u : (uint32_t)(e < 1 ? 1 : e);
}
// 1 / step as a float (0 for a group that is not finite: its q are 0 -- NaN * 0 converts to 0 too)
__device__ __forceinline__ float act8_inverse(uint32_t E) { return E == 255u ? 0.0f : __uint_as_float((254u - E) << 23); }
__device__ __forceinline__ float act8_step(uint32_t E) { return E == 255u ? __uint_as_float(0x7FFFFFFFu) : __uint_as_float(E << 23); }
// Four values as the bytes of a word: x / step, rounded to an integer by adding 1.5 * 2^23 (exactly: 1/step is a power of
// two, so the product is exact), which leaves the int8 in the low byte.  |x / step| rounds to at most 127.
__device__ __forceinline__ uint32_t act8_quant4(float a, float b, float c, float d, float inv)
{
    const float k = 12582912.0f;
    const uint32_t x = __float_as_uint(fmaf(a, inv, k)), y = __float_as_uint(fmaf(b, inv, k));
    const uint32_t z = __float_as_uint(fmaf(c, inv, k)), w = __float_as_uint(fmaf(d, inv, k));
    const uint32_t r = __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
    return inv == 0.0f ? 0u : r;                          // not finite: every q is 0
}
// the larger of m and |x|; a NaN stays
__device__ __forceinline__ float act8_max(float m, float x)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(x)));
    return r;
}
// m = max |x| of a group, any NaN as the canonical one
__device__ __forceinline__ uint32_t act8_exponent(float m) { return act8_exponent(__float_as_uint(m)); }
// the four values of a word of int8: each byte with its sign bit flipped, put behind the exponent of 2^23, is 2^23 + 128 + q
__device__ __forceinline__ void act8_value4(uint32_t w, float step, float* v)
{
    const uint32_t f = w ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (__uint_as_float(__byte_perm(f, 0x4B000000u, 0x7440 | i)) - 8388736.0f) * step;
}

// ---- gated activations
// SLOPE: also act'(g).  FAST: the slope's exponential to about 2 units in the last place of binary32, for results that are
// rounded to bfloat16 anyway (act2 has the other forms for those).
template <int ACT, bool SLOPE, bool FAST>
__device__ __forceinline__ float act(float g, float& slope)
{
    if constexpr (ACT == PALSGD_ACT_NONE) {
        if constexpr (SLOPE) slope = 1.0f;
        return g;
    } else if constexpr (ACT == PALSGD_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-g));
        const float a = g * s;
        if constexpr (SLOPE) slope = fmaf(a, 1.0f - s, s);
        return a;
    } else if constexpr (ACT == PALSGD_ACT_GELU) {
        const float cdf = fmaf(0.5f, erff(g * 0.70710678118654752f), 0.5f);
        if constexpr (SLOPE) slope = fmaf(g * 0.39894228040143268f, FAST ? __expf(-0.5f * g * g) : expf(-0.5f * g * g), cdf);
        return g * cdf;
    } else if constexpr (ACT == PALSGD_ACT_GELU_TANH) {
        // (1 + tanh z) / 2 = 1 / (1 + e^(-2z))
        const float c = 1.5957691216057308f;                     // 2 sqrt(2/pi)
        const float z2 = c * g * fmaf(0.044715f * g, g, 1.0f);
        const float s = 1.0f / (1.0f + expf(-z2));
        if constexpr (SLOPE) {                                   // (its square has to stay finite: 0 times an infinity is NaN)
            const float m = fminf(fabsf(g), 1e9f);
            slope = fmaf(g * s * (1.0f - s), c * fmaf(0.134145f * m, m, 1.0f), s);
        }
        return g * s;
    } else {
        // (a NaN stays: what overflowed in a checkpoint has to reach the gradients)
        if constexpr (SLOPE) slope = g > 0.0f ? 1.0f : g <= 0.0f ? 0.0f : g;
        return g <= 0.0f ? 0.0f : g;
    }
}

// The same for two values at a time, to a few units in the last place of binary32: for results that are rounded to
// bfloat16.  2^x and 1/x are the units' own approximations, subnormal results flushed to zero.
__device__ __forceinline__ float fast_exp2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float fast_inverse(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ f2 f2_same(float v) { return f2_of(v, v); }
__device__ __forceinline__ f2 f2_add(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
// 1 / (1 + 2^z)
__device__ __forceinline__ f2 f2_logistic(f2 z)
{
    float a, b;
    f2_get(z, a, b);
    f2_get(f2_add(f2_of(fast_exp2(a), fast_exp2(b)), f2_same(1.0f)), a, b);
    return f2_of(fast_inverse(a), fast_inverse(b));
}
template <int ACT, bool SLOPE>
__device__ __forceinline__ f2 act2(f2 g, f2& slope)
{
    if constexpr (ACT == PALSGD_ACT_SILU) {
        const f2 s = f2_logistic(f2_mul(g, f2_same(-1.4426950408889634f)));
        const f2 a = f2_mul(g, s);
        if constexpr (SLOPE) slope = f2_fma(a, f2_fma(s, f2_same(-1.0f), f2_same(1.0f)), s);
        return a;
    } else if constexpr (ACT == PALSGD_ACT_GELU_TANH) {
        const float c = 1.5957691216057308f;                     // 2 sqrt(2/pi)
        const f2 gg = f2_mul(g, g);
        const f2 s = f2_logistic(f2_mul(f2_mul(g, f2_same(-1.4426950408889634f * c)), f2_fma(gg, f2_same(0.044715f), f2_same(1.0f))));
        const f2 a = f2_mul(g, s);
        if constexpr (SLOPE) {
            float x, y;
            f2_get(gg, x, y);
            const f2 m = f2_of(fminf(x, 1e18f), fminf(y, 1e18f));
            slope = f2_fma(f2_mul(a, f2_fma(s, f2_same(-1.0f), f2_same(1.0f))), f2_fma(m, f2_same(0.134145f * c), f2_same(c)), s);
        }
        return a;
    } else {
        float x, y, sx = 0.0f, sy = 0.0f;
        f2_get(g, x, y);
        const float ax = act<ACT, SLOPE, true>(x, sx), ay = act<ACT, SLOPE, true>(y, sy);
        if constexpr (SLOPE) slope = f2_of(sx, sy);
        return f2_of(ax, ay);
    }
}

__device__ __forceinline__ float f2_total(f2 v) { float a, b; f2_get(v, a, b); return a + b; }

// ---- eight values of a row at any address, the first `n` of them inside it (the others read as 0, and are not written).
// wide: eight values of every row start on a 16-byte boundary.
template <typename T>
__device__ __forceinline__ void row8_load(const T* p, uint32_t n, bool wide, f2 (&v)[4])
{
    const unsigned char* b = reinterpret_cast<const unsigned char*>(p);
    if constexpr (sizeof(T) == 2) {
        const uint4 q = wide && n >= 8 ? __ldg(reinterpret_cast<const uint4*>(p)) : get16(b, 2 * min(n, 8u));
        v[0] = f2_wide(q.x); v[1] = f2_wide(q.y); v[2] = f2_wide(q.z); v[3] = f2_wide(q.w);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i) {
            const uint4 q = wide && n >= 8 ? __ldg(reinterpret_cast<const uint4*>(p) + i) : get16(b + 16 * i, n > 4 * i ? 4 * min(n - 4 * i, 4u) : 0);
            v[2 * i] = f2_of(__uint_as_float(q.x), __uint_as_float(q.y)); v[2 * i + 1] = f2_of(__uint_as_float(q.z), __uint_as_float(q.w));
        }
    }
}
template <typename T>
__device__ __forceinline__ void row8_store(T* p, uint32_t n, bool wide, const f2 (&v)[4])
{
    unsigned char* b = reinterpret_cast<unsigned char*>(p);
    if constexpr (sizeof(T) == 2) {
        const uint4 q = make_uint4(f2_narrow(v[0]), f2_narrow(v[1]), f2_narrow(v[2]), f2_narrow(v[3]));
        if (wide && n >= 8) *reinterpret_cast<uint4*>(p) = q;
        else put16<2>(b, 2 * min(n, 8u), q);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i) {
            float x, y, z, w;
            f2_get(v[2 * i], x, y); f2_get(v[2 * i + 1], z, w);
            const uint4 q = make_uint4(__float_as_uint(x), __float_as_uint(y), __float_as_uint(z), __float_as_uint(w));
            if (wide && n >= 8) reinterpret_cast<uint4*>(p)[i] = q;
            else put16<4>(b + 16 * i, n > 4 * i ? 4 * min(n - 4 * i, 4u) : 0, q);
        }
    }
}

}  // namespace block
}  // namespace palsgd
