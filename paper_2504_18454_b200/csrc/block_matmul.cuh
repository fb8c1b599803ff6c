// Matrix kernels of the gated feed-forward block, on the fifth-generation tensor cores.
//
// One persistent kernel serves every product of the block.  A launch carries up to four problems (the four products of
// the backward pass have the same inputs and run as one launch), each a batch of K workers' products
//     C_k[m, n] = sum over segments s and kk of A_k,s(m, kk) B_k,s(n, kk)
// with either operand contiguous along kk or along m / n (the weight gradients contract over tokens: both operands are
// read transposed, which the copy engine and the tensor core's descriptors do without a separate transpose).
//
// A pair of CTAs (a cluster, on two SMs) computes a 256 x 256 tile: each CTA stages its 128 rows of A and its half of
// B by TMA, one thread of the leading CTA issues the pair's tcgen05.mma, and each CTA holds 128 x 256 binary32 sums in
// its tensor memory, twice, so that the epilogue of one tile overlaps the products of the next.
//   warp 0: TMA producer   warp 1: MMA issue (leading CTA)   warp 2: tensor memory   warps 4..11: epilogue
// fp32 operands come as three bfloat16 parts each; the products of parts i, j with i + j <= 2 are summed as so many more
// steps of the inner axis, the small ones first.
#pragma once
#include <cuda.h>

#include "block_common.cuh"

namespace palsgd {
namespace block {

enum { MAT_PLAIN = 0, MAT_GATED = 1, MAT_HIDDEN = 2 };

constexpr uint32_t kTileM = 256, kTileN = 256, kTileK = 64;
constexpr uint32_t kStages = 6;
constexpr uint32_t kOperandBytes = 128 * kTileK * 2;                    // a CTA's half of an operand's tile
constexpr uint32_t kStageBytes = 2 * kOperandBytes;
constexpr uint32_t kMatThreads = 384;
constexpr uint32_t kBarrierBytes = 256;
constexpr uint32_t kMatSmem = kStages * kStageBytes + kBarrierBytes + 1024;   // 1024: to start on a swizzle atom
constexpr uint32_t kMaxProblems = 4;
constexpr unsigned long long kWaitLimitNs = 4000000000ull;              // how long a wait polls before it gives up

struct MatOut {
    void*   p;
    int64_t w, r;                 // worker and row stride, elements
    int64_t part;                 // 0, or the stride between the three bfloat16 parts of an fp32 value
    int     wide;                 // rows start on 16-byte boundaries
};

struct alignas(64) MatProblem {
    CUtensorMap A[2], B[2];       // by segment; the gate/up pass: B[0] gate, B[1] up
    uint32_t M, N, Kd, tiles_m, tiles_n, tiles;
    uint8_t  n_seg, a_parts, b_parts, a_mn, b_mn;
    uint8_t  a_one[2], b_one[2];  // all workers read one matrix
    MatOut   out[3];              // plain: the product; gate/up: h; hidden: dg, du, h
};

struct MatLaunch {
    MatProblem p[kMaxProblems];
    uint32_t n_problems, tiles;
    int      act, save;
    MatOut   gate, up;            // saved (gate/up pass) or read (hidden pass)
    MatOut   gate_e, up_e;
    unsigned int* gave_up;
};

// ---------------------------------------------------------------------------------------------- PTX

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive_at(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// A wait that always ends: false, and the device-wide note, if the barrier's phase does not complete.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, unsigned int* gave_up)
{
    unsigned long long start = 0;
    for (uint32_t i = 0;; ++i) {
        uint32_t done;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
        if ((i & 63) == 63) {                                           // the clock is slow to read: not at every poll
            unsigned long long now;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
            if (start == 0) start = now;
            else if (now - start > kWaitLimitNs) break;
        }
    }
    atomicExch(gave_up, 1u);
    return false;
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.aligned.release;\n barrier.cluster.wait.aligned.acquire;" ::: "memory");
}
__device__ __forceinline__ void tma_load(const CUtensorMap* map, uint32_t dst, uint32_t cluster_bar, uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3)
{
    asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(cluster_bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar)                // to this barrier of both CTAs
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32])
{
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
                   "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
                   "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared-memory operand descriptor, 128-byte swizzle.  kk contiguous: rows of 128 bytes, groups of eight 1024 apart.
// m / n contiguous: blocks of 64 m (128 bytes) by kTileK rows of kk, 8192 apart; groups of eight kk 1024 apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn)
{
    const uint64_t lead = mn ? 8192 / 16 : 1;
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (lead << 16) | ((uint64_t)(1024 / 16) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

// ---------------------------------------------------------------------------------------------- epilogue memory access

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 32 consecutive values of a row, the first `n` of them inside the matrix
__device__ __forceinline__ void store_row(float* p, const float (&v)[32], uint32_t n, bool wide)
{
    if (wide && n >= 32) {
#pragma unroll
        for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) if (i < n) p[i] = v[i];
    }
}
__device__ __forceinline__ void store_row(bf16* p, const float (&v)[32], uint32_t n, bool wide)
{
    if (wide && n >= 32) {
#pragma unroll
        for (int i = 0; i < 32; i += 8)
            *reinterpret_cast<uint4*>(p + i) = make_uint4(pack2(v[i], v[i + 1]), pack2(v[i + 2], v[i + 3]), pack2(v[i + 4], v[i + 5]), pack2(v[i + 6], v[i + 7]));
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) if (i < n) p[i] = __float2bfloat16_rn(v[i]);
    }
}
template <typename T>
__device__ __forceinline__ void load_row(const T* p, float (&v)[32], uint32_t n, bool wide)
{
    if (wide && n >= 32) {
#pragma unroll
        for (int i = 0; i < 32; i += 8) Vec<T, 8>::load(p + i, v + i);
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = i < n ? to_f(p[i]) : 0.0f;
    }
}

// The next of the three bfloat16 parts of an fp32 value; v becomes the rest, exactly.  A finite value past the largest
// bfloat16 takes that as its part; the parts behind an infinity or a NaN are zero.
__device__ __forceinline__ float next_part(float& v)
{
    float hi = __bfloat162float(__float2bfloat16_rn(v));
    const bool finite = (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
    if (finite && (__float_as_uint(hi) & 0x7F800000u) == 0x7F800000u) hi = copysignf(__uint_as_float(0x7F7F0000u), v);
    v = finite ? __fsub_rn(v, hi) : 0.0f;
    return hi;
}

// An operand of the next product: bfloat16, or (part != 0) the three parts of an fp32 value.
template <typename T>
__device__ __forceinline__ void store_operand(const MatOut& o, int64_t at, float (&v)[32], uint32_t n)
{
    bf16* p = static_cast<bf16*>(o.p) + at;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int part = 0; part < 3; ++part) {
            float hi[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) hi[i] = next_part(v[i]);
            store_row(p + part * o.part, hi, n, o.wide);
        }
    } else {
        store_row(p, v, n, o.wide);
    }
}

__device__ __forceinline__ void store_act8(const MatOut& q, const MatOut& e, int64_t qo, int64_t eo, const float (&v)[32], uint32_t n)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, i < n ? __float_as_uint(v[i]) & 0x7FFFFFFFu : 0u);
    const uint32_t E = act8_exponent(m);
    const float inv = act8_inverse(E);
    int8_t* p = static_cast<int8_t*>(q.p) + qo;
    if (q.wide && n >= 32) {
#pragma unroll
        for (int i = 0; i < 32; i += 16) {
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j / 4] |= ((uint32_t)act8_quant(v[i + j], inv) & 0xFFu) << (8 * (j & 3));
            *reinterpret_cast<uint4*>(p + i) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) if (i < n) p[i] = (int8_t)act8_quant(v[i], inv);
    }
    static_cast<uint8_t*>(e.p)[eo] = (uint8_t)E;
}

__device__ __forceinline__ void load_act8(const MatOut& q, const MatOut& e, int64_t qo, int64_t eo, float (&v)[32], uint32_t n)
{
    const float s = act8_step(static_cast<const uint8_t*>(e.p)[eo]);
    const int8_t* p = static_cast<const int8_t*>(q.p) + qo;
    if (q.wide && n >= 32) {
#pragma unroll
        for (int i = 0; i < 32; i += 16) {
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(p + i));
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int j = 0; j < 16; ++j) v[i + j] = (float)(int8_t)(w[j / 4] >> (8 * (j & 3))) * s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = i < n ? (float)p[i] * s : 0.0f;
    }
}

// v <- act(v) * u  (gate/up);  dh, g, u -> dg, du, h  (hidden).  bfloat16 results take the fast exponential.
template <int ACT, bool FAST>
__device__ __forceinline__ void gate_row(float (&g)[32], const float (&u)[32])
{
    float unused;
#pragma unroll
    for (int i = 0; i < 32; ++i) g[i] = act<ACT, false, FAST>(g[i], unused) * u[i];
}
template <int ACT, bool FAST>
__device__ __forceinline__ void hidden_row(float (&dh)[32], float (&g)[32], float (&u)[32])
{
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        float slope;
        const float a = act<ACT, true, FAST>(g[i], slope), d = dh[i];
        g[i] = d * u[i] * slope;                                        // dg
        dh[i] = a * u[i];                                               // h
        u[i] = d * a;                                                   // du
    }
}

// ---------------------------------------------------------------------------------------------- the kernel

struct Tile { uint32_t worker, m0, n0; const MatProblem* p; };

template <int MODE>
__device__ __forceinline__ Tile tile_at(const MatLaunch& a, uint32_t t)
{
    uint32_t i = 0;
    while (i + 1 < a.n_problems && t >= a.p[i].tiles) { t -= a.p[i].tiles; ++i; }
    const MatProblem& p = a.p[i];
    const uint32_t per = p.tiles_m * p.tiles_n, w = t / per, r = t - w * per, m = r % p.tiles_m, n = r / p.tiles_m;
    return Tile{w, m * kTileM, n * (MODE == MAT_GATED ? kTileN / 2 : kTileN), &p};
}

__device__ __forceinline__ uint32_t pairs_of(const MatProblem& p) { return p.a_parts == 1 ? p.b_parts : p.b_parts == 1 ? p.a_parts : 6; }

template <typename T, int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMatThreads, 1) mat_kernel(const __grid_constant__ MatLaunch a)
{
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_addr(smem_raw) + 1023) & ~1023u;
    const uint32_t bars = base + kStages * kStageBytes;
    const uint32_t full = bars, empty = bars + 8 * kStages, acc_full = bars + 16 * kStages, acc_empty = acc_full + 16, tmem_at = acc_empty + 16;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = cluster_rank();
    const uint32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < kStages; ++s) { bar_init(full + 8 * s, 1); bar_init(empty + 8 * s, 1); }
        for (uint32_t s = 0; s < 2; ++s) { bar_init(acc_full + 8 * s, 1); bar_init(acc_empty + 8 * s, 16); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_at), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_at));

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, phase = 0, used = 0;
            bool ok = true;
            for (uint32_t t = pair; ok && t < a.tiles; t += pairs) {
                const Tile tl = tile_at<MODE>(a, t);
                const MatProblem& p = *tl.p;
                const uint32_t am = tl.m0 + rank * 128;
                const uint32_t bn = MODE == MAT_GATED ? tl.n0 : tl.n0 + rank * 128;
                for (uint32_t seg = 0; ok && seg < p.n_seg; ++seg) {
                    const uint32_t bi = MODE == MAT_GATED ? rank : seg;
                    const uint32_t aw = p.a_one[seg] ? 0 : tl.worker, bw = p.b_one[bi] ? 0 : tl.worker;
                    for (int sum = 2; ok && sum >= 0; --sum)
                        for (int pa = 0; ok && pa <= sum; ++pa) {
                            const int pb = sum - pa;
                            if (pa >= p.a_parts || pb >= p.b_parts) continue;
                            for (uint32_t k = 0; k < p.Kd; k += kTileK) {
                                if (!bar_wait(empty + 8 * s, phase ^ 1, a.gave_up)) { ok = false; break; }
                                const uint32_t fb = in_cta(full + 8 * s, 0);
                                if (rank == 0) bar_expect(full + 8 * s, 2 * kStageBytes);
                                const uint32_t da = base + s * kStageBytes, db = da + kOperandBytes;
                                if (p.a_mn) {
                                    tma_load(&p.A[seg], da, fb, am, k, aw, pa);
                                    tma_load(&p.A[seg], da + 8192, fb, am + 64, k, aw, pa);
                                } else {
                                    tma_load(&p.A[seg], da, fb, k, am, aw, pa);
                                }
                                if (p.b_mn) {
                                    tma_load(&p.B[bi], db, fb, bn, k, bw, pb);
                                    tma_load(&p.B[bi], db + 8192, fb, bn + 64, k, bw, pb);
                                } else {
                                    tma_load(&p.B[bi], db, fb, k, bn, bw, pb);
                                }
                                if (used < kStages) ++used;
                                if (++s == kStages) { s = 0; phase ^= 1; }
                            }
                        }
                }
            }
            // every stage that was filled is drained before the CTA may leave: no copy or arrival is under way then
            for (uint32_t i = 0; i < used; ++i) {
                if (s == 0) { s = kStages; phase ^= 1; }
                --s;
                bar_wait(empty + 8 * s, phase, a.gave_up);
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            uint32_t s = 0, phase = 0, it = 0;
            bool ok = true;
            for (uint32_t t = pair; ok && t < a.tiles; t += pairs, ++it) {
                const Tile tl = tile_at<MODE>(a, t);
                const MatProblem& p = *tl.p;
                const uint32_t steps = p.n_seg * pairs_of(p) * ((p.Kd + kTileK - 1) / kTileK);
                // binary32 sums; bfloat16 operands; majors; N / 8; M / 16
                const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)p.a_mn << 15) | ((uint32_t)p.b_mn << 16) | ((kTileN / 8) << 17) | ((kTileM / 16) << 24);
                const uint32_t acc = it & 1, d = tmem + acc * kTileN;
                const uint64_t da = operand_desc(base, p.a_mn), db = operand_desc(base + kOperandBytes, p.b_mn);
                const uint32_t sa = p.a_mn ? 2048 / 16 : 32 / 16, sb = p.b_mn ? 2048 / 16 : 32 / 16;
                if (!bar_wait(acc_empty + 8 * acc, (it >> 1 & 1) ^ 1, a.gave_up)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (uint32_t k = 0; k < steps; ++k) {
                    if (!bar_wait(full + 8 * s, phase, a.gave_up)) { ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (uint32_t j = 0; j < kTileK / 16; ++j)
                        mma(d, da + s * (kStageBytes / 16) + j * sa, db + s * (kStageBytes / 16) + j * sb, idesc, k > 0 || j > 0);
                    mma_commit(empty + 8 * s);
                    if (++s == kStages) { s = 0; phase ^= 1; }
                }
                if (ok) mma_commit(acc_full + 8 * acc);
            }
        }
    } else if (warp >= 4) {
        const uint32_t quad = warp & 3, half = (warp - 4) >> 2;           // tensor memory rows of 32; half of the columns
        uint32_t it = 0;
        for (uint32_t t = pair; t < a.tiles; t += pairs, ++it) {
            const Tile tl = tile_at<MODE>(a, t);
            const MatProblem& p = *tl.p;
            const uint32_t acc = it & 1, src = tmem + acc * kTileN + (quad << 21);
            const uint32_t m = tl.m0 + rank * 128 + quad * 32 + lane;
            const bool row = m < p.M;
            const bool ok = bar_wait(acc_full + 8 * acc, it >> 1 & 1, a.gave_up);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            constexpr uint32_t kChunks = MODE == MAT_GATED ? 2 : 4;
#pragma unroll 1
            for (uint32_t c = 0; c < kChunks; ++c) {
                const uint32_t col = (half * kChunks + c) * 32, n = tl.n0 + col;
                const bool on = row && n < p.N;
                const uint32_t left = p.N - n;
                float v[32], u[32];
                tmem_load32(src + col, v);
                if constexpr (MODE == MAT_GATED) tmem_load32(src + kTileN / 2 + col, u);
                tmem_load_wait();
                if (on) {
                const int64_t w = tl.worker;
                const int64_t at = w * p.out[0].w + (int64_t)m * p.out[0].r + n;
                if constexpr (MODE == MAT_PLAIN) {
                    store_row(static_cast<T*>(p.out[0].p) + at, v, left, p.out[0].wide);
                } else {
                    const int64_t go = w * a.gate.w + (int64_t)m * a.gate.r + n, uo = w * a.up.w + (int64_t)m * a.up.r + n;
                    const int64_t geo = w * a.gate_e.w + (int64_t)m * a.gate_e.r + n / 32, ueo = w * a.up_e.w + (int64_t)m * a.up_e.r + n / 32;
                    constexpr bool kFast = sizeof(T) == 2;
                    if constexpr (MODE == MAT_GATED) {
                        if (a.save == PALSGD_SAVE_FULL) {
                            store_row(static_cast<T*>(a.gate.p) + go, v, left, a.gate.wide);
                            store_row(static_cast<T*>(a.up.p) + uo, u, left, a.up.wide);
                        } else if (a.save == PALSGD_SAVE_8BIT) {
                            store_act8(a.gate, a.gate_e, go, geo, v, left);
                            store_act8(a.up, a.up_e, uo, ueo, u, left);
                        }
                        switch (a.act) {
                            case PALSGD_ACT_SILU: gate_row<PALSGD_ACT_SILU, kFast>(v, u); break;
                            case PALSGD_ACT_GELU: gate_row<PALSGD_ACT_GELU, kFast>(v, u); break;
                            case PALSGD_ACT_GELU_TANH: gate_row<PALSGD_ACT_GELU_TANH, kFast>(v, u); break;
                            default: gate_row<PALSGD_ACT_RELU, kFast>(v, u);
                        }
                        store_operand<T>(p.out[0], at, v, left);
                    } else {
                        float g[32];
                        if (a.save == PALSGD_SAVE_FULL) {
                            load_row(static_cast<const T*>(a.gate.p) + go, g, left, a.gate.wide);
                            load_row(static_cast<const T*>(a.up.p) + uo, u, left, a.up.wide);
                        } else {
                            load_act8(a.gate, a.gate_e, go, geo, g, left);
                            load_act8(a.up, a.up_e, uo, ueo, u, left);
                        }
                        switch (a.act) {
                            case PALSGD_ACT_SILU: hidden_row<PALSGD_ACT_SILU, kFast>(v, g, u); break;
                            case PALSGD_ACT_GELU: hidden_row<PALSGD_ACT_GELU, kFast>(v, g, u); break;
                            case PALSGD_ACT_GELU_TANH: hidden_row<PALSGD_ACT_GELU_TANH, kFast>(v, g, u); break;
                            default: hidden_row<PALSGD_ACT_RELU, kFast>(v, g, u);
                        }
                        store_operand<T>(p.out[0], at, g, left);
                        store_operand<T>(p.out[1], at, u, left);
                        store_operand<T>(p.out[2], at, v, left);
                    }
                }
                }
                __syncwarp();                                             // the next load from tensor memory is the whole warp's
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive_at(in_cta(acc_empty + 8 * acc, 0));
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

// ---------------------------------------------------------------------------------------------- operands to copy first

// Matrices that the copy engine cannot read in place, rewritten for it: rows of bfloat16 on 16-byte boundaries; an fp32
// matrix as its three bfloat16 parts (x - hi and the next difference are exact in binary32); an 8-bit checkpoint as the
// bfloat16 values that it stands for.
enum { STAGE_BF16 = 0, STAGE_SPLIT = 1, STAGE_ACT8 = 2 };
constexpr uint32_t kMaxStaged = 5;

struct StageItem {
    const void* src; const uint8_t* e;
    int64_t  w, r, ew, er;        // strides of src and of the exponents
    bf16*    dst;
    int64_t  ld, part;            // row stride (multiple of 8) and part stride of dst; workers are rows * ld apart
    uint32_t rows, cols;
    uint64_t units;               // of 8 columns, one worker
    int      kind;
    uint32_t K;                   // workers to copy: 1 if all read one matrix
};
struct StageArgs { StageItem item[kMaxStaged]; };

__global__ void __launch_bounds__(256) stage_kernel(const __grid_constant__ StageArgs a)
{
    const StageItem& it = a.item[blockIdx.y];
    const uint32_t per = (uint32_t)(it.ld / 8);
    const int64_t k = blockIdx.z;
    if (k >= it.K) return;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < it.units; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = it.units < 0x80000000ull ? (uint32_t)i / per : i / per;
        const uint32_t c = (uint32_t)(i - row * per) * 8;
        const int64_t from = k * it.w + (int64_t)row * it.r + c;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = 0.0f;
            if (c + j < it.cols) {
                if (it.kind == STAGE_BF16) v[j] = to_f(static_cast<const bf16*>(it.src)[from + j]);
                else if (it.kind == STAGE_SPLIT) v[j] = static_cast<const float*>(it.src)[from + j];
                else v[j] = (float)static_cast<const int8_t*>(it.src)[from + j];
            }
        }
        if (it.kind == STAGE_ACT8) {
            const float s = act8_step(it.e[k * it.ew + (int64_t)row * it.er + c / 32]);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= s;
        }
        bf16* to = it.dst + (k * it.rows + (int64_t)row) * it.ld + c;
        if (it.kind == STAGE_SPLIT) {
#pragma unroll
            for (int part = 0; part < 3; ++part) {
                float hi[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) hi[j] = next_part(v[j]);
                Vec<bf16, 8>::store(to + part * it.part, hi);
            }
        } else {
            Vec<bf16, 8>::store(to, v);
        }
    }
}

struct ZeroArgs { void* p[3]; int64_t w[3], r[3]; uint32_t rows[3], cols[3]; };

template <typename T>
__global__ void __launch_bounds__(256) zero_kernel(const __grid_constant__ ZeroArgs a)
{
    const uint32_t i = blockIdx.y;
    T* p = static_cast<T*>(a.p[i]) + (int64_t)blockIdx.z * a.w[i];
    for (uint32_t r = blockIdx.x; r < a.rows[i]; r += gridDim.x)
        for (uint32_t c = threadIdx.x; c < a.cols[i]; c += 256) p[(int64_t)r * a.r[i] + c] = from_f<T>(0.0f);
}

}  // namespace block
}  // namespace palsgd
