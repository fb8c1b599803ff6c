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
//   warps 0, 3: TMA producers   warp 1: MMA issue (leading CTA)   warp 2: tensor memory   warps 4..: epilogue
// fp32 operands come as three bfloat16 parts each; the products of parts i, j with i + j <= 2 are summed as so many more
// steps of the inner axis, the small ones first.
#pragma once
#include <cuda.h>

#include "block_common.cuh"

namespace palsgd {
namespace block {

enum { MAT_PLAIN = 0, MAT_GATED = 1, MAT_HIDDEN = 2 };

constexpr uint32_t kTileM = 256, kTileN = 256, kTileK = 64;
constexpr uint32_t kOperandBytes = 128 * kTileK * 2;                    // a CTA's half of an operand's tile
constexpr uint32_t kStageBytes = 2 * kOperandBytes;
constexpr uint32_t kBarrierBytes = 256;
constexpr uint32_t kPiece = 8;                                          // fp32: steps of kTileK between two roundings to binary32

// Shared memory and warps of a kernel: 16 epilogue warps of 64 columns each (8 of 128 took three times as long in the
// hidden pass: two warps a scheduler do not cover each other's latencies).  bfloat16: they pass their results (and, in
// the hidden pass, gate and up) through blocks of 32 x 32 in shared memory.  fp32: they hold their sums in registers.
template <typename T, int MODE>
struct MatShape {
    static constexpr bool kWide = sizeof(T) == 4;
    static constexpr uint32_t kEpilogue = 16;
    static constexpr uint32_t kThreads = 128 + 32 * kEpilogue;
    static constexpr uint32_t kBlocks = kWide ? 0 : MODE == MAT_HIDDEN ? 2 : 1;   // of 2048 bytes, a warp
    static constexpr uint32_t kStages = !kWide && MODE == MAT_HIDDEN ? 5 : 6;
    static constexpr uint32_t kSmem = kStages * kStageBytes + kEpilogue * kBlocks * 2048 + kBarrierBytes + 1024;   // 1024: to start on a swizzle atom
    static_assert(kSmem <= 232448, "shared memory of a CTA");
};
constexpr uint32_t kMaxProblems = 4;
constexpr uint32_t kTileEnd = 3;                                        // what a tile costs beside its steps, in steps
constexpr unsigned long long kWaitLimitNs = 4000000000ull;              // how long a wait polls before it gives up

struct MatOut {
    void*   p;
    int64_t w, r;                 // worker and row stride, elements
    int64_t part;                 // 0, or the stride between the three bfloat16 parts of an fp32 value
    int     wide;                 // rows start on 16-byte boundaries
    uint32_t cols;                // columns that may be written: the workspace's rows have room behind their end
};

// Division of t < 2^31 by a divisor d known on the host: with s = ceil(log2 d) and m = ceil(2^(31+s) / d) < 2^32, the
// quotient is t m >> (31 + s) (m d exceeds 2^(31+s) by less than 2^s, and t times that stays below 2^(31+s)).
struct Divisor {
    uint32_t d, m, s;
    __device__ __forceinline__ uint32_t of(uint32_t t) const { return (uint32_t)(((uint64_t)t * m) >> (31 + s)); }
};

struct alignas(64) MatProblem {
    CUtensorMap A[2], B[2];       // by segment; the gate/up pass: B[0] gate, B[1] up
    uint32_t M, N, Kd, tiles;
    Divisor  tiles_m, per_worker; // tiles down, tiles of one worker
    uint8_t  n_seg, a_parts, b_parts, a_mn, b_mn;
    uint8_t  a_one[2], b_one[2];  // all workers read one matrix
    MatOut   out[3];              // plain: the product; gate/up: h; hidden: dg, du, h
};

struct MatLaunch {
    MatProblem p[kMaxProblems];
    uint32_t n_problems, tiles, heavy, lag;   // see Order
    int      save;
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
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// A wait that always ends: false, and the device-wide note, if the barrier's phase does not complete.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, unsigned int* gave_up)
{
    unsigned long long start = 0;
    for (uint32_t i = 0;; ++i) {
        uint32_t done;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
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
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16])
{
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load8(uint32_t addr, float (&v)[8])
{
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_store4(uint32_t addr, const uint32_t (&r)[4])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared-memory operand descriptor, 128-byte swizzle.  kk contiguous: rows of 128 bytes, groups of eight 1024 apart.
// m / n contiguous: blocks of 64 m (128 bytes) by kTileK rows of kk, 8192 apart; groups of eight kk 1024 apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn)
{
    const uint64_t lead = mn ? 8192 / 16 : 1;
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (lead << 16) | ((uint64_t)(1024 / 16) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

// ---------------------------------------------------------------------------------------------- epilogue memory access

__device__ __forceinline__ void lds128(uint32_t at, uint4& v)
{
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
}
__device__ __forceinline__ void sts128(uint32_t at, const uint4& v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// A block of 32 rows (one a lane) by 32 columns that a warp passes through shared memory on its way between rows and
// coalesced accesses.  ROW bytes a row; the 16-byte pieces of a row are permuted so that neither side has bank conflicts.
template <int ROW>
__device__ __forceinline__ uint32_t block_at(uint32_t base, uint32_t row, uint32_t piece)
{
    constexpr uint32_t kPieces = ROW / 16;                // 8, 4 or 2
    const uint32_t turn = kPieces == 8 ? row & 7 : kPieces == 4 ? (row >> 1) & 3 : (row >> 2) & 1;
    return base + row * ROW + ((piece ^ turn) << 4);
}

// Block -> matrix: `rows` (at most 32) rows and `cols` columns of it are inside.  E: the element type's size.
template <int ROW, int E>
__device__ __noinline__ void block_out_edge(uint32_t base, unsigned char* to, int64_t row_bytes, uint32_t rows, uint32_t cols, bool wide, uint32_t lane)
{
    constexpr uint32_t kPer = 16 / E;
    if (wide) {
        constexpr uint32_t kPieces = ROW / 16;
        const uint32_t piece = lane % kPieces;
#pragma unroll 1
        for (uint32_t row = lane / kPieces; row < rows; row += 32 / kPieces) {
            uint4 v;
            lds128(block_at<ROW>(base, row, piece), v);
            unsigned char* p = to + (int64_t)row * row_bytes + piece * 16;
            if ((piece + 1) * kPer <= cols) {
                *reinterpret_cast<uint4*>(p) = v;
            } else {                                      // the row ends inside these 16 bytes, or before them
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (uint32_t j = 0; j < kPer; ++j)
                    if (piece * kPer + j < cols) {
                        if constexpr (E == 2) reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
                        else p[j] = (unsigned char)(w[j / 4] >> (8 * (j & 3)));
                    }
            }
        }
    } else if (lane < cols) {                             // one column a lane
#pragma unroll 1
        for (uint32_t row = 0; row < rows; ++row) {
            const uint32_t at = block_at<ROW>(base, row, lane / kPer) + (lane % kPer) * E;
            unsigned char* p = to + (int64_t)row * row_bytes + lane * E;
            if constexpr (E == 2) {
                uint16_t v;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
                *reinterpret_cast<uint16_t*>(p) = v;
            } else {
                uint32_t v;
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at));
                *p = (unsigned char)v;
            }
        }
    }
}
template <int ROW, int E>
__device__ __forceinline__ void block_out(uint32_t base, unsigned char* to, int64_t row_bytes, uint32_t rows, uint32_t cols, bool wide, uint32_t lane)
{
    constexpr uint32_t kPieces = ROW / 16;
    if (rows == 32 && cols >= 32 && wide) {               // the same for the whole warp
        const uint32_t piece = lane % kPieces, row = lane / kPieces;
        unsigned char* p = to + (int64_t)row * row_bytes + piece * 16;
        const int64_t step = row_bytes * (32 / kPieces);
        uint4 v[kPieces];
#pragma unroll
        for (uint32_t i = 0; i < kPieces; ++i) lds128(block_at<ROW>(base, i * (32 / kPieces) + row, piece), v[i]);
#pragma unroll
        for (uint32_t i = 0; i < kPieces; ++i) { *reinterpret_cast<uint4*>(p) = v[i]; p += step; }
    } else if (rows && cols) {
        block_out_edge<ROW, E>(base, to, row_bytes, rows, cols, wide, lane);
    }
}

// Matrix -> block of 64-byte rows, asynchronously where the rows are aligned; zeros outside.  Complete after block_wait and
// __syncwarp.  bfloat16 fills a row; int8 its second half, so that a lane can write its bfloat16 results over its row from
// the front while it still reads.
template <int E>
__device__ __noinline__ void block_in_edge(uint32_t base, const unsigned char* from, int64_t row_bytes, uint32_t rows, uint32_t cols, bool wide, uint32_t lane)
{
    constexpr uint32_t kPieces = 2 * E, kPer = 16 / E, kFirst = E == 1 ? 2 : 0;
    if (wide) {
        const uint32_t piece = lane % kPieces;
        const uint32_t inside = piece * kPer < cols ? (cols - piece * kPer < kPer ? cols - piece * kPer : kPer) * E : 0;
#pragma unroll 1
        for (uint32_t row = lane / kPieces; row < 32; row += 32 / kPieces) {
            const uint32_t n = row < rows ? inside : 0;
            const unsigned char* p = n ? from + (int64_t)row * row_bytes + piece * 16 : from;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(block_at<64>(base, row, kFirst + piece)), "l"(p), "r"(n) : "memory");
        }
    } else {
#pragma unroll 1
        for (uint32_t row = 0; row < 32; ++row) {
            const uint32_t at = block_at<64>(base, row, kFirst + lane / kPer) + (lane % kPer) * E;
            const unsigned char* p = from + (int64_t)row * row_bytes + lane * E;
            const bool on = row < rows && lane < cols;
            if constexpr (E == 2) {
                const uint16_t v = on ? *reinterpret_cast<const uint16_t*>(p) : (uint16_t)0;
                asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(v) : "memory");
            } else {
                const uint32_t v = on ? *p : 0u;
                asm volatile("st.shared.u8 [%0], %1;" ::"r"(at), "r"(v) : "memory");
            }
        }
    }
}
template <int E>
__device__ __forceinline__ void block_in(uint32_t base, const unsigned char* from, int64_t row_bytes, uint32_t rows, uint32_t cols, bool wide, uint32_t lane)
{
    constexpr uint32_t kPieces = 2 * E, kFirst = E == 1 ? 2 : 0;
    if (rows == 32 && cols >= 32 && wide) {
        const uint32_t piece = lane % kPieces, row = lane / kPieces;
        const unsigned char* p = from + (int64_t)row * row_bytes + piece * 16;
        const int64_t step = row_bytes * (32 / kPieces);
#pragma unroll
        for (uint32_t i = 0; i < kPieces; ++i) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(block_at<64>(base, i * (32 / kPieces) + row, kFirst + piece)), "l"(p) : "memory");
            p += step;
        }
    } else if (rows && cols) {                            // (a block that is all outside is not read)
        block_in_edge<E>(base, from, row_bytes, rows, cols, wide, lane);
    }
}
__device__ __forceinline__ void block_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Eight columns of a lane's row of a bfloat16 block, as pairs of floats
__device__ __forceinline__ void row_put(uint32_t base, uint32_t lane, uint32_t j, const f2 (&v)[4])
{
    sts128(block_at<64>(base, lane, j), make_uint4(f2_narrow(v[0]), f2_narrow(v[1]), f2_narrow(v[2]), f2_narrow(v[3])));
}
__device__ __forceinline__ void row_get(uint32_t base, uint32_t lane, uint32_t j, f2 (&v)[4])
{
    uint4 a;
    lds128(block_at<64>(base, lane, j), a);
    v[0] = f2_wide(a.x); v[1] = f2_wide(a.y); v[2] = f2_wide(a.z); v[3] = f2_wide(a.w);
}
// ... of an 8-bit block: written in rows of 32 bytes, read where block_in puts it
__device__ __forceinline__ void row_put_act8(uint32_t base, uint32_t lane, uint32_t j, float inv, const float* v)
{
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(block_at<32>(base, lane, j >> 1) + (j & 1) * 8),
                 "r"(act8_quant4(v[0], v[1], v[2], v[3], inv)), "r"(act8_quant4(v[4], v[5], v[6], v[7], inv)) : "memory");
}
__device__ __forceinline__ void row_get_act8(uint32_t base, uint32_t lane, uint32_t j, float step, f2 (&v)[4])
{
    uint2 a;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(a.x), "=r"(a.y) : "r"(block_at<64>(base, lane, 2 + (j >> 1)) + (j & 1) * 8));
    float f[8];
    act8_value4(a.x, step, f);
    act8_value4(a.y, step, f + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = f2_of(f[2 * i], f[2 * i + 1]);
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

// fp32 results go out row by row, eight columns at a time (`n` of them inside): six times the products stand behind each.
__device__ __forceinline__ void store8(float* p, const float* v, uint32_t n, bool wide)
{
    if (wide && n >= 8) {
        Vec<float, 8>::store(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) p[i] = v[i];
    }
}
__device__ __forceinline__ void load8(const float* p, float* v, uint32_t n, bool wide)
{
    if (wide && n >= 8) {
        Vec<float, 8>::load(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void store8_parts(const MatOut& o, int64_t at, float* v)
{
    bf16* p = static_cast<bf16*>(o.p) + at;               // the workspace: rows are padded to eight columns
#pragma unroll
    for (int part = 0; part < 3; ++part) {
        float hi[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) hi[i] = next_part(v[i]);
        Vec<bf16, 8>::store(p + part * o.part, hi);
    }
}
__device__ __forceinline__ void store8_act8(const MatOut& q, int64_t at, const float* v, float inv, uint32_t n)
{
    int8_t* p = static_cast<int8_t*>(q.p) + at;
    const uint32_t w[2] = {act8_quant4(v[0], v[1], v[2], v[3], inv), act8_quant4(v[4], v[5], v[6], v[7], inv)};
    if (q.wide && n >= 8) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) p[i] = (int8_t)(w[i / 4] >> (8 * (i & 3)));
    }
}
__device__ __forceinline__ void load8_act8(const MatOut& q, int64_t at, float* v, float step, uint32_t n)
{
    const int8_t* p = static_cast<const int8_t*>(q.p) + at;
    uint32_t w[2] = {0, 0};
    if (q.wide && n >= 8) {
        const uint2 a = __ldg(reinterpret_cast<const uint2*>(p));
        w[0] = a.x; w[1] = a.y;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) w[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
    }
    act8_value4(w[0], step, v);
    act8_value4(w[1], step, v + 4);
}

// fp32, eight columns: g <- act(g) * u  (gate/up);  dh, g, u -> h, dg, du  (hidden)
template <int ACT>
__device__ __forceinline__ void gate8(float* g, const float* u)
{
    float unused;
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = act<ACT, false, false>(g[i], unused) * u[i];
}
template <int ACT>
__device__ __forceinline__ void hidden8(float* dh, float* g, float* u)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float slope;
        const float a = act<ACT, true, false>(g[i], slope), d = dh[i];
        g[i] = d * u[i] * slope;                                        // dg
        dh[i] = a * u[i];                                               // h
        u[i] = d * a;                                                   // du
    }
}

// ---------------------------------------------------------------------------------------------- the kernel

// The tiles of a launch in the order in which its pairs of CTAs take them up: first the `heavy` ones, then the rest.  The
// heavy ones go round the pairs; where they do not come out even, the pairs that have one less take up light ones for as
// long (`lag` of them fit beside a heavy one), so that all pairs end within a light tile of each other.  Every pair works
// out its own tiles: a pair's step `j` among the light ones is preceded by those that the others take up before that time.
// (Round and round alone left the tensor cores idle for a fifth of the backward pass of 8 workers, 768 x 2048.)
struct Order {
    uint32_t heavy, tiles, lag, pair, pairs, mine, more, j;
    __device__ __forceinline__ Order(const MatLaunch& a, uint32_t pair_, uint32_t pairs_)
        : heavy(a.heavy), tiles(a.tiles), lag(a.lag), pair(pair_), pairs(pairs_), j(0)
    {
        mine = heavy / pairs;
        more = heavy - mine * pairs;                      // this many pairs have one more
        mine += pair < more;
    }
    __device__ __forceinline__ uint32_t at(uint32_t i) const    // the pair's i-th tile; `tiles`: none
    {
        uint64_t t;
        const uint64_t k = i - mine;
        if (i < mine) t = pair + (uint64_t)i * pairs;
        else if (more == 0) t = heavy + pair + k * pairs;
        else if (pair >= more) t = heavy + (pairs - more) * k + (pair - more) + more * (k > lag ? k - lag : 0);
        else t = heavy + more * k + pair + (pairs - more) * (k + lag + 1);
        return t < tiles ? (uint32_t)t : tiles;
    }
    __device__ __forceinline__ uint32_t now() const { return at(j); }
    __device__ __forceinline__ uint32_t then() const { return at(j + 1); }
    __device__ __forceinline__ void next() { ++j; }
};

struct Tile { uint32_t worker, m0, n0; const MatProblem* p; };

template <int MODE>
__device__ __forceinline__ Tile tile_at(const MatLaunch& a, uint32_t t)
{
    uint32_t i = 0;
    while (i + 1 < a.n_problems && t >= a.p[i].tiles) { t -= a.p[i].tiles; ++i; }
    const MatProblem& p = a.p[i];
    const uint32_t w = p.per_worker.of(t), r = t - w * p.per_worker.d, n = p.tiles_m.of(r), m = r - n * p.tiles_m.d;
    return Tile{w, m * kTileM, n * (MODE == MAT_GATED ? kTileN / 2 : kTileN), &p};
}

__device__ __forceinline__ uint32_t pairs_of(const MatProblem& p) { return p.a_parts == 1 ? p.b_parts : p.b_parts == 1 ? p.a_parts : 6; }

// The inner axis of a tile in pieces, each a sum of its own in tensor memory: f(segment, first step, end, last piece).
// bfloat16: one piece a segment, joined in tensor memory.  fp32: kPiece steps (with all their parts), joined in registers
// with rounding to nearest -- the tensor cores cut off what an addition does not hold, which over long sums adds up
// (measured over 4096 steps of the inner axis in one piece: 4.4e-6 of the result's norm).
template <typename T, typename F>
__device__ __forceinline__ bool for_pieces(const MatProblem& p, F&& f)
{
    const uint32_t steps = (p.Kd + kTileK - 1) / kTileK, piece = sizeof(T) == 4 ? kPiece : steps;
    for (uint32_t seg = 0; seg < p.n_seg; ++seg)
        for (uint32_t k = 0; k < steps; k += piece)
            if (!f(seg, k, k + piece < steps ? k + piece : steps)) return false;
    return true;
}

// (The activation is a parameter of the template: with all four in one kernel the epilogue outgrew the instruction cache.)
template <typename T, int MODE, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MatShape<T, MODE>::kThreads, 1) mat_kernel(const __grid_constant__ MatLaunch a)
{
    using Shape = MatShape<T, MODE>;
    constexpr uint32_t kStages = Shape::kStages;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_addr(smem_raw) + 1023) & ~1023u;
    const uint32_t blocks = base + kStages * kStageBytes, bars = blocks + Shape::kEpilogue * Shape::kBlocks * 2048;
    const uint32_t full = bars, empty = bars + 8 * kStages, acc_full = bars + 16 * kStages, acc_empty = acc_full + 16, tmem_at = acc_empty + 16;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = cluster_rank();
    const uint32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < kStages; ++s) { bar_init(full + 8 * s, 1); bar_init(empty + 8 * s, 1); }
        for (uint32_t s = 0; s < 2; ++s) { bar_init(acc_full + 8 * s, 1); bar_init(acc_empty + 8 * s, 2 * Shape::kEpilogue); }
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

    if (warp == 0 || warp == 3) {
        // producers: warp 0 brings A, warp 3 brings B (one thread that did both held the copy engine up: 410 ns a step of
        // 32 KB, of which 120 its own)
        if (lane == 0) {
            const bool is_b = warp == 3;
            const uint32_t dst = base + (is_b ? kOperandBytes : 0), signal = in_cta(full, 0);
            uint32_t s = 0, phase = 0, used = 0;
            bool ok = true;
            for (Order o(a, pair, pairs); ok && o.now() < a.tiles; o.next()) {
                const uint32_t t = o.now();
                const Tile tl = tile_at<MODE>(a, t);
                const MatProblem& p = *tl.p;
                const uint32_t mn = is_b ? (MODE == MAT_GATED ? tl.n0 : tl.n0 + rank * 128) : tl.m0 + rank * 128;
                const bool across = is_b ? p.b_mn : p.a_mn;
                const int parts_a = p.a_parts, parts_b = p.b_parts;
                ok = for_pieces<T>(p, [&](uint32_t seg, uint32_t from, uint32_t to) {
                    const uint32_t i = is_b && MODE == MAT_GATED ? rank : seg;
                    const CUtensorMap* const map = is_b ? &p.B[i] : &p.A[i];
                    const uint32_t w = (is_b ? p.b_one[i] : p.a_one[i]) ? 0 : tl.worker;
                    for (int sum = sizeof(T) == 4 ? 2 : 0; sum >= 0; --sum)
                        for (int pa = 0; pa <= sum; ++pa) {
                            if (pa >= parts_a || sum - pa >= parts_b) continue;
                            const uint32_t part = is_b ? sum - pa : pa;
                            for (uint32_t k = from * kTileK; k < to * kTileK; k += kTileK) {
                                if (!bar_wait(empty + 8 * s, phase ^ 1, a.gave_up)) return false;
                                if (!is_b && rank == 0) bar_expect(full + 8 * s, 2 * kStageBytes);
                                const uint32_t to_s = dst + s * kStageBytes, bar = signal + 8 * s;
                                if (across) {
                                    tma_load(map, to_s, bar, mn, k, w, part);
                                    tma_load(map, to_s + 8192, bar, mn + 64, k, w, part);
                                } else {
                                    tma_load(map, to_s, bar, k, mn, w, part);
                                }
                                if (used < kStages) ++used;
                                if (++s == kStages) { s = 0; phase ^= 1; }
                            }
                        }
                    return true;
                });
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
            for (Order o(a, pair, pairs); ok && o.now() < a.tiles; o.next()) {
                const uint32_t t = o.now();
                const Tile tl = tile_at<MODE>(a, t);
                const MatProblem& p = *tl.p;
                const uint32_t n_pairs = pairs_of(p);
                // binary32 sums; bfloat16 operands; majors; N / 8; M / 16
                const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)p.a_mn << 15) | ((uint32_t)p.b_mn << 16) | ((kTileN / 8) << 17) | ((kTileM / 16) << 24);
                const uint64_t da = operand_desc(base, p.a_mn), db = operand_desc(base + kOperandBytes, p.b_mn);
                const uint32_t sa = p.a_mn ? 2048 / 16 : 32 / 16, sb = p.b_mn ? 2048 / 16 : 32 / 16;
                ok = for_pieces<T>(p, [&](uint32_t seg, uint32_t from, uint32_t to) {
                    const uint32_t acc = it & 1, d = tmem + acc * kTileN;
                    const bool begins = sizeof(T) == 4 || seg == 0, ends = sizeof(T) == 4 || seg + 1 == p.n_seg;
                    if (begins) {
                        if (!bar_wait(acc_empty + 8 * acc, (it >> 1 & 1) ^ 1, a.gave_up)) return false;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    }
                    const uint32_t steps = n_pairs * (to - from);
                    for (uint32_t k = 0; k < steps; ++k) {
                        if (!bar_wait(full + 8 * s, phase, a.gave_up)) return false;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                        for (uint32_t j = 0; j < kTileK / 16; ++j)
                            mma(d, da + s * (kStageBytes / 16) + j * sa, db + s * (kStageBytes / 16) + j * sb, idesc, !begins || k > 0 || j > 0);
                        mma_commit(empty + 8 * s);
                        if (++s == kStages) { s = 0; phase ^= 1; }
                    }
                    if (ends) { mma_commit(acc_full + 8 * acc); ++it; }
                    return true;
                });
            }
        }
    } else if (warp >= 4) {
        const uint32_t quad = warp & 3, part = (warp - 4) >> 2;           // tensor memory rows of 32; share of the columns
        uint32_t it = 0;
        auto acc_wait = [&]() {                                           // the next sum is complete
            __syncwarp();
            const bool ok = bar_wait(acc_full + 8 * (it & 1), it >> 1 & 1, a.gave_up);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            return __all_sync(0xFFFFFFFFu, ok);
        };
        auto acc_read = [&]() {                                           // ... and has been read
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive_at(in_cta(acc_empty + 8 * (it & 1), 0));
            ++it;
        };
        const int64_t gate_e_r = a.gate_e.r, up_e_r = a.up_e.r;
        if constexpr (!Shape::kWide) {
            // ---- bfloat16: blocks of 32 columns, eight at a time (in a loop: unrolled, they outgrow the instruction cache)
            constexpr uint32_t kChunks = MODE == MAT_GATED ? 1 : 2;
            const uint32_t mine = blocks + (warp - 4) * Shape::kBlocks * 2048;
            const bool eight = a.save == PALSGD_SAVE_8BIT;
            uint32_t ge = 0, ue = 0;                                      // hidden, 8 bits: exponents of the block under way
            // hidden: gate and up of block c of a tile into the warp's first two blocks
            auto fetch = [&](const Tile& tl, uint32_t c) {
                const uint32_t m = tl.m0 + rank * 128 + quad * 32, n = tl.n0 + (part * kChunks + c) * 32;
                const uint32_t M = tl.p->M, N = tl.p->N;
                const uint32_t rows = m < M ? min(M - m, 32u) : 0, cols = n < N ? N - n : 0;
                const int64_t w = tl.worker;
                const int64_t go = w * a.gate.w + (int64_t)m * a.gate.r + n, uo = w * a.up.w + (int64_t)m * a.up.r + n;
                if (eight) {
                    block_in<1>(mine, static_cast<const unsigned char*>(a.gate.p) + go, a.gate.r, rows, cols, a.gate.wide, lane);
                    block_in<1>(mine + 2048, static_cast<const unsigned char*>(a.up.p) + uo, a.up.r, rows, cols, a.up.wide, lane);
                    const bool on = lane < rows && cols;
                    ge = on ? static_cast<const uint8_t*>(a.gate_e.p)[w * a.gate_e.w + (int64_t)(m + lane) * gate_e_r + n / 32] : 0u;
                    ue = on ? static_cast<const uint8_t*>(a.up_e.p)[w * a.up_e.w + (int64_t)(m + lane) * up_e_r + n / 32] : 0u;
                } else {
                    block_in<2>(mine, static_cast<const unsigned char*>(a.gate.p) + 2 * go, 2 * a.gate.r, rows, cols, a.gate.wide, lane);
                    block_in<2>(mine + 2048, static_cast<const unsigned char*>(a.up.p) + 2 * uo, 2 * a.up.r, rows, cols, a.up.wide, lane);
                }
            };
            if constexpr (MODE == MAT_HIDDEN) { fetch(tile_at<MODE>(a, Order(a, pair, pairs).now()), 0); }
            for (Order o(a, pair, pairs); o.now() < a.tiles; o.next()) {
                const uint32_t t = o.now();
                const Tile tl = tile_at<MODE>(a, t);
                const MatProblem& p = *tl.p;
                const uint32_t src = tmem + (it & 1) * kTileN + (quad << 21);
                const uint32_t m = tl.m0 + rank * 128 + quad * 32, rows = m < p.M ? min(p.M - m, 32u) : 0;
                const int64_t w = tl.worker;
                if (!acc_wait()) break;
#pragma unroll 1
                for (uint32_t c = 0; c < kChunks; ++c) {
                    const uint32_t col = (part * kChunks + c) * 32, n = tl.n0 + col;
                    const uint32_t cols = n < p.N ? p.N - n : 0, room = n < p.out[0].cols ? p.out[0].cols - n : 0;
                    const int64_t at = 2 * (w * p.out[0].w + (int64_t)m * p.out[0].r + n), step = 2 * p.out[0].r;
                    const uint32_t b0 = mine;
                    if constexpr (MODE == MAT_PLAIN) {
#pragma unroll
                        for (uint32_t j = 0; j < 4; j += 2) {
                            float v[16];
                            tmem_load16(src + col + 8 * j, v);
                            tmem_load_wait();
                            f2 y[2][4];
#pragma unroll
                            for (int i = 0; i < 8; ++i) y[i / 4][i % 4] = f2_of(v[2 * i], v[2 * i + 1]);
                            row_put(b0, lane, j, y[0]);
                            row_put(b0, lane, j + 1, y[1]);
                        }
                        if (c + 1 == kChunks) acc_read();
                        __syncwarp();
                        block_out<64, 2>(b0, static_cast<unsigned char*>(p.out[0].p) + at, step, rows, room, p.out[0].wide, lane);
                        __syncwarp();
                    } else if constexpr (MODE == MAT_GATED) {
                        float gi = 0.0f, ui = 0.0f;                       // one over the steps of the groups
                        if (eight) {
                            float gm = 0.0f, um = 0.0f;
#pragma unroll 1
                            for (uint32_t j = 0; j < 4; ++j) {
                                float v[8], u[8];
                                tmem_load8(src + col + 8 * j, v);
                                tmem_load8(src + kTileN / 2 + col + 8 * j, u);
                                tmem_load_wait();
#pragma unroll
                                for (int i = 0; i < 8; ++i) { gm = act8_max(gm, v[i]); um = act8_max(um, u[i]); }
                            }
                            const uint32_t eg = act8_exponent(gm), eu = act8_exponent(um);
                            gi = act8_inverse(eg); ui = act8_inverse(eu);
                            if (lane < rows && cols) {
                                static_cast<uint8_t*>(a.gate_e.p)[w * a.gate_e.w + (int64_t)(m + lane) * gate_e_r + n / 32] = (uint8_t)eg;
                                static_cast<uint8_t*>(a.up_e.p)[w * a.up_e.w + (int64_t)(m + lane) * up_e_r + n / 32] = (uint8_t)eu;
                            }
                        }
                        // gate, up and h pass through one block, one after another (tensor memory is read again for each)
                        if (a.save != PALSGD_SAVE_NONE) {
#pragma unroll 1
                            for (uint32_t which = 0; which < 2; ++which) {
                                const MatOut& s = which ? a.up : a.gate;
                                const float inv = which ? ui : gi;
#pragma unroll
                                for (uint32_t j = 0; j < 4; j += 2) {
                                    float v[16];
                                    tmem_load16(src + which * (kTileN / 2) + col + 8 * j, v);
                                    tmem_load_wait();
                                    if (eight) {
                                        row_put_act8(b0, lane, j, inv, v);
                                        row_put_act8(b0, lane, j + 1, inv, v + 8);
                                    } else {
                                        f2 y[2][4];
#pragma unroll
                                        for (int i = 0; i < 8; ++i) y[i / 4][i % 4] = f2_of(v[2 * i], v[2 * i + 1]);
                                        row_put(b0, lane, j, y[0]);
                                        row_put(b0, lane, j + 1, y[1]);
                                    }
                                }
                                __syncwarp();
                                const int64_t to = w * s.w + (int64_t)m * s.r + n;
                                if (eight) block_out<32, 1>(b0, static_cast<unsigned char*>(s.p) + to, s.r, rows, cols, s.wide, lane);
                                else block_out<64, 2>(b0, static_cast<unsigned char*>(s.p) + 2 * to, 2 * s.r, rows, cols, s.wide, lane);
                                __syncwarp();
                            }
                        }
#pragma unroll 1
                        for (uint32_t j = 0; j < 4; ++j) {
                            float v[8], u[8];
                            tmem_load8(src + col + 8 * j, v);
                            tmem_load8(src + kTileN / 2 + col + 8 * j, u);
                            tmem_load_wait();
                            f2 h[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                f2 unused;
                                h[i] = f2_mul(act2<ACT, false>(f2_of(v[2 * i], v[2 * i + 1]), unused), f2_of(u[2 * i], u[2 * i + 1]));
                            }
                            row_put(b0, lane, j, h);
                        }
                        acc_read();
                        block_out<64, 2>(b0, static_cast<unsigned char*>(p.out[0].p) + at, step, rows, room, 1, lane);
                        __syncwarp();
                    } else {
                        block_wait();
                        __syncwarp();
                        const uint32_t b1 = mine + 2048;
                        const float gs = act8_step(ge), us = act8_step(ue);
#pragma unroll 1
                        for (uint32_t j = 0; j < 4; ++j) {
                            float v[8];
                            f2 g[4], q[4], dg[4], du[4], h[4];
                            tmem_load8(src + col + 8 * j, v);
                            if (eight) { row_get_act8(b0, lane, j, gs, g); row_get_act8(b1, lane, j, us, q); }
                            else { row_get(b0, lane, j, g); row_get(b1, lane, j, q); }
                            tmem_load_wait();
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                f2 slope;
                                const f2 ag = act2<ACT, true>(g[i], slope), d = f2_of(v[2 * i], v[2 * i + 1]);
                                dg[i] = f2_mul(f2_mul(d, q[i]), slope);
                                du[i] = f2_mul(d, ag);
                                h[i] = f2_mul(ag, q[i]);
                            }
                            row_put(b0, lane, j, dg);
                            row_put(b1, lane, j, du);
                            // h waits its turn in tensor memory, over sums that have been read
                            const uint32_t hw[4] = {f2_narrow(h[0]), f2_narrow(h[1]), f2_narrow(h[2]), f2_narrow(h[3])};
                            tmem_store4(src + col + 4 * j, hw);
                        }
                        tmem_store_wait();
                        __syncwarp();
                        block_out<64, 2>(b0, static_cast<unsigned char*>(p.out[0].p) + at, step, rows, room, 1, lane);
                        block_out<64, 2>(b1, static_cast<unsigned char*>(p.out[1].p) + at, step, rows, room, 1, lane);
                        __syncwarp();
                        {
                            float h[16];
                            tmem_load16(src + col, h);
                            tmem_load_wait();
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                sts128(block_at<64>(b0, lane, j), make_uint4(__float_as_uint(h[4 * j]), __float_as_uint(h[4 * j + 1]), __float_as_uint(h[4 * j + 2]), __float_as_uint(h[4 * j + 3])));
                        }
                        if (c + 1 == kChunks) acc_read();
                        __syncwarp();
                        block_out<64, 2>(b0, static_cast<unsigned char*>(p.out[2].p) + at, step, rows, room, 1, lane);
                        __syncwarp();
                        // the next block: of this tile, or the first of the warp's next tile
                        if (c + 1 < kChunks) fetch(tl, c + 1);
                        else if (o.then() < a.tiles) fetch(tile_at<MODE>(a, o.then()), 0);
                    }
                }
            }
        } else {
            // ---- fp32: sums of 64 columns in registers (gate/up: 32 of each)
            for (Order o(a, pair, pairs); o.now() < a.tiles; o.next()) {
                const uint32_t t = o.now();
                const Tile tl = tile_at<MODE>(a, t);
                const MatProblem& p = *tl.p;
                const uint32_t m = tl.m0 + rank * 128 + quad * 32 + lane;
                const int64_t w = tl.worker;
                const uint32_t col[2] = {MODE == MAT_GATED ? part * 32 : part * 64, MODE == MAT_GATED ? kTileN / 2 + part * 32 : part * 64 + 32};
                float sum[64];
#pragma unroll
                for (int i = 0; i < 64; ++i) sum[i] = 0.0f;
                const bool ok = for_pieces<T>(p, [&](uint32_t, uint32_t, uint32_t) {
                    const uint32_t src = tmem + (it & 1) * kTileN + (quad << 21);
                    if (!acc_wait()) return false;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[16];
                        tmem_load16(src + col[q / 2] + (q & 1) * 16, v);
                        tmem_load_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[q * 16 + i] += v[i];
                    }
                    acc_read();
                    return true;
                });
                if (!ok) break;
                // (nothing below is a whole warp's: rows outside have no columns, and no thread leaves the common path)
#pragma unroll
                for (int c = 0; c < (MODE == MAT_GATED ? 1 : 2); ++c) {
                    const uint32_t n = tl.n0 + col[c];
                    if (m >= p.M || n >= p.N) continue;
                    const int64_t at = w * p.out[0].w + (int64_t)m * p.out[0].r + n;
                    const int64_t go = w * a.gate.w + (int64_t)m * a.gate.r + n, uo = w * a.up.w + (int64_t)m * a.up.r + n;
                    const int64_t geo = w * a.gate_e.w + (int64_t)m * gate_e_r + n / 32, ueo = w * a.up_e.w + (int64_t)m * up_e_r + n / 32;
                    const bool eight = a.save == PALSGD_SAVE_8BIT;
                    float gs = 0.0f, us = 0.0f;                           // steps of the groups, or one over them
                    if constexpr (MODE == MAT_GATED) {
                        if (eight) {
                            float gm = 0.0f, um = 0.0f;
#pragma unroll
                            for (int i = 0; i < 32; ++i) { gm = act8_max(gm, sum[i]); um = act8_max(um, sum[32 + i]); }
                            const uint32_t eg = act8_exponent(gm), eu = act8_exponent(um);
                            static_cast<uint8_t*>(a.gate_e.p)[geo] = (uint8_t)eg;
                            static_cast<uint8_t*>(a.up_e.p)[ueo] = (uint8_t)eu;
                            gs = act8_inverse(eg); us = act8_inverse(eu);
                        }
                    } else if constexpr (MODE == MAT_HIDDEN) {
                        if (eight) {
                            gs = act8_step(static_cast<const uint8_t*>(a.gate_e.p)[geo]);
                            us = act8_step(static_cast<const uint8_t*>(a.up_e.p)[ueo]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 32; j += 8) {
                        if (n + j >= p.N) continue;
                        const uint32_t left = p.N - n - j;
                        float* v = sum + 32 * c + j;
                        if constexpr (MODE == MAT_PLAIN) {
                            store8(static_cast<float*>(p.out[0].p) + at + j, v, left, p.out[0].wide);
                        } else if constexpr (MODE == MAT_GATED) {
                            float* u = sum + 32 + j;
                            if (a.save == PALSGD_SAVE_FULL) {
                                store8(static_cast<float*>(a.gate.p) + go + j, v, left, a.gate.wide);
                                store8(static_cast<float*>(a.up.p) + uo + j, u, left, a.up.wide);
                            } else if (eight) {
                                store8_act8(a.gate, go + j, v, gs, left);
                                store8_act8(a.up, uo + j, u, us, left);
                            }
                            gate8<ACT>(v, u);
                            store8_parts(p.out[0], at + j, v);
                        } else {
                            float g[8], u[8];
                            if (eight) {
                                load8_act8(a.gate, go + j, g, gs, left);
                                load8_act8(a.up, uo + j, u, us, left);
                            } else {
                                load8(static_cast<const float*>(a.gate.p) + go + j, g, left, a.gate.wide);
                                load8(static_cast<const float*>(a.up.p) + uo + j, u, left, a.up.wide);
                            }
                            hidden8<ACT>(v, g, u);
                            store8_parts(p.out[0], at + j, g);
                            store8_parts(p.out[1], at + j, u);
                            store8_parts(p.out[2], at + j, v);
                        }
                    }
                }
            }
        }
        if constexpr (MODE == MAT_HIDDEN && !Shape::kWide) block_wait();
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
