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
//
// What bounds it (bfloat16, one B200): 8 workers of 1024 tokens, 768 x 2048 -- gate/up pass 44 us (1170 TFLOP/s: 83
// steps of 64 at 0.33 us, of which 0.29 are matrix instructions; the rest is the start, with operands from memory, and the last
// tile's epilogue: 38 us if nothing is saved, 42 in full, 44 in 8 bits), hidden pass 46 us (its epilogue: g, u in, dg, du, h
// out), dx and the weight gradients 94 us (1370 TFLOP/s).  2 workers of 8192, 2048 x 5632, back to back: forward
// 0.84-0.97 ms, backward 2.04-2.16 ms, 1050-1350 TFLOP/s at the power limit, where a library product sustains 1385.
// fp32: 8 workers of 500 tokens, 256 x 1024, backward 136-138 us, forward 69.
// One token of one worker, 2048 x 5632: forward 48 us, backward 65, for 69 and 138 MB (10.6 and 21 us): the tokens are the
// long side of every tile, which are then few and mostly zeros.
#pragma once
#include <cuda.h>

#include "block_common.cuh"

namespace palsgd {
namespace block {

// MAT_SUMS, MAT_ROWS: plain, with column sums beside the products, of partial sums or of a matrix
enum { MAT_PLAIN = 0, MAT_GATED = 1, MAT_HIDDEN = 2, MAT_LINEAR = 3, MAT_SUMS = 4, MAT_ROWS = 5 };
constexpr __host__ __device__ bool mat_plain(int mode) { return mode == MAT_PLAIN || mode == MAT_SUMS || mode == MAT_ROWS; }

constexpr uint32_t kTileM = 256, kTileN = 256, kTileK = 64;
constexpr uint32_t kOperandBytes = 128 * kTileK * 2;                    // a CTA's half of an operand's tile
constexpr uint32_t kStageBytes = 2 * kOperandBytes;
constexpr uint32_t kBarrierBytes = 256;
constexpr uint32_t kPiece = 4;                                          // fp32: steps of kTileK between two roundings to binary32

// Shared memory and warps of a kernel: 16 epilogue warps of 64 columns each (8 of 128 took 59 us where these took 49
// in the hidden pass: two warps a scheduler do not cover each other's latencies).  They pass their results (and, in the hidden
// pass, gate and up) through blocks of 32 rows of 64 bytes in shared memory: 32 columns of bfloat16, 16 of fp32.
template <typename T, int MODE>
struct MatShape {
    static constexpr bool kWide = sizeof(T) == 4;
    static constexpr uint32_t kEpilogue = 16;
    static constexpr uint32_t kThreads = 128 + 32 * kEpilogue;
    static constexpr uint32_t kBlocks = MODE == MAT_HIDDEN || MODE == MAT_LINEAR ? 2 : 1;       // a warp's
    static constexpr uint32_t kStages = kBlocks == 2 ? 5 : 6;
    static constexpr uint32_t kSmem = kStages * kStageBytes + kEpilogue * kBlocks * 2048 + kBarrierBytes + 1024;   // 1024: to start on a swizzle atom
    static_assert(kSmem <= 232448, "shared memory of a CTA");
};

constexpr uint32_t kMaxProblems = 4;
constexpr uint32_t kTileLeast = 6;                                      // steps that a tile's results take to leave: a shorter tile ends no sooner
constexpr unsigned long long kWaitLimitNs = 4000000000ull;              // how long a wait polls before it gives up

struct MatOut {
    void*   p;
    int64_t w, r;                 // worker and row stride, elements
    int64_t part;                 // the stride between the three bfloat16 parts of an fp32 value, or between shares' sums
    int     wide;                 // rows start on 16-byte boundaries
    uint32_t cols;                // columns that may be written: the workspace's rows have room behind their end
};

struct alignas(64) MatProblem {
    CUtensorMap A[2], B[2];       // by segment; the gate/up pass: B[0] gate, B[1] up
    uint32_t M, N, Kd, tiles;
    Divisor  tiles_m, per_split, per_worker; // tiles down, of one share of the inner axis, of one worker
    uint32_t splits;              // shares of the inner axis (plain): above one, out[0] takes each share's binary32 sums
    uint8_t  n_seg, a_parts, b_parts, a_mn, b_mn;
    uint8_t  a_one[2], b_one[2];  // all workers read one matrix
    MatOut   out[3];              // plain: the product; gate/up: h; hidden: dg, du, h; linear: y
};

// Column sums beside the products, in a fixed order: of rows of binary32 sums [K][parts][ld] that other CTAs have left, or of
// a matrix itself (bfloat16, rows on 16-byte boundaries).
struct MatSums {
    const float* part;            // NULL: none
    const void*  rows;            // NULL: none
    int64_t  rows_w, rows_r;
    void*    out;
    int64_t  w;                   // worker stride of out
    uint32_t parts, cols, ld, K;  // parts: rows of either
};
constexpr uint32_t kSumsCols = 64, kSumsRows = 64;        // of a matrix: columns of a warp, rows under way

struct MatLaunch {
    MatProblem p[kMaxProblems];
    MatSums  sums;                // sums, rows
    uint32_t n_problems, tiles, heavy, lag;   // see Order
    int      save;
    MatOut   gate, up;            // saved (gate/up pass) or read (hidden pass)
    MatOut   gate_e, up_e;
    MatOut   bias, residual;      // linear (gate: what is saved); p may be NULL
    CUtensorMap store[3];         // bfloat16: h (gate/up), or dg, du, h (hidden), as the copy engine writes blocks of them
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
__device__ __forceinline__ bool elect_one()                              // one thread of the warp, the same each time
{
    uint32_t p;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
    return p;
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
// A block of 32 x 32 bfloat16 (64-byte swizzle, which is the order of block_at<64>) to a matrix; what is outside is dropped.
__device__ __forceinline__ void tma_store(const CUtensorMap* map, uint32_t src, uint32_t c0, uint32_t c1, uint32_t c2)
{
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(0) : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void tma_store_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }   // the blocks may be written again
__device__ __forceinline__ void tma_store_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void block_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
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
__device__ __forceinline__ void tmem_store8(uint32_t addr, const float* v)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
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

// A block of 32 rows (one a lane) that a warp passes through shared memory on its way between rows and coalesced accesses.
// ROW bytes a row: 64, or 32 / 16 for the 8-bit form; the 16-byte pieces of a row are permuted so that neither side has
// bank conflicts.
template <int ROW>
__device__ __forceinline__ uint32_t block_at(uint32_t base, uint32_t row, uint32_t piece)
{
    constexpr uint32_t kPieces = ROW / 16;
    const uint32_t turn = kPieces == 4 ? (row >> 1) & 3 : kPieces == 2 ? (row >> 2) & 1 : 0;
    return base + row * ROW + ((piece ^ turn) << 4);
}

// Block -> matrix: `rows` (at most 32) rows and `cols` columns of it are inside.  E: the element type's size.  Elements of two
// bytes in rows off 16-byte boundaries: the whole 16-byte pieces of memory first, each of two of the block's, then the elements
// before and behind them, a row's side by side (4 x 1000 tokens, 1001 -> 777: the call 25.7 us, with every piece of the block stored in
// words where it lies 28.3; the same for fp32 67.8 and 64.5).
template <int ROW, int E>
__device__ __noinline__ void block_out_edge(uint32_t base, unsigned char* to, int64_t row_bytes, uint32_t rows, uint32_t cols, uint32_t lane)
{
    constexpr uint32_t kPieces = ROW / 16;
    const uint32_t piece = lane % kPieces, all = cols * E;
    if constexpr (E == 2) {
        if (all == ROW) {                                 // a whole row of the block: as many elements before the pieces and behind them as one holds
#pragma unroll
            for (uint32_t i = 0; i < kPieces; ++i) {
                const uint32_t row = i * (32 / kPieces) + lane / kPieces;
                unsigned char* p = to + (int64_t)row * row_bytes;
                const uint32_t s = (0u - (uint32_t)reinterpret_cast<uintptr_t>(p)) & 15;
                if (row >= rows || (s && piece + 1 == kPieces)) continue;
                uint4 a, b;
                lds128(block_at<ROW>(base, row, piece), a);
                lds128(block_at<ROW>(base, row, s ? piece + 1 : piece), b);
                *reinterpret_cast<uint4*>(p + s + 16 * piece) = shift16(a, b, s, 16);
            }
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const uint32_t row = i * 4 + lane / 8, e = (lane % 8) * 2;
                unsigned char* p = to + (int64_t)row * row_bytes;
                const uint32_t s = (0u - (uint32_t)reinterpret_cast<uintptr_t>(p)) & 15, at = e < s ? e : e + ROW - 16;
                if (row >= rows || s == 0) continue;
                uint16_t v;
                asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(block_at<ROW>(base, row, at >> 4) + (at & 15)));
                *reinterpret_cast<uint16_t*>(p + at) = v;
            }
            return;
        }
#pragma unroll 2
        for (uint32_t row = lane / kPieces; row < rows; row += 32 / kPieces) {
            unsigned char* p = to + (int64_t)row * row_bytes;
            const uint32_t s = (0u - (uint32_t)reinterpret_cast<uintptr_t>(p)) & 15, at = s + 16 * piece;
            if (at + 16 > all) continue;
            uint4 a, b;
            lds128(block_at<ROW>(base, row, piece), a);
            lds128(block_at<ROW>(base, row, s ? piece + 1 : piece), b);
            *reinterpret_cast<uint4*>(p + at) = shift16(a, b, s, 16);
        }
#pragma unroll 2
        for (uint32_t row = lane / 8; row < rows; row += 4) {
            unsigned char* p = to + (int64_t)row * row_bytes;
            const uint32_t s = (0u - (uint32_t)reinterpret_cast<uintptr_t>(p)) & 15, whole = all > s ? (all - s) & ~15u : 0;
            for (uint32_t i = (lane % 8) * 2; i + whole < all; i += 16) {
                const uint32_t at = i < s ? i : i + whole;
                uint16_t v;
                asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(block_at<ROW>(base, row, at >> 4) + (at & 15)));
                *reinterpret_cast<uint16_t*>(p + at) = v;
            }
        }
    } else {
        const uint32_t bytes = all > piece * 16 ? min(all - piece * 16, 16u) : 0;
        if (bytes == 0) return;
#pragma unroll 1
        for (uint32_t row = lane / kPieces; row < rows; row += 32 / kPieces) {
            uint4 v;
            lds128(block_at<ROW>(base, row, piece), v);
            put16<E>(to + (int64_t)row * row_bytes + piece * 16, bytes, v);
        }
    }
}
template <int ROW, int E>
__device__ __forceinline__ void block_out(uint32_t base, unsigned char* to, int64_t row_bytes, uint32_t rows, uint32_t cols, bool wide, uint32_t lane)
{
    constexpr uint32_t kPieces = ROW / 16;
    if (rows && cols >= ROW / E && wide) {                // the same for the whole warp
        const uint32_t piece = lane % kPieces, row = lane / kPieces;
        unsigned char* p = to + (int64_t)row * row_bytes + piece * 16;
        const int64_t step = row_bytes * (32 / kPieces);
        uint4 v[kPieces];
#pragma unroll
        for (uint32_t i = 0; i < kPieces; ++i) lds128(block_at<ROW>(base, i * (32 / kPieces) + row, piece), v[i]);
#pragma unroll
        for (uint32_t i = 0; i < kPieces; ++i) {
            if (i * (32 / kPieces) + row < rows) *reinterpret_cast<uint4*>(p) = v[i];
            p += step;
        }
    } else if (rows && cols) {
        block_out_edge<ROW, E>(base, to, row_bytes, rows, min(cols, (uint32_t)(ROW / E)), lane);
    }
}

// Matrix -> block of 64-byte rows, asynchronously where the rows are aligned; zeros outside.  Complete after block_wait and
// __syncwarp.  PIECES 16-byte pieces a row, the last ones of the row: int8 fills its end, so that a lane can write its
// results over its row from the front while it still reads.
template <int E, int PIECES>
__device__ __noinline__ void block_in_edge(uint32_t base, const unsigned char* from, int64_t row_bytes, uint32_t rows, uint32_t cols, uint32_t lane)
{
    const uint32_t piece = lane % PIECES, bytes = cols * E > piece * 16 ? min(cols * E - piece * 16, 16u) : 0;
#pragma unroll 4
    for (uint32_t row = lane / PIECES; row < 32; row += 32 / PIECES)
        sts128(block_at<64>(base, row, 4 - PIECES + piece), get16(from + (int64_t)row * row_bytes + piece * 16, row < rows ? bytes : 0));
}
template <int E, int PIECES>
__device__ __forceinline__ void block_in(uint32_t base, const unsigned char* from, int64_t row_bytes, uint32_t rows, uint32_t cols, bool wide, uint32_t lane)
{
    constexpr uint32_t kFirst = 4 - PIECES;
    if (rows && cols >= PIECES * 16 / E && wide) {
        const uint32_t piece = lane % PIECES, row = lane / PIECES;
        const unsigned char* p = from + (int64_t)row * row_bytes + piece * 16;
        const int64_t step = row_bytes * (32 / PIECES);
#pragma unroll
        for (uint32_t i = 0; i < PIECES; ++i) {
            const bool on = i * (32 / PIECES) + row < rows;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(block_at<64>(base, i * (32 / PIECES) + row, kFirst + piece)), "l"(on ? p : from), "r"(on ? 16u : 0u) : "memory");
            p += step;
        }
    } else if (rows && cols) {                            // (a block that is all outside is not read)
        block_in_edge<E, PIECES>(base, from, row_bytes, rows, min(cols, (uint32_t)(PIECES * 16 / E)), lane);
    }
}
__device__ __forceinline__ void block_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Eight columns of a lane's row of a block, as pairs of floats
template <typename T>
__device__ __forceinline__ void row_put(uint32_t base, uint32_t lane, uint32_t j, const f2 (&v)[4])
{
    if constexpr (sizeof(T) == 2) {
        sts128(block_at<64>(base, lane, j), make_uint4(f2_narrow(v[0]), f2_narrow(v[1]), f2_narrow(v[2]), f2_narrow(v[3])));
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
            asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(block_at<64>(base, lane, 2 * j + i)), "l"(v[2 * i]), "l"(v[2 * i + 1]) : "memory");
    }
}
template <typename T>
__device__ __forceinline__ void row_get(uint32_t base, uint32_t lane, uint32_t j, f2 (&v)[4])
{
    if constexpr (sizeof(T) == 2) {
        uint4 a;
        lds128(block_at<64>(base, lane, j), a);
        v[0] = f2_wide(a.x); v[1] = f2_wide(a.y); v[2] = f2_wide(a.z); v[3] = f2_wide(a.w);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
            asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v[2 * i]), "=l"(v[2 * i + 1]) : "r"(block_at<64>(base, lane, 2 * j + i)));
    }
}
// ... of an 8-bit block: written in rows of as many bytes as columns, read where block_in puts it
template <typename T>
__device__ __forceinline__ void row_put_act8(uint32_t base, uint32_t lane, uint32_t j, float inv, const float* v)
{
    const uint32_t at = sizeof(T) == 2 ? block_at<32>(base, lane, j >> 1) + (j & 1) * 8 : block_at<16>(base, lane, 0) + j * 8;
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(act8_quant4(v[0], v[1], v[2], v[3], inv)), "r"(act8_quant4(v[4], v[5], v[6], v[7], inv)) : "memory");
}
template <typename T>
__device__ __forceinline__ void row_get_act8(uint32_t base, uint32_t lane, uint32_t j, float step, f2 (&v)[4])
{
    const uint32_t at = sizeof(T) == 2 ? block_at<64>(base, lane, 2 + (j >> 1)) + (j & 1) * 8 : block_at<64>(base, lane, 3) + j * 8;
    uint2 a;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(a.x), "=r"(a.y) : "r"(at));
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

// N fp32 values as their three bfloat16 parts: out(part, words of two).  Where all values are finite and none rounds past
// the largest bfloat16, two at a time without a look at each (operand copies of an fp32 backward call: 18.3 -> 12.8 us).
template <int N, typename Out>
__device__ __forceinline__ void three_parts(float (&v)[N], Out&& out)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    if (top < 0x7F7F8000u) {
#pragma unroll
        for (int part = 0; part < 3; ++part) {
            uint32_t w[N / 2];
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                w[i] = f2_narrow(f2_of(v[2 * i], v[2 * i + 1]));
                v[2 * i] = __fsub_rn(v[2 * i], __uint_as_float(w[i] << 16));
                v[2 * i + 1] = __fsub_rn(v[2 * i + 1], __uint_as_float(w[i] & 0xFFFF0000u));
            }
            out(part, w);
        }
    } else {
#pragma unroll 1
        for (int part = 0; part < 3; ++part) {
            uint32_t w[N / 2];
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float lo = next_part(v[2 * i]), hi = next_part(v[2 * i + 1]);
                w[i] = f2_narrow(f2_of(lo, hi));
            }
            out(part, w);
        }
    }
}

// A block of 16 fp32 columns of an operand of the next product -> workspace, as its three parts.
template <typename T>
__device__ __forceinline__ void operand_out(uint32_t base, const MatOut& o, int64_t at, uint32_t rows, uint32_t room, uint32_t lane)
{
    static_assert(sizeof(T) == 4, "bfloat16 blocks go out by the copy engine");
    const uint32_t piece = lane & 3;
    bf16* p = static_cast<bf16*>(o.p) + at + (int64_t)(lane >> 2) * o.r + piece * 4;
#pragma unroll 1
    for (uint32_t row = lane >> 2; row < 32; row += 8) {
        float v[4];
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(block_at<64>(base, row, piece)));
        if (row < rows && piece * 4 < room) {             // (the workspace's rows hold a multiple of eight columns)
            three_parts<4>(v, [&](int part, const uint32_t (&w)[2]) { *reinterpret_cast<uint2*>(p + part * o.part) = make_uint2(w[0], w[1]); });
        }
        p += 8 * o.r;
    }
}

// The activation of a pair: fast for results that are rounded to bfloat16, accurate for fp32.
template <typename T, int ACT, bool SLOPE>
__device__ __forceinline__ f2 act_pair(f2 g, f2& slope)
{
    if constexpr (sizeof(T) == 2) {
        return act2<ACT, SLOPE>(g, slope);
    } else {
        float x, y, sx = 0.0f, sy = 0.0f;
        f2_get(g, x, y);
        const float ax = act<ACT, SLOPE, false>(x, sx), ay = act<ACT, SLOPE, false>(y, sy);
        if constexpr (SLOPE) slope = f2_of(sx, sy);
        return f2_of(ax, ay);
    }
}

// The same for the linear operator: GELU of a pair that is rounded to bfloat16 by the rational approximation of erf with one
// exponential (Abramowitz and Stegun 7.1.26, erf off by at most 1.5e-7; with the roundings of its evaluation y by some 2 and the slope by some 5
// units of 2^-24 (1 + |g|)), which is also the slope's.  (With erff for each value the pass before the activation took 27 us, so 20: 5
// workers of 4449 tokens, 144 columns.)
template <typename T, int ACT, bool SLOPE>
__device__ __forceinline__ f2 linear_act(f2 g, f2& slope)
{
    if constexpr (sizeof(T) == 2 && ACT == PALSGD_ACT_GELU) {
        float x, y;
        f2_get(g, x, y);
        const float ax = fabsf(x), ay = fabsf(y);
        f2 t = f2_fma(f2_of(ax, ay), f2_same(0.3275911f * 0.70710678118654752f), f2_same(1.0f));
        float tx, ty, ex, ey;
        f2_get(t, tx, ty);
        t = f2_of(fast_inverse(tx), fast_inverse(ty));
        f2_get(f2_mul(f2_mul(g, g), f2_same(-0.5f * 1.4426950408889634f)), ex, ey);
        const f2 e = f2_of(fast_exp2(ex), fast_exp2(ey));                // e^(-g^2 / 2)
        f2 p = f2_fma(t, f2_same(1.061405429f), f2_same(-1.453152027f));
        p = f2_fma(p, t, f2_same(1.421413741f));
        p = f2_fma(p, t, f2_same(-0.284496736f));
        p = f2_fma(p, t, f2_same(0.254829592f));
        float qx, qy;
        f2_get(f2_mul(f2_mul(f2_mul(p, t), e), f2_same(0.5f)), qx, qy);  // Phi(-|g|)
        const f2 cdf = f2_of(x > 0.0f ? 1.0f - qx : qx, y > 0.0f ? 1.0f - qy : qy);
        // (a gate beyond 10^19: its square's exponential is 0, and so is what it multiplies)
        if constexpr (SLOPE) slope = f2_fma(f2_mul(f2_of(fminf(fmaxf(x, -1e4f), 1e4f), fminf(fmaxf(y, -1e4f), 1e4f)), f2_same(0.39894228040143268f)), e, cdf);
        return f2_mul(g, cdf);
    } else if constexpr (sizeof(T) == 4 && ACT == PALSGD_ACT_GELU) {
        // fp32: the Chebyshev form of erfc that is off by at most 1.2e-7 of itself everywhere (Numerical Recipes, 6.2), as evaluated here by
        // that and about the roundings of the exponent, |E| units in the last place of e^E:
        // Phi(-|g|) = erfc(z) / 2, z = |g| / sqrt(2), erfc(z) = t e^(-z^2 + P(t)), t = 1 / (1 + z / 2)
        float x, y, tx, ty, ex, ey;
        f2_get(g, x, y);
        const f2 z = f2_of(fabsf(x) * 0.70710678118654752f, fabsf(y) * 0.70710678118654752f);
        f2_get(f2_fma(z, f2_same(0.5f), f2_same(1.0f)), tx, ty);
        const f2 t = f2_of(fast_inverse(tx), fast_inverse(ty));
        f2 p = f2_fma(t, f2_same(0.17087277f), f2_same(-0.82215223f));
        p = f2_fma(p, t, f2_same(1.48851587f));
        p = f2_fma(p, t, f2_same(-1.13520398f));
        p = f2_fma(p, t, f2_same(0.27886807f));
        p = f2_fma(p, t, f2_same(-0.18628806f));
        p = f2_fma(p, t, f2_same(0.09678418f));
        p = f2_fma(p, t, f2_same(0.37409196f));
        p = f2_fma(p, t, f2_same(1.00002368f));
        p = f2_fma(p, t, f2_same(-1.26551223f));
        const f2 zz = f2_mul(z, z);
        f2_get(f2_mul(f2_add(p, f2_neg(zz)), f2_same(1.4426950408889634f)), ex, ey);
        float qx, qy;
        f2_get(f2_mul(f2_mul(t, f2_same(0.5f)), f2_of(fast_exp2(ex), fast_exp2(ey))), qx, qy);
        const f2 cdf = f2_of(x > 0.0f ? 1.0f - qx : qx, y > 0.0f ? 1.0f - qy : qy);
        if constexpr (SLOPE) {
            float wx, wy;
            f2_get(f2_mul(zz, f2_same(-1.4426950408889634f)), wx, wy);
            slope = f2_fma(f2_mul(f2_of(fminf(fmaxf(x, -1e4f), 1e4f), fminf(fmaxf(y, -1e4f), 1e4f)), f2_same(0.39894228040143268f)),
                           f2_of(fast_exp2(wx), fast_exp2(wy)), cdf);
        }
        return f2_mul(g, cdf);
    } else {
        return act_pair<T, ACT, SLOPE>(g, slope);
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

struct Tile { uint32_t worker, m0, n0, split; const MatProblem* p; };

template <int MODE>
__device__ __forceinline__ Tile tile_at(const MatLaunch& a, uint32_t t)
{
    uint32_t i = 0;
    while (i + 1 < a.n_problems && t >= a.p[i].tiles) { t -= a.p[i].tiles; ++i; }
    const MatProblem& p = a.p[i];
    const uint32_t w = p.per_worker.of(t), i_w = t - w * p.per_worker.d, s = mat_plain(MODE) ? p.per_split.of(i_w) : 0, r = i_w - s * p.per_split.d;
    const uint32_t n = p.tiles_m.of(r), m = r - n * p.tiles_m.d;
    return Tile{w, m * kTileM, n * (MODE == MAT_GATED ? kTileN / 2 : kTileN), s, &p};
}

__device__ __forceinline__ uint32_t pairs_of(const MatProblem& p) { return p.a_parts == 1 ? p.b_parts : p.b_parts == 1 ? p.a_parts : 6; }

// bfloat16 products that go into an 8-bit checkpoint: steps of a piece.  How many of its values land on the other side of a
// rounding goes by the sums' error.  Pieces of 128 to 256 terms, three of a short inner axis where they have that many, keep it at that of
// binary32 multiply-adds (4 workers of 3000 tokens, 256 -> 600, two pieces: 22 of 7.2 million values, with one piece 49, with multiply-adds
// 13; 18.4 us, with one piece 18.1; 512 -> 600, three pieces: 44, with two 51, with multiply-adds 37; 22.2 us, with two 20.0).  Of a launch
// of few tiles, cut into shares, a share is one sum, not cut again (one worker, 512 tokens, 5632 -> 768: 20 of 1.6 million values, a product
// in binary32 27; 1024 tokens, 8192 -> 512: 59 of 2.1 million, and 55).
__device__ __forceinline__ uint32_t piece_of(uint32_t inner)
{
    const uint32_t third = (inner + 3 * kTileK - 1) / (3 * kTileK);
    return third < 2 ? 2 : third < kPiece ? third : kPiece;
}

// The inner axis of a tile -- its share of all segments' steps -- in pieces of one segment each:
// f(segment, first step, end, begins a sum, ends it).  bfloat16: the pieces of a tile are one sum.  fp32: kPiece steps (with
// all their parts) are a sum of their own, and the sums are joined in registers with rounding to nearest -- the tensor
// cores cut off what an addition does not hold, which over long sums adds up (measured over 4096 steps of the inner axis
// in one sum: 4.4e-6 of the result's norm; in pieces of 4: 2.4e-7, of 8: 4.8e-7, where the whole is 2 % faster).
// `cut`: steps of a piece, 0: sums are not cut.
template <typename F>
__device__ __forceinline__ bool for_pieces(const Tile& tl, uint32_t cut, F&& f)
{
    const MatProblem& p = *tl.p;
    const uint32_t steps = (p.Kd + kTileK - 1) / kTileK, all = p.n_seg * steps;
    uint32_t g = 0, last = all;
    if (p.splits > 1) {
        g = (uint32_t)((uint64_t)all * tl.split / p.splits);
        last = (uint32_t)((uint64_t)all * (tl.split + 1) / p.splits);
    }
    for (bool first = true; g < last; first = false) {
        const uint32_t seg = g >= steps, k = g - seg * steps;
        uint32_t n = min(steps - k, last - g);
        if (cut) n = min(n, cut);
        g += n;
        if (!f(seg, k, k + n, cut || first, cut || g == last)) return false;
    }
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
    const uint32_t warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, rank = cluster_rank();
    const uint32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    const uint32_t cut = Shape::kWide ? kPiece : MODE == MAT_LINEAR && a.save == PALSGD_SAVE_8BIT ? piece_of(a.p[0].Kd) : 0;

    let_next_start();
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
    wait_for_previous();

    if (warp == 0 || warp == 3) {
        // producers: warp 0 brings A, warp 3 brings B (one thread that did both held the copy engine up: 410 ns a step of
        // 32 KB, of which 120 its own).  The whole warp walks the loop and one thread of it issues: what it walks with stays
        // in the warp's shared registers, from where the copy engine takes it.
        {
            const bool is_b = warp == 3, one = elect_one();
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
                ok = for_pieces(tl, cut, [&](uint32_t seg, uint32_t from, uint32_t to, bool, bool) {
                    const uint32_t i = is_b && MODE == MAT_GATED ? rank : seg;
                    const CUtensorMap* const map = is_b ? &p.B[i] : &p.A[i];
                    const uint32_t w = (is_b ? p.b_one[i] : p.a_one[i]) ? 0 : tl.worker;
                    for (int sum = sizeof(T) == 4 ? 2 : 0; sum >= 0; --sum)
                        for (int pa = 0; pa <= sum; ++pa) {
                            if (pa >= parts_a || sum - pa >= parts_b) continue;
                            const uint32_t part = is_b ? sum - pa : pa;
                            for (uint32_t k = from * kTileK; k < to * kTileK; k += kTileK) {
                                if (!__all_sync(0xFFFFFFFFu, bar_wait(empty + 8 * s, phase ^ 1, a.gave_up))) return false;
                                const uint32_t to_s = dst + s * kStageBytes, bar = signal + 8 * s;
                                if (one) {
                                    if (!is_b && rank == 0) bar_expect(full + 8 * s, 2 * kStageBytes);
                                    if (across) {
                                        tma_load(map, to_s, bar, mn, k, w, part);
                                        tma_load(map, to_s + 8192, bar, mn + 64, k, w, part);
                                    } else {
                                        tma_load(map, to_s, bar, k, mn, w, part);
                                    }
                                }
                                __syncwarp();
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
        if (rank == 0) {
            const bool one = elect_one();
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
                ok = for_pieces(tl, cut, [&](uint32_t, uint32_t from, uint32_t to, bool begins, bool ends) {
                    const uint32_t acc = it & 1, d = tmem + acc * kTileN;
                    if (begins) {
                        if (!__all_sync(0xFFFFFFFFu, bar_wait(acc_empty + 8 * acc, (it >> 1 & 1) ^ 1, a.gave_up))) return false;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    }
                    const uint32_t steps = n_pairs * (to - from);
                    for (uint32_t k = 0; k < steps; ++k) {
                        if (!__all_sync(0xFFFFFFFFu, bar_wait(full + 8 * s, phase, a.gave_up))) return false;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        if (one) {
#pragma unroll
                            for (uint32_t j = 0; j < kTileK / 16; ++j)
                                mma(d, da + s * (kStageBytes / 16) + j * sa, db + s * (kStageBytes / 16) + j * sb, idesc, !begins || k > 0 || j > 0);
                            mma_commit(empty + 8 * s);
                        }
                        __syncwarp();
                        if (++s == kStages) { s = 0; phase ^= 1; }
                    }
                    if (ends) {
                        if (one) mma_commit(acc_full + 8 * acc);
                        __syncwarp();
                        ++it;
                    }
                    return true;
                });
            }
        }
    } else if (warp == 2) {
        // the sums of a bias gradient (a kernel of its own for them took 4 us, a pass over dy 6; with the code for both in the plain
        // kernel, calls without them took 8 % longer)
        const MatSums& q = a.sums;
        if constexpr (MODE == MAT_SUMS) {
            const uint32_t groups = (q.cols + 31) / 32;
            for (uint32_t g = blockIdx.x; g < groups * q.K; g += gridDim.x) {
                const uint32_t k = g / groups, c = (g - k * groups) * 32 + lane;
                if (c >= q.cols) continue;
                const float* at = q.part + (uint64_t)k * q.parts * q.ld + c;
                float v[8];
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) v[i] = 0.0f;
                for (uint32_t r = 0; r < q.parts; r += 8)
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) if (r + i < q.parts) v[i] += at[(uint64_t)(r + i) * q.ld];
                static_cast<T*>(q.out)[(int64_t)k * q.w + c] = from_f<T>(((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])));
            }
        } else if constexpr (MODE == MAT_ROWS) {
            // eight lanes have a row's 64 columns, four rows side by side, sixteen of each under way
            const uint32_t groups = (q.cols + kSumsCols - 1) / kSumsCols;
            for (uint32_t g = blockIdx.x; g < groups * q.K; g += gridDim.x) {
                const uint32_t k = g / groups, c = (g - k * groups) * kSumsCols + (lane & 7) * 8;
                const bf16* at = static_cast<const bf16*>(q.rows) + (int64_t)k * q.rows_w + c;
                const bool on = c < q.cols;
                f2 sum[4] = {0, 0, 0, 0};
                for (uint32_t r0 = lane >> 3; r0 < q.parts; r0 += kSumsRows) {
                    uint4 v[kSumsRows / 4];
#pragma unroll
                    for (uint32_t i = 0; i < kSumsRows / 4; ++i) {
                        const uint32_t r = r0 + 4 * i;
                        v[i] = !on || r >= q.parts ? make_uint4(0, 0, 0, 0)
                             : c + 8 <= q.cols ? __ldg(reinterpret_cast<const uint4*>(at + (int64_t)r * q.rows_r))
                                               : get16(reinterpret_cast<const unsigned char*>(at + (int64_t)r * q.rows_r), 2 * (q.cols - c));
                    }
#pragma unroll
                    for (uint32_t i = 0; i < kSumsRows / 4; ++i) {
                        sum[0] = f2_add(sum[0], f2_wide(v[i].x)); sum[1] = f2_add(sum[1], f2_wide(v[i].y));
                        sum[2] = f2_add(sum[2], f2_wide(v[i].z)); sum[3] = f2_add(sum[3], f2_wide(v[i].w));
                    }
                }
#pragma unroll
                for (int d = 8; d < 32; d *= 2)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = f2_add(sum[i], __shfl_xor_sync(0xFFFFFFFFu, sum[i], d));
                if (lane < 8 && on) {
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) f2_get(sum[i], f[2 * i], f[2 * i + 1]);
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) if (c + i < q.cols) static_cast<T*>(q.out)[(int64_t)k * q.w + c + i] = from_f<T>(f[i]);
                }
            }
        }
        __syncwarp();
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
        // blocks of kCols columns, eight columns at a time in a loop (unrolled, they outgrow the instruction cache)
        constexpr uint32_t E = sizeof(T), kCols = 64 / E, kOcts = kCols / 8, kMine = MODE == MAT_GATED ? 32 : 64, kChunks = kMine / kCols;
        const uint32_t b0 = blocks + (warp - 4) * Shape::kBlocks * 2048, b1 = b0 + 2048;
        const bool eight = a.save == PALSGD_SAVE_8BIT, one = elect_one();
        bool stored = false;                                              // gate/up: the block may still be read by the copy engine
        uint32_t ge = 0, ue = 0;                                          // hidden, 8 bits: exponents of the block under way
        // hidden: gate and up of block c of a tile into the warp's two blocks
        auto fetch = [&](const Tile& tl, uint32_t c) {
            const uint32_t m = tl.m0 + rank * 128 + quad * 32, n = tl.n0 + part * kMine + c * kCols;
            const uint32_t M = tl.p->M, N = tl.p->N;
            const uint32_t rows = m < M ? min(M - m, 32u) : 0, cols = n < N ? N - n : 0;
            const int64_t w = tl.worker;
            const int64_t go = w * a.gate.w + (int64_t)m * a.gate.r + n, uo = w * a.up.w + (int64_t)m * a.up.r + n;
            if (eight) {
                block_in<1, kCols / 16>(b0, static_cast<const unsigned char*>(a.gate.p) + go, a.gate.r, rows, cols, a.gate.wide, lane);
                block_in<1, kCols / 16>(b1, static_cast<const unsigned char*>(a.up.p) + uo, a.up.r, rows, cols, a.up.wide, lane);
                const bool on = lane < rows && cols;
                ge = on ? static_cast<const uint8_t*>(a.gate_e.p)[w * a.gate_e.w + (int64_t)(m + lane) * a.gate_e.r + n / 32] : 0u;
                ue = on ? static_cast<const uint8_t*>(a.up_e.p)[w * a.up_e.w + (int64_t)(m + lane) * a.up_e.r + n / 32] : 0u;
            } else {
                block_in<E, 4>(b0, static_cast<const unsigned char*>(a.gate.p) + E * go, E * a.gate.r, rows, cols, a.gate.wide, lane);
                block_in<E, 4>(b1, static_cast<const unsigned char*>(a.up.p) + E * uo, E * a.up.r, rows, cols, a.up.wide, lane);
            }
        };
        // linear: the residual of block c of a tile into the warp's second block
        auto fetch_residual = [&](const Tile& tl, uint32_t c) {
            const uint32_t m = tl.m0 + rank * 128 + quad * 32, n = tl.n0 + part * kMine + c * kCols;
            const uint32_t M = tl.p->M, N = tl.p->N;
            const int64_t at = (int64_t)tl.worker * a.residual.w + (int64_t)m * a.residual.r + n;
            block_in<E, 4>(b1, static_cast<const unsigned char*>(a.residual.p) + E * at, E * a.residual.r, m < M ? min(M - m, 32u) : 0, n < N ? N - n : 0, a.residual.wide, lane);
        };
        if constexpr (MODE == MAT_LINEAR) if (a.residual.p) fetch_residual(tile_at<MODE>(a, Order(a, pair, pairs).now()), 0);
        if constexpr (MODE == MAT_HIDDEN) fetch(tile_at<MODE>(a, Order(a, pair, pairs).now()), 0);
        for (Order o(a, pair, pairs); o.now() < a.tiles; o.next()) {
            const Tile tl = tile_at<MODE>(a, o.now());
            const MatProblem& p = *tl.p;
            const uint32_t m = tl.m0 + rank * 128 + quad * 32, rows = m < p.M ? min(p.M - m, 32u) : 0;
            const int64_t w = tl.worker;
            uint32_t src = tmem + (it & 1) * kTileN + (quad << 21) + part * kMine;
            float bias[2] = {0.0f, 0.0f};                                 // linear: of the warp's columns lane and lane + 32
            if constexpr (MODE == MAT_LINEAR) {
                if (a.bias.p) {
#pragma unroll
                    for (uint32_t i = 0; i < 2; ++i) {
                        const uint32_t n = tl.n0 + part * kMine + 32 * i + lane;
                        if (n < p.N) bias[i] = to_f(static_cast<const T*>(a.bias.p)[w * a.bias.w + n]);
                    }
                }
            }
            // (a warp whose rows or columns are all outside has nothing to do but to let the sums go)
            const bool idle = (mat_plain(MODE) || MODE == MAT_LINEAR) && (rows == 0 || tl.n0 + part * kMine >= p.N);
            if (!cut) {
                if (!acc_wait()) break;
            } else if (MODE != MAT_GATED && MODE != MAT_HIDDEN && idle) {
                bool ok = true;
                uint32_t pieces = 0;
                for_pieces(tl, cut, [&](uint32_t, uint32_t, uint32_t, bool, bool) { ++pieces; return true; });
                while (ok && --pieces) {
                    ok = acc_wait();
                    if (ok) acc_read();
                }
                if (!ok || !acc_wait()) break;
            } else if constexpr (Shape::kWide || MODE == MAT_LINEAR) {
                // the pieces' sums joined in registers, and put back for what follows (kept there through the epilogue, they spill:
                // linear in 8 bits, 1024 tokens, 768 x 2048: 43 us, and 57)
                float sum[64];
#pragma unroll
                for (int i = 0; i < 64; ++i) sum[i] = 0.0f;
                uint32_t pieces = 0;
                for_pieces(tl, cut, [&](uint32_t, uint32_t, uint32_t, bool, bool) { ++pieces; return true; });
                bool ok = true;
                for (;;) {
                    src = tmem + (it & 1) * kTileN + (quad << 21) + part * kMine;
                    if (!acc_wait()) { ok = false; break; }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[16];
                        tmem_load16(src + (MODE == MAT_GATED && q >= 2 ? kTileN / 2 + (q - 2) * 16 : q * 16), v);
                        tmem_load_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[q * 16 + i] += v[i];
                    }
                    if (--pieces == 0) break;
                    acc_read();
                }
                if (!ok) break;
#pragma unroll
                for (int q = 0; q < 8; ++q) tmem_store8(src + (MODE == MAT_GATED && q >= 4 ? kTileN / 2 + (q - 4) * 8 : q * 8), sum + 8 * q);
                tmem_store_wait();
            }
            float gi = 0.0f, ui = 0.0f, inv = 0.0f;                       // 8 bits: one over the steps of the groups (gate/up; linear)
            if constexpr (MODE == MAT_GATED) {
                const uint32_t n = tl.n0 + part * kMine;
                if (eight) {
                    float gm = 0.0f, um = 0.0f;
#pragma unroll 1
                    for (uint32_t j = 0; j < 4; ++j) {
                        float v[8], u[8];
                        tmem_load8(src + 8 * j, v);
                        tmem_load8(src + kTileN / 2 + 8 * j, u);
                        tmem_load_wait();
#pragma unroll
                        for (int i = 0; i < 8; ++i) { gm = act8_max(gm, v[i]); um = act8_max(um, u[i]); }
                    }
                    const uint32_t eg = act8_exponent(gm), eu = act8_exponent(um);
                    gi = act8_inverse(eg); ui = act8_inverse(eu);
                    if (lane < rows && n < p.N) {
                        static_cast<uint8_t*>(a.gate_e.p)[w * a.gate_e.w + (int64_t)(m + lane) * a.gate_e.r + n / 32] = (uint8_t)eg;
                        static_cast<uint8_t*>(a.up_e.p)[w * a.up_e.w + (int64_t)(m + lane) * a.up_e.r + n / 32] = (uint8_t)eu;
                    }
                }
            }
            if (idle) {
                acc_read();
                if constexpr (MODE == MAT_LINEAR) if (a.residual.p && o.then() < a.tiles) fetch_residual(tile_at<MODE>(a, o.then()), 0);
                continue;
            }
            // linear: z = the sums + bias of a block, from the tile's column j on.  (The lanes hold a bias each: loaded where it is
            // needed, its latency stood in every block's way.)
            auto linear_z = [&](uint32_t j, f2 (&z)[kCols / 2]) {
                float v[kCols];
                const float mine = j < 32 ? bias[0] : bias[1];
#pragma unroll
                for (uint32_t i = 0; i < kCols; i += 16) tmem_load16(src + j + i, *reinterpret_cast<float(*)[16]>(v + i));
                tmem_load_wait();
                if (a.bias.p) {
#pragma unroll
                    for (uint32_t i = 0; i < kCols; ++i) v[i] += __shfl_sync(0xFFFFFFFFu, mine, (j & 31) + i);
                }
#pragma unroll
                for (uint32_t i = 0; i < kCols / 2; ++i) z[i] = f2_of(v[2 * i], v[2 * i + 1]);
            };
            auto linear_top = [](float top, const f2 (&z)[kCols / 2]) {   // the largest magnitude of a block and `top`
#pragma unroll
                for (uint32_t i = 0; i < kCols / 2; ++i) {
                    float x, y;
                    f2_get(z[i], x, y);
                    top = act8_max(act8_max(top, x), y);
                }
                return top;
            };
#pragma unroll 1
            for (uint32_t c = 0; c < kChunks; ++c) {
                const uint32_t from = src + c * kCols, n = tl.n0 + part * kMine + c * kCols;
                const uint32_t cols = n < p.N ? p.N - n : 0, room = n < p.out[0].cols ? p.out[0].cols - n : 0;
                const int64_t at = w * p.out[0].w + (int64_t)m * p.out[0].r + n;
                if constexpr (mat_plain(MODE)) {
                    if (E == 2 && p.splits > 1) {                         // binary32 sums of a share: 16 columns a block
                        float* to = static_cast<float*>(p.out[0].p) + (int64_t)tl.split * p.out[0].part + at;
#pragma unroll 1
                        for (uint32_t half = 0; half < 2; ++half) {
                            float v[16];
                            tmem_load16(from + 16 * half, v);
                            tmem_load_wait();
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                sts128(block_at<64>(b0, lane, j), make_uint4(__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3])));
                            __syncwarp();
                            block_out<64, 4>(b0, reinterpret_cast<unsigned char*>(to + 16 * half), 4 * p.out[0].r, rows, room > 16 * half ? room - 16 * half : 0, true, lane);
                            __syncwarp();
                        }
                        if (c + 1 == kChunks) acc_read();
                        continue;
                    }
#pragma unroll
                    for (uint32_t j = 0; j < kOcts; j += 2) {
                        float v[16];
                        tmem_load16(from + 8 * j, v);
                        tmem_load_wait();
                        f2 y[2][4];
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i / 4][i % 4] = f2_of(v[2 * i], v[2 * i + 1]);
                        row_put<T>(b0, lane, j, y[0]);
                        row_put<T>(b0, lane, j + 1, y[1]);
                    }
                    if (c + 1 == kChunks) acc_read();
                    __syncwarp();
                    const int64_t to = E == 4 && p.splits > 1 ? at + (int64_t)tl.split * p.out[0].part : at;
                    block_out<64, E>(b0, static_cast<unsigned char*>(p.out[0].p) + E * to, E * p.out[0].r, rows, room, p.out[0].wide, lane);
                    __syncwarp();
                } else if constexpr (MODE == MAT_LINEAR) {
                    // z of the block in registers; what is saved, then y, pass through one block; the residual comes into the
                    // other one while the products of the tile, or the work on the block before, still run
                    f2 z[kCols / 2];
                    linear_z(c * kCols, z);
                    if (a.save != PALSGD_SAVE_NONE) {
                        if (eight) {
                            if (E == 2 || c % 2 == 0) {                   // a group of 32 columns begins
                                float top = linear_top(0.0f, z);
                                if constexpr (E == 4) {
                                    f2 more[kCols / 2];
                                    linear_z((c + 1) * kCols, more);
                                    top = linear_top(top, more);
                                }
                                const uint32_t e = act8_exponent(top);
                                inv = act8_inverse(e);
                                if (lane < rows && cols) static_cast<uint8_t*>(a.gate_e.p)[w * a.gate_e.w + (int64_t)(m + lane) * a.gate_e.r + n / 32] = (uint8_t)e;
                            }
#pragma unroll
                            for (uint32_t j = 0; j < kOcts; ++j) {
                                float v[8];
#pragma unroll
                                for (int i = 0; i < 4; ++i) f2_get(z[4 * j + i], v[2 * i], v[2 * i + 1]);
                                row_put_act8<T>(b0, lane, j, inv, v);
                            }
                        } else {
#pragma unroll
                            for (uint32_t j = 0; j < kOcts; ++j) row_put<T>(b0, lane, j, *reinterpret_cast<f2(*)[4]>(z + 4 * j));
                        }
                        __syncwarp();
                        const int64_t to = w * a.gate.w + (int64_t)m * a.gate.r + n;
                        if (eight) block_out<kCols, 1>(b0, static_cast<unsigned char*>(a.gate.p) + to, a.gate.r, rows, cols, a.gate.wide, lane);
                        else block_out<64, E>(b0, static_cast<unsigned char*>(a.gate.p) + E * to, E * a.gate.r, rows, cols, a.gate.wide, lane);
                    }
                    if (c + 1 == kChunks) acc_read();
                    if (a.residual.p) block_wait();
                    __syncwarp();
#pragma unroll
                    for (uint32_t j = 0; j < kOcts; ++j) {
                        f2 r[4], unused;
#pragma unroll
                        for (int i = 0; i < 4; ++i) z[4 * j + i] = linear_act<T, ACT, false>(z[4 * j + i], unused);
                        if (a.residual.p) {
                            row_get<T>(b1, lane, j, r);
#pragma unroll
                            for (int i = 0; i < 4; ++i) z[4 * j + i] = f2_add(z[4 * j + i], r[i]);
                        }
                        row_put<T>(b0, lane, j, *reinterpret_cast<f2(*)[4]>(z + 4 * j));
                    }
                    __syncwarp();
                    if (a.residual.p) {
                        if (c + 1 < kChunks) fetch_residual(tl, c + 1);
                        else if (o.then() < a.tiles) fetch_residual(tile_at<MODE>(a, o.then()), 0);
                    }
                    block_out<64, E>(b0, static_cast<unsigned char*>(p.out[0].p) + E * at, E * p.out[0].r, rows, cols, p.out[0].wide, lane);
                    __syncwarp();
                } else if constexpr (MODE == MAT_GATED) {
                    // gate, up and h pass through one block, one after another (tensor memory is read again for each); h goes
                    // out by the copy engine, and the block is free again by the time the next tile is there
                    if (E == 2 && stored) { tma_store_read(); stored = false; }
                    __syncwarp();
                    if (a.save != PALSGD_SAVE_NONE) {
#pragma unroll 1
                        for (uint32_t which = 0; which < 2; ++which) {
                            const MatOut& s = which ? a.up : a.gate;
                            const float inv = which ? ui : gi;
#pragma unroll
                            for (uint32_t j = 0; j < kOcts; j += 2) {
                                float v[16];
                                tmem_load16(from + which * (kTileN / 2) + 8 * j, v);
                                tmem_load_wait();
                                if (eight) {
                                    row_put_act8<T>(b0, lane, j, inv, v);
                                    row_put_act8<T>(b0, lane, j + 1, inv, v + 8);
                                } else {
                                    f2 y[2][4];
#pragma unroll
                                    for (int i = 0; i < 8; ++i) y[i / 4][i % 4] = f2_of(v[2 * i], v[2 * i + 1]);
                                    row_put<T>(b0, lane, j, y[0]);
                                    row_put<T>(b0, lane, j + 1, y[1]);
                                }
                            }
                            __syncwarp();
                            const int64_t to = w * s.w + (int64_t)m * s.r + n;
                            if (eight) block_out<kCols, 1>(b0, static_cast<unsigned char*>(s.p) + to, s.r, rows, cols, s.wide, lane);
                            else block_out<64, E>(b0, static_cast<unsigned char*>(s.p) + E * to, E * s.r, rows, cols, s.wide, lane);
                            __syncwarp();
                        }
                    }
#pragma unroll 1
                    for (uint32_t j = 0; j < kOcts; ++j) {
                        float v[8], u[8];
                        tmem_load8(from + 8 * j, v);
                        tmem_load8(from + kTileN / 2 + 8 * j, u);
                        tmem_load_wait();
                        f2 h[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            f2 unused;
                            h[i] = f2_mul(act_pair<T, ACT, false>(f2_of(v[2 * i], v[2 * i + 1]), unused), f2_of(u[2 * i], u[2 * i + 1]));
                        }
                        row_put<T>(b0, lane, j, h);
                    }
                    if (E == 2) block_to_async();
                    if (c + 1 == kChunks) acc_read();
                    __syncwarp();
                    if constexpr (E == 2) {
                        if (one && rows && cols) {
                            tma_store(&a.store[0], b0, n, m, tl.worker);
                            tma_store_commit();
                            stored = true;
                        }
                    } else {
                        operand_out<T>(b0, p.out[0], at, rows, room, lane);
                        __syncwarp();
                    }
                } else {
                    block_wait();
                    __syncwarp();
                    const float gs = act8_step(ge), us = act8_step(ue);
#pragma unroll 1
                    for (uint32_t j = 0; j < kOcts; ++j) {
                        float v[8];
                        f2 g[4], q[4], dg[4], du[4], h[4];
                        tmem_load8(from + 8 * j, v);
                        if (eight) { row_get_act8<T>(b0, lane, j, gs, g); row_get_act8<T>(b1, lane, j, us, q); }
                        else { row_get<T>(b0, lane, j, g); row_get<T>(b1, lane, j, q); }
                        tmem_load_wait();
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            f2 slope;
                            const f2 ag = act_pair<T, ACT, true>(g[i], slope), d = f2_of(v[2 * i], v[2 * i + 1]);
                            dg[i] = f2_mul(f2_mul(d, q[i]), slope);
                            du[i] = f2_mul(d, ag);
                            h[i] = f2_mul(ag, q[i]);
                        }
                        row_put<T>(b0, lane, j, dg);
                        row_put<T>(b1, lane, j, du);
                        // h waits its turn in tensor memory, over sums that have been read
                        if constexpr (E == 2) {
                            const uint32_t hw[4] = {f2_narrow(h[0]), f2_narrow(h[1]), f2_narrow(h[2]), f2_narrow(h[3])};
                            tmem_store4(from + 4 * j, hw);
                        } else {
                            float hv[8];
#pragma unroll
                            for (int i = 0; i < 4; ++i) f2_get(h[i], hv[2 * i], hv[2 * i + 1]);
                            tmem_store8(from + 8 * j, hv);
                        }
                    }
                    tmem_store_wait();
                    float h[16];                                          // 64 bytes of a row in either type
                    tmem_load16(from, h);
                    if constexpr (E == 2) {
                        // dg and du leave by the copy engine (100 MB of dg, du and h: 49 us through the warps, 46 so)
                        block_to_async();
                        __syncwarp();
                        if (one && rows && cols) {
                            tma_store(&a.store[0], b0, n, m, tl.worker);
                            tma_store(&a.store[1], b1, n, m, tl.worker);
                            tma_store_commit();
                        }
                        tmem_load_wait();
                        if (c + 1 == kChunks) acc_read();
                        if (one) tma_store_read();
                        __syncwarp();
                    } else {
                        tmem_load_wait();
                        if (c + 1 == kChunks) acc_read();
                        __syncwarp();
                        operand_out<T>(b0, p.out[0], at, rows, room, lane);
                        operand_out<T>(b1, p.out[1], at, rows, room, lane);
                        __syncwarp();
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        sts128(block_at<64>(b0, lane, j), make_uint4(__float_as_uint(h[4 * j]), __float_as_uint(h[4 * j + 1]), __float_as_uint(h[4 * j + 2]), __float_as_uint(h[4 * j + 3])));
                    if (E == 2) block_to_async();
                    __syncwarp();
                    if constexpr (E == 2) {
                        if (one && rows && cols) {
                            tma_store(&a.store[2], b0, n, m, tl.worker);
                            tma_store_commit();
                            tma_store_read();
                        }
                    } else {
                        operand_out<T>(b0, p.out[2], at, rows, room, lane);
                    }
                    __syncwarp();
                    // the next block: of this tile, or the first of the warp's next tile
                    if (c + 1 < kChunks) fetch(tl, c + 1);
                    else if (o.then() < a.tiles) fetch(tile_at<MODE>(a, o.then()), 0);
                }
            }
        }
        if constexpr (MODE == MAT_HIDDEN || MODE == MAT_LINEAR) block_wait();
        if (E == 2 && (MODE == MAT_GATED || MODE == MAT_HIDDEN) && one) tma_store_done();
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
    Divisor  per_row;             // ld / 8
    int      kind;
    int      wide;                // eight values of src start on a 16-byte (8 bits: 8-byte) boundary in every row
    uint32_t K;                   // workers to copy: 1 if all read one matrix
};
struct StageArgs { StageItem item[kMaxStaged]; };

// Block `block` of the `blocks` that copy worker k's part of an item: a thread has U units under way (one where the grid
// holds a thread a unit: with four, a feed-forward backward call of 4 workers of 500 tokens, 333 x 1001, took 10.4 us for
// its copies instead of 7.3).
template <uint32_t U>
__device__ __forceinline__ void stage_item(const StageItem& it, int64_t k, uint32_t block, uint32_t blocks)
{
    if (k >= it.K) return;
    const uint64_t step = (uint64_t)blocks * 256;
    for (uint64_t i0 = (uint64_t)block * 256 + threadIdx.x; i0 < it.units; i0 += U * step) {
        uint4 q[U][2];                                    // as they lie in memory; 8 bits: the exponent behind them
        int64_t to[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint64_t i = i0 + u * step;
            to[u] = -1;
            if (i >= it.units) continue;
            const uint64_t row = it.units < 0x80000000ull ? it.per_row.of((uint32_t)i) : i / it.per_row.d;
            const uint32_t c = (uint32_t)(i - row * it.per_row.d) * 8, n = c < it.cols ? min(it.cols - c, 8u) : 0;
            const int64_t from = k * it.w + (int64_t)row * it.r + c;
            to[u] = (k * it.rows + (int64_t)row) * it.ld + c;
            if (it.kind == STAGE_BF16) {
                q[u][0] = get16(static_cast<const unsigned char*>(it.src) + 2 * from, 2 * n);
            } else if (it.kind == STAGE_ACT8) {
                const unsigned char* p = static_cast<const unsigned char*>(it.src) + from;
                if (it.wide && n == 8) { const uint2 t = __ldg(reinterpret_cast<const uint2*>(p)); q[u][0] = make_uint4(t.x, t.y, 0, 0); }
                else q[u][0] = get16(p, n);
                q[u][1].x = it.e[k * it.ew + (int64_t)row * it.er + c / 32];
            } else {
                const float* p = static_cast<const float*>(it.src) + from;
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j)
                    q[u][j] = it.wide && n == 8 ? __ldg(reinterpret_cast<const uint4*>(p) + j)
                                                : get16(reinterpret_cast<const unsigned char*>(p + 4 * j), n > 4 * j ? 4 * min(n - 4 * j, 4u) : 0);
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            if (to[u] < 0) continue;
            if (it.kind == STAGE_BF16) {
                *reinterpret_cast<uint4*>(it.dst + to[u]) = q[u][0];
            } else if (it.kind == STAGE_ACT8) {
                float v[8];
                const float s = act8_step(q[u][1].x);
                act8_value4(q[u][0].x, s, v);
                act8_value4(q[u][0].y, s, v + 4);
                Vec<bf16, 8>::store(it.dst + to[u], v);
            } else {
                float v[8];
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j) {
                    v[4 * j] = __uint_as_float(q[u][j].x); v[4 * j + 1] = __uint_as_float(q[u][j].y);
                    v[4 * j + 2] = __uint_as_float(q[u][j].z); v[4 * j + 3] = __uint_as_float(q[u][j].w);
                }
                three_parts<8>(v, [&](int part, const uint32_t (&w)[4]) { *reinterpret_cast<uint4*>(it.dst + to[u] + part * it.part) = make_uint4(w[0], w[1], w[2], w[3]); });
            }
        }
    }
}

__global__ void __launch_bounds__(256) stage_kernel(const __grid_constant__ StageArgs a)
{
    let_next_start();
    wait_for_previous();
    stage_item<1>(a.item[blockIdx.y], blockIdx.z, blockIdx.x, gridDim.x);
}

// The shares' sums of a product, joined in a fixed order.
struct JoinItem {
    const float* part;            // [splits][K][M][ld]
    int64_t  w, share;            // strides of a worker and of a share
    uint32_t splits, ld, M, N;
    uint64_t units;               // of 8 columns, one worker
    Divisor  per_row;             // ld / 8
    MatOut   out;
};
struct JoinArgs { JoinItem item[kMaxProblems]; };

template <typename T>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinArgs a)
{
    let_next_start();
    wait_for_previous();
    const JoinItem& it = a.item[blockIdx.y];
    const int64_t k = blockIdx.z;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < it.units; i += (uint64_t)gridDim.x * 256) {
        const uint32_t row = it.units < 0x80000000ull ? it.per_row.of((uint32_t)i) : (uint32_t)(i / it.per_row.d);
        const uint32_t c = (uint32_t)(i - (uint64_t)row * it.per_row.d) * 8;
        if (c >= it.N) continue;
        const float* p = it.part + k * it.w + (int64_t)row * it.ld + c;
        float sum[8];
        Vec<float, 8>::load(p, sum);
        for (uint32_t s = 1; s < it.splits; s += 4) {     // (four loads under way; the order of the sums stays)
            float v[4][8];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) if (s + u < it.splits) Vec<float, 8>::load(p + (s + u) * it.share, v[u]);
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u)
                if (s + u < it.splits)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] += v[u][j];
        }
        T* to = static_cast<T*>(it.out.p) + k * it.out.w + (int64_t)row * it.out.r + c;
        const uint32_t n = min(it.N - c, 8u);
        if (it.out.wide && n == 8) {
            Vec<T, 8>::store(to, sum);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) if (j < n) to[j] = from_f<T>(sum[j]);
        }
    }
}

}  // namespace block
}  // namespace palsgd
