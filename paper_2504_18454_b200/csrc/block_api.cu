// Host side of the block operators (see include/palsgd_block.h): checks of arguments, workspaces, launches.
#include "block_common.cuh"
#include "block_matmul.cuh"
#include "block_rows.cuh"

#include <cudaTypedefs.h>

#include <cmath>
#include <mutex>

#include "block_host.h"
#include "block_overlap.h"

using namespace palsgd::block;

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
inline size_t elem(int32_t prec) { return prec == PALSGD_PREC_BF16_MASTER ? 2 : 4; }
inline bool prec_ok(int32_t p) { return p == PALSGD_PREC_FP32 || p == PALSGD_PREC_BF16_MASTER; }

constexpr uint64_t kMaxSize = 0x7FFFFFFFull;             // rows, columns, tokens: 31 bits (offsets are 64-bit)
constexpr int64_t kMaxStride = (int64_t)1 << 40;

struct Axis { uint64_t n; int64_t stride; };

// No two of n0*n1*n2 runs of `run` contiguous elements at these strides share an element (sufficient condition: sorted
// by stride, each axis steps over all of the axes inside it).
bool disjoint(Axis a, Axis b, Axis c, uint64_t run)
{
    Axis v[3] = {a, b, c};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j + 1 < 3; ++j)
            if (v[j].stride > v[j + 1].stride) { const Axis t = v[j]; v[j] = v[j + 1]; v[j + 1] = t; }
    uint64_t span = run;
    for (const Axis& x : v) {
        if (x.n <= 1) continue;
        if ((uint64_t)x.stride < span) return false;
        span += (uint64_t)x.stride * (x.n - 1);
    }
    return true;
}

// A matrix argument with the strides of axes of at most one element, which nothing steps over, as zero.
struct Mat {
    palsgd_mat m{};
    bool given;
    Mat(const palsgd_mat* p, uint32_t K, uint64_t rows) : given(p != nullptr)
    {
        if (!p) return;
        m = *p;
        if (K <= 1) m.worker_stride = 0;
        if (rows <= 1) m.row_stride = 0;
    }
    operator const palsgd_mat*() const { return given ? &m : nullptr; }
};

struct HeadsOf {
    palsgd_heads m{};
    bool given;
    HeadsOf(const palsgd_heads* p, const palsgd_qk_shape* s, uint32_t heads) : given(p != nullptr)
    {
        if (!p) return;
        m = *p;
        if (s->K <= 1) m.worker_stride = 0;
        if (s->tokens <= 1) m.token_stride = 0;
        if (heads <= 1) m.head_stride = 0;
    }
    operator const palsgd_heads*() const { return given ? &m : nullptr; }
};

// A matrix argument: EINVAL / EALIGN / OK.  Nothing is asked of a matrix without elements.
int check_mat(const palsgd_mat* m, uint32_t K, uint64_t rows, uint64_t cols, size_t es, bool output)
{
    if (!m) return PALSGD_EINVAL;
    if (m->worker_stride < 0 || m->row_stride < 0 || m->worker_stride > kMaxStride || m->row_stride > kMaxStride) return PALSGD_EINVAL;
    if (rows == 0 || cols == 0) return PALSGD_OK;
    if (!m->data) return PALSGD_EINVAL;
    if (!aligned(m->data, es)) return PALSGD_EALIGN;
    if (output && !disjoint({K, m->worker_stride}, {rows, m->row_stride}, {1, 0}, cols)) return PALSGD_EINVAL;
    return PALSGD_OK;
}

Region region(const palsgd_mat* m, uint32_t K, uint64_t rows, uint64_t cols, size_t es)
{
    if (!m) return Region(nullptr, 0);
    return Region(m->data, cols * es).axis(0, K, m->worker_stride * (int64_t)es).axis(1, rows, m->row_stride * (int64_t)es);
}

#define BLOCK_TRY(call) do { const int rc_ = (call); if (rc_ != PALSGD_OK) return rc_; } while (0)

// A launch that may start up while the stream's previous kernel still runs (the kernels wait for it: block_common.cuh).
template <typename... A, typename... B>
int launch(const char* what, void (*kernel)(A...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, const B&... args)
{
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = grid; c.blockDim = dim3(threads); c.dynamicSmemBytes = smem; c.stream = st;
    c.attrs = &early; c.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&c, kernel, args...);
    if (e == cudaSuccess) return PALSGD_OK;
    (void)cudaGetLastError();
    return palsgd_block_cuda_fail((int)e, what);
}

int sm_count()
{
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = 148;
    return n;
}

Divisor divisor(uint32_t d)
{
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return Divisor{d, (uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
}

// ------------------------------------------------------------------------------------------------ 8-bit checkpoints

int check_act8(int32_t prec, uint32_t K, uint64_t rows, uint64_t cols, const palsgd_mat* x, const palsgd_mat* q,
               const palsgd_mat* e, bool pack)
{
    if (!prec_ok(prec) || K == 0 || K > PALSGD_MAX_WORKERS || rows > kMaxSize || cols > kMaxSize) return PALSGD_EINVAL;
    BLOCK_TRY(check_mat(x, K, rows, cols, elem(prec), !pack));
    BLOCK_TRY(check_mat(q, K, rows, cols, 1, pack));
    BLOCK_TRY(check_mat(e, K, rows, ceil_div(cols, PALSGD_ACT8_GROUP), 1, pack));
    const Region rx = region(x, K, rows, cols, elem(prec)), rq = region(q, K, rows, cols, 1), re = region(e, K, rows, ceil_div(cols, PALSGD_ACT8_GROUP), 1);
    Regions all;
    if (pack) { all.reads(rx); all.writes(rq); all.writes(re); }
    else { all.reads(rq); all.reads(re); all.writes(rx); }
    return all.clash() ? PALSGD_EINVAL : PALSGD_OK;
}

template <typename T, bool PACK>
int launch_act8(uint32_t K, uint64_t rows, uint64_t cols, const palsgd_mat* x, const palsgd_mat* q, const palsgd_mat* e,
                cudaStream_t st)
{
    if (rows == 0 || cols == 0) return PALSGD_OK;
    Act8Args a{x->data, static_cast<int8_t*>(q->data), static_cast<uint8_t*>(e->data), x->worker_stride, x->row_stride,
               q->worker_stride, q->row_stride, e->worker_stride, e->row_stride, rows, cols, 0, {}};
    const bool wide = cols % 8 == 0 && aligned(x->data, 16) && (x->row_stride * sizeof(T)) % 16 == 0 && (x->worker_stride * sizeof(T)) % 16 == 0 &&
                      aligned(q->data, 8) && q->row_stride % 8 == 0 && q->worker_stride % 8 == 0;
    // rows that follow one another without gaps and end with a group: one long row
    const bool flat = wide && cols % 32 == 0 &&
                      (rows == 1 || (x->row_stride == (int64_t)cols && q->row_stride == (int64_t)cols && e->row_stride == (int64_t)(cols / 32)));
    const uint64_t per_row = ceil_div(cols, 32) * 4;
    a.units = rows * per_row;
    a.per_row = divisor((uint32_t)per_row);
    const uint64_t ctas = ceil_div(a.units, 256 * (sizeof(T) == 4 ? 2 : 4));
    if (ctas > 0x7FFFFFFFull) return PALSGD_EUNSUPPORTED;
    const dim3 grid((unsigned)ctas, K);
    return launch(PACK ? "act8 pack" : "act8 unpack",
                  flat ? act8_kernel<T, PACK, ACT8_FLAT> : wide ? act8_kernel<T, PACK, ACT8_WIDE> : act8_kernel<T, PACK, ACT8_LOOSE>, grid, 256, 0, st, a);
}

// ------------------------------------------------------------------------------------------------ feed-forward block

int check_shape(const palsgd_ffn_shape* s)
{
    if (!s || s->K == 0 || s->K > PALSGD_MAX_WORKERS || !prec_ok(s->precision)) return PALSGD_EINVAL;
    if (s->activation < PALSGD_ACT_SILU || s->activation > PALSGD_ACT_RELU) return PALSGD_EINVAL;
    if (s->save < PALSGD_SAVE_NONE || s->save > PALSGD_SAVE_8BIT) return PALSGD_EINVAL;
    if (s->d_model == 0 || s->d_ff == 0 || s->d_model > kMaxSize || s->d_ff > kMaxSize || s->tokens > kMaxSize) return PALSGD_EINVAL;
    return PALSGD_OK;
}

int check_saved(const palsgd_ffn_shape* s, const palsgd_mat* gate, const palsgd_mat* up, const palsgd_mat* gate_e,
                const palsgd_mat* up_e, bool output)
{
    const bool eight = s->save == PALSGD_SAVE_8BIT;
    const size_t es = eight ? 1 : elem(s->precision);
    BLOCK_TRY(check_mat(gate, s->K, s->tokens, s->d_ff, es, output));
    BLOCK_TRY(check_mat(up, s->K, s->tokens, s->d_ff, es, output));
    if (eight) {
        BLOCK_TRY(check_mat(gate_e, s->K, s->tokens, ceil_div(s->d_ff, PALSGD_ACT8_GROUP), 1, output));
        BLOCK_TRY(check_mat(up_e, s->K, s->tokens, ceil_div(s->d_ff, PALSGD_ACT8_GROUP), 1, output));
    }
    return PALSGD_OK;
}

void add_saved(Regions& all, const palsgd_ffn_shape* s, const palsgd_mat* gate, const palsgd_mat* up, const palsgd_mat* gate_e,
               const palsgd_mat* up_e, bool output)
{
    if (s->save == PALSGD_SAVE_NONE) return;
    const bool eight = s->save == PALSGD_SAVE_8BIT;
    const palsgd_mat* m[4] = {gate, up, eight ? gate_e : nullptr, eight ? up_e : nullptr};
    for (int i = 0; i < 4; ++i) {
        const Region r = region(m[i], s->K, s->tokens, i < 2 ? s->d_ff : ceil_div(s->d_ff, PALSGD_ACT8_GROUP), i >= 2 || eight ? 1 : elem(s->precision));
        if (output) all.writes(r);
        else all.reads(r);
    }
}

// Hands out 256-byte aligned pieces of the workspace; with base = nullptr it only counts.
struct Arena {
    char* base;
    size_t used;
    void* take(size_t bytes)
    {
        void* p = base ? base + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return p;
    }
    // Never 0: a caller's buffer of no bytes may be NULL, and NULL asks for the size.
    size_t need() const { return used ? used : 256; }
};

int check_workspace(const void* ws, const size_t* bytes)
{
    if (!bytes) return PALSGD_EINVAL;
    if (ws && !aligned(ws, 256)) return PALSGD_EALIGN;
    return PALSGD_OK;
}

// The workspace's size is asked for or checked, and that nothing that the call writes overlaps.
int settle(const Arena& ws, size_t* bytes, Regions& all)
{
    if (ws.base && *bytes < ws.need()) { *bytes = ws.need(); return PALSGD_EINVAL; }
    all.writes(Region(ws.base, ws.used));
    if (all.clash()) return PALSGD_EINVAL;
    if (!ws.base) *bytes = ws.need();
    return PALSGD_OK;
}

// Set by a kernel whose wait gave up (see palsgd_block_status).
__device__ unsigned int g_gave_up;

constexpr int kMaxDevices = 64;

// What the matrix kernels need of a device, looked up on its first call.
struct Device {
    bool ready;
    int sms;
    unsigned int* gave_up;
};
Device g_device[kMaxDevices];
PFN_cuTensorMapEncodeTiled_v12000 g_encode;
std::mutex g_mutex;

template <typename T, int MODE, int ACT>
cudaError_t allow_smem() { return cudaFuncSetAttribute(mat_kernel<T, MODE, ACT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MatShape<T, MODE>::kSmem); }

template <typename T>
cudaError_t allow_smem_all()
{
    const cudaError_t e[9] = {allow_smem<T, MAT_PLAIN, 0>(),
                              allow_smem<T, MAT_GATED, 0>(), allow_smem<T, MAT_GATED, 1>(), allow_smem<T, MAT_GATED, 2>(), allow_smem<T, MAT_GATED, 3>(),
                              allow_smem<T, MAT_HIDDEN, 0>(), allow_smem<T, MAT_HIDDEN, 1>(), allow_smem<T, MAT_HIDDEN, 2>(), allow_smem<T, MAT_HIDDEN, 3>()};
    for (cudaError_t r : e) if (r != cudaSuccess) return r;
    return cudaSuccess;
}

int device_of(Device& out)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return palsgd_block_cuda_fail((int)e, "cudaGetDevice");
    if (dev < 0 || dev >= kMaxDevices) return PALSGD_EUNSUPPORTED;
    // The device's context has to be current in this thread before the driver is asked for tensor maps: a thread that has
    // made no call of the runtime's yet (autograd's, say) has none.
    e = cudaSetDevice(dev);
    if (e != cudaSuccess) return palsgd_block_cuda_fail((int)e, "cudaSetDevice");
    std::lock_guard<std::mutex> lock(g_mutex);
    Device& d = g_device[dev];
    if (!d.ready) {
        if (!g_encode) {
            void* f = nullptr;
            cudaDriverEntryPointQueryResult found;
            e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
            if (e == cudaSuccess && (found != cudaDriverEntryPointSuccess || !f)) e = cudaErrorSymbolNotFound;
            if (e != cudaSuccess) return palsgd_block_cuda_fail((int)e, "cuTensorMapEncodeTiled");
            g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
        }
        void* p = nullptr;
        e = cudaGetSymbolAddress(&p, g_gave_up);
        if (e == cudaSuccess) e = allow_smem_all<float>();
        if (e == cudaSuccess) e = allow_smem_all<bf16>();
        if (e != cudaSuccess) return palsgd_block_cuda_fail((int)e, "matrix kernel set-up");
        d.gave_up = static_cast<unsigned int*>(p);
        d.sms = sm_count();
        d.ready = true;
    }
    out = d;
    return PALSGD_OK;
}

// An operand as the copy engine reads it: bfloat16 [parts][K][rows][cols], in the caller's memory or the workspace.
struct Operand {
    const void* p;
    int64_t w, r, part;
    uint64_t rows, cols;
    uint32_t K, parts;
    bool one;                                            // all workers read one matrix
};

struct Stage {
    StageArgs a{};
    uint32_t n = 0;
};

// Rows in the workspace: bfloat16 in rows of a multiple of 16 bytes.
Operand own_operand(Arena& ws, uint32_t K, uint64_t rows, uint64_t cols, uint32_t parts)
{
    const int64_t ld = (int64_t)(ceil_div(cols, 8) * 8);
    Operand o{nullptr, ld * (int64_t)rows, ld, ld * (int64_t)rows * K, rows, cols, K, parts, false};
    o.p = ws.take((size_t)parts * o.part * 2);
    return o;
}

// Reads m in place where the copy engine can (bfloat16, 16-byte boundaries), else puts it on the list of copies.
Operand input_operand(Arena& ws, Stage& st, const palsgd_mat* m, const palsgd_mat* e, int32_t prec, uint32_t K, uint64_t rows, uint64_t cols)
{
    const bool one = K == 1 || m->worker_stride == 0;
    const int64_t w = one ? 0 : m->worker_stride, r = rows == 1 ? (int64_t)(ceil_div(cols, 8) * 8) : m->row_stride;
    if (!e && prec == PALSGD_PREC_BF16_MASTER && aligned(m->data, 16) && r % 8 == 0 && w % 8 == 0 && r >= (int64_t)cols &&
        r < kMaxStride / 2 && w < kMaxStride / 2)
        return Operand{m->data, w, r, 0, rows, cols, K, 1, one};
    const int kind = e ? STAGE_ACT8 : prec == PALSGD_PREC_FP32 ? STAGE_SPLIT : STAGE_BF16;
    const uint32_t copies = one && (!e || K == 1 || e->worker_stride == 0) ? 1 : K;
    Operand o = own_operand(ws, copies, rows, cols, kind == STAGE_SPLIT ? 3 : 1);
    o.K = K;
    o.one = copies == 1;
    const int64_t unit = kind == STAGE_SPLIT ? 4 : 8;    // elements between the boundaries of wide loads
    const bool wide = aligned(m->data, kind == STAGE_ACT8 ? 8 : 16) && m->row_stride % unit == 0 && w % unit == 0;
    StageItem& it = st.a.item[st.n++];
    it = StageItem{m->data, e ? static_cast<const uint8_t*>(e->data) : nullptr, w, m->row_stride, e ? e->worker_stride : 0, e ? e->row_stride : 0,
                   static_cast<bf16*>(const_cast<void*>(o.p)), o.r, o.part, (uint32_t)rows, (uint32_t)cols, rows * (uint64_t)(o.r / 8), divisor((uint32_t)(o.r / 8)), kind, wide, copies};
    return o;
}

int run_stage(const Stage& st, uint32_t K, int sms, cudaStream_t stream)
{
    if (st.n == 0) return PALSGD_OK;
    uint64_t most = 1;
    for (uint32_t i = 0; i < st.n; ++i) most = st.a.item[i].units > most ? st.a.item[i].units : most;
    const uint64_t want = ceil_div(most, 256), cap = 32ull * sms;
    return launch("operand copies", stage_kernel, dim3((unsigned)(want < cap ? want : cap), st.n, K), 256, 0, stream, st.a);
}

// box: columns and rows of one copy, its order in shared memory
int encode(CUtensorMap* map, const Operand& o, uint32_t box_cols, uint32_t box_rows, CUtensorMapSwizzle order)
{
    const cuuint64_t dims[4] = {o.cols, o.rows, o.one ? 1u : o.K, o.parts};
    // a dimension of one element is never stepped over, but its stride has to be a valid one
    const cuuint64_t row = (cuuint64_t)o.r * 2, w = o.one ? row : (cuuint64_t)o.w * 2, part = o.parts > 1 ? (cuuint64_t)o.part * 2 : row;
    const cuuint64_t strides[3] = {row, w, part};
    const cuuint32_t box[4] = {box_cols, box_rows, 1, 1}, unit[4] = {1, 1, 1, 1};
    const CUresult rc = g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(o.p), dims, strides, box, unit,
                                 CU_TENSOR_MAP_INTERLEAVE_NONE, order, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (rc == CUDA_SUCCESS) return PALSGD_OK;
    return palsgd_block_cuda_fail((int)rc, "cuTensorMapEncodeTiled");   // (the runtime's codes are the driver's)
}

int encode(CUtensorMap* map, const Operand& o, bool mn) { return encode(map, o, 64, mn ? kTileK : 128, CU_TENSOR_MAP_SWIZZLE_128B); }
int encode_store(CUtensorMap* map, const Operand& o) { return encode(map, o, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B); }

MatOut out_of(const palsgd_mat* m, uint64_t cols, size_t es)
{
    MatOut o{m->data, m->worker_stride, m->row_stride, 0, 0, (uint32_t)cols};
    o.wide = aligned(m->data, 16) && (m->worker_stride * es) % 16 == 0 && (m->row_stride * es) % 16 == 0;
    return o;
}
MatOut out_of(const Operand& o) { return MatOut{const_cast<void*>(o.p), o.w, o.r, o.part, 1, (uint32_t)o.r}; }

// One product appended to a launch; B1/A1: the second segment, or (gate/up) the up weights as B1.
int add_problem(MatLaunch& L, uint64_t M, uint64_t N, uint64_t Kd, uint32_t K, const Operand* A0, const Operand* A1, bool amn,
                const Operand* B0, const Operand* B1, bool bmn, uint32_t n_step)
{
    MatProblem& p = L.p[L.n_problems++];
    p.M = (uint32_t)M; p.N = (uint32_t)N; p.Kd = (uint32_t)Kd;
    const uint64_t down = ceil_div(M, kTileM), across = ceil_div(N, n_step), tiles = down * across * K;
    if (down * across > 0x7FFFFFFFull || L.tiles + tiles > 0x7FFFFFFFull) return PALSGD_EUNSUPPORTED;
    p.tiles_m = divisor((uint32_t)down);
    p.per_split = p.per_worker = divisor((uint32_t)(down * across));
    p.splits = 1;
    p.tiles = (uint32_t)tiles;
    L.tiles += p.tiles;
    p.n_seg = A1 ? 2 : 1;
    p.a_parts = (uint8_t)A0->parts; p.b_parts = (uint8_t)B0->parts; p.a_mn = amn; p.b_mn = bmn;
    const Operand *A[2] = {A0, A1}, *B[2] = {B0, B1};
    for (int i = 0; i < 2; ++i) {
        if (A[i]) { p.a_one[i] = A[i]->one; BLOCK_TRY(encode(&p.A[i], *A[i], amn)); }
        if (B[i]) { p.b_one[i] = B[i]->one; BLOCK_TRY(encode(&p.B[i], *B[i], bmn)); }
    }
    return PALSGD_OK;
}

// One product of a plain launch as the host plans it.
struct Product {
    uint64_t M, N, Kd;
    const Operand *A0, *A1, *B0, *B1;
    bool amn, bmn;
    const palsgd_mat* out;
    uint32_t splits;
    const float* part;
    uint64_t tiles(uint32_t K) const { return ceil_div(M, kTileM) * ceil_div(N, kTileN) * K; }
    uint64_t steps(uint32_t parts) const { return (A1 ? 2 : 1) * ceil_div(Kd, kTileK) * (parts == 3 ? 6 : 1); }
    static uint64_t length_of(uint64_t steps) { return (steps > kTileLeast ? steps : kTileLeast) + 1; }
    uint64_t length(uint32_t parts) const { return length_of(ceil_div(steps(parts), splits)); }
    int64_t ld() const { return (int64_t)(ceil_div(N, 8) * 8); }
};

// Cuts long inner axes into shares where a launch has too few tiles for the pairs of CTAs: the shares' binary32 sums go
// to the workspace and one more small kernel joins them (kJoin: what that costs, in steps of about 0.35 us; kStepBytes: the
// sums that are written and read again in a step's time).  Of a few cuts -- shares of the average load of a pair, or up to
// three times that -- the one that should end first, if it ends before no cut at all.  (One worker, one token, 2048 x
// 5632: the second product is 8 tiles of 88 steps, the forward call 68 us uncut and 48 us cut.)
constexpr uint64_t kJoin = 26, kStepBytes = 4000000;
constexpr uint32_t kMaxSplits = 32;

void plan_splits(Product* p, int n, uint32_t K, uint32_t parts, uint64_t pairs)
{
    uint64_t work = 0;
    for (int i = 0; i < n; ++i) { p[i].splits = 1; work += p[i].tiles(K) * p[i].length(parts); }
    const uint64_t least = work / pairs > 8 ? work / pairs : 8;
    // when the last tile ends, the longer tiles being taken up first
    auto end_of = [&](uint64_t share) {
        uint64_t tiles = 0, all = 0, longest = 0, shortest = ~0ull, rounds = 0, bytes = 0;
        bool joins = false;
        for (int i = 0; i < n; ++i) {
            const uint64_t s = p[i].steps(parts), c = share ? ceil_div(s, share) : 1, split = c > kMaxSplits ? kMaxSplits : c;
            const uint64_t len = Product::length_of(ceil_div(s, split)), count = p[i].tiles(K) * split;
            tiles += count; all += count * len;
            rounds = ceil_div(tiles, pairs) * len;       // (of products that are alike)
            longest = len > longest ? len : longest;
            shortest = len < shortest ? len : shortest;
            if (split > 1) { joins = true; bytes += 8 * split * K * p[i].M * (uint64_t)p[i].ld(); }
        }
        uint64_t e = longest == shortest ? rounds : all / pairs + shortest;
        if (e < longest) e = longest;
        return e + (joins ? kJoin + bytes / kStepBytes : 0);
    };
    uint64_t best = end_of(0), share = 0;
    for (uint64_t quarter = 4; quarter <= 12; ++quarter) {
        const uint64_t s = least * quarter / 4, e = end_of(s);
        if (e < best) { best = e; share = s; }
    }
    for (int i = 0; share && i < n; ++i) {
        const uint64_t c = ceil_div(p[i].steps(parts), share);
        // (fp32: a share is of whole steps of the inner axis)
        const uint64_t most = p[i].steps(1);
        p[i].splits = (uint32_t)(c > kMaxSplits ? kMaxSplits : c);
        if (p[i].splits > most) p[i].splits = (uint32_t)most;
    }
}

template <typename T, int MODE, int ACT>
int launch_mat(const MatLaunch& L, uint32_t pairs, cudaStream_t st)
{
    return launch("matrix kernel", mat_kernel<T, MODE, ACT>, dim3(2 * pairs), MatShape<T, MODE>::kThreads, MatShape<T, MODE>::kSmem, st, L);
}

template <typename T, int MODE>
int launch_mat(const MatLaunch& L, int act, uint32_t pairs, cudaStream_t st)
{
    if constexpr (MODE == MAT_PLAIN) {
        return launch_mat<T, MODE, 0>(L, pairs, st);
    } else {
        switch (act) {
            case PALSGD_ACT_SILU: return launch_mat<T, MODE, PALSGD_ACT_SILU>(L, pairs, st);
            case PALSGD_ACT_GELU: return launch_mat<T, MODE, PALSGD_ACT_GELU>(L, pairs, st);
            case PALSGD_ACT_GELU_TANH: return launch_mat<T, MODE, PALSGD_ACT_GELU_TANH>(L, pairs, st);
            default: return launch_mat<T, MODE, PALSGD_ACT_RELU>(L, pairs, st);
        }
    }
}

template <int MODE>
int run_mat(MatLaunch& L, const palsgd_ffn_shape* s, const Device& d, cudaStream_t st)
{
    if (L.tiles == 0) return PALSGD_OK;
    L.gave_up = d.gave_up;
    const uint32_t pairs = (uint32_t)(d.sms / 2) < L.tiles ? (uint32_t)(d.sms / 2) : L.tiles;
    return s->precision == PALSGD_PREC_FP32 ? launch_mat<float, MODE>(L, s->activation, pairs, st) : launch_mat<bf16, MODE>(L, s->activation, pairs, st);
}

// Decides on the shares and takes the workspace for their sums (the same decision in both calls of an entry point: it
// goes by sizes alone, for the device's pairs of CTAs).
void take_shares(Arena& ws, Product* p, int n, uint32_t K, uint32_t parts)
{
    plan_splits(p, n, K, parts, (uint64_t)sm_count() / 2);
    for (int i = 0; i < n; ++i)
        if (p[i].splits > 1) p[i].part = static_cast<const float*>(ws.take((size_t)p[i].splits * K * p[i].M * (size_t)p[i].ld() * sizeof(float)));
}

// The products of a call in one launch, the longer ones first, and the kernel that joins what was cut.
int run_products(Product* p, int n, const palsgd_ffn_shape* s, const Device& d, size_t es, uint32_t parts, cudaStream_t st)
{
    MatLaunch L{};
    JoinArgs join{};
    uint32_t joins = 0;
    uint64_t units = 0;
    int heavy = 0;                                       // products whose tiles are the longer ones (Order)
    if (n == 4) {                                        // dx and the three weight gradients, which are alike
        heavy = 1;
        if (p[0].length(parts) < p[1].length(parts)) {
            const Product x = p[0];
            for (int i = 0; i < 3; ++i) p[i] = p[i + 1];
            p[3] = x;
            heavy = 3;
        }
    }
    for (int i = 0; i < n; ++i) {
        BLOCK_TRY(add_problem(L, p[i].M, p[i].N, p[i].Kd, s->K, p[i].A0, p[i].A1, p[i].amn, p[i].B0, p[i].B1, p[i].bmn, kTileN));
        MatProblem& q = L.p[i];
        q.out[0] = out_of(p[i].out, p[i].N, es);
        if (p[i].splits > 1) {
            JoinItem& j = join.item[joins++];
            const int64_t ld = p[i].ld(), w = ld * (int64_t)p[i].M;
            j = JoinItem{p[i].part, w, w * s->K, p[i].splits, (uint32_t)ld, (uint32_t)p[i].M, (uint32_t)p[i].N, p[i].M * (uint64_t)(ld / 8), divisor((uint32_t)(ld / 8)), q.out[0]};
            if (j.units > units) units = j.units;
            q.out[0] = MatOut{const_cast<float*>(p[i].part), w, ld, w * s->K, 1, (uint32_t)ld};
            q.splits = p[i].splits;
            const uint64_t per = (uint64_t)q.per_split.d * q.splits, tiles = per * s->K;
            if (per > 0x7FFFFFFFull || L.tiles - q.tiles + tiles > 0x7FFFFFFFull) return PALSGD_EUNSUPPORTED;
            q.per_worker = divisor((uint32_t)per);
            L.tiles += (uint32_t)tiles - q.tiles;
            q.tiles = (uint32_t)tiles;
        }
        if (i + 1 == heavy) L.heavy = L.tiles;
    }
    if (heavy) L.lag = (uint32_t)(p[0].length(parts) / p[n - 1].length(parts));
    BLOCK_TRY(run_mat<MAT_PLAIN>(L, s, d, st));
    if (joins == 0) return PALSGD_OK;
    const uint64_t want = ceil_div(units, 256), cap = 16ull * d.sms;
    const dim3 grid((unsigned)(want < cap ? want : cap), joins, s->K);
    return launch("joined shares", es == 4 ? join_kernel<float> : join_kernel<bf16>, grid, 256, 0, st, join);
}

void set_saved(MatLaunch& L, const palsgd_ffn_shape* s, const palsgd_mat* gate, const palsgd_mat* up, const palsgd_mat* gate_e, const palsgd_mat* up_e)
{
    L.save = s->save;
    if (s->save == PALSGD_SAVE_NONE) return;
    const size_t es = s->save == PALSGD_SAVE_8BIT ? 1 : elem(s->precision);
    L.gate = out_of(gate, s->d_ff, es);
    L.up = out_of(up, s->d_ff, es);
    if (s->save == PALSGD_SAVE_8BIT) { L.gate_e = out_of(gate_e, 0, 1); L.up_e = out_of(up_e, 0, 1); }
}

// ------------------------------------------------------------------------------------------------ q/k norm + rotation

int check_heads(const palsgd_heads* h, const palsgd_qk_shape* s, uint32_t heads, bool output)
{
    if (heads == 0) return PALSGD_OK;
    if (!h || h->worker_stride < 0 || h->token_stride < 0 || h->head_stride < 0) return PALSGD_EINVAL;
    if (h->worker_stride > kMaxStride || h->token_stride > kMaxStride || h->head_stride > kMaxStride) return PALSGD_EINVAL;
    if (s->tokens == 0) return PALSGD_OK;
    if (!h->data) return PALSGD_EINVAL;
    if (!aligned(h->data, elem(s->precision))) return PALSGD_EALIGN;
    if (output && !disjoint({s->K, h->worker_stride}, {s->tokens, h->token_stride}, {heads, h->head_stride}, s->head_dim)) return PALSGD_EINVAL;
    return PALSGD_OK;
}

int check_qk(const palsgd_qk_shape* s, const float* cos_t, const float* sin_t, const int32_t* pos)
{
    if (!s || s->K == 0 || s->K > PALSGD_MAX_WORKERS || !prec_ok(s->precision) || s->reserved_ != 0) return PALSGD_EINVAL;
    if (s->tokens > kMaxSize || s->heads_q > 65535u || s->heads_k > 65535u) return PALSGD_EINVAL;
    if (s->head_dim == 0 || s->rotary_dim > s->head_dim || s->rotary_dim % 2) return PALSGD_EINVAL;
    if (s->interleaved != 0 && s->interleaved != 1) return PALSGD_EINVAL;
    if (!(std::isfinite(s->eps) && s->eps >= 0.0)) return PALSGD_EINVAL;
    if (s->pos_worker_stride < 0 || s->pos_worker_stride > kMaxStride || s->table_rows > kMaxSize) return PALSGD_EINVAL;
    if (s->rotary_dim && s->tokens) {
        if (!pos || (s->table_rows && (!cos_t || !sin_t))) return PALSGD_EINVAL;
        if (!aligned(pos, 4) || !aligned(cos_t, 4) || !aligned(sin_t, 4)) return PALSGD_EALIGN;
    }
    if (s->head_dim > 512) return PALSGD_EUNSUPPORTED;
    return PALSGD_OK;
}

Region region(const palsgd_heads* h, const palsgd_qk_shape* s, uint32_t heads)
{
    const int64_t es = (int64_t)elem(s->precision);
    if (!h || heads == 0) return Region(nullptr, 0);
    return Region(h->data, s->head_dim * (uint64_t)es).axis(0, s->K, h->worker_stride * es).axis(1, s->tokens, h->token_stride * es).axis(2, heads, h->head_stride * es);
}

// The tables and positions of a call
void add_angles(Regions& all, const palsgd_qk_shape* s, const float* cos_t, const float* sin_t, const int32_t* pos)
{
    if (s->rotary_dim == 0 || s->tokens == 0) return;
    all.reads(Region(cos_t, s->table_rows * (s->rotary_dim / 2) * 4));
    all.reads(Region(sin_t, s->table_rows * (s->rotary_dim / 2) * 4));
    all.reads(Region(pos, s->tokens * 4).axis(0, s->K, s->pos_worker_stride * 4));
}

bool heads_wide(const void* p, int64_t w, int64_t t, int64_t h, size_t es)
{
    return aligned(p, 16) && (w * es) % 16 == 0 && (t * es) % 16 == 0 && (h * es) % 16 == 0;
}

struct QkPlan { QkArgs a; int V, NS, pairs; };

// CTAs by the workers, and by q and k as their heads are.  Needs nothing of the operands: the workspace goes by it.
void share_out(QkArgs& a, const palsgd_qk_shape* s, bool back)
{
    const uint32_t heads[2] = {s->heads_q, s->heads_k}, all = heads[0] + heads[1];
    const uint64_t slots = (uint64_t)qk_ctas_per_sm(back) * sm_count() / s->K;
    for (int i = 0; i < 2; ++i) {
        uint64_t n = all ? slots * heads[i] / all : 0;
        const uint64_t most = ceil_div(s->tokens, kQkThreads / 32);
        if (n > most) n = most;
        if (heads[i] && n == 0) n = 1;
        a.ctas[i] = (uint32_t)n;
    }
}

QkPlan plan_qk(const palsgd_qk_shape* s, const float* cos_t, const float* sin_t, const int32_t* pos, bool back)
{
    QkPlan p{};
    QkArgs& a = p.a;
    a.cos_t = cos_t; a.sin_t = sin_t; a.pos = pos; a.pos_w = s->pos_worker_stride;
    a.tokens = s->tokens; a.table_rows = s->table_rows; a.head_dim = s->head_dim; a.rot = s->rotary_dim;
    a.eps = (float)s->eps;
    a.table_wide = s->rotary_dim % 8 == 0 && aligned(cos_t, 16) && aligned(sin_t, 16);
    a.side[0].heads = s->heads_q; a.side[1].heads = s->heads_k;
    share_out(a, s, back);
    return p;
}

void finish_qk(QkPlan& p, const palsgd_qk_shape* s, bool back)
{
    QkArgs& a = p.a;
    const size_t es = elem(s->precision);
    const int v = (int)(16 / es);
    bool wide = s->head_dim % v == 0;
    for (const HeadsArg& h : a.side)
        if (h.heads)
            wide = wide && heads_wide(h.x, h.xw, h.xt, h.xh, es) && heads_wide(h.out, h.ow, h.ot, h.oh, es) &&
                   (!back || heads_wide(h.d, h.dw, h.dt, h.dh, es));
    p.V = wide ? v : 1;
    const uint32_t half = s->rotary_dim / 2, n_vec = s->head_dim / p.V;
    p.pairs = s->interleaved ? QK_INTER : half % p.V ? QK_CROSS : QK_SPLIT;
    a.pair_slots = p.pairs == QK_SPLIT || p.V == 1 ? half / p.V : 0;
    a.slots = p.pairs == QK_SPLIT ? half / p.V + (n_vec - 2 * (half / p.V) + 1) / 2 : (n_vec + 1) / 2;
    a.lanes = 1;
    while (a.lanes < 32 && a.lanes < a.slots) a.lanes *= 2;
    p.NS = 1;
    while ((uint32_t)p.NS * a.lanes < a.slots) p.NS *= 2;
    // Heads abreast: the most that divide the heads evenly and leave each group four in a row, over which it forms the
    // token's products once; more where there are too few tokens to keep every warp busy.
    const uint32_t groups = 32 / a.lanes;
    for (int i = 0; i < 2; ++i) {
        const uint32_t heads = a.side[i].heads;
        uint32_t n = 1;
        while (n < groups && n < heads &&
               ((heads % (2 * n) == 0 && heads / (2 * n) >= 4) || s->tokens * s->K * n < (uint64_t)(qk_ctas_per_sm(back) * (kQkThreads / 32)) * sm_count() * groups))
            n *= 2;
        a.abreast[i] = n;
    }
}

template <typename T, bool BACK, int PAIRS>
int launch_qk(const QkPlan& p, const palsgd_qk_shape* s, cudaStream_t st)
{
    const dim3 grid(p.a.ctas[0] + p.a.ctas[1], s->K);
    constexpr int W = 16 / (int)sizeof(T);
    const char* what = "q/k norm + rotation";
    auto run = [&](void (*kernel)(const QkArgs), int V, int NS) { return launch(what, kernel, grid, kQkThreads, qk_smem(V, NS, BACK, s->head_dim), st, p.a); };
    if (p.V == W && p.NS == 1) {
        switch (p.a.lanes) {
            case 4: return run(qk_kernel<T, W, 1, BACK, PAIRS, 4>, W, 1);
            case 8: return run(qk_kernel<T, W, 1, BACK, PAIRS, 8>, W, 1);
            case 16: return run(qk_kernel<T, W, 1, BACK, PAIRS, 16>, W, 1);
            default: return run(qk_kernel<T, W, 1, BACK, PAIRS, 0>, W, 1);
        }
    }
    if constexpr (W == 4) {                              // (bfloat16: 512 values are 32 slots, one a lane)
        if (p.V == W) return run(qk_kernel<T, W, 2, BACK, PAIRS, 32>, W, 2);
    }
    if constexpr (PAIRS != QK_CROSS) {                   // (one value a vector is never across)
        if (p.NS <= 2) return run(qk_kernel<T, 1, 2, BACK, PAIRS, 0>, 1, 2);
        return run(qk_kernel<T, 1, 8, BACK, PAIRS, 32>, 1, 8);
    }
    return PALSGD_EUNSUPPORTED;
}

template <typename T, bool BACK>
int launch_qk(const QkPlan& p, const palsgd_qk_shape* s, cudaStream_t st)
{
    return p.pairs == QK_INTER ? launch_qk<T, BACK, QK_INTER>(p, s, st) : p.pairs == QK_CROSS ? launch_qk<T, BACK, QK_CROSS>(p, s, st) : launch_qk<T, BACK, QK_SPLIT>(p, s, st);
}

template <bool BACK>
int run_qk(const QkPlan& p, const palsgd_qk_shape* s, cudaStream_t st)
{
    return s->precision == PALSGD_PREC_FP32 ? launch_qk<float, BACK>(p, s, st) : launch_qk<bf16, BACK>(p, s, st);
}

}  // namespace

extern "C" int palsgd_act8_pack(int32_t precision, uint32_t K, uint64_t rows, uint64_t cols, const palsgd_mat* x_,
                                const palsgd_mat* q_, const palsgd_mat* e_, void* stream)
{
    const Mat x(x_, K, rows), q(q_, K, rows), e(e_, K, rows);
    BLOCK_TRY(check_act8(precision, K, rows, cols, x, q, e, true));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return precision == PALSGD_PREC_FP32 ? launch_act8<float, true>(K, rows, cols, x, q, e, st)
                                         : launch_act8<bf16, true>(K, rows, cols, x, q, e, st);
}

extern "C" int palsgd_act8_unpack(int32_t precision, uint32_t K, uint64_t rows, uint64_t cols, const palsgd_mat* q_,
                                  const palsgd_mat* e_, const palsgd_mat* x_, void* stream)
{
    const Mat x(x_, K, rows), q(q_, K, rows), e(e_, K, rows);
    BLOCK_TRY(check_act8(precision, K, rows, cols, x, q, e, false));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return precision == PALSGD_PREC_FP32 ? launch_act8<float, false>(K, rows, cols, x, q, e, st)
                                         : launch_act8<bf16, false>(K, rows, cols, x, q, e, st);
}

extern "C" int palsgd_ffn_forward(const palsgd_ffn_shape* s, const palsgd_mat* x_, const palsgd_mat* w_gate_,
                                  const palsgd_mat* w_up_, const palsgd_mat* w_down_, const palsgd_mat* y_,
                                  const palsgd_mat* gate_, const palsgd_mat* up_, const palsgd_mat* gate_e_,
                                  const palsgd_mat* up_e_, void* workspace, size_t* workspace_bytes, void* stream)
{
    BLOCK_TRY(check_shape(s));
    const Mat x(x_, s->K, s->tokens), w_gate(w_gate_, s->K, s->d_ff), w_up(w_up_, s->K, s->d_ff), w_down(w_down_, s->K, s->d_model);
    const Mat y(y_, s->K, s->tokens), gate(gate_, s->K, s->tokens), up(up_, s->K, s->tokens), gate_e(gate_e_, s->K, s->tokens), up_e(up_e_, s->K, s->tokens);
    const uint64_t M = s->tokens, D = s->d_model, F = s->d_ff;
    const size_t es = elem(s->precision);
    BLOCK_TRY(check_mat(x, s->K, M, D, es, false));
    BLOCK_TRY(check_mat(w_gate, s->K, F, D, es, false));
    BLOCK_TRY(check_mat(w_up, s->K, F, D, es, false));
    BLOCK_TRY(check_mat(w_down, s->K, D, F, es, false));
    BLOCK_TRY(check_mat(y, s->K, M, D, es, true));
    if (s->save != PALSGD_SAVE_NONE) BLOCK_TRY(check_saved(s, gate, up, gate_e, up_e, true));
    BLOCK_TRY(check_workspace(workspace, workspace_bytes));
    Arena ws{static_cast<char*>(workspace), 0};
    Stage stage;
    const uint32_t parts = s->precision == PALSGD_PREC_FP32 ? 3 : 1;
    Operand ox, og, ou, od, oh;
    if (M) {
        ox = input_operand(ws, stage, x, nullptr, s->precision, s->K, M, D);
        og = input_operand(ws, stage, w_gate, nullptr, s->precision, s->K, F, D);
        ou = input_operand(ws, stage, w_up, nullptr, s->precision, s->K, F, D);
        od = input_operand(ws, stage, w_down, nullptr, s->precision, s->K, D, F);
        oh = own_operand(ws, s->K, M, F, parts);
    }
    Product down{M, D, F, &oh, nullptr, &od, nullptr, false, false, y, 1, nullptr};
    if (M) take_shares(ws, &down, 1, s->K, parts);
    Regions all;
    all.reads(region(x, s->K, M, D, es));
    all.reads(region(w_gate, s->K, F, D, es)); all.reads(region(w_up, s->K, F, D, es)); all.reads(region(w_down, s->K, D, F, es));
    all.writes(region(y, s->K, M, D, es));
    add_saved(all, s, gate, up, gate_e, up_e, true);
    BLOCK_TRY(settle(ws, workspace_bytes, all));
    if (!workspace) return PALSGD_OK;
    if (M == 0) return PALSGD_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Device dev{};
    BLOCK_TRY(device_of(dev));
    MatLaunch gated{};
    BLOCK_TRY(add_problem(gated, M, F, D, s->K, &ox, nullptr, false, &og, &ou, false, kTileN / 2));
    gated.p[0].out[0] = out_of(oh);
    if (parts == 1) BLOCK_TRY(encode_store(&gated.store[0], oh));
    set_saved(gated, s, gate, up, gate_e, up_e);
    BLOCK_TRY(run_stage(stage, s->K, dev.sms, st));
    BLOCK_TRY(run_mat<MAT_GATED>(gated, s, dev, st));
    return run_products(&down, 1, s, dev, es, parts, st);
}

extern "C" int palsgd_ffn_backward(const palsgd_ffn_shape* s, const palsgd_mat* dy_, const palsgd_mat* x_, const palsgd_mat* x_e_,
                                   const palsgd_mat* w_gate_, const palsgd_mat* w_up_, const palsgd_mat* w_down_,
                                   const palsgd_mat* gate_, const palsgd_mat* up_, const palsgd_mat* gate_e_,
                                   const palsgd_mat* up_e_, const palsgd_mat* dx_, const palsgd_mat* dw_gate_,
                                   const palsgd_mat* dw_up_, const palsgd_mat* dw_down_, void* workspace,
                                   size_t* workspace_bytes, void* stream)
{
    BLOCK_TRY(check_shape(s));
    const Mat dy(dy_, s->K, s->tokens), x(x_, s->K, s->tokens), x_e(x_e_, s->K, s->tokens), dx(dx_, s->K, s->tokens);
    const Mat w_gate(w_gate_, s->K, s->d_ff), w_up(w_up_, s->K, s->d_ff), w_down(w_down_, s->K, s->d_model);
    const Mat gate(gate_, s->K, s->tokens), up(up_, s->K, s->tokens), gate_e(gate_e_, s->K, s->tokens), up_e(up_e_, s->K, s->tokens);
    const Mat dw_gate(dw_gate_, s->K, s->d_ff), dw_up(dw_up_, s->K, s->d_ff), dw_down(dw_down_, s->K, s->d_model);
    if (s->save == PALSGD_SAVE_NONE || (x_e && s->save != PALSGD_SAVE_8BIT)) return PALSGD_EINVAL;
    const uint64_t M = s->tokens, D = s->d_model, F = s->d_ff;
    const size_t es = elem(s->precision);
    BLOCK_TRY(check_mat(dy, s->K, M, D, es, false));
    BLOCK_TRY(check_mat(x, s->K, M, D, x_e ? 1 : es, false));
    if (x_e) BLOCK_TRY(check_mat(x_e, s->K, M, ceil_div(D, PALSGD_ACT8_GROUP), 1, false));
    BLOCK_TRY(check_mat(w_gate, s->K, F, D, es, false));
    BLOCK_TRY(check_mat(w_up, s->K, F, D, es, false));
    BLOCK_TRY(check_mat(w_down, s->K, D, F, es, false));
    BLOCK_TRY(check_saved(s, gate, up, gate_e, up_e, false));
    if (dx) BLOCK_TRY(check_mat(dx, s->K, M, D, es, true));
    BLOCK_TRY(check_mat(dw_gate, s->K, F, D, es, true));
    BLOCK_TRY(check_mat(dw_up, s->K, F, D, es, true));
    BLOCK_TRY(check_mat(dw_down, s->K, D, F, es, true));
    BLOCK_TRY(check_workspace(workspace, workspace_bytes));
    Arena ws{static_cast<char*>(workspace), 0};
    Stage stage;
    const uint32_t parts = s->precision == PALSGD_PREC_FP32 ? 3 : 1;
    Operand ody, ox, og, ou, od, hid[3];                 // hid: dg, du, h
    if (M) {
        ody = input_operand(ws, stage, dy, nullptr, s->precision, s->K, M, D);
        ox = input_operand(ws, stage, x, x_e, s->precision, s->K, M, D);
        od = input_operand(ws, stage, w_down, nullptr, s->precision, s->K, D, F);
        if (dx) {
            og = input_operand(ws, stage, w_gate, nullptr, s->precision, s->K, F, D);
            ou = input_operand(ws, stage, w_up, nullptr, s->precision, s->K, F, D);
        }
        for (Operand& o : hid) o = own_operand(ws, s->K, M, F, parts);
    }
    // dx contracts over both halves of the hidden axis, the weight gradients over the tokens
    const Product all[4] = {{M, D, F, &hid[0], &hid[1], &og, &ou, false, true, dx, 1, nullptr},
                            {F, D, M, &hid[0], nullptr, &ox, nullptr, true, true, dw_gate, 1, nullptr},
                            {F, D, M, &hid[1], nullptr, &ox, nullptr, true, true, dw_up, 1, nullptr},
                            {D, F, M, &ody, nullptr, &hid[2], nullptr, true, true, dw_down, 1, nullptr}};
    Product products[4];
    const int n_products = dx ? 4 : 3;
    for (int i = 0; i < n_products; ++i) products[i] = all[dx ? i : i + 1];
    if (M) take_shares(ws, products, n_products, s->K, parts);
    Regions mem;
    mem.reads(region(dy, s->K, M, D, es));
    mem.reads(region(x, s->K, M, D, x_e ? 1 : es));
    mem.reads(region(x_e, s->K, M, ceil_div(D, PALSGD_ACT8_GROUP), 1));
    mem.reads(region(w_gate, s->K, F, D, es)); mem.reads(region(w_up, s->K, F, D, es)); mem.reads(region(w_down, s->K, D, F, es));
    add_saved(mem, s, gate, up, gate_e, up_e, false);
    mem.writes(region(dx, s->K, M, D, es));
    mem.writes(region(dw_gate, s->K, F, D, es)); mem.writes(region(dw_up, s->K, F, D, es)); mem.writes(region(dw_down, s->K, D, F, es));
    BLOCK_TRY(settle(ws, workspace_bytes, mem));
    if (!workspace) return PALSGD_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (M == 0) {
        const palsgd_mat* w[3] = {dw_gate, dw_up, dw_down};
        ZeroArgs z{};
        for (int i = 0; i < 3; ++i) {
            z.p[i] = w[i]->data; z.w[i] = w[i]->worker_stride; z.r[i] = w[i]->row_stride;
            z.rows[i] = (uint32_t)(i < 2 ? F : D); z.cols[i] = (uint32_t)(i < 2 ? D : F);
        }
        const dim3 grid((unsigned)(F > D ? F : D) < 1024u ? (unsigned)(F > D ? F : D) : 1024u, 3, s->K);
        return launch("zero weight gradients", es == 4 ? zero_kernel<float> : zero_kernel<bf16>, grid, 256, 0, st, z);
    }
    Device dev{};
    BLOCK_TRY(device_of(dev));
    MatLaunch hidden{};
    BLOCK_TRY(add_problem(hidden, M, F, D, s->K, &ody, nullptr, false, &od, nullptr, true, kTileN));
    for (int i = 0; i < 3; ++i) {
        hidden.p[0].out[i] = out_of(hid[i]);
        if (parts == 1) BLOCK_TRY(encode_store(&hidden.store[i], hid[i]));
    }
    set_saved(hidden, s, gate, up, gate_e, up_e);
    BLOCK_TRY(run_stage(stage, s->K, dev.sms, st));
    BLOCK_TRY(run_mat<MAT_HIDDEN>(hidden, s, dev, st));
    return run_products(products, n_products, s, dev, es, parts, st);
}

extern "C" int palsgd_block_status(void* stream)
{
    Device dev{};
    BLOCK_TRY(device_of(dev));
    unsigned int v = 0;
    cudaError_t e = cudaMemcpyAsync(&v, dev.gave_up, sizeof v, cudaMemcpyDeviceToHost, static_cast<cudaStream_t>(stream));
    if (e == cudaSuccess) e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
    if (e == cudaSuccess && v) {
        e = cudaMemsetAsync(dev.gave_up, 0, sizeof v, static_cast<cudaStream_t>(stream));
        if (e == cudaSuccess) return palsgd_block_cuda_fail((int)cudaErrorLaunchTimeout, "a matrix kernel's wait gave up");
    }
    return e == cudaSuccess ? PALSGD_OK : palsgd_block_cuda_fail((int)e, "palsgd_block_status");
}

extern "C" int palsgd_qk_norm_rope_forward(const palsgd_qk_shape* s, const palsgd_heads* q, const palsgd_heads* k,
                                           const palsgd_mat* w_q, const palsgd_mat* w_k, const float* cos_table,
                                           const float* sin_table, const int32_t* positions, const palsgd_heads* q_out,
                                           const palsgd_heads* k_out, void* stream)
{
    BLOCK_TRY(check_qk(s, cos_table, sin_table, positions));
    const uint32_t heads[2] = {s->heads_q, s->heads_k};
    const HeadsOf given[4] = {{q, s, heads[0]}, {k, s, heads[1]}, {q_out, s, heads[0]}, {k_out, s, heads[1]}};
    const Mat weights[2] = {{w_q, s->K, 1}, {w_k, s->K, 1}};
    const palsgd_heads *in[2] = {given[0], given[1]}, *out[2] = {given[2], given[3]};
    const palsgd_mat* w[2] = {weights[0], weights[1]};
    for (int i = 0; i < 2; ++i) {
        BLOCK_TRY(check_heads(in[i], s, heads[i], false));
        BLOCK_TRY(check_heads(out[i], s, heads[i], true));
        if (heads[i]) BLOCK_TRY(check_mat(w[i], s->K, 1, s->head_dim, elem(s->precision), false));
    }
    Regions all;
    add_angles(all, s, cos_table, sin_table, positions);
    for (int i = 0; i < 2; ++i) {
        if (heads[i]) all.reads(region(w[i], s->K, 1, s->head_dim, elem(s->precision)));
        all.writes(region(out[i], s, heads[i]), all.reads(region(in[i], s, heads[i])));
    }
    if (all.clash()) return PALSGD_EINVAL;
    if (s->tokens == 0 || (heads[0] | heads[1]) == 0) return PALSGD_OK;
    QkPlan p = plan_qk(s, cos_table, sin_table, positions, false);
    for (int i = 0; i < 2; ++i) {
        if (!heads[i]) continue;
        HeadsArg& h = p.a.side[i];
        h.x = in[i]->data; h.xw = in[i]->worker_stride; h.xt = in[i]->token_stride; h.xh = in[i]->head_stride;
        h.out = out[i]->data; h.ow = out[i]->worker_stride; h.ot = out[i]->token_stride; h.oh = out[i]->head_stride;
        h.w = w[i]->data; h.ww = w[i]->worker_stride;
    }
    finish_qk(p, s, false);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return run_qk<false>(p, s, st);
}

extern "C" int palsgd_qk_norm_rope_backward(const palsgd_qk_shape* s, const palsgd_heads* dq_out, const palsgd_heads* dk_out,
                                            const palsgd_heads* q, const palsgd_heads* k, const palsgd_mat* w_q,
                                            const palsgd_mat* w_k, const float* cos_table, const float* sin_table,
                                            const int32_t* positions, const palsgd_heads* dq, const palsgd_heads* dk,
                                            const palsgd_mat* dw_q, const palsgd_mat* dw_k, void* workspace,
                                            size_t* workspace_bytes, void* stream)
{
    BLOCK_TRY(check_qk(s, cos_table, sin_table, positions));
    const uint32_t heads[2] = {s->heads_q, s->heads_k};
    const HeadsOf given[6] = {{q, s, heads[0]}, {k, s, heads[1]}, {dq_out, s, heads[0]}, {dk_out, s, heads[1]}, {dq, s, heads[0]}, {dk, s, heads[1]}};
    const Mat weights[4] = {{w_q, s->K, 1}, {w_k, s->K, 1}, {dw_q, s->K, 1}, {dw_k, s->K, 1}};
    const palsgd_heads *in[2] = {given[0], given[1]}, *grad[2] = {given[2], given[3]}, *out[2] = {given[4], given[5]};
    const palsgd_mat *w[2] = {weights[0], weights[1]}, *dw[2] = {weights[2], weights[3]};
    for (int i = 0; i < 2; ++i) {
        BLOCK_TRY(check_heads(grad[i], s, heads[i], false));
        BLOCK_TRY(check_heads(in[i], s, heads[i], false));
        BLOCK_TRY(check_heads(out[i], s, heads[i], true));
        if (!heads[i] && (!dw[i] || !dw[i]->data)) { dw[i] = nullptr; continue; }
        BLOCK_TRY(check_mat(dw[i], s->K, 1, s->head_dim, elem(s->precision), true));
        if (heads[i]) BLOCK_TRY(check_mat(w[i], s->K, 1, s->head_dim, elem(s->precision), false));
    }
    BLOCK_TRY(check_workspace(workspace, workspace_bytes));
    QkPlan p = plan_qk(s, cos_table, sin_table, positions, true);
    Arena ws{static_cast<char*>(workspace), 0};
    float* part[2] = {nullptr, nullptr};
    for (int i = 0; i < 2; ++i)
        if (heads[i]) part[i] = static_cast<float*>(ws.take((size_t)s->K * p.a.ctas[i] * s->head_dim * sizeof(float)));
    Regions all;
    add_angles(all, s, cos_table, sin_table, positions);
    for (int i = 0; i < 2; ++i) {
        if (heads[i]) all.reads(region(w[i], s->K, 1, s->head_dim, elem(s->precision)));
        const int x = all.reads(region(in[i], s, heads[i])), d = all.reads(region(grad[i], s, heads[i]));
        all.writes(region(out[i], s, heads[i]), x, d);
        all.writes(region(dw[i], s->K, 1, s->head_dim, elem(s->precision)));
    }
    BLOCK_TRY(settle(ws, workspace_bytes, all));
    if (!workspace) return PALSGD_OK;
    QkSumArgs sum{};
    for (int i = 0; i < 2; ++i) {
        if (dw[i]) { sum.dw[i] = dw[i]->data; sum.dww[i] = dw[i]->worker_stride; }
        if (!heads[i]) continue;                         // no parts: a gradient that is given becomes zero
        HeadsArg& h = p.a.side[i];
        h.x = in[i]->data; h.xw = in[i]->worker_stride; h.xt = in[i]->token_stride; h.xh = in[i]->head_stride;
        h.d = grad[i]->data; h.dw = grad[i]->worker_stride; h.dt = grad[i]->token_stride; h.dh = grad[i]->head_stride;
        h.out = out[i]->data; h.ow = out[i]->worker_stride; h.ot = out[i]->token_stride; h.oh = out[i]->head_stride;
        h.w = w[i]->data; h.ww = w[i]->worker_stride;
        h.part = part[i];
        sum.part[i] = part[i];
        sum.parts[i] = s->tokens ? p.a.ctas[i] : 0;
    }
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    sum.head_dim = s->head_dim;
    const dim3 grid((unsigned)ceil_div(s->head_dim, 32), 2, s->K);
    if (s->tokens && (heads[0] | heads[1])) {
        finish_qk(p, s, true);
        BLOCK_TRY(run_qk<true>(p, s, st));
    }
    return launch("q/k weight gradient", s->precision == PALSGD_PREC_FP32 ? qk_sum_kernel<float> : qk_sum_kernel<bf16>, grid, 256, 0, st, sum);
}
