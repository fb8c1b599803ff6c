// Host side of the block operators, what their entry points share: checks of arguments, workspaces, launches.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/palsgd_block.h"
#include "block_common.cuh"
#include "block_host.h"
#include "block_overlap.h"

namespace palsgd {
namespace block {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
inline size_t elem(int32_t prec) { return prec == PALSGD_PREC_BF16_MASTER ? 2 : 4; }
inline bool prec_ok(int32_t p) { return p == PALSGD_PREC_FP32 || p == PALSGD_PREC_BF16_MASTER; }

constexpr uint64_t kMaxSize = 0x7FFFFFFFull;             // rows, columns, tokens: 31 bits (offsets are 64-bit)
constexpr int64_t kMaxStride = (int64_t)1 << 40;

struct Axis { uint64_t n; int64_t stride; };

// No two of n0*n1*n2 runs of `run` contiguous elements at these strides share an element (sufficient condition: sorted
// by stride, each axis steps over all of the axes inside it).
inline bool disjoint(Axis a, Axis b, Axis c, uint64_t run)
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

// A matrix argument: EINVAL / EALIGN / OK.  Nothing is asked of a matrix without elements.
inline int check_mat(const palsgd_mat* m, uint32_t K, uint64_t rows, uint64_t cols, size_t es, bool output)
{
    if (!m) return PALSGD_EINVAL;
    if (m->worker_stride < 0 || m->row_stride < 0 || m->worker_stride > kMaxStride || m->row_stride > kMaxStride) return PALSGD_EINVAL;
    if (rows == 0 || cols == 0) return PALSGD_OK;
    if (!m->data) return PALSGD_EINVAL;
    if (!aligned(m->data, es)) return PALSGD_EALIGN;
    if (output && !disjoint({K, m->worker_stride}, {rows, m->row_stride}, {1, 0}, cols)) return PALSGD_EINVAL;
    return PALSGD_OK;
}

inline Region region(const palsgd_mat* m, uint32_t K, uint64_t rows, uint64_t cols, size_t es)
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

// A kernel's dynamic shared memory beyond what every kernel may have.  (An attribute of the function on the current device;
// 0.2 us a call.)
inline int allow_smem(const void* kernel, size_t bytes)
{
    if (bytes <= 32 * 1024) return PALSGD_OK;             // (48 KB, a kernel's own static memory among them)
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) return PALSGD_OK;
    (void)cudaGetLastError();
    return palsgd_block_cuda_fail((int)e, "shared memory of a kernel");
}

inline int sm_count()
{
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = 148;
    return n;
}

inline Divisor divisor(uint32_t d)
{
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return Divisor{d, (uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
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

inline int check_workspace(const void* ws, const size_t* bytes)
{
    if (!bytes) return PALSGD_EINVAL;
    if (ws && !aligned(ws, 256)) return PALSGD_EALIGN;
    return PALSGD_OK;
}

// The workspace's size is asked for or checked, and that nothing that the call writes overlaps.
inline int settle(const Arena& ws, size_t* bytes, Regions& all)
{
    if (ws.base && *bytes < ws.need()) { *bytes = ws.need(); return PALSGD_EINVAL; }
    all.writes(Region(ws.base, ws.used));
    if (all.clash()) return PALSGD_EINVAL;
    if (!ws.base) *bytes = ws.need();
    return PALSGD_OK;
}

}  // namespace block
}  // namespace palsgd
