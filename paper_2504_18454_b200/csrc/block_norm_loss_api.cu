// Host side of the layer norm and the cross entropy (see include/palsgd_block.h): checks of arguments, workspaces, launches.
#include "block_columns.cuh"
#include "block_common.cuh"
#include "block_loss.cuh"
#include "block_norm.cuh"

#include <cmath>

#include "block_args.h"

using namespace palsgd::block;

namespace {

// ------------------------------------------------------------------------------------------------ layer norm

constexpr uint64_t kNormMostWidth = 16384;               // a row in the registers of at most 1024 lanes

int check_norm(const palsgd_norm_shape* s)
{
    if (!s || s->K == 0 || s->K > PALSGD_MAX_WORKERS || !prec_ok(s->precision)) return PALSGD_EINVAL;
    if (s->width == 0 || s->width > kMaxSize || s->tokens > kMaxSize) return PALSGD_EINVAL;
    if (!(std::isfinite(s->eps) && s->eps >= 0.0)) return PALSGD_EINVAL;
    return s->width > kNormMostWidth ? PALSGD_EUNSUPPORTED : PALSGD_OK;
}

// Rows on 16-byte boundaries, of whole pieces
bool norm_wide(const palsgd_mat* m, size_t es)
{
    return !m || (aligned(m->data, 16) && (m->worker_stride * es) % 16 == 0 && (m->row_stride * es) % 16 == 0);
}

// Lanes of a team, pieces a lane: the fewest lanes of up to 8 warps that hold a row in `most` pieces each, narrow rows in one
// piece a lane (several rows a warp); beyond that 16 or 32 warps, with two pieces a lane of bfloat16 and four of fp32 (16
// values: what 1024 threads have the registers for).
struct Team { uint32_t lanes, pieces; };
Team team_of(uint64_t width, size_t es, uint32_t most)
{
    const uint64_t pieces = ceil_div(width * es, 16);
    Team t{pieces <= 32 ? 4u : 32u, 0};
    while (t.lanes < 256 && pieces > (uint64_t)t.lanes * (pieces <= 32 ? 1 : most)) t.lanes *= 2;
    if (pieces > 256ull * most) t.lanes = pieces > 512 * es ? 1024 : 512;
    t.pieces = (uint32_t)ceil_div(pieces, t.lanes);
    return t;
}
uint64_t teams_of(Team t) { return t.lanes <= 256 ? 256 / t.lanes : 1; }

// CTAs of a worker: as many as run at a time, each team with as many rows as any other (but for the last turn).
uint32_t norm_ctas(const palsgd_norm_shape* s, Team t, uint32_t per_sm)
{
    uint64_t most = (uint64_t)(t.lanes > 256 ? 1 : per_sm) * sm_count() / s->K;
    if (most == 0) most = 1;
    const uint64_t turns = ceil_div(s->tokens, most * teams_of(t));
    const uint64_t n = turns ? ceil_div(s->tokens, turns * teams_of(t)) : 1;
    return (uint32_t)(n ? n : 1);
}

// CTAs an SM that the kernel's registers are fitted to; the ring of a lane, 16 bytes a place.
template <bool BACK> constexpr uint32_t norm_ctas_per_sm(uint32_t pieces) { return BACK || pieces > 2 ? 2 : 3; }
template <bool BACK> constexpr uint32_t norm_most() { return BACK ? 2 : 3; }        // pieces a lane

template <typename T, bool BACK, int N, bool WIDE, bool ADD, int WARPS>
int launch_norm(const NormArgs& a, dim3 grid, cudaStream_t st)
{
    constexpr int kCtas = WARPS > 8 ? 1 : (int)norm_ctas_per_sm<BACK>(N);
    void (*kernel)(NormArgs);
    if constexpr (BACK) kernel = norm_backward_kernel<T, N, WIDE, ADD, WARPS, kCtas>;
    else kernel = norm_forward_kernel<T, N, WIDE, ADD, WARPS, kCtas>;
    const unsigned threads = WARPS == 8 ? 256 : WARPS * 32;
    constexpr int kArrays = BACK ? ADD ? 3 : 2 : ADD ? 2 : 1;
    constexpr uint32_t kStage = norm_stage_bytes<T, WIDE, N>(kArrays, WARPS), kStages = norm_stages<T, WIDE, N>(kArrays, WARPS, kCtas);
    static_assert(kStages >= 1, "room for a row");
    static_assert(!BACK || WARPS > 8 || kStage * kStages >= 2 * sizeof(float) * (WARPS / 2) * 32 * N * kPieceValues<T>, "room for the sums of two teams or more");
    const size_t smem = (size_t)kStage * kStages;
    BLOCK_TRY(allow_smem(reinterpret_cast<const void*>(kernel), smem));
    return launch(BACK ? "layer norm backward" : "layer norm", kernel, grid, threads, smem, st, a);
}

template <typename T, bool BACK, bool WIDE, bool ADD>
int launch_norm(const NormArgs& a, Team t, dim3 grid, cudaStream_t st)
{
    if (t.lanes == 512) return launch_norm<T, BACK, (int)sizeof(T), WIDE, ADD, 16>(a, grid, st);
    if (t.lanes == 1024) return launch_norm<T, BACK, (int)sizeof(T), WIDE, ADD, 32>(a, grid, st);
    if (t.pieces == 1) return launch_norm<T, BACK, 1, WIDE, ADD, 8>(a, grid, st);
    if constexpr (norm_most<BACK>() == 2) {
        return launch_norm<T, BACK, 2, WIDE, ADD, 8>(a, grid, st);
    } else {
        switch (t.pieces) {
            case 2: return launch_norm<T, BACK, 2, WIDE, ADD, 8>(a, grid, st);
            default: return launch_norm<T, BACK, 3, WIDE, ADD, 8>(a, grid, st);
        }
    }
}

template <typename T, bool BACK>
int launch_norm(const NormArgs& a, Team t, bool wide, bool add, dim3 grid, cudaStream_t st)
{
    if (wide) return add ? launch_norm<T, BACK, true, true>(a, t, grid, st) : launch_norm<T, BACK, true, false>(a, t, grid, st);
    return add ? launch_norm<T, BACK, false, true>(a, t, grid, st) : launch_norm<T, BACK, false, false>(a, t, grid, st);
}

// ------------------------------------------------------------------------------------------------ cross entropy

int check_loss(const palsgd_loss_shape* s, const int32_t* targets)
{
    if (!s || s->K == 0 || s->K > PALSGD_MAX_WORKERS || !prec_ok(s->precision)) return PALSGD_EINVAL;
    if (s->vocab == 0 || s->vocab > kMaxSize || s->tokens > kMaxSize) return PALSGD_EINVAL;
    if (s->target_worker_stride < 0 || s->target_worker_stride > kMaxStride) return PALSGD_EINVAL;
    if (s->tokens && !targets) return PALSGD_EINVAL;
    if (!aligned(targets, 4)) return PALSGD_EALIGN;
    return PALSGD_OK;
}

Region target_region(const palsgd_loss_shape* s, const int32_t* targets)
{
    return Region(targets, s->tokens * 4).axis(0, s->K, s->target_worker_stride * 4);
}

}  // namespace

extern "C" int palsgd_layer_norm_forward(const palsgd_norm_shape* s, const palsgd_mat* x_, const palsgd_mat* residual_,
                                         const palsgd_mat* w_, const palsgd_mat* b_, const palsgd_mat* y_, const palsgd_mat* total_,
                                         const palsgd_mat* mean_, const palsgd_mat* rstd_, void* stream)
{
    BLOCK_TRY(check_norm(s));
    const uint64_t M = s->tokens, D = s->width;
    const size_t es = elem(s->precision);
    const Mat x(x_, s->K, M), r(residual_, s->K, M), w(w_, s->K, 1), b(b_, s->K, 1), y(y_, s->K, M), total(total_, s->K, M), mean(mean_, s->K, 1), rstd(rstd_, s->K, 1);
    if (r.given != total.given) return PALSGD_EINVAL;
    BLOCK_TRY(check_mat(x, s->K, M, D, es, false));
    BLOCK_TRY(check_mat(w, s->K, 1, D, es, false));
    BLOCK_TRY(check_mat(b, s->K, 1, D, es, false));
    BLOCK_TRY(check_mat(y, s->K, M, D, es, true));
    if (r.given) {
        BLOCK_TRY(check_mat(r, s->K, M, D, es, false));
        BLOCK_TRY(check_mat(total, s->K, M, D, es, true));
    }
    if (mean.given) BLOCK_TRY(check_mat(mean, s->K, 1, M, 4, true));
    if (rstd.given) BLOCK_TRY(check_mat(rstd, s->K, 1, M, 4, true));
    Regions all;
    all.reads(region(x, s->K, M, D, es)); all.reads(region(r, s->K, M, D, es));
    all.reads(region(w, s->K, 1, D, es)); all.reads(region(b, s->K, 1, D, es));
    all.writes(region(y, s->K, M, D, es)); all.writes(region(total, s->K, M, D, es));
    all.writes(region(mean, s->K, 1, M, 4)); all.writes(region(rstd, s->K, 1, M, 4));
    if (all.clash()) return PALSGD_EINVAL;
    if (M == 0) return PALSGD_OK;
    NormArgs a{};
    a.x = x.m.data; a.xw = x.m.worker_stride; a.xr = x.m.row_stride;
    a.r = r.m.data; a.rw = r.m.worker_stride; a.rr = r.m.row_stride;
    a.w = w.m.data; a.ww = w.m.worker_stride; a.b = b.m.data; a.bw = b.m.worker_stride;
    a.y = y.m.data; a.yw = y.m.worker_stride; a.yr = y.m.row_stride;
    a.total = total.m.data; a.tw = total.m.worker_stride; a.tr = total.m.row_stride;
    a.mean = static_cast<float*>(mean.m.data); a.mw = mean.m.worker_stride;
    a.rstd = static_cast<float*>(rstd.m.data); a.sw = rstd.m.worker_stride;
    a.rows = M; a.width = (uint32_t)D; a.eps = (float)s->eps;
    const bool wide = (D * es) % 16 == 0 && norm_wide(x, es) && norm_wide(r, es) && norm_wide(w, es) && norm_wide(b, es) && norm_wide(y, es) && norm_wide(total, es);
    const Team t = team_of(D, es, norm_most<false>());
    a.lanes = t.lanes;
    const dim3 grid(norm_ctas(s, t, norm_ctas_per_sm<false>(t.pieces)), s->K);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return es == 4 ? launch_norm<float, false>(a, t, wide, r.given, grid, st) : launch_norm<bf16, false>(a, t, wide, r.given, grid, st);
}

extern "C" int palsgd_layer_norm_backward(const palsgd_norm_shape* s, const palsgd_mat* dy_, const palsgd_mat* x_, const palsgd_mat* w_,
                                          const palsgd_mat* mean_, const palsgd_mat* rstd_, const palsgd_mat* dtotal_, const palsgd_mat* dx_,
                                          const palsgd_mat* dw_, const palsgd_mat* db_, void* workspace, size_t* workspace_bytes,
                                          void* stream)
{
    BLOCK_TRY(check_norm(s));
    const uint64_t M = s->tokens, D = s->width;
    const size_t es = elem(s->precision);
    const Mat dy(dy_, s->K, M), x(x_, s->K, M), w(w_, s->K, 1), mean(mean_, s->K, 1), rstd(rstd_, s->K, 1), past(dtotal_, s->K, M);
    const Mat dx(dx_, s->K, M), dw(dw_, s->K, 1), db(db_, s->K, 1);
    BLOCK_TRY(check_mat(dy, s->K, M, D, es, false));
    BLOCK_TRY(check_mat(x, s->K, M, D, es, false));
    BLOCK_TRY(check_mat(w, s->K, 1, D, es, false));
    BLOCK_TRY(check_mat(mean, s->K, 1, M, 4, false));
    BLOCK_TRY(check_mat(rstd, s->K, 1, M, 4, false));
    if (past.given) BLOCK_TRY(check_mat(past, s->K, M, D, es, false));
    BLOCK_TRY(check_mat(dx, s->K, M, D, es, true));
    BLOCK_TRY(check_mat(dw, s->K, 1, D, es, true));
    BLOCK_TRY(check_mat(db, s->K, 1, D, es, true));
    BLOCK_TRY(check_workspace(workspace, workspace_bytes));
    const Team t = team_of(D, es, norm_most<true>());
    // (four rows a team: as long as the launch of the kernel that joins what several CTAs leave)
    const uint32_t ctas = s->tokens <= 4 * teams_of(t) ? 1 : norm_ctas(s, t, norm_ctas_per_sm<true>(t.pieces));
    Arena ws{static_cast<char*>(workspace), 0};
    const uint32_t part_ld = (uint32_t)ceil_div(2 * D, 4) * 4;
    float* part = ctas > 1 ? static_cast<float*>(ws.take((size_t)s->K * ctas * part_ld * sizeof(float))) : nullptr;
    Regions all;
    all.reads(region(dy, s->K, M, D, es)); all.reads(region(x, s->K, M, D, es)); all.reads(region(w, s->K, 1, D, es));
    all.reads(region(mean, s->K, 1, M, 4)); all.reads(region(rstd, s->K, 1, M, 4)); all.reads(region(past, s->K, M, D, es));
    all.writes(region(dx, s->K, M, D, es)); all.writes(region(dw, s->K, 1, D, es)); all.writes(region(db, s->K, 1, D, es));
    BLOCK_TRY(settle(ws, workspace_bytes, all));
    if (!workspace) return PALSGD_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (M == 0) {                                         // (addresses of matrices without rows may be anything)
        ZeroArgs z{};
        z.p[0] = dw.m.data; z.w[0] = dw.m.worker_stride;
        z.p[1] = db.m.data; z.w[1] = db.m.worker_stride;
        z.rows[0] = z.rows[1] = 1;
        z.cols[0] = z.cols[1] = (uint32_t)D;
        return launch("zero weight gradients", es == 4 ? zero_kernel<float> : zero_kernel<bf16>, dim3(1, 2, s->K), 256, 0, st, z);
    }
    NormArgs a{};
    a.x = x.m.data; a.xw = x.m.worker_stride; a.xr = x.m.row_stride;
    a.r = past.m.data; a.rw = past.m.worker_stride; a.rr = past.m.row_stride;
    a.dy = dy.m.data; a.dw = dy.m.worker_stride; a.dr = dy.m.row_stride;
    a.w = w.m.data; a.ww = w.m.worker_stride;
    a.y = dx.m.data; a.yw = dx.m.worker_stride; a.yr = dx.m.row_stride;
    a.mean = static_cast<float*>(mean.m.data); a.mw = mean.m.worker_stride;
    a.rstd = static_cast<float*>(rstd.m.data); a.sw = rstd.m.worker_stride;
    a.part = part; a.part_ld = part_ld;
    a.dw_out = dw.m.data; a.dwo = dw.m.worker_stride; a.db_out = db.m.data; a.dbo = db.m.worker_stride;
    a.rows = M; a.width = (uint32_t)D; a.lanes = t.lanes;
    const bool wide = (D * es) % 16 == 0 && norm_wide(dy, es) && norm_wide(x, es) && norm_wide(w, es) && norm_wide(past, es) && norm_wide(dx, es);
    const dim3 grid(ctas, s->K);
    BLOCK_TRY((es == 4 ? launch_norm<float, true>(a, t, wide, past.given, grid, st) : launch_norm<bf16, true>(a, t, wide, past.given, grid, st)));
    if (!part) return PALSGD_OK;
    ColumnSumArgs c{part, {dw.m.data, db.m.data}, {dw.m.worker_stride, db.m.worker_stride}, ctas, (uint32_t)(2 * D), part_ld, (uint32_t)D, (uint32_t)D, (uint32_t)D, 0};
    const dim3 columns((unsigned)ceil_div(2 * D, 128), s->K);
    return launch("layer norm weight gradients", es == 4 ? column_sum_kernel<float> : column_sum_kernel<bf16>, columns, 256, 0, st, c);
}

extern "C" int palsgd_cross_entropy_forward(const palsgd_loss_shape* s, const palsgd_mat* logits_, const int32_t* targets,
                                            const palsgd_mat* loss_, const palsgd_mat* lse_, void* stream)
{
    BLOCK_TRY(check_loss(s, targets));
    const uint64_t M = s->tokens, V = s->vocab;
    const size_t es = elem(s->precision);
    const Mat z(logits_, s->K, M), loss(loss_, s->K, 1), lse(lse_, s->K, 1);
    BLOCK_TRY(check_mat(z, s->K, M, V, es, false));
    BLOCK_TRY(check_mat(loss, s->K, 1, M, 4, true));
    BLOCK_TRY(check_mat(lse, s->K, 1, M, 4, true));
    Regions all;
    all.reads(region(z, s->K, M, V, es)); all.reads(target_region(s, targets));
    all.writes(region(loss, s->K, 1, M, 4)); all.writes(region(lse, s->K, 1, M, 4));
    if (all.clash()) return PALSGD_EINVAL;
    if (M == 0) return PALSGD_OK;
    LossArgs a{};
    a.z = z.m.data; a.zw = z.m.worker_stride; a.zr = z.m.row_stride;
    a.target = targets; a.tw = s->K > 1 ? s->target_worker_stride : 0;
    a.loss = static_cast<float*>(loss.m.data); a.lw = loss.m.worker_stride;
    a.lse = static_cast<float*>(lse.m.data); a.sw = lse.m.worker_stride;
    a.rows = M; a.vocab = (uint32_t)V;
    // A team with at least eight pieces a lane, or, where rows are few, as many lanes as there are pieces
    const uint64_t pieces = ceil_div(V * es, 16), least = M * s->K < (uint64_t)sm_count() * 4 ? 1 : 8;
    a.warps = 1;
    while (a.warps < (least == 1 ? 32u : 8u) && pieces >= least * a.warps * 64) a.warps *= 2;
    const uint64_t teams = a.warps <= 8 ? 8 / a.warps : 1;
    // as many CTAs as run at a time, each team with as many rows as any other (but for the last turn)
    const uint64_t run = (a.warps <= 8 ? 4ull : 1ull) * sm_count() / s->K, turns = ceil_div(M, (run ? run : 1) * teams);
    return launch("cross entropy", es == 4 ? loss_forward_kernel<float> : loss_forward_kernel<bf16>, dim3((unsigned)ceil_div(M, turns * teams), s->K), (unsigned)(teams * a.warps * 32), 0,
                  static_cast<cudaStream_t>(stream), a);
}

extern "C" int palsgd_cross_entropy_backward(const palsgd_loss_shape* s, const palsgd_mat* dloss_, const palsgd_mat* logits_,
                                             const int32_t* targets, const palsgd_mat* lse_, const palsgd_mat* dlogits_, void* stream)
{
    BLOCK_TRY(check_loss(s, targets));
    const uint64_t M = s->tokens, V = s->vocab;
    const size_t es = elem(s->precision);
    const Mat dloss(dloss_, s->K, 1), z(logits_, s->K, M), lse(lse_, s->K, 1), dz(dlogits_, s->K, M);
    BLOCK_TRY(check_mat(dloss, s->K, 1, M, 4, false));
    BLOCK_TRY(check_mat(z, s->K, M, V, es, false));
    BLOCK_TRY(check_mat(lse, s->K, 1, M, 4, false));
    BLOCK_TRY(check_mat(dz, s->K, M, V, es, true));
    Regions all;
    all.reads(region(dloss, s->K, 1, M, 4)); all.reads(target_region(s, targets)); all.reads(region(lse, s->K, 1, M, 4));
    all.writes(region(dz, s->K, M, V, es), all.reads(region(z, s->K, M, V, es)));
    if (all.clash()) return PALSGD_EINVAL;
    if (M == 0) return PALSGD_OK;
    LossArgs a{};
    a.z = z.m.data; a.zw = z.m.worker_stride; a.zr = z.m.row_stride;
    a.target = targets; a.tw = s->K > 1 ? s->target_worker_stride : 0;
    a.dloss = static_cast<const float*>(dloss.m.data); a.gw = dloss.m.worker_stride;
    a.lse = static_cast<float*>(lse.m.data); a.sw = lse.m.worker_stride;
    a.dz = dz.m.data; a.dw = dz.m.worker_stride; a.dr = dz.m.row_stride;
    a.rows = M; a.vocab = (uint32_t)V;
    const uint64_t pieces = ceil_div(V * es, 16) + 1;     // (a row that starts inside a piece has one more)
    a.warps = 1;
    while (a.warps < 8 && pieces >= a.warps * 64) a.warps *= 2;
    const uint64_t parts = ceil_div(pieces, a.warps * 32 * kLossPieces), units = parts * M;
    if (units > 0x7FFFFFFFull) return PALSGD_EUNSUPPORTED;
    const LossGrid g{divisor((uint32_t)parts), (uint32_t)units};
    return launch("cross entropy gradient", es == 4 ? loss_backward_kernel<float> : loss_backward_kernel<bf16>,
                  dim3((unsigned)ceil_div(units, 8 / a.warps), s->K), 256, 0, static_cast<cudaStream_t>(stream), a, g);
}
