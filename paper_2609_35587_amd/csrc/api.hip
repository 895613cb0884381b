// C-ABI entry points: host-side argument checks, then one launch each.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <numeric>

#include "internal.hpp"

namespace {

thread_local char g_err[512];

int fail(int status, const char *fn, const char *fmt, ...) __attribute__((format(printf, 3, 4)));

int fail(int status, const char *fn, const char *fmt, ...)
{
    int n = snprintf(g_err, sizeof g_err, "%s: ", fn);
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err + n, sizeof g_err - (size_t)n, fmt, ap);
    va_end(ap);
    return status;
}

int launched(hipError_t e, const char *fn)
{
    if (e != hipSuccess) return fail(HWSEL_EHIP, fn, "launch failed: %s", hipGetErrorString(e));
    g_err[0] = 0;
    return HWSEL_OK;
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// Memory that a call reads or writes, [at, end): runs of `width` bytes, `step` bytes from one to the next (0: one run).
struct Region {
    uintptr_t at, end;
    int64_t width, step;
};

Region region_of(const void *p, int64_t bytes)
{
    const uintptr_t at = p ? (uintptr_t)p : 0;
    return {at, at + (p ? (uintptr_t)bytes : 0), p ? bytes : 0, 0};
}

// rows x cols of a matrix.
Region region_of(const hwsel_matrix_t &m, int64_t rows, int64_t cols)
{
    const int64_t each = m.dtype == HWSEL_DTYPE_BF16 ? 2 : 4;
    Region r = region_of(m.data, cols * each);
    if (!m.data || rows == 1) return r;
    r.step = m.ld * each;                                   // (at most 2^42, rows below 2^31)
    const __int128 end = (__int128)r.end + (__int128)(rows - 1) * r.step;
    r.end = end < (__int128)UINTPTR_MAX ? (uintptr_t)end : UINTPTR_MAX;
    return r;
}

// Whether two regions may share a byte.  Both repeat with the greatest common divisor of their steps, within which columns
// of one buffer, each matrix its own, lie apart.
bool overlap(const Region &a, const Region &b)
{
    if (a.end <= b.at || b.end <= a.at || a.width == 0 || b.width == 0) return false;
    const int64_t period = std::gcd(a.step, b.step);
    if (period == 0) return true;
    const int64_t from = (int64_t)((((__int128)b.at - (__int128)a.at) % period + period) % period);
    return a.width > from || from + b.width > period;
}

// Results overlap nothing else that the call reads or writes, but result `whole` (-1: none) the first operand.
struct Named {
    const char *name;
    Region region;
};

template <int N, int M>
int check_apart(const Named (&outs)[N], const Region (&ins)[M], int whole, const char *fn)
{
    for (int o = 0; o < N; ++o) {
        bool apart = true;
        for (int i = o == whole; i < M; ++i) apart = apart && !overlap(outs[o].region, ins[i]);
        for (int i = 0; i < o; ++i) apart = apart && !overlap(outs[o].region, outs[i].region);
        if (!apart) return fail(HWSEL_EINVAL, fn, "%s in the place of another operand or result", outs[o].name);
    }
    return HWSEL_OK;
}

}  // namespace

extern "C" {

const char *hwsel_status_string(int status)
{
    switch (status) {
    case HWSEL_OK: return "ok";
    case HWSEL_EINVAL: return "invalid argument";
    case HWSEL_EUNSUPPORTED: return "unsupported";
    case HWSEL_EHIP: return "HIP runtime error";
    default: return "unknown status";
    }
}

const char *hwsel_last_error(void) { return g_err; }

static int check_hw(const hwsel_hw_t &hw, const char *fn, hwsel::HwDev *h)
{
    const int64_t positive[] = {hw.n_sm, hw.smem_per_sm, hw.smem_per_block_max, hw.regs_per_sm,
                                hw.max_regs_per_thread, hw.max_blocks_per_sm, hw.max_threads_per_sm,
                                hw.arch_id, hw.llc_bytes, hw.hbm_bw_gbps, hw.peak_gflops[0],
                                hw.peak_gflops[1], hw.peak_gflops[2]};
    for (int64_t v : positive)
        if (v < 1) return fail(HWSEL_EINVAL, fn, "hardware field %lld < 1", (long long)v);
    if (hw.smem_reserved < 0) return fail(HWSEL_EINVAL, fn, "smem_reserved < 0");
    *h = hwsel::HwDev{hw.n_sm, hw.smem_per_sm, hw.smem_per_block_max, hw.smem_reserved, hw.regs_per_sm,
                      hw.max_regs_per_thread, hw.max_blocks_per_sm, hw.max_threads_per_sm, hw.arch_id,
                      hw.llc_bytes, hw.hbm_bw_gbps, {hw.peak_gflops[0], hw.peak_gflops[1], hw.peak_gflops[2]}};
    return HWSEL_OK;
}

// Shared checks of the problem/candidate inputs; fills the kernel views.
static int check_rows(const hwsel_hw_t &hw, const hwsel_problem_t *problems, int32_t P, const int64_t *seg_offsets,
                      const hwsel_cands_t *cands, int64_t R, const char *fn, hwsel::HwDev *h, hwsel::CandsDev *c)
{
    if (!problems || !seg_offsets || !cands) return fail(HWSEL_EINVAL, fn, "null pointer");
    const void *fields[] = {cands->tile_m, cands->tile_n, cands->tile_k, cands->inst_n, cands->stages,
                            cands->cluster_m, cands->cluster_n, cands->swizzle, cands->inst_m_div16,
                            cands->inst_k, cands->kernel_sched, cands->epi_sched, cands->tile_sched};
    for (const void *f : fields)
        if (!f) return fail(HWSEL_EINVAL, fn, "null candidate field");
    if (P < 1 || R < 1) return fail(HWSEL_EINVAL, fn, "P=%d R=%lld must be >= 1", P, (long long)R);
    if (int st = check_hw(hw, fn, h)) return st;
    *c = hwsel::CandsDev{cands->tile_m, cands->tile_n, cands->tile_k, cands->inst_n, cands->stages,
                         cands->cluster_m, cands->cluster_n, cands->swizzle, cands->inst_m_div16,
                         cands->inst_k, cands->kernel_sched, cands->epi_sched, cands->tile_sched};
    return HWSEL_OK;
}

int hwsel_features(hwsel_hw_t hw, const hwsel_problem_t *problems, int32_t P, const int64_t *seg_offsets,
                   const hwsel_cands_t *cands, int64_t R, int32_t n_features, float *X, int64_t ld,
                   void *stream)
{
    static const char *fn = "hwsel_features";
    hwsel::HwDev h;
    hwsel::CandsDev c;
    if (int st = check_rows(hw, problems, P, seg_offsets, cands, R, fn, &h, &c)) return st;
    if (!X) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (n_features != 64 && n_features != 96 && n_features != 128)
        return fail(HWSEL_EUNSUPPORTED, fn, "n_features=%d (supported: 64, 96, 128)", n_features);
    if (ld < n_features || ld % 4 != 0) return fail(HWSEL_EINVAL, fn, "ld=%lld", (long long)ld);
    if (!aligned16(X)) return fail(HWSEL_EINVAL, fn, "X not 16-byte aligned");
    return launched(hwsel::launch_features(h, problems, P, seg_offsets, c, R, n_features, X, ld,
                                           (hipStream_t)stream),
                    fn);
}

int hwsel_sample_score(hwsel_hw_t hw, const hwsel_problem_t *problems, int32_t P, const int64_t *seg_offsets,
                       const hwsel_cands_t *cands, int64_t R, float *scores, void *stream)
{
    static const char *fn = "hwsel_sample_score";
    hwsel::HwDev h;
    hwsel::CandsDev c;
    if (int st = check_rows(hw, problems, P, seg_offsets, cands, R, fn, &h, &c)) return st;
    if (!scores) return fail(HWSEL_EINVAL, fn, "null pointer");
    return launched(hwsel::launch_sample_score(h, problems, P, seg_offsets, c, R, scores, (hipStream_t)stream), fn);
}

int hwsel_linear_score(const hwsel_linear_t *lin, const float *X, int64_t R, int64_t ld, float *scores,
                       void *stream)
{
    static const char *fn = "hwsel_linear_score";
    if (!lin || !X || !scores || !lin->mean || !lin->inv_std || !lin->w || !lin->w_onehot)
        return fail(HWSEL_EINVAL, fn, "null pointer");
    if (lin->n_features != 64 && lin->n_features != 96 && lin->n_features != 128)
        return fail(HWSEL_EUNSUPPORTED, fn, "n_features=%d (supported: 64, 96, 128)", lin->n_features);
    if (R < 1) return fail(HWSEL_EINVAL, fn, "R=%lld", (long long)R);
    if (ld < lin->n_features || ld % 4 != 0) return fail(HWSEL_EINVAL, fn, "ld=%lld", (long long)ld);
    if (!aligned16(X)) return fail(HWSEL_EINVAL, fn, "X not 16-byte aligned");
    return launched(hwsel::launch_linear(*lin, X, R, ld, scores, (hipStream_t)stream), fn);
}

int hwsel_evaluate_workspace_bytes(int32_t P, size_t *bytes)
{
    static const char *fn = "hwsel_evaluate_workspace_bytes";
    if (!bytes) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (P < 1) return fail(HWSEL_EINVAL, fn, "P=%d", P);
    *bytes = hwsel::evaluate_workspace_bytes(P);
    g_err[0] = 0;
    return HWSEL_OK;
}

int hwsel_evaluate(const float *runtimes, const int64_t *seg_offsets, int32_t P, const int32_t *idx, int32_t k,
                   double *out, double *regret, int32_t *rank, double *ybar, void *workspace,
                   size_t workspace_bytes, void *stream)
{
    static const char *fn = "hwsel_evaluate";
    if (!runtimes || !seg_offsets || !idx || !out || !workspace) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (P < 1) return fail(HWSEL_EINVAL, fn, "P=%d", P);
    if (k < 1 || k > 64) return fail(HWSEL_EINVAL, fn, "k=%d (1..64)", k);
    const size_t need = hwsel::evaluate_workspace_bytes(P);
    if (workspace_bytes < need) return fail(HWSEL_EINVAL, fn, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (((uintptr_t)workspace & 255u) != 0) return fail(HWSEL_EINVAL, fn, "workspace not 256-byte aligned");
    return launched(hwsel::launch_evaluate(runtimes, seg_offsets, P, idx, k, out, regret, rank, ybar, workspace,
                                           (hipStream_t)stream),
                    fn);
}

int hwsel_evaluate_noalloc(const float *runtimes, const int64_t *seg_offsets, int32_t P, const int32_t *idx,
                           int32_t k, double *out, double *regret, int32_t *rank, double *ybar, void *stream)
{
    static const char *fn = "hwsel_evaluate_noalloc";
    if (!runtimes || !seg_offsets || !idx || !out) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (P < 1 || P > HWSEL_EVAL_NOALLOC_MAX_P)
        return fail(HWSEL_EINVAL, fn, "P=%d (1..%d)", P, HWSEL_EVAL_NOALLOC_MAX_P);
    if (k < 1 || k > 64) return fail(HWSEL_EINVAL, fn, "k=%d (1..64)", k);
    void *scratch = nullptr;
    size_t scratch_bytes = 0;
    const hipError_t e = hwsel::evaluate_noalloc_scratch(&scratch, &scratch_bytes);
    if (e != hipSuccess) return fail(HWSEL_EHIP, fn, "scratch address: %s", hipGetErrorString(e));
    if (scratch_bytes < hwsel::evaluate_workspace_bytes(P) || scratch_bytes != HWSEL_EVAL_NOALLOC_SCRATCH_BYTES)
        return fail(HWSEL_EHIP, fn, "scratch of %zu bytes", scratch_bytes);
    return launched(hwsel::launch_evaluate(runtimes, seg_offsets, P, idx, k, out, regret, rank, ybar, scratch,
                                           (hipStream_t)stream),
                    fn);
}

int hwsel_static_config_workspace_bytes(int32_t P, int32_t n_configs, size_t *bytes)
{
    static const char *fn = "hwsel_static_config_workspace_bytes";
    if (!bytes) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (P < 1 || n_configs < 1) return fail(HWSEL_EINVAL, fn, "P=%d n_configs=%d", P, n_configs);
    *bytes = hwsel::static_config_workspace_bytes(P, n_configs);
    g_err[0] = 0;
    return HWSEL_OK;
}

int hwsel_static_config(const float *runtimes, const int64_t *seg_offsets, int32_t P, const int32_t *config_id,
                        int32_t n_configs, int32_t *best, double *mean_y, void *workspace, size_t workspace_bytes,
                        void *stream)
{
    static const char *fn = "hwsel_static_config";
    if (!runtimes || !seg_offsets || !config_id || !best || !mean_y || !workspace)
        return fail(HWSEL_EINVAL, fn, "null pointer");
    if (P < 1 || n_configs < 1) return fail(HWSEL_EINVAL, fn, "P=%d n_configs=%d", P, n_configs);
    const size_t need = hwsel::static_config_workspace_bytes(P, n_configs);
    if (workspace_bytes < need) return fail(HWSEL_EINVAL, fn, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (((uintptr_t)workspace & 255u) != 0) return fail(HWSEL_EINVAL, fn, "workspace not 256-byte aligned");
    return launched(hwsel::launch_static_config(runtimes, seg_offsets, P, config_id, n_configs, best, mean_y,
                                                workspace, (hipStream_t)stream),
                    fn);
}

int hwsel_catalogue_mask(hwsel_hw_t hw, const hwsel_problem_t *problems, int32_t P, uint32_t flags, uint8_t *mask,
                         int64_t *n_valid, void *stream)
{
    static const char *fn = "hwsel_catalogue_mask";
    hwsel::HwDev h;
    if (!problems || !mask || !n_valid) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (P < 1) return fail(HWSEL_EINVAL, fn, "P=%d", P);
    if (((uintptr_t)mask & 3u) != 0) return fail(HWSEL_EINVAL, fn, "mask not 4-byte aligned");
    if (int st = check_hw(hw, fn, &h)) return st;
    return launched(hwsel::launch_catalogue_mask(h, problems, P, flags, mask, n_valid, (hipStream_t)stream), fn);
}

int hwsel_catalogue_compact(const uint8_t *mask, const int64_t *n_valid, int32_t P, int64_t *seg_offsets,
                            int32_t *point, int64_t capacity, void *stream)
{
    static const char *fn = "hwsel_catalogue_compact";
    if (!mask || !n_valid || !seg_offsets || (!point && capacity > 0)) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (P < 1 || capacity < 0) return fail(HWSEL_EINVAL, fn, "P=%d capacity=%lld", P, (long long)capacity);
    if (((uintptr_t)mask & 3u) != 0) return fail(HWSEL_EINVAL, fn, "mask not 4-byte aligned");
    return launched(hwsel::launch_catalogue_compact(mask, n_valid, P, seg_offsets, point, capacity,
                                                    (hipStream_t)stream),
                    fn);
}

int hwsel_catalogue_candidates(const hwsel_problem_t *problems, int32_t P, const int64_t *seg_offsets,
                               const int32_t *point, int64_t R, const hwsel_cands_out_t *out, void *stream)
{
    static const char *fn = "hwsel_catalogue_candidates";
    if (!problems || !seg_offsets || !out) return fail(HWSEL_EINVAL, fn, "null pointer");
    const void *fields[] = {out->tile_m, out->tile_n, out->tile_k, out->inst_n, out->stages, out->cluster_m,
                            out->cluster_n, out->swizzle, out->inst_m_div16, out->inst_k, out->kernel_sched,
                            out->epi_sched, out->tile_sched};
    for (const void *f : fields)
        if (!f) return fail(HWSEL_EINVAL, fn, "null candidate field");
    if (P < 1 || R < 1) return fail(HWSEL_EINVAL, fn, "P=%d R=%lld", P, (long long)R);
    return launched(hwsel::launch_catalogue_candidates(problems, P, seg_offsets, point, R, *out,
                                                       (hipStream_t)stream),
                    fn);
}

static int check_forest(const hwsel_forest_t *f, const float *X, int64_t R, int64_t ld, const char *fn)
{
    if (!f || !X || !f->node_feature || !f->node_threshold || !f->leaf_value)
        return fail(HWSEL_EINVAL, fn, "null pointer");
    if (R < 1 || f->n_trees < 1) return fail(HWSEL_EINVAL, fn, "R=%lld n_trees=%d", (long long)R, f->n_trees);
    if (f->depth < 1 || f->depth > 12) return fail(HWSEL_EUNSUPPORTED, fn, "depth=%d (1..12)", f->depth);
    if (f->n_features < 1 || f->n_features > 256)
        return fail(HWSEL_EUNSUPPORTED, fn, "n_features=%d (1..256)", f->n_features);
    if (ld < f->n_features) return fail(HWSEL_EINVAL, fn, "ld=%lld < n_features", (long long)ld);
    return HWSEL_OK;
}

int hwsel_forest_pack_bytes(const hwsel_forest_t *f, size_t *bytes)
{
    static const char *fn = "hwsel_forest_pack_bytes";
    if (!f || !bytes) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (f->n_trees < 1) return fail(HWSEL_EINVAL, fn, "n_trees=%d", f->n_trees);
    if (!hwsel::packable(*f))
        return fail(HWSEL_EUNSUPPORTED, fn, "depth=%d n_features=%d (packed: depth <= 10, n_features <= 128)",
                    f->depth, f->n_features);
    *bytes = hwsel::packed_bytes(*f);
    g_err[0] = 0;
    return HWSEL_OK;
}

int hwsel_forest_pack(const hwsel_forest_t *f, void *packed, size_t bytes, void *stream)
{
    static const char *fn = "hwsel_forest_pack";
    size_t need = 0;
    if (int s = hwsel_forest_pack_bytes(f, &need)) return s;
    if (!packed || !f->node_feature || !f->node_threshold || !f->leaf_value)
        return fail(HWSEL_EINVAL, fn, "null pointer");
    if (f->n_features < 1 || f->depth < 1) return fail(HWSEL_EINVAL, fn, "empty forest shape");
    if (bytes < need) return fail(HWSEL_EINVAL, fn, "bytes=%zu < %zu", bytes, need);
    if (!aligned16(packed)) return fail(HWSEL_EINVAL, fn, "packed not 16-byte aligned");
    switch (hwsel::pack_forest(*f, packed, (hipStream_t)stream)) {
    case hwsel::PackStatus::ok: g_err[0] = 0; return HWSEL_OK;
    case hwsel::PackStatus::bad_feature: return fail(HWSEL_EINVAL, fn, "node feature >= n_features");
    case hwsel::PackStatus::nan_threshold: return fail(HWSEL_EINVAL, fn, "NaN threshold");
    case hwsel::PackStatus::too_many_thresholds:
        return fail(HWSEL_EUNSUPPORTED, fn, "a feature has more than 255 distinct thresholds");
    default: return fail(HWSEL_EHIP, fn, "copy failed: %s", hipGetErrorString(hipGetLastError()));
    }
}

int hwsel_forest_pack_host(const hwsel_forest_t *f, void *image, size_t bytes)
{
    static const char *fn = "hwsel_forest_pack_host";
    size_t need = 0;
    if (int s = hwsel_forest_pack_bytes(f, &need)) return s;
    if (!image || !f->node_feature || !f->node_threshold || !f->leaf_value)
        return fail(HWSEL_EINVAL, fn, "null pointer");
    if (f->n_features < 1 || f->depth < 1) return fail(HWSEL_EINVAL, fn, "empty forest shape");
    if (bytes < need) return fail(HWSEL_EINVAL, fn, "bytes=%zu < %zu", bytes, need);
    switch (hwsel::build_image(*f, f->node_feature, f->node_threshold, f->leaf_value, static_cast<uint8_t *>(image))) {
    case hwsel::PackStatus::ok: g_err[0] = 0; return HWSEL_OK;
    case hwsel::PackStatus::bad_feature: return fail(HWSEL_EINVAL, fn, "node feature >= n_features");
    case hwsel::PackStatus::nan_threshold: return fail(HWSEL_EINVAL, fn, "NaN threshold");
    case hwsel::PackStatus::too_many_thresholds:
        return fail(HWSEL_EUNSUPPORTED, fn, "a feature has more than 255 distinct thresholds");
    default: return fail(HWSEL_EINVAL, fn, "cannot pack");
    }
}

int hwsel_forest_workspace_bytes(const hwsel_forest_t *f, int64_t R, size_t *bytes)
{
    static const char *fn = "hwsel_forest_workspace_bytes";
    size_t dummy = 0;
    if (int s = hwsel_forest_pack_bytes(f, &dummy)) return s;
    if (R < 1) return fail(HWSEL_EINVAL, fn, "R=%lld", (long long)R);
    *bytes = hwsel::packed_workspace_bytes(*f, R);
    return HWSEL_OK;
}

int hwsel_forest_score(const hwsel_forest_t *f, const void *packed, const float *X, int64_t R, int64_t ld,
                       float *scores, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *fn = "hwsel_forest_score";
    if (int s = check_forest(f, X, R, ld, fn)) return s;
    if (!scores) return fail(HWSEL_EINVAL, fn, "null scores");
    if (!packed) return launched(hwsel::launch_forest_score(*f, X, R, ld, scores, (hipStream_t)stream), fn);
    if (!hwsel::packable(*f)) return fail(HWSEL_EUNSUPPORTED, fn, "forest shape cannot be packed");
    if (!aligned16(packed)) return fail(HWSEL_EINVAL, fn, "packed not 16-byte aligned");
    const size_t need = hwsel::packed_workspace_bytes(*f, R);
    if (!workspace || workspace_bytes < need)
        return fail(HWSEL_EINVAL, fn, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (((uintptr_t)workspace & 255u) != 0) return fail(HWSEL_EINVAL, fn, "workspace not 256-byte aligned");
    return launched(hwsel::launch_forest_packed(*f, packed, X, R, ld, scores, workspace, (hipStream_t)stream), fn);
}

int hwsel_forest_score_checked(const hwsel_forest_t *f, const void *packed, const float *X, int64_t R, int64_t ld,
                               float *scores, void *workspace, size_t workspace_bytes, uint64_t *leaf_hash,
                               uint16_t *leaf_idx, int64_t leaf_row0, int64_t leaf_rows, void *stream)
{
    static const char *fn = "hwsel_forest_score_checked";
    if (int s = check_forest(f, X, R, ld, fn)) return s;
    if (!scores || !packed) return fail(HWSEL_EINVAL, fn, "null scores or packed image");
    if (!hwsel::packable(*f)) return fail(HWSEL_EUNSUPPORTED, fn, "forest shape cannot be packed");
    if (!aligned16(packed)) return fail(HWSEL_EINVAL, fn, "packed not 16-byte aligned");
    const size_t need = hwsel::packed_workspace_bytes(*f, R);
    if (!workspace || workspace_bytes < need)
        return fail(HWSEL_EINVAL, fn, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (((uintptr_t)workspace & 255u) != 0) return fail(HWSEL_EINVAL, fn, "workspace not 256-byte aligned");
    if (((uintptr_t)leaf_hash & 7u) != 0) return fail(HWSEL_EINVAL, fn, "leaf_hash not 8-byte aligned");
    if (leaf_idx && (leaf_row0 < 0 || leaf_rows < 1 || leaf_row0 > R - leaf_rows))
        return fail(HWSEL_EINVAL, fn, "leaf rows [%lld, %lld + %lld) outside [0, %lld)", (long long)leaf_row0,
                    (long long)leaf_row0, (long long)leaf_rows, (long long)R);
    return launched(hwsel::launch_forest_checked(*f, packed, X, R, ld, scores, workspace, leaf_hash, leaf_idx,
                                                 leaf_row0, leaf_rows, (hipStream_t)stream),
                    fn);
}

int hwsel_forest_leaves(const hwsel_forest_t *f, const float *X, int64_t R, int64_t ld, const int64_t *rows,
                        int64_t n_rows, uint16_t *leaf_idx, void *stream)
{
    static const char *fn = "hwsel_forest_leaves";
    if (int s = check_forest(f, X, R, ld, fn)) return s;
    if (!rows || !leaf_idx) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (n_rows < 1) return fail(HWSEL_EINVAL, fn, "n_rows=%lld", (long long)n_rows);
    return launched(hwsel::launch_forest_leaves(*f, X, R, ld, rows, n_rows, leaf_idx, (hipStream_t)stream), fn);
}

int hwsel_select_forest_workspace_bytes(const hwsel_forest_t *f, int64_t R, size_t *bytes)
{
    static const char *fn = "hwsel_select_forest_workspace_bytes";
    size_t dummy = 0;
    if (int s = hwsel_forest_pack_bytes(f, &dummy)) return s;
    if (!bytes) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (R < 1) return fail(HWSEL_EINVAL, fn, "R=%lld", (long long)R);
    *bytes = hwsel::packed_workspace_bytes(*f, R) + ((size_t)R * sizeof(float) + 255) / 256 * 256;
    return HWSEL_OK;
}

int hwsel_select_forest(hwsel_hw_t hw, const hwsel_problem_t *problems, int32_t P, const int64_t *seg_offsets,
                        const hwsel_cands_t *cands, int64_t R, int32_t n_features, const hwsel_forest_t *f,
                        const void *packed, int32_t k, int32_t *idx, float *vals, float *scores, void *workspace,
                        size_t workspace_bytes, void *stream)
{
    static const char *fn = "hwsel_select_forest";
    hwsel::HwDev h;
    hwsel::CandsDev c;
    if (int st = check_rows(hw, problems, P, seg_offsets, cands, R, fn, &h, &c)) return st;
    if (n_features != 64 && n_features != 96 && n_features != 128)
        return fail(HWSEL_EUNSUPPORTED, fn, "n_features=%d (supported: 64, 96, 128)", n_features);
    if (!f || !packed || !idx || !workspace || !f->node_feature || !f->node_threshold || !f->leaf_value)
        return fail(HWSEL_EINVAL, fn, "null pointer");
    if (f->n_trees < 1) return fail(HWSEL_EINVAL, fn, "n_trees=%d", f->n_trees);
    if (!hwsel::packable(*f)) return fail(HWSEL_EUNSUPPORTED, fn, "forest shape cannot be packed");
    if (f->n_features < 1 || f->n_features > n_features)
        return fail(HWSEL_EINVAL, fn, "forest n_features=%d, feature map has %d", f->n_features, n_features);
    if (k < 1 || k > 64) return fail(HWSEL_EINVAL, fn, "k=%d (1..64)", k);
    if (!aligned16(packed)) return fail(HWSEL_EINVAL, fn, "packed not 16-byte aligned");
    const size_t base = hwsel::packed_workspace_bytes(*f, R);
    const size_t need = base + ((size_t)R * sizeof(float) + 255) / 256 * 256;
    if (workspace_bytes < need)
        return fail(HWSEL_EINVAL, fn, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (((uintptr_t)workspace & 255u) != 0) return fail(HWSEL_EINVAL, fn, "workspace not 256-byte aligned");
    hipStream_t s = (hipStream_t)stream;
    float *sc = scores ? scores : reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + base);
    hipError_t e = hwsel::launch_features_bins(h, problems, P, seg_offsets, c, R, n_features,
                                               packed, hwsel::packed_image_id(*f), f->n_features,
                                               hwsel::packed_nan_bin(*f), static_cast<uint8_t *>(workspace),
                                               hwsel::packed_bin_stride(*f), s);
    if (e == hipSuccess) e = hwsel::launch_forest_from_bins(*f, packed, R, sc, workspace, s);
    if (e == hipSuccess) e = hwsel::launch_topk(sc, seg_offsets, P, k, idx, vals, s);
    return launched(e, fn);
}

static int check_mlp(const hwsel_mlp_t *m, const char *fn)
{
    if (!m || !m->mean || !m->inv_std || !m->W1 || !m->W2 || !m->W3 || !m->W4 || !m->b1 || !m->b2 || !m->b3 ||
        !m->b4)
        return fail(HWSEL_EINVAL, fn, "null pointer");
    if (m->n_in != 128 || m->h1 != 512 || m->h2 != 512 || m->h3 != 256)
        return fail(HWSEL_EUNSUPPORTED, fn, "widths %d-%d-%d-%d (supported: 128-512-512-256)", m->n_in, m->h1,
                    m->h2, m->h3);
    return HWSEL_OK;
}

int hwsel_mlp_pack_bytes(const hwsel_mlp_t *m, size_t *bytes)
{
    static const char *fn = "hwsel_mlp_pack_bytes";
    if (!bytes) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (int s = check_mlp(m, fn)) return s;
    *bytes = hwsel::mlp_packed_bytes();
    g_err[0] = 0;
    return HWSEL_OK;
}

int hwsel_mlp_pack(const hwsel_mlp_t *m, void *packed, size_t bytes, void *stream)
{
    static const char *fn = "hwsel_mlp_pack";
    if (int s = check_mlp(m, fn)) return s;
    if (!packed) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (bytes < hwsel::mlp_packed_bytes()) return fail(HWSEL_EINVAL, fn, "bytes=%zu < %zu", bytes, hwsel::mlp_packed_bytes());
    if (!aligned16(packed)) return fail(HWSEL_EINVAL, fn, "packed not 16-byte aligned");
    return launched(hwsel::launch_mlp_pack(*m, packed, (hipStream_t)stream), fn);
}

int hwsel_mlp_score(const hwsel_mlp_t *m, const void *packed, const float *X, int64_t R, int64_t ld, float *scores,
                    void *stream)
{
    static const char *fn = "hwsel_mlp_score";
    if (int s = check_mlp(m, fn)) return s;
    if (!X || !scores) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (R < 1) return fail(HWSEL_EINVAL, fn, "R=%lld", (long long)R);
    if (ld < 128 || ld % 4 != 0) return fail(HWSEL_EINVAL, fn, "ld=%lld", (long long)ld);
    if (!aligned16(X)) return fail(HWSEL_EINVAL, fn, "X not 16-byte aligned");
    if (!packed) return launched(hwsel::launch_mlp(*m, X, R, ld, scores, (hipStream_t)stream), fn);
    if (!aligned16(packed) || !aligned16(m->mean) || !aligned16(m->inv_std) || !aligned16(m->b1) ||
        !aligned16(m->b2) || !aligned16(m->b3) || ((uintptr_t)m->W4 & 7u) != 0)
        return fail(HWSEL_EINVAL, fn, "misaligned packed weights, statistics or biases");
    return launched(hwsel::launch_mlp_packed(*m, packed, X, R, ld, scores, (hipStream_t)stream), fn);
}

int hwsel_topk_per_problem(const float *scores, const int64_t *seg_offsets, int32_t P, int32_t k, int32_t *idx,
                           float *vals, void *stream)
{
    static const char *fn = "hwsel_topk_per_problem";
    if (!scores || !seg_offsets || !idx) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (P < 1) return fail(HWSEL_EINVAL, fn, "P=%d", P);
    if (k < 1 || k > 64) return fail(HWSEL_EINVAL, fn, "k=%d (1..64)", k);
    return launched(hwsel::launch_topk(scores, seg_offsets, P, k, idx, vals, (hipStream_t)stream), fn);
}

int hwsel_regret(const float *runtimes, const int64_t *seg_offsets, int32_t P, const int32_t *idx, int32_t k,
                 float *regret_top1, float *regret_bestk, int32_t *best_idx, void *stream)
{
    static const char *fn = "hwsel_regret";
    if (!runtimes || !seg_offsets || !idx || !regret_top1) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (P < 1) return fail(HWSEL_EINVAL, fn, "P=%d", P);
    if (k < 1 || k > 64) return fail(HWSEL_EINVAL, fn, "k=%d (1..64)", k);
    return launched(hwsel::launch_regret(runtimes, seg_offsets, P, idx, k, regret_top1, regret_bestk, best_idx,
                                         (hipStream_t)stream),
                    fn);
}

// Largest sizes of an 8-bit matrix: row numbers within an int32 with room to
// step past the end, and columns whose
// blocks fit a grid's second dimension (of 2^16 - 1 groups of four blocks)
// and 256 rows of which lie within 2^32 bytes.
static constexpr int64_t kFp8MaxRows = (int64_t)1 << 30, kFp8MaxCols = (int64_t)1 << 23;

static int check_fp8(const hwsel_fp8_t *x, const char *name, const char *fn)
{
    if (!x || !x->q || !x->scale) return fail(HWSEL_EINVAL, fn, "%s: null pointer", name);
    if (x->rows < 1 || x->cols < 1)
        return fail(HWSEL_EINVAL, fn, "%s: %lld x %lld", name, (long long)x->rows, (long long)x->cols);
    if (x->format != HWSEL_FP8_E4M3 && x->format != HWSEL_FP8_E5M2)
        return fail(HWSEL_EINVAL, fn, "%s: format %d", name, x->format);
    if (x->block_rows != 1 && x->block_rows != HWSEL_FP8_BLOCK)
        return fail(HWSEL_EINVAL, fn, "%s: block_rows %d (1 or 128)", name, x->block_rows);
    if (x->rows > kFp8MaxRows || x->cols > kFp8MaxCols)
        return fail(HWSEL_EUNSUPPORTED, fn, "%s: %lld x %lld (at most %lld x %lld)", name, (long long)x->rows,
                    (long long)x->cols, (long long)kFp8MaxRows, (long long)kFp8MaxCols);
    const int64_t nkb = (x->cols + HWSEL_FP8_BLOCK - 1) / HWSEL_FP8_BLOCK;
    if (x->ld < nkb * HWSEL_FP8_BLOCK || x->ld % 16 != 0 || !aligned16(x->q))
        return fail(HWSEL_EINVAL, fn, "%s: codes misaligned or ld=%lld short", name, (long long)x->ld);
    if (x->ld >= (int64_t)1 << 24) return fail(HWSEL_EUNSUPPORTED, fn, "%s: ld=%lld", name, (long long)x->ld);
    if (x->ld_scale < nkb || x->ld_scale % 4 != 0 || ((uintptr_t)x->scale & 3u) != 0)
        return fail(HWSEL_EINVAL, fn, "%s: scales misaligned or ld_scale=%lld short", name, (long long)x->ld_scale);
    return HWSEL_OK;
}

// A plain matrix beside an 8-bit one: dtype, row length and element alignment.
static int check_plain(const void *X, int32_t dtype, int64_t ld, int64_t cols, const char *fn)
{
    if (!X) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (dtype != HWSEL_DTYPE_FP32 && dtype != HWSEL_DTYPE_BF16)
        return fail(HWSEL_EUNSUPPORTED, fn, "dtype %d (fp32 or bf16)", dtype);
    if (ld < cols) return fail(HWSEL_EINVAL, fn, "ld=%lld < %lld", (long long)ld, (long long)cols);
    if ((uintptr_t)X % (dtype == HWSEL_DTYPE_FP32 ? 4 : 2) != 0) return fail(HWSEL_EINVAL, fn, "matrix misaligned");
    return HWSEL_OK;
}

int hwsel_fp8_quantise(const void *X, int32_t dtype, int64_t ld, int32_t transposed, const float *mean,
                       const float *inv_std, const hwsel_fp8_t *out, void *stream)
{
    static const char *fn = "hwsel_fp8_quantise";
    if (int st = check_fp8(out, "out", fn)) return st;
    if (transposed != 0 && transposed != 1) return fail(HWSEL_EINVAL, fn, "transposed=%d", transposed);
    if (int st = check_plain(X, dtype, ld, transposed ? out->rows : out->cols, fn)) return st;
    if (!mean != !inv_std) return fail(HWSEL_EINVAL, fn, "mean and inv_std go together");
    if (mean && (transposed || out->block_rows != 1))
        return fail(HWSEL_EUNSUPPORTED, fn, "standardising goes with rows as they are and block_rows 1");
    return launched(hwsel::launch_fp8_quantise(X, dtype == HWSEL_DTYPE_BF16, ld, transposed != 0, mean, inv_std, *out,
                                               (hipStream_t)stream),
                    fn);
}

int hwsel_fp8_dequantise(const hwsel_fp8_t *in, void *X, int32_t dtype, int64_t ld, void *stream)
{
    static const char *fn = "hwsel_fp8_dequantise";
    if (int st = check_fp8(in, "in", fn)) return st;
    if (int st = check_plain(X, dtype, ld, in->cols, fn)) return st;
    return launched(hwsel::launch_fp8_dequantise(*in, X, dtype == HWSEL_DTYPE_BF16, ld, (hipStream_t)stream), fn);
}

int hwsel_fp8_transpose(const hwsel_fp8_t *in, const hwsel_fp8_t *out, void *stream)
{
    static const char *fn = "hwsel_fp8_transpose";
    if (int st = check_fp8(in, "in", fn)) return st;
    if (int st = check_fp8(out, "out", fn)) return st;
    if (in->rows != out->cols || in->cols != out->rows)
        return fail(HWSEL_EINVAL, fn, "%lld x %lld transposed is not %lld x %lld", (long long)in->rows,
                    (long long)in->cols, (long long)out->rows, (long long)out->cols);
    return launched(hwsel::launch_fp8_transpose(*in, *out, (hipStream_t)stream), fn);
}

static int check_product(const hwsel_fp8_t *A, const hwsel_fp8_t *B, const char *fn)
{
    if (int st = check_fp8(A, "A", fn)) return st;
    if (int st = check_fp8(B, "B", fn)) return st;
    if (A->cols != B->cols)
        return fail(HWSEL_EINVAL, fn, "summed sizes %lld and %lld differ", (long long)A->cols, (long long)B->cols);
    if (B->format != HWSEL_FP8_E4M3) return fail(HWSEL_EUNSUPPORTED, fn, "B in E5M2");
    return HWSEL_OK;
}

static int check_product_call(const hwsel_fp8_t *A, const hwsel_fp8_t *B, const float *bias, int32_t activation,
                              const void *workspace, size_t workspace_bytes, bool fp32, bool codes, const char *fn)
{
    if (int st = check_product(A, B, fn)) return st;
    if (!hwsel::fp8_product_fits(A->rows, B->rows, A->cols, fp32, codes))
        return fail(HWSEL_EUNSUPPORTED, fn, "a result of %lld x %lld", (long long)A->rows, (long long)B->rows);
    if ((uintptr_t)bias & 3u) return fail(HWSEL_EINVAL, fn, "bias misaligned");
    if (activation != HWSEL_ACT_NONE && activation != HWSEL_ACT_GELU)
        return fail(HWSEL_EINVAL, fn, "activation %d", activation);
    const size_t need = hwsel::fp8_matmul_workspace_bytes(A->rows, B->rows, A->cols);
    if (need && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need))
        return fail(HWSEL_EINVAL, fn, "workspace of %zu bytes, %zu needed, 256-byte aligned", workspace_bytes, need);
    return HWSEL_OK;
}

int hwsel_fp8_matmul_workspace_bytes(const hwsel_fp8_t *A, const hwsel_fp8_t *B, size_t *bytes)
{
    static const char *fn = "hwsel_fp8_matmul_workspace_bytes";
    if (!bytes) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (int st = check_product(A, B, fn)) return st;
    *bytes = hwsel::fp8_matmul_workspace_bytes(A->rows, B->rows, A->cols);
    g_err[0] = 0;
    return HWSEL_OK;
}

int hwsel_fp8_matmul(const hwsel_fp8_t *A, const hwsel_fp8_t *B, const float *bias, int32_t activation, void *C,
                     int32_t dtype, int64_t ldc, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *fn = "hwsel_fp8_matmul";
    if (int st = check_product_call(A, B, bias, activation, workspace, workspace_bytes, dtype == HWSEL_DTYPE_FP32, false, fn))
        return st;
    if (int st = check_plain(C, dtype, ldc, B->rows, fn)) return st;
    return launched(hwsel::launch_fp8_matmul(*A, *B, bias, activation == HWSEL_ACT_GELU, C, dtype == HWSEL_DTYPE_BF16, ldc,
                                             workspace, (hipStream_t)stream),
                    fn);
}

int hwsel_fp8_layer(const hwsel_fp8_t *A, const hwsel_fp8_t *B, const float *bias, int32_t activation,
                    const hwsel_fp8_t *C, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *fn = "hwsel_fp8_layer";
    if (int st = check_product_call(A, B, bias, activation, workspace, workspace_bytes, false, true, fn)) return st;
    if (int st = check_fp8(C, "C", fn)) return st;
    if (C->rows != A->rows || C->cols != B->rows)
        return fail(HWSEL_EINVAL, fn, "C is %lld x %lld, the product %lld x %lld", (long long)C->rows, (long long)C->cols,
                    (long long)A->rows, (long long)B->rows);
    if (C->format != HWSEL_FP8_E4M3 || C->block_rows != 1)
        return fail(HWSEL_EUNSUPPORTED, fn, "C: format %d block_rows %d (E4M3, 1)", C->format, C->block_rows);
    return launched(hwsel::launch_fp8_layer(*A, *B, bias, activation == HWSEL_ACT_GELU, *C, workspace, (hipStream_t)stream), fn);
}

static int check_sample_sizes(int64_t R, int32_t P, int32_t n_draws, const char *fn)
{
    if (R < 0 || P < 1 || n_draws < 1)
        return fail(HWSEL_EINVAL, fn, "R=%lld P=%d n_draws=%d", (long long)R, P, n_draws);
    if (R > (int64_t)1 << 30) return fail(HWSEL_EUNSUPPORTED, fn, "R=%lld (at most 2^30)", (long long)R);
    return HWSEL_OK;
}

int hwsel_sample_workspace_bytes(int64_t R, int32_t P, int32_t n_draws, size_t *bytes)
{
    static const char *fn = "hwsel_sample_workspace_bytes";
    if (!bytes) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (int st = check_sample_sizes(R, P, n_draws, fn)) return st;
    *bytes = hwsel::sample_workspace_bytes(R, P, n_draws);
    g_err[0] = 0;
    return HWSEL_OK;
}

int hwsel_sample_per_problem(const float *scores, int64_t R, const int64_t *seg_offsets, int32_t P,
                             const hwsel_sampling_t *how, const float *u, int32_t n_draws, int32_t *idx, float *prob,
                             int32_t *kept, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *fn = "hwsel_sample_per_problem";
    if (int st = check_sample_sizes(R, P, n_draws, fn)) return st;
    if ((!scores && R > 0) || !seg_offsets || !how || !u || !idx) return fail(HWSEL_EINVAL, fn, "null pointer");
    const size_t need = hwsel::sample_workspace_bytes(R, P, n_draws);
    if (need && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need))
        return fail(HWSEL_EINVAL, fn, "workspace of %zu bytes, %zu needed, 256-byte aligned", workspace_bytes, need);
    return launched(hwsel::launch_sample(scores, R, seg_offsets, P, *how, u, n_draws, idx, prob, kept, workspace,
                                         (hipStream_t)stream),
                    fn);
}

static int check_logprob_sizes(int64_t R, int32_t P, const char *fn)
{
    if (R < 0 || P < 1) return fail(HWSEL_EINVAL, fn, "R=%lld P=%d", (long long)R, P);
    if (R > (int64_t)1 << 30) return fail(HWSEL_EUNSUPPORTED, fn, "R=%lld (at most 2^30)", (long long)R);
    return HWSEL_OK;
}

static int check_top(int32_t top, const char *fn)
{
    return top < 0 || top > 64 ? fail(HWSEL_EINVAL, fn, "top=%d (0..64)", top) : HWSEL_OK;
}

int hwsel_logprob_workspace_bytes(int64_t R, int32_t P, int32_t top, size_t *bytes)
{
    static const char *fn = "hwsel_logprob_workspace_bytes";
    if (!bytes) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (int st = check_logprob_sizes(R, P, fn)) return st;
    if (int st = check_top(top, fn)) return st;
    *bytes = hwsel::logprob_workspace_bytes(R, P, top);
    g_err[0] = 0;
    return HWSEL_OK;
}

int hwsel_logprob_per_problem(const float *scores, int64_t R, const int64_t *seg_offsets, int32_t P, float temperature,
                              const float *temperature_of, const int32_t *picks, int32_t n_picks, int32_t top,
                              float *logp, float *entropy, float *norm, int32_t *top_idx, float *top_logp,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *fn = "hwsel_logprob_per_problem";
    if (int st = check_logprob_sizes(R, P, fn)) return st;
    if (n_picks < 0) return fail(HWSEL_EINVAL, fn, "n_picks=%d", n_picks);
    if (int st = check_top(top, fn)) return st;
    if ((!scores && R > 0) || !seg_offsets || (n_picks > 0 && (!picks || !logp)) || (top > 0 && (!top_idx || !top_logp)))
        return fail(HWSEL_EINVAL, fn, "null pointer");
    const size_t need = hwsel::logprob_workspace_bytes(R, P, top);
    if (need && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need))
        return fail(HWSEL_EINVAL, fn, "workspace of %zu bytes, %zu needed, 256-byte aligned", workspace_bytes, need);
    const Region ins[] = {region_of(scores, 4 * R), region_of(seg_offsets, 8 * ((int64_t)P + 1)), region_of(temperature_of, 4 * (int64_t)P),
                          region_of(n_picks ? picks : nullptr, 4 * (int64_t)P * n_picks)};
    const Named outs[] = {{"logp", region_of(n_picks ? logp : nullptr, 4 * (int64_t)P * n_picks)}, {"entropy", region_of(entropy, 4 * (int64_t)P)},
                          {"norm", region_of(norm, 8 * (int64_t)P)}, {"top_idx", region_of(top ? top_idx : nullptr, 4 * (int64_t)P * top)},
                          {"top_logp", region_of(top ? top_logp : nullptr, 4 * (int64_t)P * top)}, {"the workspace", region_of(workspace, (int64_t)need)}};
    if (int st = check_apart(outs, ins, -1, fn)) return st;
    return launched(hwsel::launch_logprob(scores, R, seg_offsets, P, temperature, temperature_of, picks, n_picks, top, logp, entropy,
                                          norm, top_idx, top_logp, workspace, (hipStream_t)stream),
                    fn);
}

int hwsel_logprob_gradient(const float *scores, int64_t R, const int64_t *seg_offsets, int32_t P, float temperature,
                           const float *temperature_of, const float *norm, const int32_t *picks, int32_t n_picks,
                           const float *d_logp, const float *entropy, const float *d_entropy, float *d_scores, void *stream)
{
    static const char *fn = "hwsel_logprob_gradient";
    if (int st = check_logprob_sizes(R, P, fn)) return st;
    if (n_picks < 0) return fail(HWSEL_EINVAL, fn, "n_picks=%d", n_picks);
    if (((!scores || !d_scores) && R > 0) || !seg_offsets || !norm || (n_picks > 0 && (!picks || !d_logp)))
        return fail(HWSEL_EINVAL, fn, "null pointer");
    if (!entropy != !d_entropy) return fail(HWSEL_EINVAL, fn, "entropy and d_entropy go together");
    if (scores < d_scores + R && d_scores < scores + R) return fail(HWSEL_EINVAL, fn, "d_scores overlaps the scores");
    const int64_t of_problems = 4 * (int64_t)P, of_picks = 4 * (int64_t)P * n_picks;
    const Region ins[] = {region_of(seg_offsets, 8 * ((int64_t)P + 1)), region_of(temperature_of, of_problems), region_of(norm, 2 * of_problems),
                          region_of(n_picks ? picks : nullptr, of_picks), region_of(n_picks ? d_logp : nullptr, of_picks),
                          region_of(entropy, of_problems), region_of(d_entropy, of_problems)};
    const Named outs[] = {{"d_scores", region_of(d_scores, 4 * R)}};
    if (int st = check_apart(outs, ins, -1, fn)) return st;
    return launched(hwsel::launch_logprob_gradient(scores, R, seg_offsets, P, temperature, temperature_of, norm, picks, n_picks,
                                                   d_logp, entropy, d_entropy, d_scores, (hipStream_t)stream),
                    fn);
}

static const hwsel_matrix_t kNoMatrix = {nullptr, 0, HWSEL_DTYPE_FP32};

static const hwsel_matrix_t &or_none(const hwsel_matrix_t *m) { return m && m->data ? *m : kNoMatrix; }

// Rows and columns of plain matrices are 32-bit numbers in the kernels, with room to step past the last column.
static int check_plain_sizes(int64_t rows, int64_t cols, const char *fn)
{
    if (rows < 1 || cols < 1) return fail(HWSEL_EINVAL, fn, "%lld x %lld", (long long)rows, (long long)cols);
    if (rows > INT32_MAX || cols > (int64_t)1 << 30)
        return fail(HWSEL_EUNSUPPORTED, fn, "%lld x %lld (rows below 2^31, at most 2^30 columns)", (long long)rows, (long long)cols);
    return HWSEL_OK;
}

// A matrix that may be absent; its dtype is `dtype` where that is not negative.
static int check_matrix(const hwsel_matrix_t &m, const char *name, int64_t cols, int32_t dtype, const char *fn)
{
    if (!m.data) return HWSEL_OK;
    if (int st = check_plain(m.data, m.dtype, m.ld, cols, fn)) return st;
    if (m.ld > (int64_t)1 << 40) return fail(HWSEL_EINVAL, fn, "%s: ld=%lld", name, (long long)m.ld);
    if (dtype >= 0 && m.dtype != dtype) return fail(HWSEL_EINVAL, fn, "%s: dtype %d, not %d", name, m.dtype, dtype);
    return HWSEL_OK;
}

// A result in the place of an operand lies as that does.
static int check_in_place(const hwsel_matrix_t &out, const hwsel_matrix_t &in, const char *name, const char *fn)
{
    if (out.data && out.data == in.data && (out.ld != in.ld || out.dtype != in.dtype))
        return fail(HWSEL_EINVAL, fn, "%s in place, with another ld or dtype", name);
    return HWSEL_OK;
}

static int check_dropout(const hwsel_dropout_t &d, const char *fn)
{
    if (!(d.p >= 0.0f && d.p <= 1.0f)) return fail(HWSEL_EINVAL, fn, "p=%g (0..1)", (double)d.p);
    if ((uintptr_t)d.state & 7u) return fail(HWSEL_EINVAL, fn, "state misaligned");
    return HWSEL_OK;
}

int hwsel_dropout(const hwsel_dropout_t *how, int64_t rows, int64_t cols, const hwsel_matrix_t *X, const hwsel_matrix_t *residual,
                  const hwsel_matrix_t *Y, void *stream)
{
    static const char *fn = "hwsel_dropout";
    if (!how || !X || !X->data || !Y || !Y->data) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (int st = check_plain_sizes(rows, cols, fn)) return st;
    if (int st = check_dropout(*how, fn)) return st;
    if (int st = check_matrix(*X, "X", cols, -1, fn)) return st;
    if (int st = check_matrix(*Y, "Y", cols, -1, fn)) return st;
    if (int st = check_matrix(or_none(residual), "residual", cols, Y->dtype, fn)) return st;
    const hwsel_matrix_t &r = or_none(residual);
    if (int st = check_in_place(*Y, *X, "Y", fn)) return st;
    if (int st = check_in_place(*Y, r, "Y", fn)) return st;
    const Region ins[] = {Y->data == X->data ? Region{} : region_of(*X, rows, cols), Y->data == r.data ? Region{} : region_of(r, rows, cols),
                          region_of(how->state, 16)};
    const Named outs[] = {{"Y", region_of(*Y, rows, cols)}};
    if (int st = check_apart(outs, ins, -1, fn)) return st;
    return launched(hwsel::launch_dropout(*how, rows, cols, *X, r, *Y, (hipStream_t)stream), fn);
}

// What both passes of a join share.
static int check_join(const hwsel_join_t *j, const char *fn)
{
    if (!j) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (int st = check_plain_sizes(j->rows, j->cols, fn)) return st;
    if (int st = check_dropout(j->dropout, fn)) return st;
    if (!(j->eps > 0.0f) || j->eps > 3.4028235e38f) return fail(HWSEL_EINVAL, fn, "eps=%g", (double)j->eps);
    if (!(__builtin_fabsf(j->stream_scale) <= 3.4028235e38f) || !(__builtin_fabsf(j->branch_scale) <= 3.4028235e38f))
        return fail(HWSEL_EINVAL, fn, "scales %g and %g", (double)j->stream_scale, (double)j->branch_scale);
    if ((j->post_norm != 0 && j->post_norm != 1) || (j->gate_sigmoid != 0 && j->gate_sigmoid != 1))
        return fail(HWSEL_EINVAL, fn, "post_norm=%d gate_sigmoid=%d", j->post_norm, j->gate_sigmoid);
    if (j->gate_cols != 0 && j->gate_cols != 1 && j->gate_cols != j->cols)
        return fail(HWSEL_EINVAL, fn, "gate_cols=%lld (0, 1 or %lld)", (long long)j->gate_cols, (long long)j->cols);
    if (((uintptr_t)j->w_branch & 3u) || ((uintptr_t)j->w_pre & 3u)) return fail(HWSEL_EINVAL, fn, "weights misaligned");
    return HWSEL_OK;
}

static int check_branch(const hwsel_join_t *j, const hwsel_matrix_t &y, const hwsel_matrix_t &gate, const char *fn)
{
    if (!y.data && (j->gate_cols != 0 || j->w_branch)) return fail(HWSEL_EINVAL, fn, "a gate or w_branch without y");
    if ((j->gate_cols != 0) != (gate.data != nullptr)) return fail(HWSEL_EINVAL, fn, "gate_cols=%lld and gate", (long long)j->gate_cols);
    return HWSEL_OK;
}

int hwsel_block_join(const hwsel_join_t *j, const hwsel_matrix_t *x, const hwsel_matrix_t *y_, const hwsel_matrix_t *gate_,
                     const hwsel_matrix_t *x1_, const hwsel_matrix_t *z_, void *stream)
{
    static const char *fn = "hwsel_block_join";
    if (int st = check_join(j, fn)) return st;
    const hwsel_matrix_t &y = or_none(y_), &gate = or_none(gate_), &x1 = or_none(x1_), &z = or_none(z_);
    if (!x || !x->data || (!x1.data && !z.data)) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (int st = check_branch(j, y, gate, fn)) return st;
    const int32_t block = y.data ? y.dtype : -1;
    if (int st = check_matrix(*x, "x", j->cols, -1, fn)) return st;
    if (int st = check_matrix(y, "y", j->cols, -1, fn)) return st;
    if (int st = check_matrix(gate, "gate", j->gate_cols, block, fn)) return st;
    if (int st = check_matrix(x1, "x1", j->cols, x->dtype, fn)) return st;
    if (int st = check_matrix(z, "z", j->cols, block, fn)) return st;
    if (int st = check_in_place(x1, *x, "x1", fn)) return st;
    auto at = [&](const hwsel_matrix_t &m, int64_t width) { return region_of(m, j->rows, width); };
    const Region ins[] = {at(*x, j->cols), at(y, j->cols), at(gate, j->gate_cols), region_of(j->w_branch, 4 * j->cols),
                          region_of(j->w_pre, 4 * j->cols), region_of(j->dropout.state, 16)};
    const Named outs[] = {{"z", at(z, j->cols)}, {"x1", at(x1, j->cols)}};
    if (int st = check_apart(outs, ins, x1.data == x->data ? 1 : -1, fn)) return st;
    const bool bbf = (y.data ? y.dtype : z.dtype) == HWSEL_DTYPE_BF16;
    return launched(hwsel::launch_block_join(*j, *x, y, gate, x1, z, x->dtype == HWSEL_DTYPE_BF16, bbf, (hipStream_t)stream), fn);
}

int hwsel_block_join_gradient_workspace_bytes(const hwsel_join_t *j, size_t *bytes)
{
    static const char *fn = "hwsel_block_join_gradient_workspace_bytes";
    if (!bytes) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (int st = check_join(j, fn)) return st;
    *bytes = hwsel::join_gradient_workspace_bytes(*j);
    g_err[0] = 0;
    return HWSEL_OK;
}

int hwsel_block_join_gradient(const hwsel_join_t *j, const hwsel_matrix_t *x1, const hwsel_matrix_t *y_, const hwsel_matrix_t *gate_,
                              const hwsel_matrix_t *d_x1_, const hwsel_matrix_t *d_z_, const hwsel_matrix_t *dx_,
                              const hwsel_matrix_t *dy_, const hwsel_matrix_t *dgate_, float *dw_branch, float *dw_pre, void *workspace,
                              size_t workspace_bytes, void *stream)
{
    static const char *fn = "hwsel_block_join_gradient";
    if (int st = check_join(j, fn)) return st;
    const hwsel_matrix_t &y = or_none(y_), &gate = or_none(gate_), &d_x1 = or_none(d_x1_), &d_z = or_none(d_z_), &dx = or_none(dx_),
                         &dy = or_none(dy_), &dgate = or_none(dgate_);
    if (!x1 || !x1->data || (!d_x1.data && !d_z.data)) return fail(HWSEL_EINVAL, fn, "null pointer");
    if (!dx.data && !dy.data && !dgate.data && !dw_branch && !dw_pre) return fail(HWSEL_EINVAL, fn, "no output");
    if (int st = check_branch(j, y, gate, fn)) return st;
    if ((!y.data && (dy.data || dw_branch)) || (!gate.data && dgate.data) || (!d_z.data && dw_pre))
        return fail(HWSEL_EINVAL, fn, "an output without its input");
    const int32_t block = y.data ? y.dtype : -1;
    if (int st = check_matrix(*x1, "x1", j->cols, -1, fn)) return st;
    if (int st = check_matrix(y, "y", j->cols, -1, fn)) return st;
    if (int st = check_matrix(gate, "gate", j->gate_cols, block, fn)) return st;
    if (int st = check_matrix(d_x1, "d_x1", j->cols, x1->dtype, fn)) return st;
    if (int st = check_matrix(d_z, "d_z", j->cols, block, fn)) return st;
    if (int st = check_matrix(dx, "dx", j->cols, x1->dtype, fn)) return st;
    if (int st = check_matrix(dy, "dy", j->cols, block, fn)) return st;
    if (int st = check_matrix(dgate, "dgate", j->gate_cols, block, fn)) return st;
    if (int st = check_in_place(dx, d_x1, "dx", fn)) return st;
    if (((uintptr_t)dw_branch & 3u) || ((uintptr_t)dw_pre & 3u)) return fail(HWSEL_EINVAL, fn, "weights' gradients misaligned");
    const size_t need = hwsel::join_gradient_workspace_bytes(*j);
    if (need && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need))
        return fail(HWSEL_EINVAL, fn, "workspace of %zu bytes, %zu needed, 256-byte aligned", workspace_bytes, need);
    const int64_t cols = j->cols;
    auto at = [&](const hwsel_matrix_t &m, int64_t width) { return region_of(m, j->rows, width); };
    const Named outs[] = {{"dx", at(dx, cols)}, {"dy", at(dy, cols)}, {"dgate", at(dgate, j->gate_cols)}, {"dw_branch", region_of(dw_branch, 4 * cols)},
                          {"dw_pre", region_of(dw_pre, 4 * cols)}, {"the workspace", region_of(workspace, (int64_t)need)}};
    const Region ins[] = {at(d_x1, cols), at(*x1, cols), at(y, cols), at(gate, j->gate_cols), at(d_z, cols), region_of(j->w_branch, 4 * cols),
                          region_of(j->w_pre, 4 * cols), region_of(j->dropout.state, 16)};
    if (int st = check_apart(outs, ins, dx.data == d_x1.data ? 0 : -1, fn)) return st;
    const bool bbf = (y.data ? y.dtype : d_z.dtype) == HWSEL_DTYPE_BF16;
    return launched(hwsel::launch_block_join_gradient(*j, *x1, y, gate, d_x1, d_z, dx, dy, dgate, dw_branch, dw_pre, workspace,
                                                      x1->dtype == HWSEL_DTYPE_BF16, bbf, (hipStream_t)stream),
                    fn);
}

}  // extern "C"
