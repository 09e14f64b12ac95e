// C-ABI of the row operators (declarations and contract: include/fragscan.h):
// argument checks, workspace sizes and launches.  Every check is done before
// anything is enqueued.
#include "../../include/fragscan.h"

#include <cstdarg>
#include <cstdio>

#include "rows.h"

using namespace fs;

namespace {

fs_status fail(fs_status s, const char *fmt, ...)
{
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return (fs_status)row_error(s, buf);
}

int elem(int dtype) { return dtype == FS_BF16 ? 2 : 4; }

bool aligned(const void *p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// One array of rows: stride within the limits, total extent below 2^62 bytes.
fs_status check_rows(const char *name, const void *p, int64_t rows, int64_t len, int64_t stride, int es, bool out)
{
    if (!p) return fail(FS_ERR_INVALID_ARG, "%s is NULL", name);
    if (!aligned(p, es)) return fail(FS_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    if (stride < 0 || (out && rows > 1 && stride < len))
        return fail(FS_ERR_INVALID_ARG, "%s: row stride %lld, rows of %lld", name, (long long)stride, (long long)len);
    if (stride > ((int64_t)1 << 60) / (rows > 1 ? rows : 1))
        return fail(FS_ERR_UNSUPPORTED, "%s: %lld rows of stride %lld", name, (long long)rows, (long long)stride);
    return FS_OK;
}

fs_status check_common(int64_t rows, int32_t dtype)
{
    if (rows < 0) return fail(FS_ERR_INVALID_ARG, "rows is %lld", (long long)rows);
    if (rows >= ((int64_t)1 << 31)) return fail(FS_ERR_UNSUPPORTED, "%lld rows: 2^31 or more", (long long)rows);
    if (dtype != FS_F32 && dtype != FS_BF16) return fail(FS_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    return FS_OK;
}

fs_status check_scores(int64_t rows, int32_t classes, int32_t dtype, int32_t n_top)
{
    fs_status st = check_common(rows, dtype);
    if (st != FS_OK) return st;
    if (classes < 1 || classes > FS_MAX_CLASSES) return fail(FS_ERR_INVALID_ARG, "classes is %d", classes);
    if (n_top < 0 || n_top > FS_MAX_TOP) return fail(FS_ERR_INVALID_ARG, "n_top is %d, at most %d", n_top, FS_MAX_TOP);
    return FS_OK;
}

fs_status check_temperature(float t)
{
    if (!(t >= 1e-30f && t <= 1e30f))
        return fail(FS_ERR_INVALID_ARG, "temperature %g: 1e-30 to 1e30", (double)t);
    return FS_OK;
}

fs_status check_floats(const char *name, const void *p)
{
    return aligned(p, 4) ? FS_OK : fail(FS_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
}

fs_status check_workspace(const void *ws, size_t have, size_t need)
{
    if (have < need) return fail(FS_ERR_WORKSPACE, "workspace of %zu bytes, the call needs %zu", have, need);
    if (need && !ws) return fail(FS_ERR_INVALID_ARG, "workspace pointer is NULL");
    if (need && !aligned(ws, 256)) return fail(FS_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    return FS_OK;
}

fs_status launched(hipError_t e, const char *what)
{
    return e == hipSuccess ? FS_OK : fail(FS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Sizes and pointers of a projection; `sizes` checks only what workspace sizes depend on.
fs_status check_projection(const fs_projection *p, bool sizes, ProjArgs &a)
{
    if (!p) return fail(FS_ERR_INVALID_ARG, "projection is NULL");
    fs_status st = check_common(p->rows, p->dtype);
    if (st != FS_OK) return st;
    if (p->k < 1 || p->k > FS_MAX_FEATURES || p->m < 1 || p->m > FS_MAX_FEATURES)
        return fail(FS_ERR_INVALID_ARG, "k is %d, m is %d: 1 to %d", p->k, p->m, FS_MAX_FEATURES);
    if (p->n_adapters < 0 || p->n_adapters > (1 << 20))
        return fail(FS_ERR_INVALID_ARG, "n_adapters is %d: 0 to %d", p->n_adapters, 1 << 20);
    if (p->n_adapters == 0 ? p->rank != 0 : (p->rank < 1 || p->rank > FS_MAX_RANK))
        return fail(FS_ERR_INVALID_ARG, "rank is %d with %d adapters: 1 to %d, 0 without adapters", p->rank,
                    p->n_adapters, FS_MAX_RANK);
    a = ProjArgs{p->rows, p->k, p->m, p->n_adapters, p->rank, p->d_x, p->d_w, p->x_stride, p->w_stride,
                 p->d_bias, p->d_a, p->d_b, p->d_scale, p->d_ids};
    if (sizes) return FS_OK;
    const int es = elem(p->dtype);
    if ((st = check_rows("d_w", p->d_w, p->m, p->k, p->w_stride, es, false)) != FS_OK) return st;
    if ((st = check_floats("d_bias", p->d_bias)) != FS_OK) return st;
    if (p->n_adapters) {
        if (!p->d_a || !p->d_b) return fail(FS_ERR_INVALID_ARG, "d_a or d_b is NULL with %d adapters", p->n_adapters);
        if (!aligned(p->d_a, es) || !aligned(p->d_b, es))
            return fail(FS_ERR_INVALID_ARG, "d_a or d_b is not aligned to its elements");
        if ((st = check_floats("d_scale", p->d_scale)) != FS_OK) return st;
        if ((st = check_floats("d_ids", p->d_ids)) != FS_OK) return st;
    } else if (p->d_a || p->d_b || p->d_scale || p->d_ids) {
        return fail(FS_ERR_INVALID_ARG, "adapter pointers given with no adapters");
    }
    if (p->rows) {
        if ((st = check_rows("d_x", p->d_x, p->rows, p->k, p->x_stride, es, false)) != FS_OK) return st;
        if (p->n_adapters && !p->d_ids) return fail(FS_ERR_INVALID_ARG, "d_ids is NULL with adapters");
    }
    return FS_OK;
}

}  // namespace

extern "C" {

fs_status fs_logprobs_workspace(int64_t rows, int32_t classes, int32_t dtype, int32_t n_top, size_t *bytes)
{
    if (!bytes) return fail(FS_ERR_INVALID_ARG, "bytes is NULL");
    fs_status st = check_scores(rows, classes, dtype, n_top);
    if (st != FS_OK) return st;
    *bytes = rows ? logprobs_workspace(rows, classes, dtype, n_top) : 0;
    return FS_OK;
}

fs_status fs_logprobs(const void *d_scores, int64_t rows, int32_t classes, int64_t stride, int32_t dtype,
                      float temperature, const int32_t *d_labels, int32_t n_top, float *d_logp, float *d_entropy,
                      float *d_norm, int32_t *d_top_id, float *d_top_logp, void *d_workspace,
                      size_t workspace_bytes, void *stream)
{
    fs_status st = check_scores(rows, classes, dtype, n_top);
    if (st != FS_OK) return st;
    if ((st = check_temperature(temperature)) != FS_OK) return st;
    if (!rows) return FS_OK;
    if ((st = check_rows("d_scores", d_scores, rows, classes, stride, elem(dtype), false)) != FS_OK) return st;
    if (!d_logp && !d_entropy && !d_norm && !d_top_id && !d_top_logp)
        return fail(FS_ERR_INVALID_ARG, "no output is wanted");
    if (d_logp && !d_labels) return fail(FS_ERR_INVALID_ARG, "d_logp needs d_labels");
    if ((d_top_id || d_top_logp) && !n_top) return fail(FS_ERR_INVALID_ARG, "a list of best classes with n_top 0");
    const void *floats[] = {d_labels, d_logp, d_entropy, d_norm, d_top_id, d_top_logp};
    for (const void *p : floats)
        if ((st = check_floats("a label or output array", p)) != FS_OK) return st;
    if ((st = check_workspace(d_workspace, workspace_bytes, logprobs_workspace(rows, classes, dtype, n_top))) != FS_OK)
        return st;
    const LogprobArgs a{d_scores, rows, stride, classes, 1.0f / temperature, d_labels,
                        d_top_id || d_top_logp ? n_top : 0, d_logp, d_entropy, d_norm, d_top_id, d_top_logp};
    return launched(launch_logprobs(a, dtype, d_workspace, static_cast<hipStream_t>(stream)), "fs_logprobs");
}

fs_status fs_logprobs_grad(const void *d_scores, int64_t rows, int32_t classes, int64_t stride, int32_t dtype,
                           float temperature, const int32_t *d_labels, const float *d_norm, const float *d_entropy,
                           const float *d_g_logp, const float *d_g_entropy, void *d_g_scores, int64_t g_stride,
                           void *stream)
{
    fs_status st = check_scores(rows, classes, dtype, 0);
    if (st != FS_OK) return st;
    if ((st = check_temperature(temperature)) != FS_OK) return st;
    if (!rows) return FS_OK;
    if ((st = check_rows("d_scores", d_scores, rows, classes, stride, elem(dtype), false)) != FS_OK) return st;
    if ((st = check_rows("d_g_scores", d_g_scores, rows, classes, g_stride, elem(dtype), true)) != FS_OK) return st;
    if (d_g_scores == d_scores && rows > 1 && stride != g_stride)
        return fail(FS_ERR_INVALID_ARG, "in place the two row strides must be equal");
    if (!d_norm) return fail(FS_ERR_INVALID_ARG, "d_norm is NULL");
    if (!d_g_logp && !d_g_entropy) return fail(FS_ERR_INVALID_ARG, "no gradient is given");
    if (d_g_logp && !d_labels) return fail(FS_ERR_INVALID_ARG, "d_g_logp needs d_labels");
    if (d_g_entropy && !d_entropy) return fail(FS_ERR_INVALID_ARG, "d_g_entropy needs d_entropy");
    const void *floats[] = {d_labels, d_norm, d_entropy, d_g_logp, d_g_entropy};
    for (const void *p : floats)
        if ((st = check_floats("a label or gradient array", p)) != FS_OK) return st;
    const LogprobGradArgs a{d_scores, rows, stride, classes, 1.0f / temperature, d_g_logp ? d_labels : nullptr, d_norm,
                            d_entropy, d_g_logp, d_g_entropy, d_g_scores, g_stride};
    return launched(launch_logprobs_grad(a, dtype, static_cast<hipStream_t>(stream)), "fs_logprobs_grad");
}

fs_status fs_project_workspace(const fs_projection *p, size_t *bytes)
{
    if (!bytes) return fail(FS_ERR_INVALID_ARG, "bytes is NULL");
    ProjArgs a;
    fs_status st = check_projection(p, true, a);
    if (st != FS_OK) return st;
    *bytes = project_workspace(a, p->dtype);
    return FS_OK;
}

fs_status fs_project(const fs_projection *p, void *d_y, int64_t y_stride, float *d_hidden, void *d_workspace,
                     size_t workspace_bytes, void *stream)
{
    ProjArgs a;
    fs_status st = check_projection(p, false, a);
    if (st != FS_OK) return st;
    if (!a.rows) return FS_OK;
    if ((st = check_rows("d_y", d_y, a.rows, a.M, y_stride, elem(p->dtype), true)) != FS_OK) return st;
    if (d_hidden && !a.n) return fail(FS_ERR_INVALID_ARG, "d_hidden given with no adapters");
    if ((st = check_floats("d_hidden", d_hidden)) != FS_OK) return st;
    if ((st = check_workspace(d_workspace, workspace_bytes, project_workspace(a, p->dtype))) != FS_OK) return st;
    return launched(launch_project(a, p->dtype, d_y, y_stride, d_hidden, d_workspace,
                                   static_cast<hipStream_t>(stream)), "fs_project");
}

fs_status fs_project_grad_workspace(const fs_projection *p, size_t *bytes)
{
    if (!bytes) return fail(FS_ERR_INVALID_ARG, "bytes is NULL");
    ProjArgs a;
    fs_status st = check_projection(p, true, a);
    if (st != FS_OK) return st;
    *bytes = project_grad_workspace(a, p->dtype);
    return FS_OK;
}

fs_status fs_project_grad(const fs_projection *p, const void *d_g, int64_t g_stride, const float *d_hidden,
                          void *d_gx, int64_t gx_stride, void *d_ga, void *d_gb, void *d_workspace,
                          size_t workspace_bytes, void *stream)
{
    ProjArgs a;
    fs_status st = check_projection(p, false, a);
    if (st != FS_OK) return st;
    const int es = elem(p->dtype);
    if (!d_gx && !d_ga && !d_gb) return fail(FS_ERR_INVALID_ARG, "no gradient is wanted");
    if (!d_ga != !d_gb) return fail(FS_ERR_INVALID_ARG, "d_ga and d_gb come together");
    if (d_ga && !a.n) return fail(FS_ERR_INVALID_ARG, "d_ga and d_gb given with no adapters");
    if (!aligned(d_ga, es) || !aligned(d_gb, es))
        return fail(FS_ERR_INVALID_ARG, "d_ga or d_gb is not aligned to its elements");
    if (d_hidden && !a.n) return fail(FS_ERR_INVALID_ARG, "d_hidden given with no adapters");
    if ((st = check_floats("d_hidden", d_hidden)) != FS_OK) return st;
    if (a.rows) {
        if ((st = check_rows("d_g", d_g, a.rows, a.M, g_stride, es, false)) != FS_OK) return st;
        if (d_gx && (st = check_rows("d_gx", d_gx, a.rows, a.K, gx_stride, es, true)) != FS_OK) return st;
    } else if (!d_ga) {
        return FS_OK;
    }
    if ((st = check_workspace(d_workspace, workspace_bytes, project_grad_workspace(a, p->dtype))) != FS_OK) return st;
    return launched(launch_project_grad(a, p->dtype, d_g, g_stride, d_hidden, d_gx, gx_stride, d_ga, d_gb,
                                        d_workspace, static_cast<hipStream_t>(stream)), "fs_project_grad");
}

}  // extern "C"
