// Entry points of aet_ops.h: the checks of what a caller hands over, and the errors.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <initializer_list>

#include "ops_internal.h"

namespace aet_ops {

static thread_local char g_error[256] = "";

static aet_status fail(aet_status st, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof g_error, fmt, ap);
    va_end(ap);
    return st;
}

static aet_status done(hipError_t e) {
    return e == hipSuccess ? AET_OK : fail(AET_EHIP, "%s", hipGetErrorString(e));
}

Drop make_drop(double p, uint64_t seed, int64_t first_row, int64_t cols) {
    Drop d;
    d.key = aet::splitmix_at(seed, 3);
    d.half = (uint64_t)(cols + 1) / 2;
    d.first = (uint64_t)first_row * d.half;
    const double least = floor(p * 4294967296.0 + 0.5);
    d.least = least >= 4294967295.0 ? 4294967295u : (uint32_t)least;
    d.scale = (float)(1 / (1 - p));
    return d;
}

// What a matrix per client (or maps: three strides) may look like.  Sizes and strides are bounded so that no
// offset leaves 63 bits.
constexpr int64_t kMost = INT64_C(1) << 46;   // elements between the first and the last of a tensor

static bool in_reach(int64_t count, int64_t stride) {
    return stride >= 0 && (count <= 1 || stride <= kMost / (count - 1));
}
static int64_t esize(int dtype) { return dtype == AET_F32 ? 4 : 2; }

static const char *bad_ptr(const void *p, int dtype) {
    if (!p) return "is NULL";
    return (uintptr_t)p % (uintptr_t)esize(dtype) ? "is not aligned to its type" : nullptr;
}
// nd strides of an input, outermost first, and how many there are of each
static const char *bad_in(const void *p, int dtype, int nd, const int64_t *count, const int64_t *stride) {
    for (int i = 0; i < nd; ++i)
        if (!in_reach(count[i], stride[i])) return "has a stride that is negative or too large";
    return bad_ptr(p, dtype);
}
// An output's places must be distinct: each stride reaches past all that lies inside it.
static const char *bad_out(const void *p, int dtype, int nd, const int64_t *count, const int64_t *stride, int64_t cols) {
    if (const char *why = bad_in(p, dtype, nd, count, stride)) return why;
    int64_t span = cols;
    for (int i = nd - 1; i >= 0; --i) {
        if (count[i] > 1 && stride[i] < span) return "overlaps itself";
        span = (count[i] - 1) * stride[i] + span;
    }
    return nullptr;
}

constexpr int kMostSize = 1 << 30;
static bool bad_sizes(std::initializer_list<int64_t> sizes, const char **why) {
    for (int64_t v : sizes)
        if (v < 0 || v > kMostSize) {
            *why = "a size is negative or over 2^30";
            return true;
        }
    return false;
}
static bool bad_common(int dtype, int act, const char **why) {
    if (dtype != AET_F32 && dtype != AET_BF16) *why = "dtype is neither AET_F32 nor AET_BF16";
    else if (act < AET_ACT_NONE || act > AET_ACT_GELU) *why = "act is none of the AET_ACT_ values";
    else return false;
    return true;
}
static bool bad_drop(double p, int64_t first_row, int64_t rows, const char **why) {
    if (!(p >= 0 && p < 1)) *why = "p is not in [0, 1)";
    else if (first_row < 0 || first_row > INT64_MAX - rows) *why = "first_row is out of range";
    else return false;
    return true;
}
static bool bad_workspace(const void *ws, size_t have, size_t need) {
    return need && (!ws || have < need || (uintptr_t)ws % 256);
}

#define AET_CHECK(name, expr)                                                    \
    do {                                                                         \
        if (const char *why_ = (expr)) return fail(AET_EINVAL, name " %s", why_); \
    } while (0)

// ---- linear ------------------------------------------------------------------------------

static aet_status check(const aet_linear *a) {
    const char *why;
    if (!a) return fail(AET_EINVAL, "the record is NULL");
    if (bad_common(a->dtype, a->act, &why)) return fail(AET_EINVAL, "%s", why);
    if (bad_sizes({a->n, a->rows, a->in, a->out}, &why)) return fail(AET_EINVAL, "%s", why);
    if (bad_drop(a->p, a->first_row, (int64_t)a->n * a->rows, &why)) return fail(AET_EINVAL, "%s", why);
    if (!a->n || !a->rows || !a->out) return AET_OK;
    const int64_t nr[2] = {a->n, a->rows}, no[2] = {a->n, a->out};
    auto in = [&](const aet_in &t, const int64_t *count) { const int64_t st[2] = {t.client, t.row}; return bad_in(t.p, a->dtype, 2, count, st); };
    auto out = [&](const aet_out &t, const int64_t *count, int64_t cols) { const int64_t st[2] = {t.client, t.row}; return bad_out(t.p, a->dtype, 2, count, st, cols); };
    if (a->in) {
        AET_CHECK("x", in(a->x, nr));
        AET_CHECK("w", in(a->w, no));
    }
    if (a->bias.p) {
        const int64_t st[1] = {a->bias.client};
        AET_CHECK("bias", bad_in(a->bias.p, a->dtype, 1, nr, st));
    }
    if (a->residual.p) AET_CHECK("residual", in(a->residual, nr));
    AET_CHECK("y", out(a->y, nr, a->out));
    if (a->pre.p) AET_CHECK("pre", out(a->pre, nr, a->out));
    return AET_OK;
}

// One W for all clients and rows that lie in one piece: the clients are one.
static void fold(aet_linear &a) {
    if (a.n <= 1) return;
    auto flat = [&](const void *p, int64_t client, int64_t row) { return !p || client == a.rows * row; };
    if (a.w.client || (a.bias.p && a.bias.client) || (int64_t)a.n * a.rows > kMostSize) return;
    if (!flat(a.x.p, a.x.client, a.x.row) || !flat(a.residual.p, a.residual.client, a.residual.row) ||
        !flat(a.y.p, a.y.client, a.y.row) || !flat(a.pre.p, a.pre.client, a.pre.row))
        return;
    a.rows *= a.n;
    a.n = 1;
}

static aet_status check(const aet_linear_grad *a, bool *shared) {
    const char *why;
    if (!a) return fail(AET_EINVAL, "the record is NULL");
    if (bad_common(a->dtype, a->act, &why)) return fail(AET_EINVAL, "%s", why);
    if (bad_sizes({a->n, a->rows, a->in, a->out}, &why)) return fail(AET_EINVAL, "%s", why);
    if (bad_drop(a->p, a->first_row, (int64_t)a->n * a->rows, &why)) return fail(AET_EINVAL, "%s", why);
    *shared = a->n != 1 && ((a->dw.p && !a->dw.client) || (a->db.p && !a->db.client));
    const int64_t n = *shared ? 1 : a->n;   // gradients of parameters
    const int64_t nr[2] = {a->n, a->rows}, no[2] = {a->n, a->out}, go[2] = {n, a->out};
    auto in = [&](const aet_in &t, const int64_t *count) { const int64_t st[2] = {t.client, t.row}; return bad_in(t.p, a->dtype, 2, count, st); };
    auto out = [&](const aet_out &t, const int64_t *count, int64_t cols) { const int64_t st[2] = {t.client, t.row}; return bad_out(t.p, a->dtype, 2, count, st, cols); };
    const bool wants = a->dx.p || a->dw.p || a->db.p;
    if (a->n && a->rows && a->out && wants) {
        AET_CHECK("dy", in(a->dy, nr));
        if (a->act != AET_ACT_NONE) AET_CHECK("pre", in(a->pre, nr));
        if (a->dw.p && a->in) AET_CHECK("x", in(a->x, nr));
        if (a->dx.p && a->in) AET_CHECK("w", in(a->w, no));
    }
    if (a->dx.p) AET_CHECK("dx", out(a->dx, nr, a->in));
    if (a->dw.p) AET_CHECK("dw", out(a->dw, go, a->in));
    if (a->db.p) {
        const int64_t st[1] = {a->db.client};
        AET_CHECK("db", bad_out(a->db.p, a->dtype, 1, go, st, a->out));
    }
    if (*shared) {
        if ((a->dx.p && a->w.client) || (a->dw.p && a->dw.client) || (a->db.p && a->db.client))
            return fail(AET_EINVAL, "w, dw and db: either all or none are the same for all clients (client = 0)");
        // (of those that are read or written; up to one row a client, there is nothing that a row's stride would say)
        auto flat = [&](const void *p, int64_t client, int64_t row) { return !p || a->rows <= 1 || client == a->rows * row; };
        if (a->n && (!flat(a->dy.p, a->dy.client, a->dy.row) || (a->dw.p && !flat(a->x.p, a->x.client, a->x.row)) ||
                     (a->act != AET_ACT_NONE && !flat(a->pre.p, a->pre.client, a->pre.row)) || !flat(a->dx.p, a->dx.client, a->dx.row)))
            return fail(AET_EINVAL, "one W for all clients: rows have to lie client after client (client = rows * row)");
        if ((int64_t)a->n * a->rows > kMostSize) return fail(AET_EINVAL, "one W for all clients: more than 2^30 rows");
    }
    return AET_OK;
}

static void fold(aet_linear_grad &a, bool shared) {
    if (!shared) return;
    if (a.rows == 1) {
        a.dy.row = a.dy.client;
        a.x.row = a.x.client;
        a.pre.row = a.pre.client;
        a.dx.row = a.dx.client;
    }
    a.rows *= a.n;
    a.n = 1;
}

// ---- group norm --------------------------------------------------------------------------

template <class A>
static aet_status check_norm(const A *a) {
    const char *why;
    if (bad_common(a->dtype, a->act, &why)) return fail(AET_EINVAL, "%s", why);
    if (bad_sizes({a->n, a->batch, a->positions}, &why)) return fail(AET_EINVAL, "%s", why);
    if (a->groups < 1 || a->width < 1 || (int64_t)a->groups * a->width > (1 << 24))
        return fail(AET_EINVAL, "groups and width have to be positive, with at most 2^24 channels");
    const int64_t one[1] = {a->n};
    if (a->gamma.p) AET_CHECK("gamma", bad_in(a->gamma.p, a->dtype, 1, one, &a->gamma.client));
    if (a->beta.p) AET_CHECK("beta", bad_in(a->beta.p, a->dtype, 1, one, &a->beta.client));
    return AET_OK;
}
template <class M>
static const char *bad_maps(const M &t, int dtype, int64_t n, int64_t batch, int64_t positions, int64_t channels, bool out) {
    const int64_t count[3] = {n, batch, positions}, st[3] = {t.client, t.sample, t.row};
    return out ? bad_out(t.p, dtype, 3, count, st, channels) : bad_in(t.p, dtype, 3, count, st);
}
static const char *bad_stats(const float *p) { return (uintptr_t)p % 4 ? "is not aligned to its type" : nullptr; }

static aet_status check(const aet_group_norm *a) {
    if (!a) return fail(AET_EINVAL, "the record is NULL");
    if (const aet_status st = check_norm(a)) return st;
    if (!(a->eps >= 0)) return fail(AET_EINVAL, "eps is negative");
    AET_CHECK("mean", bad_stats(a->mean));
    AET_CHECK("rstd", bad_stats(a->rstd));
    if (!a->n || !a->batch || !a->positions) return AET_OK;
    const int64_t C = (int64_t)a->groups * a->width;
    AET_CHECK("x", bad_maps(a->x, a->dtype, a->n, a->batch, a->positions, C, false));
    AET_CHECK("y", bad_maps(a->y, a->dtype, a->n, a->batch, a->positions, C, true));
    return AET_OK;
}
static aet_status check(const aet_group_norm_grad *a) {
    if (!a) return fail(AET_EINVAL, "the record is NULL");
    if (const aet_status st = check_norm(a)) return st;
    const int64_t C = (int64_t)a->groups * a->width;
    auto param = [&](const aet_out &t) {
        const int64_t count[1] = {t.client ? a->n : 1};
        return bad_out(t.p, a->dtype, 1, count, &t.client, C);
    };
    if (a->dgamma.p) AET_CHECK("dgamma", param(a->dgamma));
    if (a->dbeta.p) AET_CHECK("dbeta", param(a->dbeta));
    if (a->n != 1 && a->dgamma.p && a->dbeta.p && !a->dgamma.client != !a->dbeta.client)
        return fail(AET_EINVAL, "dgamma and dbeta: either both or none are the same for all clients (client = 0)");
    if (!a->n || !a->batch || !a->positions) return AET_OK;
    AET_CHECK("dy", bad_maps(a->dy, a->dtype, a->n, a->batch, a->positions, C, false));
    AET_CHECK("x", bad_maps(a->x, a->dtype, a->n, a->batch, a->positions, C, false));
    if (a->dx.p) AET_CHECK("dx", bad_maps(a->dx, a->dtype, a->n, a->batch, a->positions, C, true));
    if (!a->mean || !a->rstd) return fail(AET_EINVAL, "mean or rstd is NULL");
    AET_CHECK("mean", bad_stats(a->mean));
    AET_CHECK("rstd", bad_stats(a->rstd));
    return AET_OK;
}

// ---- dropout -----------------------------------------------------------------------------

static aet_status run_dropout(const aet_dropout *a, bool residual, void *hip_stream) {
    const char *why;
    if (!a) return fail(AET_EINVAL, "the record is NULL");
    if (bad_common(a->dtype, AET_ACT_NONE, &why)) return fail(AET_EINVAL, "%s", why);
    if (bad_sizes({a->n, a->rows, a->cols}, &why)) return fail(AET_EINVAL, "%s", why);
    if (bad_drop(a->p, a->first_row, (int64_t)a->n * a->rows, &why)) return fail(AET_EINVAL, "%s", why);
    if (!residual && a->residual.p) return fail(AET_EINVAL, "the gradient takes no residual");
    if (!a->n || !a->rows || !a->cols) return AET_OK;
    const int64_t nr[2] = {a->n, a->rows}, xs[2] = {a->x.client, a->x.row}, rs[2] = {a->residual.client, a->residual.row},
                  ys[2] = {a->y.client, a->y.row};
    AET_CHECK("x", bad_in(a->x.p, a->dtype, 2, nr, xs));
    if (a->residual.p) AET_CHECK("residual", bad_in(a->residual.p, a->dtype, 2, nr, rs));
    AET_CHECK("y", bad_out(a->y.p, a->dtype, 2, nr, ys, a->cols));
    aet_dropout b = *a;
    auto flat = [&](const void *p, int64_t client, int64_t row) { return !p || client == b.rows * row; };
    if (b.n > 1 && (int64_t)b.n * b.rows <= kMostSize && flat(b.x.p, b.x.client, b.x.row) && flat(b.y.p, b.y.client, b.y.row) &&
        flat(b.residual.p, b.residual.client, b.residual.row)) {
        b.rows *= b.n;
        b.n = 1;
    }
    return done(launch_dropout(b, (hipStream_t)hip_stream));
}

}  // namespace aet_ops

using namespace aet_ops;

extern "C" {

const char *aet_ops_last_error(void) { return g_error; }

aet_status aet_dropout_forward(const aet_dropout *a, void *hip_stream) { return run_dropout(a, true, hip_stream); }
aet_status aet_dropout_backward(const aet_dropout *a, void *hip_stream) { return run_dropout(a, false, hip_stream); }

size_t aet_linear_workspace_bytes(const aet_linear *a) {
    if (check(a) != AET_OK) return 0;
    aet_linear b = *a;
    fold(b);
    return b.n && b.rows && b.out ? linear_forward_workspace(b) : 0;
}
aet_status aet_linear_forward(const aet_linear *a, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (const aet_status st = check(a)) return st;
    aet_linear b = *a;
    fold(b);
    if (!b.n || !b.rows || !b.out) return AET_OK;
    const size_t need = linear_forward_workspace(b);
    if (bad_workspace(workspace, workspace_bytes, need))
        return fail(AET_ENOMEM, "the workspace needs %zu bytes, 256-byte aligned; got %zu", need, workspace_bytes);
    return done(launch_linear_forward(b, workspace, (hipStream_t)hip_stream));
}

size_t aet_linear_backward_workspace_bytes(const aet_linear_grad *a) {
    bool shared;
    if (check(a, &shared) != AET_OK) return 0;
    aet_linear_grad b = *a;
    fold(b, shared);
    return b.n ? linear_backward_workspace(b) : 0;
}
aet_status aet_linear_backward(const aet_linear_grad *a, void *workspace, size_t workspace_bytes, void *hip_stream) {
    bool shared;
    if (const aet_status st = check(a, &shared)) return st;
    aet_linear_grad b = *a;
    fold(b, shared);
    if (!b.n) return AET_OK;
    const size_t need = linear_backward_workspace(b);
    if (bad_workspace(workspace, workspace_bytes, need))
        return fail(AET_ENOMEM, "the workspace needs %zu bytes, 256-byte aligned; got %zu", need, workspace_bytes);
    return done(launch_linear_backward(b, workspace, (hipStream_t)hip_stream));
}

size_t aet_group_norm_workspace_bytes(const aet_group_norm *a) {
    return check(a) == AET_OK ? group_norm_forward_workspace(*a) : 0;
}
aet_status aet_group_norm_forward(const aet_group_norm *a, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (const aet_status st = check(a)) return st;
    if (!a->n || !a->batch) return AET_OK;
    const size_t need = group_norm_forward_workspace(*a);
    if (bad_workspace(workspace, workspace_bytes, need))
        return fail(AET_ENOMEM, "the workspace needs %zu bytes, 256-byte aligned; got %zu", need, workspace_bytes);
    return done(launch_group_norm_forward(*a, workspace, (hipStream_t)hip_stream));
}

size_t aet_group_norm_backward_workspace_bytes(const aet_group_norm_grad *a) {
    return check(a) == AET_OK ? group_norm_backward_workspace(*a) : 0;
}
aet_status aet_group_norm_backward(const aet_group_norm_grad *a, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (const aet_status st = check(a)) return st;
    const size_t need = group_norm_backward_workspace(*a);
    if (bad_workspace(workspace, workspace_bytes, need))
        return fail(AET_ENOMEM, "the workspace needs %zu bytes, 256-byte aligned; got %zu", need, workspace_bytes);
    return done(launch_group_norm_backward(*a, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
