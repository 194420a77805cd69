// The linear layer with bias, activation, dropout and residual in its epilogue, and its gradient.
#include "ops_internal.h"
#include "ops_tiles.h"

namespace aet_ops {

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

static Product forward_product(const aet_linear &a) {
    Product p = {};
    p.a = {a.x.p, a.x.client, a.x.row, false};
    p.b = {a.w.p, a.w.client, a.w.row, false};
    p.clients = a.n;
    p.M = a.rows;
    p.N = a.out;
    p.K = a.in;
    p.e = {a.bias, a.residual, a.y, a.pre, a.rows, a.act, make_drop(a.p, a.seed, a.first_row, a.out)};
    return p;
}
size_t linear_forward_workspace(const aet_linear &a) { return product_workspace(a.dtype, forward_product(a)); }
hipError_t launch_linear_forward(const aet_linear &a, void *workspace, hipStream_t s) {
    return launch_product(a.dtype, forward_product(a), workspace, s);
}

// dz, and db: a thread per column.
template <typename T>
__global__ __launch_bounds__(256) void k_dz(aet_linear_grad a, Drop d, T *dz, int64_t dz_row) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)a.n * a.out) return;
    const int64_t c = i / a.out;
    const int col = (int)(i - c * a.out);
    float sum = 0;
    for (int r = 0; r < a.rows; ++r) {
        float v[1] = {(float)((const T *)a.dy.p)[c * a.dy.client + r * a.dy.row + col]};
        if (d.least) drop_apply(d, drop_row(d, c * a.rows + r), col, v);
        if (a.act) {
            const float z = (float)((const T *)a.pre.p)[c * a.pre.client + r * a.pre.row + col];
            v[0] *= a.act == AET_ACT_RELU ? act_slope<AET_ACT_RELU>(z) : a.act == AET_ACT_SILU ? act_slope<AET_ACT_SILU>(z) : act_slope<AET_ACT_GELU>(z);
        }
        sum += v[0];
        if (dz) dz[(c * a.rows + r) * dz_row + col] = (T)v[0];
    }
    if (a.db.p) ((T *)a.db.p)[c * a.db.client + col] = (T)sum;
}

// dz has a place of its own unless it is dy.
struct BackwardPlan {
    bool own_dz;
    int64_t dz_row;
    Product dx, dw;
    size_t dz_bytes, bytes;
};
static BackwardPlan plan(const aet_linear_grad &a, char *workspace) {
    BackwardPlan b = {};
    b.own_dz = a.p > 0 || a.act != AET_ACT_NONE;
    const int e = a.dtype == AET_F32 ? 4 : 2;
    b.dz_row = ceil_div((int64_t)a.out * e, 16) * 16 / e;
    b.dz_bytes = b.own_dz && (a.dx.p || a.dw.p) ? up256((size_t)a.n * a.rows * b.dz_row * e) : 0;
    Operand dz = {a.dy.p, a.dy.client, a.dy.row, false};
    if (b.own_dz) dz = {workspace, a.rows * b.dz_row, b.dz_row, false};
    const Drop none = {};
    if (a.dx.p) {
        b.dx.a = dz;
        b.dx.b = {a.w.p, a.w.client, a.w.row, true};
        b.dx.clients = a.n;
        b.dx.M = a.rows;
        b.dx.N = a.in;
        b.dx.K = a.out;
        b.dx.e = {{}, {}, a.dx, {}, a.rows, AET_ACT_NONE, none};
    }
    if (a.dw.p) {
        dz.by_columns = true;
        b.dw.a = dz;
        b.dw.b = {a.x.p, a.x.client, a.x.row, true};
        b.dw.clients = a.n;
        b.dw.M = a.out;
        b.dw.N = a.in;
        b.dw.K = a.rows;
        b.dw.e = {{}, {}, a.dw, {}, a.out, AET_ACT_NONE, none};
    }
    const size_t x = product_workspace(a.dtype, b.dx), w = product_workspace(a.dtype, b.dw);
    b.bytes = b.dz_bytes + (x > w ? x : w);
    return b;
}

size_t linear_backward_workspace(const aet_linear_grad &a) { return plan(a, nullptr).bytes; }

template <typename T>
static hipError_t backward(const aet_linear_grad &a, char *workspace, hipStream_t s) {
    const BackwardPlan b = plan(a, workspace);
    const int64_t columns = (int64_t)a.n * a.out;
    if (columns && (b.dz_bytes || a.db.p))
        k_dz<T><<<(int)ceil_div(columns, 256), 256, 0, s>>>(a, make_drop(a.p, a.seed, a.first_row, a.out), b.dz_bytes ? (T *)workspace : nullptr, b.dz_row);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.dx.p) e = launch_product(a.dtype, b.dx, workspace + b.dz_bytes, s);
    if (e == hipSuccess && a.dw.p) e = launch_product(a.dtype, b.dw, workspace + b.dz_bytes, s);
    return e;
}
hipError_t launch_linear_backward(const aet_linear_grad &a, void *workspace, hipStream_t s) {
    return a.dtype == AET_F32 ? backward<float>(a, (char *)workspace, s) : backward<bf16>(a, (char *)workspace, s);
}

}  // namespace aet_ops
