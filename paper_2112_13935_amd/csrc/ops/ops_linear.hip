// The linear layer with bias, activation, dropout and residual in its epilogue, and its gradient.
#include "ops_internal.h"

namespace aet_ops {

// C[m][n] = sum over k of A(m, k) B(n, k) for each client; what is done with a sum is the epilogue's.
struct Operand {
    const void *p;
    int64_t client, row, k;   // strides
};

struct ForwardEpilogue {
    aet_in bias, residual;
    aet_out y, pre;
    int rows, act;
    Drop d;
};
struct StoreEpilogue {
    aet_out c;
};

__device__ __forceinline__ float act_any(int act, float z) {
    switch (act) {
    case AET_ACT_RELU: return act_value<AET_ACT_RELU>(z);
    case AET_ACT_SILU: return act_value<AET_ACT_SILU>(z);
    case AET_ACT_GELU: return act_value<AET_ACT_GELU>(z);
    default: return z;
    }
}
__device__ __forceinline__ float slope_any(int act, float z) {
    switch (act) {
    case AET_ACT_RELU: return act_slope<AET_ACT_RELU>(z);
    case AET_ACT_SILU: return act_slope<AET_ACT_SILU>(z);
    case AET_ACT_GELU: return act_slope<AET_ACT_GELU>(z);
    default: return 1.0f;
    }
}

template <typename T>
__device__ __forceinline__ void finish(const ForwardEpilogue &e, int c, int m, int n, float v) {
    if (e.bias.p) v += (float)((const T *)e.bias.p)[c * e.bias.client + n];
    if (e.pre.p) ((T *)e.pre.p)[c * e.pre.client + m * e.pre.row + n] = (T)v;
    float w[1] = {act_any(e.act, v)};
    if (e.d.least) drop_apply(e.d, drop_row(e.d, (int64_t)c * e.rows + m), n, w);
    if (e.residual.p) w[0] += (float)((const T *)e.residual.p)[c * e.residual.client + m * e.residual.row + n];
    ((T *)e.y.p)[c * e.y.client + m * e.y.row + n] = (T)w[0];
}
template <typename T>
__device__ __forceinline__ void finish(const StoreEpilogue &e, int c, int m, int n, float v) {
    ((T *)e.c.p)[c * e.c.client + m * e.c.row + n] = (T)v;
}

// 16 x 16 values a workgroup, one a thread.
template <typename T, class E>
__global__ __launch_bounds__(256) void k_product(Operand a, Operand b, int M, int N, int K, E e) {
    __shared__ float sa[16][17], sb[16][17];
    const int tn = (N + 15) / 16, tm = (M + 15) / 16;
    const int c = blockIdx.x / (tn * tm), t = blockIdx.x % (tn * tm), m0 = t / tn * 16, n0 = t % tn * 16;
    const int i = threadIdx.x / 16, j = threadIdx.x % 16;
    float acc = 0;
    for (int k0 = 0; k0 < K; k0 += 16) {
        sa[i][j] = m0 + i < M && k0 + j < K ? (float)((const T *)a.p)[c * a.client + (m0 + i) * a.row + (k0 + j) * a.k] : 0.0f;
        sb[i][j] = n0 + i < N && k0 + j < K ? (float)((const T *)b.p)[c * b.client + (n0 + i) * b.row + (k0 + j) * b.k] : 0.0f;
        __syncthreads();
        for (int k = 0; k < 16; ++k) acc += sa[i][k] * sb[j][k];
        __syncthreads();
    }
    if (m0 + i < M && n0 + j < N) finish<T>(e, c, m0 + i, n0 + j, acc);
}

template <typename T, class E>
static void product(const Operand &a, const Operand &b, int n, int M, int N, int K, const E &e, hipStream_t s) {
    const int64_t blocks = n * ceil_div(M, 16) * ceil_div(N, 16);
    if (blocks) k_product<T><<<(int)blocks, 256, 0, s>>>(a, b, M, N, K, e);
}

size_t linear_forward_workspace(const aet_linear &) { return 0; }
hipError_t launch_linear_forward(const aet_linear &a, void *, hipStream_t s) {
    const Operand x = {a.x.p, a.x.client, a.x.row, 1}, w = {a.w.p, a.w.client, a.w.row, 1};
    const ForwardEpilogue e = {a.bias, a.residual, a.y, a.pre, a.rows, a.act, make_drop(a.p, a.seed, a.first_row, a.out)};
    a.dtype == AET_F32 ? product<float>(x, w, a.n, a.rows, a.out, a.in, e, s) : product<bf16>(x, w, a.n, a.rows, a.out, a.in, e, s);
    return hipGetLastError();
}

// dz, and db: a thread per column.
template <typename T>
__global__ __launch_bounds__(256) void k_dz(aet_linear_grad a, Drop d, T *dz) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)a.n * a.out) return;
    const int64_t c = i / a.out;
    const int col = (int)(i - c * a.out);
    float sum = 0;
    for (int r = 0; r < a.rows; ++r) {
        float v[1] = {(float)((const T *)a.dy.p)[c * a.dy.client + r * a.dy.row + col]};
        if (d.least) drop_apply(d, drop_row(d, c * a.rows + r), col, v);
        if (a.act) v[0] *= slope_any(a.act, (float)((const T *)a.pre.p)[c * a.pre.client + r * a.pre.row + col]);
        sum += v[0];
        dz[(c * a.rows + r) * a.out + col] = (T)v[0];
    }
    if (a.db.p) ((T *)a.db.p)[c * a.db.client + col] = (T)sum;
}

size_t linear_backward_workspace(const aet_linear_grad &a) {
    return (size_t)a.n * a.rows * a.out * (a.dtype == AET_F32 ? 4 : 2);
}
template <typename T>
static void backward(const aet_linear_grad &a, T *dz, hipStream_t s) {
    const int64_t columns = (int64_t)a.n * a.out;
    if (columns) k_dz<T><<<(int)ceil_div(columns, 256), 256, 0, s>>>(a, make_drop(a.p, a.seed, a.first_row, a.out), dz);
    const int64_t client = (int64_t)a.rows * a.out;
    if (a.dx.p) product<T>({dz, client, a.out, 1}, {a.w.p, a.w.client, 1, a.w.row}, a.n, a.rows, a.in, a.out, StoreEpilogue{a.dx}, s);
    if (a.dw.p) product<T>({dz, client, 1, a.out}, {a.x.p, a.x.client, 1, a.x.row}, a.n, a.out, a.in, a.rows, StoreEpilogue{a.dw}, s);
}
hipError_t launch_linear_backward(const aet_linear_grad &a, void *workspace, hipStream_t s) {
    a.dtype == AET_F32 ? backward<float>(a, (float *)workspace, s) : backward<bf16>(a, (bf16 *)workspace, s);
    return hipGetLastError();
}

}  // namespace aet_ops
