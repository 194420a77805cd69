// The linear layer with bias, activation, dropout and residual in its epilogue, and its gradient.
#include <type_traits>

#include "ops_internal.h"
#include "ops_tiles.h"

namespace aet_ops {

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

static Product forward_product(const aet_linear &a) {
    Product p = {};
    p.a = {a.x.p, a.x.client, a.x.row};
    p.b = {a.w.p, a.w.client, a.w.row};
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

// dz = dropout'(dy) * act'(z), and its sums over rows.  A workgroup has 32 pieces of 16 bytes of a strip of a client's rows,
// eight rows at a time, and four times that on the way; the sums of several strips go to `partial` and are added by k_db,
// in their order.  Bound by memory: 4 x 4096 rows of 8192 in bf16, two
// values read and two written, 199 us, 5.4 TB/s.  Inside the products it would be worked out again for each column of
// tiles, and for the second product.
// bf16: dz is kept as the nearest bf16 value and the nearest to what that leaves, 16 bits, for two products of the matrix
// unit each.  One value alone adds an error of the size of the outputs' own rounding to them (relative 2-norm of dx and dw 1.4 times
// as large); a second leaves 2^-8 of that, which no output shows.
struct DzShape {
    int across, strips, strip;   // workgroups: side by side, one below the other; rows of a strip
    int64_t dz_row, low;         // low: bf16, where the second parts begin
    float *partial;              // [strip][client][out]
};

template <typename T, int ACT, bool DROP>
__global__ __launch_bounds__(256) void k_dz(aet_linear_grad a, Drop d, DzShape s, T *dz) {
    constexpr int V = 16 / sizeof(T);
    __shared__ float lds[8][32 * V];
    const int per = s.across * s.strips;
    const int64_t client = blockIdx.x / per;
    const int b = blockIdx.x % per, strip = b / s.across, tx = threadIdx.x % 32, ty = threadIdx.x / 32;
    // A row's last piece is moved back to end with it and shares columns with the one before, whose values both work out and
    // store: nobody has to look where pieces end (57 rows of 50 for 19 clients in bf16: 24 us with the look, 7 without).  Only what is a
    // thread's own, from `own` on, is counted.  Rows of less than a piece have `rest`.
    const int place = (b % s.across * 32 + tx) * V, col = place + V <= a.out ? place : a.out > V ? a.out - V : 0, own = place - col;
    const int rest = a.out < V ? a.out : V;
    const bool ends = sizeof(T) == 2 && place < a.out && place + V > a.out;
    const int64_t first = (int64_t)strip * s.strip, end = first + s.strip < a.rows ? first + s.strip : a.rows;
    const T *dy = (const T *)a.dy.p + client * a.dy.client + col;
    const T *pre = (const T *)a.pre.p + client * a.pre.client + col;
    float sum[V] = {};
    const auto one = [&](int64_t r, const wide<T, V> &rd, const wide<T, V> &rz, int count) {
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = (float)rd[e];
        if (ACT) {
            float z[V];
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] = (float)rz[e];
            slope_each<ACT>(z, v);
        }
        // last, so that what the forward pass took out has a gradient of 0 whatever z was
        if (DROP) {
            const uint64_t q = drop_row(d, client * a.rows + r);
            if (a.out & 1) drop_apply_any(d, q, col, v);
            else drop_apply(d, q, col, v);
        }
        if (dz) {
            T *const to = dz + (client * a.rows + r) * s.dz_row;
            if (ends) *(wide<T, V> *)(to + s.dz_row - V) = wide<T, V>{};   // zeros up to the next row, for the products
            if constexpr (sizeof(T) == 2) {
                float high[V], low[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    high[e] = (float)(T)v[e];
                    // what would round to infinity has the largest value; infinities and NaN are in the first part alone
                    const bool finite = __builtin_fabsf(v[e]) <= __FLT_MAX__;
                    if (finite && __builtin_fabsf(high[e]) > __FLT_MAX__) high[e] = __builtin_copysignf(0x1.fep127f, v[e]);
                    low[e] = finite ? v[e] - high[e] : 0.0f;
                }
                if (ends) *(wide<T, V> *)(to + s.low + s.dz_row - V) = wide<T, V>{};
                store_some(to + col, count, high);
                store_some(to + s.low + col, count, low);
            } else {
                store_some(to + col, count, v);
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += v[e];
    };
    // N rows at a time
    const auto rows = [&](auto n, int count) {
        constexpr int N = n;
#pragma unroll 1
        for (int64_t r0 = first + ty; r0 < end; r0 += 8 * N) {
            wide<T, V> rd[N], rz[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int64_t r = r0 + 8 * i < end ? r0 + 8 * i : end - 1;
                rd[i] = load_raw<T, V>(dy + r * a.dy.row, count);
                if (ACT) rz[i] = load_raw<T, V>(pre + r * a.pre.row, count);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int64_t r = r0 + 8 * i;
                if (r < end) one(r, rd[i], rz[i], count);
            }
        }
    };
    if (rest < V) {
        if (place == 0) rows(std::integral_constant<int, 1>(), rest);
    } else if (own < V) {
        rows(std::integral_constant<int, 4>(), V);
    }
    if (!a.db.p) return;
    if (own < V) {   // (own is 0 or more; V and more: no piece)
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e >= own) lds[ty][tx * V + e - own] = sum[e];
    }
    __syncthreads();
    const int mine = b % s.across * (32 * V) + threadIdx.x;
    if (threadIdx.x >= 32 * V || mine >= a.out) return;
    float total = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) total += lds[i][threadIdx.x];
    if (s.strips == 1) ((T *)a.db.p)[client * a.db.client + mine] = (T)total;
    else s.partial[((int64_t)strip * a.n + client) * a.out + mine] = total;
}

template <typename T>
__global__ __launch_bounds__(256) void k_db(aet_linear_grad a, DzShape s) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (int64_t)a.n * a.out;
    if (i >= all) return;
    float total = 0;
#pragma unroll 8
    for (int k = 0; k < s.strips; ++k) total += s.partial[k * all + i];
    ((T *)a.db.p)[i / a.out * a.db.client + i % a.out] = (T)total;
}

// dz has a place of its own unless it is dy.
struct BackwardPlan {
    DzShape dz;
    Product dx, dw;
    size_t dz_bytes, db_bytes, bytes;
};
static BackwardPlan plan(const aet_linear_grad &a, char *workspace) {
    BackwardPlan b = {};
    const bool own = (a.p > 0 || a.act != AET_ACT_NONE) && (a.dx.p || a.dw.p);
    const int e = a.dtype == AET_F32 ? 4 : 2;
    b.dz.dz_row = ceil_div((int64_t)a.out * e, 16) * 16 / e;
    b.dz.across = (int)ceil_div(a.out, 32 * 16 / e);
    // strips of at least 64 rows, as many as give every compute unit several workgroups; up to 128 rows one, which takes no
    // longer than the launch that adds several
    const int64_t wanted = ceil_div(2048, (int64_t)a.n * b.dz.across + 1), most = a.rows <= 128 ? 1 : ceil_div(a.rows, 64);
    b.dz.strip = (int)ceil_div(ceil_div(a.rows, wanted < most ? wanted : most > 0 ? most : 1), 8) * 8;
    b.dz.strips = a.rows ? (int)ceil_div(a.rows, b.dz.strip) : 1;
    const size_t part = own ? up256((size_t)a.n * a.rows * b.dz.dz_row * e) : 0;
    b.dz.low = e == 2 ? (int64_t)(part / e) : 0;
    b.dz_bytes = part * (e == 2 ? 2 : 1);
    b.db_bytes = a.db.p && b.dz.strips > 1 ? up256((size_t)b.dz.strips * a.n * a.out * sizeof(float)) : 0;
    b.dz.partial = (float *)(workspace + b.dz_bytes);
    Operand dz = {a.dy.p, a.dy.client, a.dy.row};
    if (own) dz = {workspace, a.rows * b.dz.dz_row, b.dz.dz_row, false, true, b.dz.low};
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
    b.bytes = b.dz_bytes + b.db_bytes + (x > w ? x : w);
    return b;
}

size_t linear_backward_workspace(const aet_linear_grad &a) { return plan(a, nullptr).bytes; }

template <typename T>
static hipError_t backward(const aet_linear_grad &a, char *workspace, hipStream_t s) {
    const BackwardPlan b = plan(a, workspace);
    char *const more = workspace + b.dz_bytes + b.db_bytes;
    hipError_t e = hipSuccess;
    if (a.out && (b.dz_bytes || a.db.p)) {
        const int64_t blocks = (int64_t)a.n * b.dz.across * b.dz.strips;
        if (!grid_fits(blocks, 256) || (a.db.p && b.dz.strips > 1 && !grid_fits(ceil_div((int64_t)a.n * a.out, 256), 256))) return hipErrorInvalidConfiguration;
        const Drop d = make_drop(a.p, a.seed, a.first_row, a.out);
        const auto dz = [&](auto act) {
            const auto kernel = d.least ? k_dz<T, act, true> : k_dz<T, act, false>;
            kernel<<<(int)blocks, 256, 0, s>>>(a, d, b.dz, b.dz_bytes ? (T *)workspace : nullptr);
        };
        switch (a.act) {
        case AET_ACT_RELU: dz(std::integral_constant<int, AET_ACT_RELU>()); break;
        case AET_ACT_SILU: dz(std::integral_constant<int, AET_ACT_SILU>()); break;
        case AET_ACT_GELU: dz(std::integral_constant<int, AET_ACT_GELU>()); break;
        default: dz(std::integral_constant<int, AET_ACT_NONE>());
        }
        if (a.db.p && b.dz.strips > 1) k_db<T><<<(int)ceil_div((int64_t)a.n * a.out, 256), 256, 0, s>>>(a, b.dz);
        e = hipGetLastError();
    }
    bool both = false;
    if (e == hipSuccess && a.dx.p && a.dw.p) e = launch_pair(a.dtype, b.dx, b.dw, s, &both);
    if (both) return e;
    if (e == hipSuccess && a.dx.p) e = launch_product(a.dtype, b.dx, more, s);
    if (e == hipSuccess && a.dw.p) e = launch_product(a.dtype, b.dw, more, s);
    return e;
}
hipError_t launch_linear_backward(const aet_linear_grad &a, void *workspace, hipStream_t s) {
    return a.dtype == AET_F32 ? backward<float>(a, (char *)workspace, s) : backward<bf16>(a, (char *)workspace, s);
}

}  // namespace aet_ops
