// Layer normalisation of rows, the residual stream joined in, and its gradient.
//
// Bound by memory.  A row lies in the registers of 4, 16 or 64 lanes of a wave, or of 4 to 16 waves, in pieces of 16 bytes;
// it is read once: mean first, then the squares of the differences from it.  Rows too long for that (16384 values in fp32, 32768
// in bf16; half as many in a gradient with sums by column) are read again for each pass (k_ln_long).
//   16384 rows of 4096 in bf16: 46 us (5.8 TB/s), with the residual and h 97 (5.5); gradient with dh joined in 123 (4.4; without sums
//   over rows 107: the rest are the sums of 512 strips, written and read).  A row of 784 in fp32: 6.1 us, the call.
#include "ops_internal.h"

#include <type_traits>

namespace aet_ops {

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Piece p of a row: values col .. col + V - 1, of which [lo, hi) are the thread's own.  A row's last piece is moved back to
// end with the row, so that nobody has to look where pieces end; rows of less than a piece have hi values.
template <int V>
struct Piece {
    int col, lo, hi;
    __device__ __forceinline__ Piece(int p, int cols) {
        const int place = p * V;
        col = place + V <= cols ? place : cols > V ? cols - V : 0;
        lo = place < cols ? place - col : 0;
        hi = place < cols ? (cols < V ? cols : V) : 0;
    }
    // ODD: some pieces are not whole
    template <bool ODD>
    __device__ __forceinline__ bool has(int e) const { return ODD ? e >= lo && e < hi : hi > 0; }
};
template <typename T, int V, bool ODD>
__device__ __forceinline__ wide<T, V> load_piece(const T *row, const Piece<V> &p, int cols) {
    if (ODD && cols < V) return load_raw<T, V>(row, p.hi);
    return *(const wide<T, V> *)(row + p.col);
}
template <typename T, int V, bool ODD>
__device__ __forceinline__ void store_piece(T *row, const Piece<V> &p, int cols, const float (&v)[V]) {
    if (p.hi == 0) return;
    store_some<T, V>(row + p.col, ODD && cols < V ? p.hi : V, v);
}

// Sums of N values over the lanes and waves that share a row.  lds: N * WAVES floats that nobody reads any more.
template <int L, int WAVES, int N, typename S>
__device__ __forceinline__ void row_sums(S (&v)[N], S *lds) {
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] += __shfl_xor(v[n], off, 64);
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x / 64;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) lds[n * WAVES + wave] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            S sum = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += lds[n * WAVES + w];
            v[n] = sum;
        }
    }
}

constexpr int threads_of(int waves) { return waves > 4 ? 64 * waves : 256; }

template <typename T, int L, int WAVES, int NP, bool ODD>
__global__ __launch_bounds__(threads_of(WAVES)) void k_ln(aet_layer_norm a, float inv) {
    constexpr int V = 16 / sizeof(T), THREADS = threads_of(WAVES), G = L * WAVES, R = THREADS / G;
    __shared__ float lds[2][WAVES];
    const int64_t at = (int64_t)blockIdx.x * R + threadIdx.x / G;
    const int64_t client = at / a.rows, row = at - client * a.rows;
    const int t = threadIdx.x % G;
    if (client >= a.n) return;   // (whole rows: WAVES > 1 has one a workgroup)
    const T *x = (const T *)a.x.p + client * a.x.client + row * a.x.row;
    const T *res = a.residual.p ? (const T *)a.residual.p + client * a.residual.client + row * a.residual.row : nullptr;
    wide<T, V> rx[NP], rr[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) rx[i] = load_piece<T, V, ODD>(x, Piece<V>(t + i * G, a.cols), a.cols);
    if (res)
#pragma unroll
        for (int i = 0; i < NP; ++i) rr[i] = load_piece<T, V, ODD>(res, Piece<V>(t + i * G, a.cols), a.cols);
    float v[NP][V], s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const Piece<V> p(t + i * G, a.cols);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            v[i][e] = (float)rx[i][e];
            if (res) v[i][e] += (float)rr[i][e];
            s[0] += p.template has<ODD>(e) ? v[i][e] : 0.0f;
        }
    }
    row_sums<L, WAVES, 1>(s, lds[0]);
    const float mean = s[0] * inv;
    s[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const Piece<V> p(t + i * G, a.cols);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = p.template has<ODD>(e) ? v[i][e] - mean : 0.0f;
            s[0] = __builtin_fmaf(d, d, s[0]);
        }
    }
    row_sums<L, WAVES, 1>(s, lds[1]);
    const float rstd = 1.0f / __builtin_sqrtf(s[0] * inv + a.eps);
    if (t == 0) {
        if (a.mean) a.mean[at] = mean;
        if (a.rstd) a.rstd[at] = rstd;
    }
    // Everything of the row has been read: y and h may be x or the residual.
    T *y = (T *)a.y.p + client * a.y.client + row * a.y.row;
    T *h = a.h.p ? (T *)a.h.p + client * a.h.client + row * a.h.row : nullptr;
    const T *gamma = a.gamma.p ? (const T *)a.gamma.p + client * a.gamma.client : nullptr;
    const T *beta = a.beta.p ? (const T *)a.beta.p + client * a.beta.client : nullptr;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const Piece<V> p(t + i * G, a.cols);
        if (h) store_piece<T, V, ODD>(h, p, a.cols, v[i]);
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = (v[i][e] - mean) * rstd;
        if (gamma) {
            const wide<T, V> g = load_piece<T, V, ODD>(gamma, p, a.cols);
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] *= (float)g[e];
        }
        if (beta) {
            const wide<T, V> b = load_piece<T, V, ODD>(beta, p, a.cols);
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] += (float)b[e];
        }
        store_piece<T, V, ODD>(y, p, a.cols, o);
    }
}

// Rows of any length, read once for each sum and once more.  Their sums are in 64 bits.
constexpr int kLong = 1024;
template <typename T>
__global__ __launch_bounds__(kLong) void k_ln_long(aet_layer_norm a, double inv) {
    constexpr int V = 16 / sizeof(T);
    __shared__ double lds[2][kLong / 64];
    const int64_t at = blockIdx.x, client = at / a.rows, row = at - client * a.rows;
    const T *x = (const T *)a.x.p + client * a.x.client + row * a.x.row;
    const T *res = a.residual.p ? (const T *)a.residual.p + client * a.residual.client + row * a.residual.row : nullptr;
    const auto read = [&](int64_t col, float (&v)[V]) {
        load_some(x + col, (int)(a.cols - col < V ? a.cols - col : V), v);
        if (res) {
            float r[V];
            load_some(res + col, (int)(a.cols - col < V ? a.cols - col : V), r);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] += r[e];
        }
    };
    double s[1] = {0};
    for (int64_t col = threadIdx.x * V; col < a.cols; col += kLong * V) {
        float v[V], part = 0;
        read(col, v);
#pragma unroll
        for (int e = 0; e < V; ++e) part += v[e];   // (0 past the end)
        s[0] += part;
    }
    row_sums<64, kLong / 64, 1>(s, lds[0]);
    const float mean = (float)(s[0] * inv);
    s[0] = 0;
    for (int64_t col = threadIdx.x * V; col < a.cols; col += kLong * V) {
        float v[V], part = 0;
        read(col, v);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = col + e < a.cols ? v[e] - mean : 0.0f;
            part = __builtin_fmaf(d, d, part);
        }
        s[0] += part;
    }
    row_sums<64, kLong / 64, 1>(s, lds[1]);
    const float rstd = 1.0f / __builtin_sqrtf((float)(s[0] * inv) + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[at] = mean;
        if (a.rstd) a.rstd[at] = rstd;
    }
    T *y = (T *)a.y.p + client * a.y.client + row * a.y.row;
    T *h = a.h.p ? (T *)a.h.p + client * a.h.client + row * a.h.row : nullptr;
    for (int64_t col = threadIdx.x * V; col < a.cols; col += kLong * V) {
        const int count = (int)(a.cols - col < V ? a.cols - col : V);
        float v[V], o[V], g[V];
        read(col, v);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = (v[e] - mean) * rstd;
        if (a.gamma.p) {
            load_some((const T *)a.gamma.p + client * a.gamma.client + col, count, g);
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] *= g[e];
        }
        if (a.beta.p) {
            load_some((const T *)a.beta.p + client * a.beta.client + col, count, g);
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] += g[e];
        }
        if (h) store_some(h + col, count, v);
        store_some(y + col, count, o);
    }
}

// Calls f(L, WAVES, NP) for the smallest group that holds a row of so many pieces; false: none does.  (Sixteen waves have too few
// registers for sums by column.)
template <bool SUMS, class F>
static bool for_width(int64_t pieces, F f) {
#define AET_WIDTH(L, W, NP) \
    if (pieces <= (L) * (W) * (NP)) return f(std::integral_constant<int, L>(), std::integral_constant<int, W>(), std::integral_constant<int, NP>()), true
    AET_WIDTH(4, 1, 1);
    AET_WIDTH(16, 1, 1);
    AET_WIDTH(64, 1, 1);
    AET_WIDTH(64, 1, 2);
    AET_WIDTH(64, 4, 1);
    AET_WIDTH(64, 4, 2);
    AET_WIDTH(64, 4, 4);
    AET_WIDTH(64, 8, 4);
    if constexpr (!SUMS) AET_WIDTH(64, 16, 4);
#undef AET_WIDTH
    return false;
}

template <typename T>
static hipError_t forward(const aet_layer_norm &a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const int64_t rows = (int64_t)a.n * a.rows;
    const float inv = a.cols ? (float)(1.0 / a.cols) : 0.0f;
    hipError_t e = hipSuccess;
    const bool held = a.cols > 0 && for_width<false>(ceil_div(a.cols, V), [&](auto L, auto W, auto NP) {
        constexpr int threads = threads_of(W), R = threads / (L * W);
        const int64_t blocks = ceil_div(rows, R);
        if (!grid_fits(blocks, threads)) {
            e = hipErrorInvalidConfiguration;
            return;
        }
        const auto kernel = a.cols % V ? k_ln<T, L, W, NP, true> : k_ln<T, L, W, NP, false>;
        kernel<<<(int)blocks, threads, 0, s>>>(a, inv);
    });
    if (!held) {
        if (!grid_fits(rows, kLong)) return hipErrorInvalidConfiguration;
        k_ln_long<T><<<(int)rows, kLong, 0, s>>>(a, a.cols ? 1.0 / a.cols : 0.0);
    }
    return e != hipSuccess ? e : hipGetLastError();
}
hipError_t launch_layer_norm_forward(const aet_layer_norm &a, hipStream_t s) {
    return a.dtype == AET_F32 ? forward<float>(a, s) : forward<bf16>(a, s);
}

// ---- the gradient ------------------------------------------------------------------------

// xh = (x - mean) rstd, e = dy gamma:  dx = rstd (e - mean of e - xh mean of (e xh)) + dh.  The sums of dy xh and dy
// over rows are kept by column by the threads that have the column in a strip of rows, and go to `partial`, which
// k_ln_join adds in the strips' order.
struct StripShape {
    int strips, strip;      // of a client; rows of one
    int line;               // floats between the lines of partial
    float *partial;         // [client][strip][dgamma, dbeta][line]
    bool direct;            // one strip: straight to dgamma and dbeta
};

template <typename T>
__device__ __forceinline__ void put_sum(const aet_layer_norm_grad &a, const StripShape &s, int64_t client, int strip, int col, float dgamma, float dbeta) {
    if (s.direct) {
        if (a.dgamma.p) ((T *)a.dgamma.p)[client * a.dgamma.client + col] = (T)dgamma;
        if (a.dbeta.p) ((T *)a.dbeta.p)[client * a.dbeta.client + col] = (T)dbeta;
    } else {
        float *const to = s.partial + (client * s.strips + strip) * 2 * s.line + col;
        to[0] = dgamma;
        to[s.line] = dbeta;
    }
}

template <typename T, int L, int WAVES, int NP, bool ODD, bool PARAMS>
__global__ __launch_bounds__(threads_of(WAVES)) void k_ln_back(aet_layer_norm_grad a, StripShape s, float inv) {
    constexpr int V = 16 / sizeof(T), THREADS = threads_of(WAVES), G = L * WAVES, R = THREADS / G;
    __shared__ float lds[2][2 * WAVES];
    __shared__ float sums[PARAMS && R > 1 ? 2 * THREADS * V : 1];
    const int64_t client = blockIdx.x / s.strips;
    const int strip = blockIdx.x % s.strips, t = threadIdx.x % G, group = threadIdx.x / G;
    const int64_t first = (int64_t)strip * s.strip, end = first + s.strip < a.rows ? first + s.strip : a.rows;
    const T *dy = (const T *)a.dy.p + client * a.dy.client, *x = (const T *)a.x.p + client * a.x.client;
    const T *dh = a.dh.p ? (const T *)a.dh.p + client * a.dh.client : nullptr;
    float dg[PARAMS ? NP : 1][V] = {}, db[PARAMS ? NP : 1][V] = {};
    wide<T, V> gamma[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        if (a.gamma.p) gamma[i] = load_piece<T, V, ODD>((const T *)a.gamma.p + client * a.gamma.client, Piece<V>(t + i * G, a.cols), a.cols);
        else
#pragma unroll
            for (int e = 0; e < V; ++e) gamma[i][e] = (T)1.0f;
    }
    struct Row {
        wide<T, V> d[NP], x[NP], h[NP];
        float mean, rstd;
        int64_t at;
        bool in;
    };
    // the group's row of the turn from r0 on (its last one again behind the end)
    const auto load = [&](Row &row, int64_t r0) {
        row.in = r0 + group < end;
        row.at = row.in ? r0 + group : end - 1;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const Piece<V> p(t + i * G, a.cols);
            row.d[i] = load_piece<T, V, ODD>(dy + row.at * a.dy.row, p, a.cols);
            row.x[i] = load_piece<T, V, ODD>(x + row.at * a.x.row, p, a.cols);
            if (dh) row.h[i] = load_piece<T, V, ODD>(dh + row.at * a.dh.row, p, a.cols);
        }
        row.mean = a.mean[client * a.rows + row.at];
        row.rstd = a.rstd[client * a.rows + row.at];
    };
    int turn = 0;
    const auto work = [&](Row &row) {
        float v[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const Piece<V> p(t + i * G, a.cols);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool own = p.template has<ODD>(e);
                const float d = own ? (float)row.d[i][e] : 0.0f, xh = own ? ((float)row.x[i][e] - row.mean) * row.rstd : 0.0f, g = d * (float)gamma[i][e];
                v[0] += own ? g : 0.0f;
                v[1] = __builtin_fmaf(own ? g : 0.0f, xh, v[1]);
                if (PARAMS && row.in) {
                    dg[i][e] = __builtin_fmaf(d, xh, dg[i][e]);
                    db[i][e] += d;
                }
            }
        }
        if (!a.dx.p) return;
        // dx may be dh, and a row's last two pieces share columns: what is loaded of dh has arrived before anybody stores
        if (dh)
#pragma unroll
            for (int i = 0; i < NP; ++i) asm volatile("" ::"v"(row.h[i]));
        row_sums<L, WAVES, 2>(v, lds[turn]);
        turn ^= 1;
        if (NP > 2)   // kept as they were read, not as fp32
#pragma unroll
            for (int i = 0; i < NP; ++i) asm volatile("" : "+v"(row.d[i]), "+v"(row.x[i]));
        const float m1 = v[0] * inv, m2 = v[1] * inv;
        T *dx = (T *)a.dx.p + client * a.dx.client + row.at * a.dx.row;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const Piece<V> p(t + i * G, a.cols);
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xh = ((float)row.x[i][e] - row.mean) * row.rstd;
                o[e] = ((float)row.d[i][e] * (float)gamma[i][e] - m1 - xh * m2) * row.rstd;
                if (dh) o[e] += (float)row.h[i][e];
            }
            if (row.in) store_piece<T, V, ODD>(dx, p, a.cols, o);
        }
    };
    // The next turn's rows are on their way while this one's are worked on, where the registers hold them (all groups of a workgroup
    // have as many turns).  dx may be dy or dh: a row is stored only where it is read, in its own turn.
    Row row[2];
    if constexpr (WAVES > 4) {
        for (int64_t r0 = first; r0 < end; r0 += R) {
            load(row[0], r0);
            work(row[0]);
        }
    } else {
        load(row[0], first);
        int64_t r0 = first;
        for (; r0 + 2 * R < end; r0 += 2 * R) {
            load(row[1], r0 + R);
            work(row[0]);
            load(row[0], r0 + 2 * R);
            work(row[1]);
        }
        if (r0 + R < end) load(row[1], r0 + R);
        work(row[0]);
        if (r0 + R < end) work(row[1]);
    }
    if constexpr (PARAMS) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const Piece<V> p(t + i * G, a.cols);
            if constexpr (R > 1) {
                if (i) __syncthreads();
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    sums[threadIdx.x * V + e] = dg[i][e];
                    sums[(THREADS + threadIdx.x) * V + e] = db[i][e];
                }
                __syncthreads();
                if (group == 0)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float g = 0, b = 0;
                        for (int k = 0; k < R; ++k) {
                            g += sums[(k * G + t) * V + e];
                            b += sums[(THREADS + k * G + t) * V + e];
                        }
                        if (p.template has<ODD>(e)) put_sum<T>(a, s, client, strip, p.col + e, g, b);
                    }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (p.template has<ODD>(e)) put_sum<T>(a, s, client, strip, p.col + e, dg[i][e], db[i][e]);
            }
        }
    }
}

// Rows of any length: dx row by row, and the sums column by column.
template <typename T>
__global__ __launch_bounds__(kLong) void k_ln_back_long(aet_layer_norm_grad a, double inv) {
    constexpr int V = 16 / sizeof(T);
    __shared__ double lds[2 * kLong / 64];
    const int64_t at = blockIdx.x, client = at / a.rows, row = at - client * a.rows;
    const T *dy = (const T *)a.dy.p + client * a.dy.client + row * a.dy.row, *x = (const T *)a.x.p + client * a.x.client + row * a.x.row;
    const float mean = a.mean[at], rstd = a.rstd[at];
    const auto read = [&](int64_t col, int count, float (&e)[V], float (&xh)[V]) {
        float g[V];
        load_some(dy + col, count, e);
        load_some(x + col, count, xh);
        if (a.gamma.p) {
            load_some((const T *)a.gamma.p + client * a.gamma.client + col, count, g);
#pragma unroll
            for (int i = 0; i < V; ++i) e[i] *= g[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) xh[i] = (xh[i] - mean) * rstd;
    };
    double v[2] = {0, 0};
    for (int64_t col = threadIdx.x * V; col < a.cols; col += kLong * V) {
        const int count = (int)(a.cols - col < V ? a.cols - col : V);
        float e[V], xh[V], s1 = 0, s2 = 0;
        read(col, count, e, xh);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s1 += i < count ? e[i] : 0.0f;
            s2 = __builtin_fmaf(i < count ? e[i] : 0.0f, i < count ? xh[i] : 0.0f, s2);
        }
        v[0] += s1;
        v[1] += s2;
    }
    row_sums<64, kLong / 64, 2>(v, lds);
    const float m1 = (float)(v[0] * inv), m2 = (float)(v[1] * inv);
    T *dx = (T *)a.dx.p + client * a.dx.client + row * a.dx.row;
    for (int64_t col = threadIdx.x * V; col < a.cols; col += kLong * V) {
        const int count = (int)(a.cols - col < V ? a.cols - col : V);
        float e[V], xh[V], h[V] = {};
        read(col, count, e, xh);
        if (a.dh.p) load_some((const T *)a.dh.p + client * a.dh.client + row * a.dh.row + col, count, h);
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = (e[i] - m1 - xh[i] * m2) * rstd + h[i];
        store_some(dx + col, count, e);
    }
}
template <typename T>
__global__ __launch_bounds__(256) void k_ln_params_long(aet_layer_norm_grad a, StripShape s, int across) {
    constexpr int V = 16 / sizeof(T);
    const int64_t block = blockIdx.x, client = block / ((int64_t)across * s.strips);
    const int in = (int)(block - client * across * s.strips), strip = in / across;
    const int64_t col = ((int64_t)(in % across) * 256 + threadIdx.x) * V;
    if (col >= a.cols) return;
    const int count = (int)(a.cols - col < V ? a.cols - col : V);
    const int64_t first = (int64_t)strip * s.strip, end = first + s.strip < a.rows ? first + s.strip : a.rows;
    float dg[V] = {}, db[V] = {};
    for (int64_t row = first; row < end; ++row) {
        const float mean = a.mean[client * a.rows + row], rstd = a.rstd[client * a.rows + row];
        float d[V], x[V];
        load_some((const T *)a.dy.p + client * a.dy.client + row * a.dy.row + col, count, d);
        load_some((const T *)a.x.p + client * a.x.client + row * a.x.row + col, count, x);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            dg[e] = __builtin_fmaf(d[e], (x[e] - mean) * rstd, dg[e]);
            db[e] += d[e];
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e < count) put_sum<T>(a, s, client, strip, (int)col + e, dg[e], db[e]);
}

// Adds the strips' sums: 32 runs of them side by side, in their order, then the runs by twos.  A workgroup has 32 columns.
template <typename T>
__global__ __launch_bounds__(256) void k_ln_join(aet_layer_norm_grad a, StripShape s, int64_t count, int across) {
    __shared__ f4 lds[32][8];
    const int which = blockIdx.x % 2;
    const int64_t client = blockIdx.x / 2 / across;
    const int piece = blockIdx.x / 2 % across * 8 + threadIdx.x % 8, run = threadIdx.x / 8;
    const int64_t each = (count + 31) / 32, first = run * each, end = first + each < count ? first + each : count;
    const aet_out &out = which ? a.dbeta : a.dgamma;
    f4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (out.p && piece * 4 < s.line) {
        const float *from = s.partial + client * count * 2 * s.line + which * s.line + piece * 4;
#pragma unroll 4
        for (int64_t k = first; k < end; ++k) sum += *(const f4 *)(from + k * 2 * s.line);
    }
    lds[run][threadIdx.x % 8] = sum;
    __syncthreads();
    const int col = blockIdx.x / 2 % across * 32 + threadIdx.x;
    if (threadIdx.x >= 32 || !out.p || col >= a.cols) return;
    float total[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) total[k] = lds[k][threadIdx.x / 4][threadIdx.x % 4];
#pragma unroll
    for (int off = 16; off > 0; off /= 2)
#pragma unroll
        for (int k = 0; k < off; ++k) total[k] += total[k + off];
    ((T *)out.p)[client * out.client + col] = (T)total[0];
}

// Parameters' gradients over nothing.
template <typename T>
__global__ __launch_bounds__(256) void k_ln_none(aet_layer_norm_grad a, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, client = i / a.cols, col = i - client * a.cols;
    if (client >= n) return;
    if (a.dgamma.p) ((T *)a.dgamma.p)[client * a.dgamma.client + col] = (T)0.0f;
    if (a.dbeta.p) ((T *)a.dbeta.p)[client * a.dbeta.client + col] = (T)0.0f;
}

static bool shared_of(const aet_layer_norm_grad &a) { return a.n != 1 && ((a.dgamma.p && !a.dgamma.client) || (a.dbeta.p && !a.dbeta.client)); }
// Strips: as many workgroups as the compute units hold (what a group of four waves with a piece a lane leaves room for is four a unit, with
// two pieces two, else one), since every strip's sums are written and read again; each with four or more turns where there are
// rows enough.  16384 rows of 4096 in bf16, dh joined in: 512 strips 123 us, 1024 133, 256 138.
static StripShape strips_of(const aet_layer_norm_grad &a, void *workspace) {
    const int V = a.dtype == AET_F32 ? 4 : 8;
    int at_once = 1, all = 512;
    const bool params = a.dgamma.p || a.dbeta.p;
    const auto group = [&](auto L, auto W, auto NP) {
        at_once = threads_of(W) / (L * W);
        all = NP == 4 ? 256 : W == 4 && NP == 1 ? 1024 : 512;
    };
    const bool held = params ? for_width<true>(ceil_div(a.cols, V), group) : for_width<false>(ceil_div(a.cols, V), group);
    StripShape s = {};
    const int64_t per = held ? a.n : a.n * ceil_div(a.cols, 256 * V);
    const int64_t wanted = ceil_div(all, per > 0 ? per : 1), most = ceil_div(a.rows, 4 * (int64_t)at_once);
    int64_t strips = wanted < most ? wanted : most;
    if (strips * per < 256) strips = wanted < ceil_div(a.rows, at_once) ? wanted : ceil_div(a.rows, at_once);
    s.strip = (int)(ceil_div(ceil_div(a.rows, strips > 0 ? strips : 1), at_once) * at_once);
    s.strips = s.strip ? (int)ceil_div(a.rows, s.strip) : 1;
    s.line = (int)(ceil_div(a.cols, 4) * 4);
    s.partial = (float *)workspace;
    s.direct = s.strips == 1 && !(shared_of(a) && a.n > 1);
    return s;
}
size_t layer_norm_backward_workspace(const aet_layer_norm_grad &a) {
    if (!a.n || !a.rows || !a.cols || !(a.dgamma.p || a.dbeta.p)) return 0;
    const StripShape s = strips_of(a, nullptr);
    return s.direct ? 0 : up256((size_t)a.n * s.strips * 2 * s.line * sizeof(float));
}

template <typename T>
static hipError_t backward(const aet_layer_norm_grad &a, void *workspace, hipStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    const bool params = a.dgamma.p || a.dbeta.p;
    const int64_t sums = shared_of(a) ? 1 : a.n;   // of parameters
    if (!a.cols) return hipSuccess;
    if (!a.n || !a.rows) {
        const int64_t blocks = ceil_div(sums * a.cols, 256);
        if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
        if (params && blocks) k_ln_none<T><<<(int)blocks, 256, 0, stream>>>(a, sums);
        return hipGetLastError();
    }
    if (!params && !a.dx.p) return hipSuccess;
    const StripShape s = strips_of(a, workspace);
    const float inv = (float)(1.0 / a.cols);
    const int64_t blocks = (int64_t)a.n * s.strips;
    hipError_t e = hipSuccess;
    const auto go = [&](auto sums, auto L, auto W, auto NP) {
        if (!grid_fits(blocks, threads_of(W))) {
            e = hipErrorInvalidConfiguration;
            return;
        }
        const auto kernel = a.cols % V ? k_ln_back<T, L, W, NP, true, sums> : k_ln_back<T, L, W, NP, false, sums>;
        kernel<<<(int)blocks, threads_of(W), 0, stream>>>(a, s, inv);
    };
    const bool held = params ? for_width<true>(ceil_div(a.cols, V), [&](auto... g) { go(std::true_type(), g...); })
                             : for_width<false>(ceil_div(a.cols, V), [&](auto... g) { go(std::false_type(), g...); });
    if (!held) {
        const int64_t rows = (int64_t)a.n * a.rows, across = ceil_div(a.cols, 256 * V);
        if ((a.dx.p && !grid_fits(rows, kLong)) || (params && !grid_fits(blocks * across, 256))) return hipErrorInvalidConfiguration;
        // first, while dy has its values (dx may be dy)
        if (params) k_ln_params_long<T><<<(int)(blocks * across), 256, 0, stream>>>(a, s, (int)across);
        if (a.dx.p) k_ln_back_long<T><<<(int)rows, kLong, 0, stream>>>(a, 1.0 / a.cols);
    }
    if (e != hipSuccess) return e;
    if (params && !s.direct) {
        const int64_t across = ceil_div(a.cols, 32), joins = 2 * across * sums;
        if (!grid_fits(joins, 256)) return hipErrorInvalidConfiguration;
        k_ln_join<T><<<(int)joins, 256, 0, stream>>>(a, s, a.n * s.strips / sums, (int)across);
    }
    return hipGetLastError();
}
hipError_t launch_layer_norm_backward(const aet_layer_norm_grad &a, void *workspace, hipStream_t s) {
    return a.dtype == AET_F32 ? backward<float>(a, workspace, s) : backward<bf16>(a, workspace, s);
}

}  // namespace aet_ops
