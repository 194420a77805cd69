// The orthogonalised update: X = G / (|G| + eps), then X <- a X + (b A + c A A) X with A = X X^T, some steps of it, which take
// the singular values s of X to a s + b s^3 + c s^5 and leave the vectors.
//
// Bound by the matrix cores: of a matrix of m x k (m <= k, else its transpose) a step is the products X X^T and A A, of which
// the upper half of the tiles is worked out and stored twice, and B X.  Every matrix is held as a sum of two fp16 values, scaled by a
// power of two that its bound allows (the singular values of X begin at no more than 1 and stay below the polynomial's largest
// value, which is followed from step to step): 22 bits of a value, down to 2^-39 of that bound.  A product is three of the
// matrix unit's, high high + high low + low high.  Relative 2-norm against 64 bits, five steps of 64 x 64 to 512 x 512 matrices:
// 4e-7 to 3e-6 where products in fp32 give 1e-6 to 2e-5; with one fp16 value 1e-3 to 3e-3, with one bf16 value 5e-3 to 2e-2,
// as much as or more than the rounding of a bf16 result (1.7e-3).
//
// Where X is wide and the result bf16, several steps go by the matrices of m x m alone: X X^T once, then with P = a + b A + c A A
// of each step Q <- Q P and A <- (A P) P, all of them polynomials of the first A, which commute and are symmetric; at the end
// X <- Q X.  What A is off by is not corrected there, and grows as the square of what small singular values do, so X is worked out in
// between before that has come to 200: two steps a run with the default polynomial.  Relative 2-norm against 64 bits before the result is
// rounded, five steps of gradients with bf16's noise, of rank 1, of rank 16 to all, and over five decades: 4e-5 to 1e-4, 3e-6 to 4e-5, and 5e-6
// to 8e-6, with products in fp32 6e-5 to 1.7e-4, 1e-6 to 5e-5, and 4e-6 to 7e-6.  (Up to 2e3, three steps a run, it was up to four times that, and with
// other polynomials and more steps up to 50 times what products in fp32 are off by; a run of all five 3e-2.)
//
// All matrices of a call lie in the workspace with zeros up to whole tiles, so that no product has to look where they end.
//
// Five steps, y = keep w + scale X: 4096 x 4096 of fp32 4.2 to 4.5 ms (the matrix unit at 920 to 990 TF/s), 4 x 1024 x 4096 in bf16 820 to 930 us
// (step by step 1120; the products of 1024^3 in tiles of 64, whose operands come from the L2s at 12.7 TB/s: 22 of 31 us each), 3 x 1001 x 515
// of fp32 182 to 200 (18 launches: 4 us each to begin and to end), 16 x 128 x 784 of fp32 109 (13 launches).
#include <math.h>

#include <type_traits>

#include "ops_internal.h"
#include "ops_stage.h"

namespace aet_ops {

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// A matrix per client in two parts, 32 columns of the one next to those of the other, which makes a line of memory:
// [client][rows][cols / 32][high, low][32].  line: values of a row, 2 cols.
struct Parts {
    _Float16 *p;
    int64_t client;
    int line;
    // of 8 columns from col on; the second parts are 32 further
    __device__ __forceinline__ _Float16 *at(int64_t c, int row, int col) const { return p + c * client + (int64_t)row * line + col / 32 * 64 + col % 32; }
};

// high + low = v to within 2^-22 of it
__device__ __forceinline__ void split_half(const float (&v)[8], half8 &high, half8 &low) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        high[e] = (_Float16)v[e];
        low[e] = (_Float16)(v[e] - (float)high[e]);
    }
}

__device__ __forceinline__ void put_parts(const Parts &x, int64_t client, int row, int col, const float (&v)[8]) {
    half8 high, low;
    split_half(v, high, low);
    _Float16 *const to = x.at(client, row, col);
    *(half8 *)to = high;
    *(half8 *)(to + 32) = low;
}
__device__ __forceinline__ void get_parts(const Parts &x, int64_t client, int row, int col, float (&v)[8]) {
    const _Float16 *from = x.at(client, row, col);
    const half8 high = *(const half8 *)from, low = *(const half8 *)(from + 32);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)high[e] + (float)low[e];
}

// ---- bounds and scales -------------------------------------------------------------------

// The largest |a s + b s^3 + c s^5| over s in [0, top]
__host__ __device__ inline double largest(double a, double b, double c, double top) {
    const auto f = [&](double s) { return fabs(s * (a + s * s * (b + s * s * c))); };
    double most = f(top);
    // where the slope a + 3 b q + 5 c q^2 of q = s^2 is 0
    const double d = 9 * b * b - 20 * a * c;
    if (c != 0 && d >= 0) {
        for (int sign = -1; sign <= 1; sign += 2) {
            const double q = (-3 * b + sign * sqrt(d)) / (10 * c);
            if (q > 0 && q < top * top) most = fmax(most, f(sqrt(q)));
        }
    }
    if (b != 0) {
        const double q = -a / (3 * b);   // (c = 0; else a value more)
        if (q > 0 && q < top * top) most = fmax(most, f(sqrt(q)));
    }
    return most;
}
constexpr double kRoom = 1.02;   // for what the products are off
// A step from singular values up to x: bounds of A's and B's, and of the next X's
struct Bounds {
    double a, b, next;
};
__host__ __device__ inline Bounds bounds_of(const aet_orthogonal &o, double x) {
    const double q = x * x;
    return {q, q * (fabs(o.b) + fabs(o.c) * q), kRoom * largest(o.a, o.b, o.c, x)};
}
bool orthogonal_bounded(const aet_orthogonal &o) {
    double x = kRoom;
    for (int i = 0; i < o.steps; ++i) {
        const Bounds b = bounds_of(o, x);
        if (!(b.b < 0x1p60) || !(b.next < 0x1p30)) return false;
        x = b.next;
    }
    return true;
}
// The exponent of a power of two that takes a value of this bound to 2^14 or more and less than 2^15, of a type whose largest value is nearly 2^16.
// (Below 2^-400 no more: what is multiplied with it stays in 64 bits' range, and is nothing in the result.)
__device__ inline int room_of(double bound) {
    int e = -400;
    if (bound > 0) frexp(bound, &e);
    return 15 - (e > -400 ? e : -400);
}

// The largest |a + b q + c q^2| over q in [0, top^2]: how much a step makes of a singular value, at most
__host__ __device__ inline double most_growth(double a, double b, double c, double top) {
    const auto p = [&](double q) { return fabs(a + q * (b + q * c)); };
    double most = fmax(p(0), p(top * top));
    if (c != 0) {
        const double q = -b / (2 * c);
        if (q > 0 && q < top * top) most = fmax(most, p(q));
    }
    return kRoom * most;
}

// What the products of a step multiply by, with the scales of what they take and make.
struct Scales {
    float a_by;                                     // A = X X^T
    float b_by, b_plus, x_plus;                     // a step by itself: B = b A + c A A, X = a X + B X
    float ax_by, x_ax, x_aax;                       // the same as a X + b (A X) + c A (A X)
    float p_by, p_plus, p_diagonal;                 // several by A alone: P
    float q_by, t_by, n_by;                         // Q P, A P, (A P) P
    float x_by;                                     // B X or Q X
};
// The steps in runs that go by A alone: where a run ends.  (A run of one step is a step by itself.)
struct Runs {
    uint64_t ends[2];
    __host__ __device__ bool end(int i) const { return ends[i / 64] >> (i % 64) & 1; }
};
// Of a client whose X begins with singular values up to x; the last X's own scale is taken out of *y_by.  (A thread's time, about as much as
// a launch: powers of two are divided by as exponents.)
__device__ inline void scales_of(const aet_orthogonal &o, const Runs &runs, double x, Scales *to, double *y_by) {
    int sx = room_of(x), sa = 0, sq = 0;
    double q = 0;
    bool first = true;   // of a run
    const auto times = [](double v, int e) { return (float)ldexp(v, e); };
    for (int i = 0; i < o.steps; ++i) {
        const Bounds b = bounds_of(o, x);
        const int next = room_of(b.next);
        Scales t = {};
        if (first) {
            sa = room_of(b.a);
            t.a_by = times(1, sa - 2 * sx);
        }
        if (first && runs.end(i)) {
            const int sb = room_of(b.b), st = room_of(x * b.a);
            t.b_by = times(o.c, sb - 2 * sa);
            t.b_plus = times(o.b, sb - sa);
            t.x_by = times(1, next - sb - sx);
            t.x_plus = times(o.a, next - sx);
            t.ax_by = times(1, st - sa - sx);
            t.x_ax = times(o.b, next - sa - sx);
            t.x_aax = times(o.c, next - sa - st);
            sx = next;
        } else {
            const double p = most_growth(o.a, o.b, o.c, x);
            const int sp = room_of(p), st = room_of(x * b.next), sn = room_of(b.next * b.next);
            t.p_by = times(o.c, sp - 2 * sa);
            t.p_plus = times(o.b, sp - sa);
            t.p_diagonal = times(o.a, sp);
            const double more = first ? p : kRoom * q * p;
            const int s = first ? sp : room_of(more);
            t.q_by = first ? 0.0f : times(1, s - sq - sp);
            t.t_by = times(1, st - sa - sp);
            t.n_by = times(1, sn - st - sp);
            q = more;
            sq = s;
            sa = sn;
            if (runs.end(i)) {
                t.x_by = times(1, next - sq - sx);
                sx = next;
            }
        }
        to[i] = t;
        first = runs.end(i);
        x = b.next;
    }
    *y_by = ldexp(o.scale, -sx);
}

// ---- the norm, the first X, and the result -----------------------------------------------

struct Whole {
    int m, k;           // of X
    int mp, kp;         // with the zeros
    bool tall;          // X is G's transpose
    int parts;          // of the sum of squares
    Runs runs;
    double *sums;       // [client][parts]
    Scales *scales;     // [client][steps]
    double *y_by;       // [client]
};

template <typename T>
__global__ __launch_bounds__(256) void k_ortho_norm(aet_orthogonal a, Whole w) {
    constexpr int V = 16 / sizeof(T);
    __shared__ double lds[4];
    const int64_t client = blockIdx.x / w.parts, part = blockIdx.x % w.parts;
    const T *g = (const T *)a.g.p + client * a.g.client;
    const int64_t across = (a.cols + V - 1) / V, all = across * a.rows;
    double sum = 0;
    for (int64_t i = part * 256 + threadIdx.x; i < all; i += (int64_t)w.parts * 256) {
        const int64_t row = i / across, col = (i - row * across) * V;
        float v[V];
        load_some(g + row * a.g.row + col, (int)(a.cols - col < V ? a.cols - col : V), v);
#pragma unroll
        for (int e = 0; e < V; ++e) sum = __builtin_fma((double)v[e], (double)v[e], sum);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) w.sums[blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// A tile of 64 x 64 of G per workgroup, with zeros behind its ends: X or its transpose, and through LDS the other.
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_first(aet_orthogonal a, Whole w, Parts straight, Parts turned) {
    __shared__ double lds[4];
    __shared__ float tile[64][65];
    // the first workgroups, one a client, work out the scales
    const int rows = w.tall ? w.kp : w.mp, cols = w.tall ? w.mp : w.kp, across = cols / 64, tiles = across * (rows / 64);
    const bool scales = blockIdx.x < (unsigned)a.n;
    const int64_t client = scales ? blockIdx.x : (blockIdx.x - a.n) / tiles;
    const int t = scales ? 0 : (blockIdx.x - a.n) % tiles, r0 = t / across * 64, c0 = t % across * 64;
    double sum = threadIdx.x < w.parts ? w.sums[client * w.parts + threadIdx.x] : 0;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = sum;
    __syncthreads();
    const double own = __builtin_sqrt((lds[0] + lds[1]) + (lds[2] + lds[3])), norm = own + a.eps;
    // singular values are at most the norm's share of norm + eps, and the scales go by that: also a gradient far below eps keeps its bits
    const double top = own > 0 && norm < INFINITY ? kRoom * own / norm : 0;
    if (scales) {
        if (threadIdx.x == 0) scales_of(a, w.runs, top, w.scales + client * a.steps, w.y_by + client);
        return;
    }
    // (values that are not finite: all of X is NaN)
    const double by = own < INFINITY ? (top > 0 ? ldexp(1.0, room_of(top)) / norm : 0) : __builtin_nan("");
    const T *g = (const T *)a.g.p + client * a.g.client;
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int r = i / 8, c = i % 8 * 8;
        float v[8];
        load_some(g + (int64_t)(r0 + r) * a.g.row + c0 + c, r0 + r < a.rows ? a.cols - c0 - c : 0, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = r0 + r < a.rows && c0 + c + e < a.cols ? (float)((double)v[e] * by) : 0.0f;
            tile[r][c + e] = v[e];
        }
        if (straight.p) put_parts(straight, client, r0 + r, c0 + c, v);
    }
    if (!turned.p) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int c = i / 8, r = i % 8 * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[r + e][c];
        put_parts(turned, client, c0 + c, r0 + r, v);
    }
}

// y = keep w + scale X
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_last(aet_orthogonal a, Whole w, Parts x) {
    __shared__ float tile[64][65];
    const int across = (w.k + 63) / 64, tiles = across * ((w.m + 63) / 64);
    const int64_t client = blockIdx.x / tiles;
    const int t = blockIdx.x % tiles, r0 = t / across * 64, c0 = t % across * 64;
    const T *old = a.w.p ? (const T *)a.w.p + client * a.w.client : nullptr;
    T *y = (T *)a.y.p + client * a.y.client;
    const double by = w.y_by[client];
    const float keep = (float)a.keep;
    const auto value = [&](int r, int c, float (&v)[8]) {
        get_parts(x, client, r0 + r, c0 + c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)(v[e] * by);
    };
    if (w.tall) {
        for (int i = threadIdx.x; i < 64 * 8; i += 256) {
            const int r = i / 8, c = i % 8 * 8;
            float v[8];
            value(r, c, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[r][c + e] = v[e];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 64 * 64; i += 256) {
            const int c = i / 64, r = i % 64;
            if (r0 + r >= w.m || c0 + c >= w.k) continue;
            const int64_t row = c0 + c, col = r0 + r;
            float v = tile[r][c];
            if (old) v = __builtin_fmaf(keep, (float)old[row * a.w.row + col], v);
            y[row * a.y.row + col] = (T)v;
        }
        return;
    }
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int r = i / 8, c = i % 8 * 8, count = w.k - c0 - c;
        if (r0 + r >= w.m || count <= 0) continue;
        float v[8], o[8];
        value(r, c, v);
        if (old) {
            load_some(old + (int64_t)(r0 + r) * a.w.row + c0 + c, count, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(keep, o[e], v[e]);
        }
        store_some(y + (int64_t)(r0 + r) * a.y.row + c0 + c, count, v);
    }
}

// ---- products ----------------------------------------------------------------------------

// C = by sum over k of A(m, k) B(n, k), plus `plus` times what lies in the same place of `add`, plus `diagonal` where row and column
// are the same; or two products of the same sizes in one launch.
struct Side {
    Parts a, b, c, add;
    Parts turned;                           // where C's transpose goes to too; p = NULL: nowhere
    const float *by, *plus, *diagonal;      // of the first client; `apart` between clients; plus, diagonal: or NULL
};
struct HalfProduct {
    Side side[2];
    int each, apart;               // clients of a side
    int M, N, K, clients;          // clients: of all sides
    int tiles_m, tiles_n, tiles;   // tiles: of a client; SYM: of the upper half
    int slices, slice_k, blocks;   // parts of the sum; partial sums go to `partial` where there are several
    float *partial;                // [slice][client][M][N]
};

// The place of tile t of the upper half, row after row, of n x n tiles
__device__ __forceinline__ void upper_tile(int t, int n, int &i, int &j) {
    const double q = 2.0 * n + 1;
    i = (int)((q - __builtin_sqrt(q * q - 8.0 * t)) * 0.5);
    // (the root may be off by a rounding)
    if (t < i * n - i * (i - 1) / 2) --i;
    else if (t >= (i + 1) * n - (i + 1) * i / 2) ++i;
    j = i + t - (i * n - i * (i - 1) / 2);
}

// What C's sums are multiplied with
struct Factors {
    float by, plus, diagonal;
    __device__ __forceinline__ Factors(const Side &d, int64_t at) : by(d.by[at]), plus(d.plus ? d.plus[at] : 0.0f), diagonal(d.diagonal ? d.diagonal[at] : 0.0f) {}
};
// 8 columns of C from their sums
__device__ __forceinline__ void finish_half(const Side &d, int64_t client, int row, int col, const Factors &f, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= f.by;
    if (d.add.p) {
        float o[8];
        get_parts(d.add, client, row, col, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(o[e], f.plus, v[e]);
    }
    if (d.diagonal)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += row == col + e ? f.diagonal : 0.0f;
    put_parts(d.c, client, row, col, v);
}

// T x T tiles of C, WR x WC waves, NB stages of 32 k in use or on their way.  SYM: C is symmetric: only tiles of the upper half are
// worked out, and are C's other half's when turned.  TB: B by columns, which takes longer to read from LDS (B X of 1024 x 1024 x 1024 21
// us, with X's transpose by rows 14) but saves making the transpose: for large tiles.
template <int T, int WR, int WC, int NB, bool SYM, bool TB>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_half(HalfProduct p) {
    constexpr int THREADS = 64 * WR * WC, FM = T / WR / 32, FN = T / WC / 32;
    // (as values of one part: a line has 32 k of both; by columns a row of the stage has T columns of both)
    using SA = Stage<T, 64, false>;
    using SB = std::conditional_t<TB, Stage<2 * T, 32, true>, Stage<T, 64, false>>;
    constexpr int kStage = SA::kBytes + SB::kBytes;
    extern __shared__ __attribute__((aligned(1024))) char lds_[];
    const lds_ptr lds = (lds_ptr)lds_;
    int id = xcd_order(blockIdx.x, p.blocks);
    const int tile = id % p.tiles;
    id /= p.tiles;
    const int slice = id % p.slices, all = id / p.slices;   // all: the client's number among those of all sides
    const Side &d = p.side[all >= p.each];
    const int64_t client = all >= p.each ? all - p.each : all;
    const Factors factors(d, client * p.apart);
    int ti, tj;
    if constexpr (SYM) {
        upper_tile(tile, p.tiles_m, ti, tj);
    } else {   // eight rows of tiles at a time, column after column
        const int group = tile / (8 * p.tiles_n) * 8, high = p.tiles_m - group < 8 ? p.tiles_m - group : 8, in = tile - group * p.tiles_n;
        ti = group + in % high;
        tj = in / high;
    }
    const int m0 = ti * T, n0 = tj * T, k0 = slice * p.slice_k, k1 = k0 + p.slice_k < p.K ? k0 + p.slice_k : p.K;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wr = wave / WC, wc = wave % WC;

    DirectStage<T, 64, false, THREADS> la;
    std::conditional_t<TB, DirectStage<2 * T, 32, true, THREADS>, DirectStage<T, 64, false, THREADS>> lb;
    la.begin({d.a.p, d.a.client, d.a.line, false, true, 0}, client, m0, 1 << 30, 2 * k0, 0);
    lb.begin({d.b.p, d.b.client, d.b.line, TB, true, 0}, client, TB ? 2 * n0 : n0, 1 << 30, TB ? k0 : 2 * k0, 0);
    const auto fetch = [&](int i) {
        const lds_ptr to = lds + i % NB * kStage;
        la.load(to);
        lb.load(to + SA::kBytes);
    };
    struct Fragments {
        half8 a[FM][2], b[FN][2];
    };
    const auto read = [&](Fragments &f, int stage, int ks) {
        const lds_ptr at = lds + stage % NB * kStage;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
#pragma unroll
            for (int i = 0; i < FN; ++i)
                f.b[i][q] = __builtin_bit_cast(half8, TB ? SB::fragment(at + SA::kBytes, 2 * (wc * FN + i) + q, ks, lane) : SB::fragment(at + SA::kBytes, wc * FN + i, ks + 2 * q, lane));
#pragma unroll
            for (int j = 0; j < FM; ++j) f.a[j][q] = __builtin_bit_cast(half8, SA::fragment(at, wr * FM + j, ks + 2 * q, lane));
        }
    };
    // Where the registers have room the small products, high low and low high, are summed apart from high high, so that they are
    // rounded at their own size: results are nearer by 10 to 25 % (130 x 1400 of rank 12: 1.4e-5 -> 1.2e-5), at the same time.
    constexpr int kSums = FM * FN < 4 ? 2 : 1;
    f16v acc[kSums][FN][FM];
#pragma unroll
    for (int h = 0; h < kSums; ++h)
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[h][i][j] = f16v{};
    const auto multiply = [&](const Fragments &f) {
#pragma unroll
        for (int q = 0; q < 3; ++q)   // low high, high high, high low
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    f16v &c = acc[kSums == 2 && q != 1][i][j];
                    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.b[i][q == 0], f.a[j][q == 2], c, 0, 0, 0);
                }
    };
    // All but the last `still` of what is on its way to LDS has arrived, and what was read of it, everywhere.
    const auto arrived = [&](auto still) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | (still & 15) | (still >> 4) << 14);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The fragments of the next 16 k are read while the matrix unit has the last ones, also across the barrier that says that the
    // next stage has arrived everywhere and that this one's place may be written again.
    const int stages = (k1 - k0) / 32;
    constexpr int kLoads = decltype(la)::kCount + decltype(lb)::kCount, kReads = 2 * ((TB ? 2 : 1) * FN + FM);
    typedef std::integral_constant<int, 0> None;
    Fragments f[2];
    for (int i = 0; i < NB && i < stages; ++i) fetch(i);
    if (stages >= NB) arrived(std::integral_constant<int, (NB - 1) * kLoads>());
    else arrived(None());
    read(f[0], 0, 0);
    const auto stage = [&](int i, auto more, auto still, auto get) {
        read(f[1], i, 1);
        multiply(f[0]);
        interleave<3 * FM * FN, kReads>();
        arrived(still);
        get(i);
        if constexpr (more) read(f[0], i + 1, 0);
        multiply(f[1]);
        interleave<3 * FM * FN, kReads>();
    };
    int i = 0;
    for (; i + NB < stages; ++i) stage(i, std::true_type(), std::integral_constant<int, (NB - 2) * kLoads>(), [&](int i) { fetch(i + NB); });
    for (; i + 1 < stages; ++i) stage(i, std::true_type(), None(), [](int) {});
    stage(i, std::false_type(), None(), [](int) {});
    __syncthreads();

    // A lane has, of row m0 + lane % 32 of a fragment, four columns at a time: through LDS, a wave for itself, to lanes with 8 columns.
    constexpr int W = FN * 32, LINE = W + 4, ACROSS = W / 8, DOWN = 64 / ACROSS;
    __attribute__((address_space(3))) float *mine = (__attribute__((address_space(3))) float *)lds + wave * (32 * LINE);
    const bool turn = d.turned.p && !(SYM && ti == tj) && p.slices == 1;
    const auto settle = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    };
#pragma unroll
    for (int j = 0; j < FM; ++j) {
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f4 v;
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = kSums == 2 ? acc[0][i][j][4 * q + x] + acc[kSums - 1][i][j][4 * q + x] : acc[0][i][j][4 * q + x];
                *(__attribute__((address_space(3))) f4 *)(mine + (lane & 31) * LINE + i * 32 + 8 * q + 4 * (lane >> 5)) = v;
            }
        settle();
        const int row0 = m0 + (wr * FM + j) * 32, col0 = n0 + wc * W;
#pragma unroll 1
        for (int r = 0; r < 32; r += DOWN) {
            const int line = r + lane / ACROSS, c = lane % ACROSS * 8;
            float v[8];
            __attribute__((address_space(3))) f4 *const at = (__attribute__((address_space(3))) f4 *)(mine + line * LINE + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = at[e / 4][e % 4];
            if (p.slices > 1) {
                float *const to = p.partial + (((int64_t)slice * p.clients + all) * p.M + row0 + line) * p.N + col0 + c;
                *(f4 *)to = f4{v[0], v[1], v[2], v[3]};
                *(f4 *)(to + 4) = f4{v[4], v[5], v[6], v[7]};
                continue;
            }
            finish_half(d, client, row0 + line, col0 + c, factors, v);
            if (turn) {
                at[0] = f4{v[0], v[1], v[2], v[3]};
                at[1] = f4{v[4], v[5], v[6], v[7]};
            }
        }
        if (turn) {
            settle();
#pragma unroll 1
            for (int c = lane / 4; c < W; c += 16) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = mine[(lane % 4 * 8 + e) * LINE + c];
                put_parts(d.turned, client, col0 + c, row0 + lane % 4 * 8, v);
            }
        }
        settle();
    }
}

// Y = a X + b T + c A T, T = A X, of small A, all of which lies in LDS: 64 columns a workgroup.  A launch instead of two (B, and B X).  Five
// steps: 1 x 64 x 64 73 -> 50 us, 300 x 64 x 512 257 -> 225, 16 x 128 x 784 128 -> 112; 64 x 128 x 784, four workgroups a unit one after the
// other, 224 -> 256.
struct HalfApply {
    Parts a, xt, x, y, yt;         // yt.p = NULL: not wanted
    const Scales *by;              // of the first client
    int steps, tiles, blocks;      // steps: between clients' scales
};
template <int M>
struct ApplyTile {
    using SA = Stage<M, 64, false>;
    using SB = Stage<64, 64, false>;
    static constexpr int kDeep = M / 32, FM = M / 64, LINE = 36;
    static constexpr int kX = kDeep * SA::kBytes, kTurn = kX + kDeep * SB::kBytes, kLds = kTurn + 4 * 32 * LINE * 4;
};
template <int M>
__global__ __launch_bounds__(256) void k_half_apply(HalfApply p) {
    using L = ApplyTile<M>;
    using SA = typename L::SA;
    using SB = typename L::SB;
    constexpr int FM = L::FM, LINE = L::LINE;
    extern __shared__ __attribute__((aligned(1024))) char lds_[];
    const lds_ptr lds = (lds_ptr)lds_;
    const int id = xcd_order(blockIdx.x, p.blocks), n0 = id % p.tiles * 64;
    const int64_t client = id / p.tiles;
    const Scales &by = p.by[client * p.steps];
    const float ax_by = by.ax_by, x_ax = by.x_ax, x_aax = by.x_aax, plus = by.x_plus;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wr = wave / 2, wc = wave % 2;

    DirectStage<M, 64, false, 256> la;
    DirectStage<64, 64, false, 256> lb;
    la.begin({p.a.p, p.a.client, p.a.line, false, true, 0}, client, 0, 1 << 30, 0, 0);
    lb.begin({p.xt.p, p.xt.client, p.xt.line, false, true, 0}, client, n0, 1 << 30, 0, 0);
#pragma unroll
    for (int i = 0; i < L::kDeep; ++i) {
        la.load(lds + i * SA::kBytes);
        lb.load(lds + L::kX + i * SB::kBytes);
    }
    const auto arrived = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // the small products apart from high high
    struct Sums {
        f16v s[2][FM];
        __device__ __forceinline__ float at(int j, int e) const { return s[0][j][e] + s[1][j][e]; }
    };
    const auto multiply = [&](Sums &c) {
#pragma unroll
        for (int j = 0; j < FM; ++j) c.s[0][j] = c.s[1][j] = f16v{};
#pragma unroll
        for (int i = 0; i < 2 * L::kDeep; ++i) {
            half8 a[FM][2], b[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                b[q] = __builtin_bit_cast(half8, SB::fragment(lds + L::kX + i / 2 * SB::kBytes, wc, i % 2 + 2 * q, lane));
#pragma unroll
                for (int j = 0; j < FM; ++j) a[j][q] = __builtin_bit_cast(half8, SA::fragment(lds + i / 2 * SA::kBytes, wr * FM + j, i % 2 + 2 * q, lane));
            }
#pragma unroll
            for (int q = 0; q < 3; ++q)   // low high, high high, high low
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    f16v &o = c.s[q != 1][j];
                    o = __builtin_amdgcn_mfma_f32_32x32x16_f16(b[q == 0], a[j][q == 2], o, 0, 0, 0);
                }
        }
    };
    // A lane has, of row lane % 32 of a fragment, four columns at a time: through LDS, a wave for itself, by columns or by rows
    __attribute__((address_space(3))) float *const mine = (__attribute__((address_space(3))) float *)(lds + L::kTurn) + wave * (32 * LINE);
    const auto settle = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    };
    const auto put = [&](auto value) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *(__attribute__((address_space(3))) f4 *)(mine + (lane & 31) * LINE + 8 * q + 4 * (lane >> 5)) = f4{value(4 * q), value(4 * q + 1), value(4 * q + 2), value(4 * q + 3)};
        settle();
    };
    // calls f(column, 8 rows' values)
    const auto turned = [&](auto f) {
#pragma unroll
        for (int c = lane / 4; c < 32; c += 16) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = mine[(lane % 4 * 8 + e) * LINE + c];
            f(c, v);
        }
        settle();
    };
    Sums t, u;
    arrived();
    multiply(t);
    arrived();   // T takes X's place
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        put([&](int e) { return t.at(j, e) * ax_by; });
        turned([&](int c, const float (&v)[8]) {
            half8 high, low;
            split_half(v, high, low);
            const lds_ptr to = lds + L::kX + (wr * FM + j) * SB::kBytes;
            *(__attribute__((address_space(3))) half8 *)(to + SB::slot(wc * 32 + c, lane % 4) * 16) = high;
            *(__attribute__((address_space(3))) half8 *)(to + SB::slot(wc * 32 + c, 4 + lane % 4) * 16) = low;
        });
    }
    arrived();
    multiply(u);
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        put([&](int e) { return __builtin_fmaf(u.at(j, e), x_aax, t.at(j, e) * x_ax); });
        const int row0 = (wr * FM + j) * 32, col0 = n0 + wc * 32;
#pragma unroll
        for (int r = 0; r < 32; r += 16) {
            const int line = r + lane / 4, c = lane % 4 * 8;
            __attribute__((address_space(3))) f4 *const at = (__attribute__((address_space(3))) f4 *)(mine + line * LINE + c);
            float v[8], o[8];
            get_parts(p.x, client, row0 + line, col0 + c, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(o[e], plus, at[e / 4][e % 4]);
            put_parts(p.y, client, row0 + line, col0 + c, v);
            at[0] = f4{v[0], v[1], v[2], v[3]};
            at[1] = f4{v[4], v[5], v[6], v[7]};
        }
        settle();
        if (p.yt.p) turned([&](int c, const float (&v)[8]) { put_parts(p.yt, client, col0 + c, row0 + lane % 4 * 8, v); });
    }
}

// Adds the slices of a split sum, in their order, and ends it: 64 x 64 of C a workgroup.
template <bool SYM>
__global__ __launch_bounds__(256) void k_half_join(HalfProduct p, int tiles) {
    __shared__ float turned[64][65];
    const int all = blockIdx.x / tiles, tile = blockIdx.x % tiles, across = p.N / 64;
    const Side &d = p.side[all >= p.each];
    const int64_t client = all >= p.each ? all - p.each : all;
    const Factors factors(d, client * p.apart);
    int ti = tile / across, tj = tile % across;
    if constexpr (SYM) upper_tile(tile, across, ti, tj);
#pragma unroll
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int r = i / 8, c = i % 8 * 8;
        float v[8] = {};
        const float *from = p.partial + ((int64_t)all * p.M + ti * 64 + r) * p.N + tj * 64 + c;
        for (int k = 0; k < p.slices; ++k, from += (int64_t)p.clients * p.M * p.N) {
            const f4 x = *(const f4 *)from, y = *(const f4 *)(from + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] += x[e];
                v[4 + e] += y[e];
            }
        }
        finish_half(d, client, ti * 64 + r, tj * 64 + c, factors, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) turned[c + e][r] = v[e];
    }
    if (!d.turned.p || (SYM && ti == tj)) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int r = i / 8, c = i % 8 * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = turned[r][c + e];
        put_parts(d.turned, client, tj * 64 + r, ti * 64 + c, v);
    }
}

// ---- the steps ---------------------------------------------------------------------------

// Kinds of tiles: microseconds for 32 k where a compute unit has one workgroup (`busy`: more when all units have one), for each further
// one up to the `fit` that it holds, and for a workgroup's beginning and end.  Measured on products of 64 to 4096.  (Tiles of 64 with three
// stages on their way, of which a unit holds three: 1024 x 1024 3 % slower than with four.  With twice the waves, each of a pair with every
// other 16 k: 16 x 128 x 784 130 us, 3 x 1001 x 515 188, as with one.)
struct Kind {
    int tile, fit;
    float alone, busy, more, end;
};
static const Kind kKinds[] = {{256, 1, 1.7f, 0.8f, 0.0f, 8.0f}, {128, 2, 0.58f, 0.2f, 0.62f, 5.0f}, {64, 2, 0.22f, 0.0f, 0.13f, 3.5f}};
struct Choice {
    const Kind *kind;
    int slices;
    float time;
};
static Choice choose(int64_t clients, int64_t M, int64_t N, int64_t K, bool sym) {
    Choice best = {};
    for (const Kind &k : kKinds) {
        if (M % k.tile || N % k.tile) continue;
        const int64_t tm = M / k.tile, tiles = clients * (sym ? tm * (tm + 1) / 2 : tm * (N / k.tile)), stages = K / 32;
        // what is read and written beside the operands, at 5 TB/s: 4 bytes of each place a value
        const float ends = (float)clients * (float)M * (float)N * (sym ? 8 : k.tile == 256 ? 8 : 12) / 5e6f;
        for (int64_t slices = 1; slices == 1 || (slices <= 32 && stages / slices >= 4); slices *= 2) {
            const int64_t blocks = tiles * slices;
            const float waves = blocks <= 256 ? 1.0f : (float)ceil_div(blocks, 128) * 0.5f, fit = (float)k.fit;
            const float alone = k.alone + k.busy * (blocks < 256 ? (float)blocks / 256 : 1.0f);
            const float stage = waves <= fit ? alone + (waves - 1) * k.more : (alone + (fit - 1) * k.more) * waves / fit;
            float t = (float)ceil_div(stages, slices) * stage;
            // the L2s bring operands at some 12.7 TB/s
            const float bring = (float)blocks * (float)ceil_div(stages, slices) * (float)(256 * k.tile) / 12.7e6f;
            t = (t > bring ? t : bring) + k.end + ends;
            // partial sums are written and read at about 6 TB/s, and the launch that adds them takes 5
            if (slices > 1) t += 5.0f + (float)blocks * (float)(8 * k.tile * k.tile) / 6e6f;
            if (!best.kind || t < best.time) best = {&k, (int)slices, t};
        }
    }
    return best;
}

static int64_t up(int64_t v, int64_t to) { return ceil_div(v, to) * to; }

struct OrthoPlan {
    Whole w;
    Choice gram, square, pair, times;   // X X^T, A A, two of those, B X
    bool runs;                          // several steps by A alone
    bool apply;                         // steps by themselves without B
    Parts x[2], xt[2], a[2], b, p[2], q[2], t;   // xt: X's transpose, where B X wants that
    bool turned() const { return times.kind->tile < 256; }
    float *partial;
    size_t bytes;
};
// Where runs end, if there are any.
static Runs runs_of(const aet_orthogonal &o, bool any) {
    Runs r = {};
    double x = kRoom, grown = 1;
    for (int i = 0; i < o.steps; ++i) {
        const auto square = [](double v) { return v > 1 ? v * v : 1.0; };
        grown *= square(most_growth(o.a, o.b, o.c, x));
        x = bounds_of(o, x).next;
        // (the last step is one, too)
        const bool end = !any || i + 1 == o.steps || grown * square(most_growth(o.a, o.b, o.c, x)) > 200;
        if (end) {
            r.ends[i / 64] |= UINT64_C(1) << (i % 64);
            grown = 1;
        }
    }
    return r;
}
// The time of the products
static float time_of(const OrthoPlan &p, int steps, const Runs &runs) {
    float t = 0;
    for (int i = 0, first = 0; i < steps; ++i) {
        if (!runs.end(i)) continue;
        const int len = i + 1 - first;
        first = i + 1;
        t += p.gram.time + p.times.time + (float)len * p.square.time;
        // A P and (A P) P of all but the last; Q P of all but the first: with A P where a step has both
        if (len > 1) t += (float)(len + 1) * p.square.time + (float)(len - 2) * p.pair.time;
    }
    return t;
}
static OrthoPlan plan(const aet_orthogonal &o, char *workspace) {
    OrthoPlan p = {};
    p.w.tall = o.rows > o.cols;
    p.w.m = p.w.tall ? o.cols : o.rows;
    p.w.k = p.w.tall ? o.rows : o.cols;
    const Runs one = runs_of(o, false), several = runs_of(o, true);
    // sides up to whole tiles of one kind, the one that is the fastest in all
    float best = 0;
    for (const Kind &k : kKinds) {
        const int64_t mp = up(p.w.m, k.tile), kp = up(p.w.k, k.tile);
        OrthoPlan q = p;
        q.w.mp = (int)mp;
        q.w.kp = (int)kp;
        q.gram = choose(o.n, mp, mp, kp, true);
        q.square = choose(o.n, mp, mp, mp, true);
        q.pair = choose(2 * (int64_t)o.n, mp, mp, mp, true);
        q.times = choose(o.n, mp, kp, mp, false);
        const float a = time_of(q, o.steps, one), b = time_of(q, o.steps, several);
        q.runs = o.dtype == AET_BF16 && b < a;
        q.w.runs = q.runs ? several : one;
        if (p.gram.kind && (q.runs ? b : a) >= best) continue;
        best = q.runs ? b : a;
        p = q;
    }
    // (128 rows fill a compute unit's LDS: where that is more than one round of workgroups, products by themselves are faster)
    p.apply = o.steps && !p.runs && (p.w.mp == 64 || (p.w.mp == 128 && (int64_t)o.n * (p.w.kp / 64) <= 256));
    // parts of the sum of squares: some 2048 workgroups, each with values for its threads
    const int64_t pieces = ceil_div(o.cols, o.dtype == AET_F32 ? 4 : 8) * o.rows, wanted = ceil_div(2048, o.n > 0 ? o.n : 1);
    p.w.parts = (int)(wanted < 256 ? wanted : 256);
    if (p.w.parts > ceil_div(pieces, 256)) p.w.parts = (int)ceil_div(pieces, 256);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        char *const q = workspace + at;
        at += up256(bytes);
        return q;
    };
    const auto parts = [&](int64_t rows, int64_t cols) {
        return Parts{(_Float16 *)take((size_t)o.n * 2 * rows * cols * sizeof(_Float16)), 2 * rows * cols, (int)(2 * cols)};
    };
    p.x[0] = parts(p.w.mp, p.w.kp);
    if (o.steps) {
        p.x[1] = parts(p.w.mp, p.w.kp);
        if (p.turned()) for (Parts &t : p.xt) t = parts(p.w.kp, p.w.mp);
        const auto squares = [&](Parts &t) { t = parts(p.w.mp, p.w.mp); };
        squares(p.a[0]);
        if (!p.apply) squares(p.b);
        if (p.runs) {
            squares(p.a[1]);
            for (int i = 0; i < 2; ++i) squares(p.p[i]), squares(p.q[i]);
            squares(p.t);
        }
        size_t most = 0;
        const auto split = [&](const Choice &c, int64_t clients, int64_t cols) {
            const size_t values = c.slices > 1 ? (size_t)c.slices * clients * p.w.mp * cols : 0;
            most = values > most ? values : most;
        };
        split(p.gram, o.n, p.w.mp);
        split(p.square, o.n, p.w.mp);
        if (p.runs) split(p.pair, 2 * (int64_t)o.n, p.w.mp);
        split(p.times, o.n, p.w.kp);
        p.partial = (float *)take(most * sizeof(float));
    }
    p.w.sums = (double *)take((size_t)o.n * p.w.parts * sizeof(double));
    p.w.scales = (Scales *)take((size_t)o.n * o.steps * sizeof(Scales));
    p.w.y_by = (double *)take((size_t)o.n * sizeof(double));
    p.bytes = at;
    return p;
}
size_t orthogonal_workspace(const aet_orthogonal &o) { return plan(o, nullptr).bytes; }

template <int T, int WR, int WC, int NB, bool SYM, bool TB>
static hipError_t run_half(const HalfProduct &p, hipStream_t stream) {
    const auto kernel = k_half<T, WR, WC, NB, SYM, TB>;
    constexpr int stages = NB * 2 * T * 128, ends = WR * WC * 32 * (T / WC + 4) * 4, lds = stages > ends ? stages : ends;
    if constexpr (lds > 64 * 1024) {
        static aet::PerDevice allowed;
        int dev = 0, ok = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        e = allowed.get(dev, &ok, [&](int *v) {
            *v = 1;
            return hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        });
        if (e != hipSuccess) return e;
    }
    kernel<<<p.blocks, 64 * WR * WC, lds, stream>>>(p);
    return hipGetLastError();
}
template <int M>
static hipError_t run_apply(const HalfApply &p, hipStream_t stream) {
    const auto kernel = k_half_apply<M>;
    constexpr int lds = ApplyTile<M>::kLds;
    if constexpr (lds > 64 * 1024) {
        static aet::PerDevice allowed;
        int dev = 0, ok = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        e = allowed.get(dev, &ok, [&](int *v) {
            *v = 1;
            return hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        });
        if (e != hipSuccess) return e;
    }
    kernel<<<p.blocks, 256, lds, stream>>>(p);
    return hipGetLastError();
}

template <bool SYM>   // SYM: A = B
static hipError_t product(const Choice &c, HalfProduct p, hipStream_t s) {
    const int t = c.kind->tile;
    const int64_t tm = p.M / t, tn = p.N / t, tiles = SYM ? tm * (tm + 1) / 2 : tm * tn;
    const int64_t am = p.M / 64, joins = SYM ? am * (am + 1) / 2 : am * (p.N / 64);
    if (!grid_fits(tiles * p.clients * c.slices, t == 256 ? 512 : 256) || !grid_fits(joins * p.clients, 256)) return hipErrorInvalidConfiguration;
    p.tiles_m = (int)tm;
    p.tiles_n = (int)tn;
    p.tiles = (int)tiles;
    p.slices = c.slices;
    p.slice_k = (int)ceil_div(p.K / 32, c.slices) * 32;
    p.slices = (int)ceil_div(p.K, p.slice_k);
    p.blocks = (int)(tiles * p.clients * p.slices);
    hipError_t e;
    if (t == 256) e = run_half<256, 2, 4, 2, SYM, !SYM>(p, s);
    else if (t == 128) e = run_half<128, 2, 2, 2, SYM, false>(p, s);
    else e = run_half<64, 2, 2, 4, SYM, false>(p, s);
    if (e != hipSuccess || p.slices == 1) return e;
    k_half_join<SYM><<<(int)(joins * p.clients), 256, 0, s>>>(p, (int)joins);
    return hipGetLastError();
}

template <typename T>
static hipError_t run(const aet_orthogonal &o, char *workspace, hipStream_t s) {
    const OrthoPlan p = plan(o, workspace);
    const int64_t norms = (int64_t)o.n * p.w.parts, firsts = (int64_t)o.n * (p.w.mp / 64) * (p.w.kp / 64),
                  lasts = (int64_t)o.n * ceil_div(p.w.m, 64) * ceil_div(p.w.k, 64);
    if (!grid_fits(norms, 256) || !grid_fits(firsts + o.n, 256)) return hipErrorInvalidConfiguration;
    k_ortho_norm<T><<<(int)norms, 256, 0, s>>>(o, p.w);
    k_ortho_first<T><<<(int)(o.n + firsts), 256, 0, s>>>(o, p.w, p.w.tall ? p.xt[0] : p.x[0], p.w.tall ? p.x[0] : p.xt[0]);
    hipError_t e = hipGetLastError();
    const Parts none = {};
    const int apart = o.steps * (int)(sizeof(Scales) / sizeof(float)), mp = p.w.mp, kp = p.w.kp;
    const auto one = [&](const Side &d, int N, int K) {
        HalfProduct h = {{d, d}, o.n, apart, mp, N, K, o.n};
        h.partial = p.partial;
        return h;
    };
    const auto step = [&](hipError_t now) {
        if (e == hipSuccess) e = now;
        return e == hipSuccess;
    };
    int now = 0, at = 0;   // of x and xt, and of a: the one that has the present values
    const Parts *q = nullptr;
    for (int i = 0, first = 0; i < o.steps; ++i) {
        const Scales *by = p.w.scales + i;
        const Parts &x = p.x[now], &xt = p.turned() ? p.xt[now] : x, &y = p.x[now ^ 1], &yt = i + 1 < o.steps && p.turned() ? p.xt[now ^ 1] : none;
        const bool end = p.w.runs.end(i);
        if (i == first && !step(product<true>(p.gram, one({x, x, p.a[at], none, p.a[at], &by->a_by}, mp, kp), s))) return e;
        const Parts &a = p.a[at];
        if (i == first && end && p.apply) {
            const int tiles = kp / 64, blocks = o.n * tiles;   // (no more than `firsts`)
            const HalfApply h = {a, xt, x, y, yt, by, o.steps, tiles, blocks};
            if (!step(mp == 64 ? run_apply<64>(h, s) : run_apply<128>(h, s))) return e;
        } else if (i == first && end) {   // a step by itself
            if (!step(product<true>(p.square, one({a, a, p.b, a, p.b, &by->b_by, &by->b_plus}, mp, mp), s))) return e;
            if (!step(product<false>(p.times, one({p.b, xt, y, x, yt, &by->x_by, &by->x_plus}, kp, mp), s))) return e;
        } else {
            const Parts &pp = p.p[i % 2], &next = p.a[at ^ 1];
            if (!step(product<true>(p.square, one({a, a, pp, a, pp, &by->p_by, &by->p_plus, &by->p_diagonal}, mp, mp), s))) return e;
            const Side qs = {q ? *q : a, pp, p.q[i % 2], none, p.q[i % 2], &by->q_by}, ts = {a, pp, p.t, none, p.t, &by->t_by};
            if (i == first) {
                q = &pp;
                if (!step(product<true>(p.square, one(ts, mp, mp), s))) return e;
            } else {
                q = &p.q[i % 2];
                HalfProduct h = one(qs, mp, mp);
                if (!end) {
                    h.side[1] = ts;
                    h.clients = 2 * o.n;
                }
                if (!step(product<true>(end ? p.square : p.pair, h, s))) return e;
            }
            if (!end) {
                if (!step(product<true>(p.square, one({p.t, pp, next, none, next, &by->n_by}, mp, mp), s))) return e;
                at ^= 1;
            } else if (!step(product<false>(p.times, one({*q, xt, y, none, yt, &by->x_by}, kp, mp), s))) {
                return e;
            }
        }
        if (end) {
            now ^= 1;
            first = i + 1;
            q = nullptr;
        }
    }
    if (e != hipSuccess) return e;
    k_ortho_last<T><<<(int)lasts, 256, 0, s>>>(o, p.w, p.x[now]);
    return hipGetLastError();
}
hipError_t launch_orthogonalise(const aet_orthogonal &o, void *workspace, hipStream_t s) {
    return o.dtype == AET_F32 ? run<float>(o, (char *)workspace, s) : run<bf16>(o, (char *)workspace, s);
}

}  // namespace aet_ops
