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
// All matrices of a call lie in the workspace with zeros up to whole tiles, so that no product has to look where they end.
#include <math.h>

#include <type_traits>

#include "ops_internal.h"
#include "ops_stage.h"

namespace aet_ops {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// A matrix per client in two parts: [client][high, low][rows][cols]
struct Planes {
    _Float16 *p;
    int64_t client, low;   // low: from the first part to the second
    int cols;
};

// high + low = v to within 2^-23 of it
__device__ __forceinline__ void split_half(const float (&v)[8], half8 &high, half8 &low) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        high[e] = (_Float16)v[e];
        low[e] = (_Float16)(v[e] - (float)high[e]);
    }
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
// A power of two that takes a value of this bound to 2^14 or more and less than 2^15, of a type whose largest value is nearly 2^16.
__device__ inline double room_of(double bound) {
    if (!(bound > 0)) return 1;
    int e;
    frexp(bound, &e);
    return ldexp(1.0, 15 - e);
}

// What the products of a step multiply by, with the scales of what they take and make.
struct Scales {
    float a_by, b_by, b_plus, x_by, x_plus;
};
// Of a client whose X begins with singular values up to x; the last X's own scale is taken out of *y_by.
__device__ inline void scales_of(const aet_orthogonal &o, double x, Scales *to, double *y_by) {
    double sx = room_of(x);
    for (int i = 0; i < o.steps; ++i) {
        const Bounds b = bounds_of(o, x);
        const double sa = room_of(b.a), sb = room_of(b.b), next = room_of(b.next);
        to[i] = {(float)(sa / (sx * sx)), (float)(o.c * sb / (sa * sa)), (float)(o.b * sb / sa), (float)(next / (sb * sx)), (float)(o.a * next / sx)};
        x = b.next;
        sx = next;
    }
    *y_by = o.scale / sx;
}

// ---- the norm, the first X, and the result -----------------------------------------------

struct Whole {
    int m, k;           // of X
    int mp, kp;         // with the zeros
    bool tall;          // X is G's transpose
    int parts;          // of the sum of squares
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

// A tile of 64 x 64 of X per workgroup, from G by rows or columns, through LDS where X is the transpose.
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_first(aet_orthogonal a, Whole w, Planes x) {
    __shared__ double lds[4];
    __shared__ float tile[64][65];
    const int across = w.kp / 64, tiles = across * (w.mp / 64);
    const int64_t client = blockIdx.x / tiles;
    const int t = blockIdx.x % tiles, r0 = t / across * 64, c0 = t % across * 64;
    double sum = threadIdx.x < w.parts ? w.sums[client * w.parts + threadIdx.x] : 0;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = sum;
    __syncthreads();
    const double own = __builtin_sqrt((lds[0] + lds[1]) + (lds[2] + lds[3])), norm = own + a.eps;
    // singular values are at most the norm's share of norm + eps, and the scales go by that: also a gradient far below eps keeps its bits
    const double top = own > 0 && norm < INFINITY ? kRoom * own / norm : 0;
    if (t == 0 && threadIdx.x == 0) scales_of(a, top, w.scales + client * a.steps, w.y_by + client);
    // (values that are not finite: all of X is NaN)
    const double by = own < INFINITY ? (top > 0 ? room_of(top) / norm : 0) : __builtin_nan("");
    const T *g = (const T *)a.g.p + client * a.g.client;
    if (w.tall) {
        for (int i = threadIdx.x; i < 64 * 64; i += 256) {
            const int c = i / 64, r = i % 64;   // of X
            tile[r][c] = r0 + r < w.m && c0 + c < w.k ? (float)((double)(float)g[(int64_t)(c0 + c) * a.g.row + r0 + r] * by) : 0.0f;
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int r = i / 8, c = i % 8 * 8;
        float v[8];
        if (w.tall) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = tile[r][c + e];
        } else {
            load_some(g + (int64_t)(r0 + r) * a.g.row + c0 + c, r0 + r < w.m ? w.k - c0 - c : 0, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = r0 + r < w.m && c0 + c + e < w.k ? (float)((double)v[e] * by) : 0.0f;
        }
        half8 high, low;
        split_half(v, high, low);
        _Float16 *const to = x.p + client * x.client + (int64_t)(r0 + r) * x.cols + c0 + c;
        *(half8 *)to = high;
        *(half8 *)(to + x.low) = low;
    }
}

// y = keep w + scale X
template <typename T>
__global__ __launch_bounds__(256) void k_ortho_last(aet_orthogonal a, Whole w, Planes x) {
    __shared__ float tile[64][65];
    const int across = (w.k + 63) / 64, tiles = across * ((w.m + 63) / 64);
    const int64_t client = blockIdx.x / tiles;
    const int t = blockIdx.x % tiles, r0 = t / across * 64, c0 = t % across * 64;
    const T *old = a.w.p ? (const T *)a.w.p + client * a.w.client : nullptr;
    T *y = (T *)a.y.p + client * a.y.client;
    const double by = w.y_by[client];
    const float keep = (float)a.keep;
    const auto value = [&](int r, int c, float (&v)[8]) {
        const _Float16 *from = x.p + client * x.client + (int64_t)(r0 + r) * x.cols + c0 + c;
        const half8 high = *(const half8 *)from, low = *(const half8 *)(from + x.low);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)(((float)high[e] + (float)low[e]) * by);
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

// C = by sum over k of A(m, k) B(n, k), plus `plus` times what lies in the same place of `add`, in two parts.
struct HalfProduct {
    Planes a, b, c, add;
    int tiles_m, tiles_n, tiles;   // tiles: of a client; SYM: of the upper half
    int k, blocks;
    const float *by, *plus;        // of the first client; steps apart
    int apart;
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

// T x T tiles of C, W x W' waves.  SYM: C is symmetric; TB: B by columns.
template <int T, int BK, int WR, int WC, bool SYM>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_half(HalfProduct p) {
    constexpr bool TB = !SYM;
    constexpr int THREADS = 64 * WR * WC, FM = T / WR / 32, FN = T / WC / 32, KS = BK / 16;
    using SA = Stage<T, BK, false>;
    using SB = Stage<T, BK, TB>;
    constexpr int kPart = SA::kBytes, kStage = 4 * kPart;   // A high, A low, B high, B low
    static_assert(SA::kBytes == SB::kBytes, "square tiles");
    extern __shared__ __attribute__((aligned(1024))) char lds_[];
    const lds_ptr lds = (lds_ptr)lds_;
    const int id = xcd_order(blockIdx.x, p.blocks);
    const int64_t client = id / p.tiles;
    const int tile = id % p.tiles;
    int ti, tj;
    if constexpr (SYM) {
        upper_tile(tile, p.tiles_m, ti, tj);
    } else {   // eight rows of tiles at a time, column after column
        const int group = tile / (8 * p.tiles_n) * 8, high = p.tiles_m - group < 8 ? p.tiles_m - group : 8, in = tile - group * p.tiles_n;
        ti = group + in % high;
        tj = in / high;
    }
    const int m0 = ti * T, n0 = tj * T;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wr = wave / WC, wc = wave % WC;

    DirectStage<T, BK, false, THREADS> la, la2;
    DirectStage<T, BK, TB, THREADS> lb, lb2;
    la.begin({p.a.p, p.a.client, p.a.cols, false, true, 0}, client, m0, 1 << 30, 0, 0);
    lb.begin({p.b.p, p.b.client, p.b.cols, TB, true, 0}, client, n0, 1 << 30, 0, 0);
    la2 = la;
    lb2 = lb;
    la2.p += p.a.low * 2;
    lb2.p += p.b.low * 2;
    const auto fetch = [&](int i) {
        const lds_ptr to = lds + i % 2 * kStage;
        la.load(to);
        la2.load(to + kPart);
        lb.load(to + 2 * kPart);
        lb2.load(to + 3 * kPart);
    };
    const float by = p.by[client * p.apart], plus = p.plus ? p.plus[client * p.apart] : 0.0f;
    f16v acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = f16v{};
    const int stages = p.k / BK;
    fetch(0);
    for (int s = 0; s < stages; ++s) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);   // all that is on its way to LDS, and what was read of it
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + 1 < stages) fetch(s + 1);
        const lds_ptr at = lds + s % 2 * kStage;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            half8 a[FM][2], b[FN][2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
#pragma unroll
                for (int i = 0; i < FN; ++i) b[i][q] = __builtin_bit_cast(half8, SB::fragment(at + (2 + q) * kPart, wc * FN + i, ks, lane));
#pragma unroll
                for (int j = 0; j < FM; ++j) a[j][q] = __builtin_bit_cast(half8, SA::fragment(at + q * kPart, wr * FM + j, ks, lane));
            }
#pragma unroll
            for (int q = 0; q < 3; ++q)
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int j = 0; j < FM; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(b[i][q == 0], a[j][q == 1], acc[i][j], 0, 0, 0);
        }
    }
    __syncthreads();

    // A lane has, of row m0 + lane % 32 of a fragment, four columns at a time: through LDS, a wave for itself, to lanes with 8 columns.
    constexpr int W = FN * 32, LINE = W + 4, ACROSS = W / 8, DOWN = 64 / ACROSS;
    __attribute__((address_space(3))) float *mine = (__attribute__((address_space(3))) float *)lds + wave * (32 * LINE);
    const auto settle = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    };
    const auto put = [&](const float (&v)[8], int row, int col) {
        half8 high, low;
        split_half(v, high, low);
        _Float16 *const to = p.c.p + client * p.c.client + (int64_t)row * p.c.cols + col;
        *(half8 *)to = high;
        *(half8 *)(to + p.c.low) = low;
    };
#pragma unroll
    for (int j = 0; j < FM; ++j) {
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f4 v;
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = acc[i][j][4 * q + x] * by;
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
            if (p.add.p) {
                const _Float16 *from = p.add.p + client * p.add.client + (int64_t)(row0 + line) * p.add.cols + col0 + c;
                const half8 high = *(const half8 *)from, low = *(const half8 *)(from + p.add.low);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf((float)high[e] + (float)low[e], plus, v[e]);
                if (SYM && ti != tj) {
                    at[0] = f4{v[0], v[1], v[2], v[3]};
                    at[1] = f4{v[4], v[5], v[6], v[7]};
                }
            }
            put(v, row0 + line, col0 + c);
        }
        if (SYM && ti != tj) {   // the same values on the other side
            settle();
#pragma unroll 1
            for (int c = lane / 4; c < W; c += 16) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = mine[(lane % 4 * 8 + e) * LINE + c];
                put(v, col0 + c, row0 + lane % 4 * 8);
            }
        }
        settle();
    }
}

// ---- the steps ---------------------------------------------------------------------------

struct Kind {
    int tile;
    float stage, end;   // microseconds of 32 k of all workgroups that a compute unit holds, and of an epilogue
    int fit;
};
static const Kind kKinds[] = {{256, 1.9f, 8.0f, 1}, {128, 1.1f, 3.0f, 2}, {64, 0.8f, 2.0f, 4}};

static int64_t up(int64_t v, int64_t to) { return ceil_div(v, to) * to; }

struct OrthoPlan {
    Whole w;
    const Kind *kind;
    Planes x[2], a, b;
    size_t bytes;
};
static OrthoPlan plan(const aet_orthogonal &o, char *workspace) {
    OrthoPlan p = {};
    p.w.tall = o.rows > o.cols;
    p.w.m = p.w.tall ? o.cols : o.rows;
    p.w.k = p.w.tall ? o.rows : o.cols;
    float best = 0;
    for (const Kind &k : kKinds) {
        const int64_t tm = ceil_div(p.w.m, k.tile), tk = ceil_div(p.w.k, k.tile);
        const auto time = [&](int64_t tiles, int64_t sum) { return (float)ceil_div(tiles * o.n, 256 * k.fit) * ((float)ceil_div(sum, 32) * k.stage + k.end); };
        const int64_t half = tm * (tm + 1) / 2;
        const float t = time(half, tk * k.tile) + time(half, tm * k.tile) + time(tm * tk, tm * k.tile);
        if (!p.kind || t < best) {
            best = t;
            p.kind = &k;
        }
    }
    p.w.mp = (int)up(p.w.m, p.kind->tile);
    p.w.kp = (int)up(p.w.k, p.kind->tile);
    // parts of the sum of squares: some 2048 workgroups, each with values for its threads
    const int64_t pieces = ceil_div(o.cols, o.dtype == AET_F32 ? 4 : 8) * o.rows, wanted = ceil_div(2048, o.n > 0 ? o.n : 1);
    p.w.parts = (int)(wanted < 256 ? wanted : 256);
    if (p.w.parts > ceil_div(pieces, 256)) p.w.parts = (int)ceil_div(pieces, 256);
    size_t at = 0;
    const auto planes = [&](int64_t rows, int64_t cols) {
        const Planes q = {(_Float16 *)(workspace + at), 2 * rows * cols, rows * cols, (int)cols};
        at += up256((size_t)o.n * 2 * rows * cols * sizeof(_Float16));
        return q;
    };
    p.x[0] = planes(p.w.mp, p.w.kp);
    if (o.steps) {
        p.x[1] = planes(p.w.mp, p.w.kp);
        p.a = planes(p.w.mp, p.w.mp);
        p.b = planes(p.w.mp, p.w.mp);
    }
    p.w.sums = (double *)(workspace + at);
    at += up256((size_t)o.n * p.w.parts * sizeof(double));
    p.w.scales = (Scales *)(workspace + at);
    at += up256((size_t)o.n * o.steps * sizeof(Scales));
    p.w.y_by = (double *)(workspace + at);
    at += up256((size_t)o.n * sizeof(double));
    p.bytes = at;
    return p;
}
size_t orthogonal_workspace(const aet_orthogonal &o) { return plan(o, nullptr).bytes; }

template <int T, int BK, int WR, int WC, bool SYM>
static hipError_t run_half(const HalfProduct &p, hipStream_t stream) {
    const auto kernel = k_half<T, BK, WR, WC, SYM>;
    constexpr int stages = 2 * 4 * T * BK * 2, FN = T / WC / 32, ends = WR * WC * 32 * (FN * 32 + 4) * 4, lds = stages > ends ? stages : ends;
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
// sym: C and A = B are symmetric, or A = B and C = A A^T; else B is by columns
static hipError_t product(const OrthoPlan &plan, int64_t n, HalfProduct p, int64_t M, int64_t N, int64_t K, bool sym, hipStream_t s) {
    const int t = plan.kind->tile;
    const int64_t tm = M / t, tn = N / t, tiles = sym ? tm * (tm + 1) / 2 : tm * tn;
    if (tiles * n > INT32_MAX) return hipErrorInvalidConfiguration;
    p.tiles_m = (int)tm;
    p.tiles_n = (int)tn;
    p.tiles = (int)tiles;
    p.blocks = (int)(tiles * n);
    p.k = (int)K;
    if (t == 256) return sym ? run_half<256, 32, 2, 4, true>(p, s) : run_half<256, 32, 2, 4, false>(p, s);
    if (t == 128) return sym ? run_half<128, 32, 2, 2, true>(p, s) : run_half<128, 32, 2, 2, false>(p, s);
    return sym ? run_half<64, 32, 2, 2, true>(p, s) : run_half<64, 32, 2, 2, false>(p, s);
}

template <typename T>
static hipError_t run(const aet_orthogonal &o, char *workspace, hipStream_t s) {
    const OrthoPlan p = plan(o, workspace);
    const int64_t norms = (int64_t)o.n * p.w.parts, firsts = (int64_t)o.n * (p.w.mp / 64) * (p.w.kp / 64),
                  lasts = (int64_t)o.n * ceil_div(p.w.m, 64) * ceil_div(p.w.k, 64);
    if (norms > INT32_MAX || firsts > INT32_MAX) return hipErrorInvalidConfiguration;
    k_ortho_norm<T><<<(int)norms, 256, 0, s>>>(o, p.w);
    k_ortho_first<T><<<(int)firsts, 256, 0, s>>>(o, p.w, p.x[0]);
    hipError_t e = hipGetLastError();
    for (int i = 0; i < o.steps && e == hipSuccess; ++i) {
        const Planes &x = p.x[i % 2], &y = p.x[(i + 1) % 2], none = {};
        const Scales *by = p.w.scales + i;
        const int apart = o.steps * (int)(sizeof(Scales) / sizeof(float));
        e = product(p, o.n, {x, x, p.a, none, 0, 0, 0, 0, 0, &by->a_by, nullptr, apart}, p.w.mp, p.w.mp, p.w.kp, true, s);
        if (e == hipSuccess) e = product(p, o.n, {p.a, p.a, p.b, p.a, 0, 0, 0, 0, 0, &by->b_by, &by->b_plus, apart}, p.w.mp, p.w.mp, p.w.mp, true, s);
        if (e == hipSuccess) e = product(p, o.n, {p.b, x, y, x, 0, 0, 0, 0, 0, &by->x_by, &by->x_plus, apart}, p.w.mp, p.w.kp, p.w.mp, false, s);
    }
    if (e != hipSuccess) return e;
    k_ortho_last<T><<<(int)lasts, 256, 0, s>>>(o, p.w, p.x[o.steps % 2]);
    return hipGetLastError();
}
hipError_t launch_orthogonalise(const aet_orthogonal &o, void *workspace, hipStream_t s) {
    return o.dtype == AET_F32 ? run<float>(o, (char *)workspace, s) : run<bf16>(o, (char *)workspace, s);
}

}  // namespace aet_ops
