// The gradient of the linear layer of values held in 4 bits.
//
// dx = dz W and dw = dz^T x, dz = dropout'(dy) act'(z), in fp32.  W and x have two bits a value and dz more, so a product takes W and x in
// one part, and dz in two (22 bits).  fp16 has few exponents, so that both operands are scaled by powers of two that
// move from one to the other: a row of the contraction in W by the exponent that its largest block has, which its column of dz is
// multiplied by; then a row of dz so that its largest value is near 2^15, which the row of the result is multiplied by.  What is lost
// of a value is below 2^-39 of the largest of its row, and blocks of W (or x) less than 2^-36 of the largest of their row.
//
// 8192 x 4096 x 4096 behind SiLU 1.37 ms.  In bf16 one fp16 value would do it in 660 us, but is 2^-11 of dz off, which shows where terms
// cancel; two bf16 values take 1.01 ms, and no more by the linear layer's own way.
#include "ops_internal.h"
#include "ops_mx4.h"
#include "ops_stage.h"

#include <limits.h>

#include <type_traits>

namespace aet_ops {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));

constexpr int kNone = kNoExponent;

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Rows of held values as fp16, times 2^-exps[row], where exps is the exponent of the row's largest block that has a value, less 13
// (magnitudes up to 6 become up to 49152); zeros up to a multiple of 8.
struct HalfRows {
    Held from;
    _Float16 *to;
    int32_t *exps;
    int64_t rows, all;   // of a client, and of all
};
// W's rows and x's, a wave each, and the places of the maxima that come next.
__global__ __launch_bounds__(256) void k_mx4_half(HalfRows w, HalfRows x, int cols, int line, int32_t *tops, int64_t count) {
    int64_t at = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    const int64_t thread = (int64_t)blockIdx.x * 256 + threadIdx.x, threads = (int64_t)gridDim.x * 256;
    for (int64_t i = thread; i < count; i += threads) tops[i] = INT_MIN;
    const HalfRows &r = at < w.all ? w : x;
    if (at >= w.all) at -= w.all;
    if (at >= r.all) return;
    const int lane = threadIdx.x % 64;
    const int64_t client = at / r.rows, row = at - client * r.rows;
    const uint8_t *codes = (const uint8_t *)r.from.codes.p + client * r.from.codes.client + row * r.from.codes.row;
    const uint8_t *scales = (const uint8_t *)r.from.scales.p + client * r.from.scales.client + row * r.from.scales.row;
    const int blocks = (cols + 31) / 32, pieces = line / 8;
    // 8 codes from column 8 i on; past the end 0
    const auto read = [&](int i) {
        const int left = cols - 8 * i, bytes = (left + 1) / 2;
        const uint8_t *p = codes + (int64_t)i * 4;
        uint32_t v = 0;
        if (left >= 8) {
            v = __builtin_bit_cast(uint32_t, (uint8_t __attribute__((ext_vector_type(4))))(*(const wide<uint8_t, 4> *)p));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v |= e < bytes ? (uint32_t)p[e] << (8 * e) : 0;
            if (left > 0) v &= (1u << (4 * left)) - 1;
        }
        return v;
    };
    int top = INT_MIN;
#pragma unroll 4
    for (int i = lane; i < pieces; i += 64) {
        const int scale = i / 4 < blocks ? scales[i / 4] : 255;
        const uint32_t code = read(i);
        if (scale != 255 && (code & 0x77777777u)) top = scale > top ? scale : top;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const int o = __shfl_xor(top, off, 64);
        top = o > top ? o : top;
    }
    const int shift = (top == INT_MIN ? 127 : top) - 13;   // scales become scale - shift + 127
    if (lane == 0) r.exps[at] = top == INT_MIN ? kNone : shift - 127;   // (a row of zeros weighs nothing)
#pragma unroll 4
    for (int i = lane; i < pieces; i += 64) {
        // (a block that has a value is moved to no more than 2^13; zeros may have any scale, which must not become 255, NaN)
        const int scale = i / 4 < blocks ? scales[i / 4] : 127, moved = scale - shift + 127, most = 127 + 13;
        const float by = __builtin_bit_cast(float, (uint32_t)(scale == 255 ? 255 : moved < 0 ? 0 : moved < most ? moved : most) << 23);
        const uint32_t code = read(i);
        const half2v c0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, by, 0), c1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, by, 1),
                     c2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, by, 2), c3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, by, 3);
        *(half8 *)(r.to + at * line + (int64_t)i * 8) = half8{c0[0], c0[1], c1[0], c1[1], c2[0], c2[1], c3[0], c3[1]};
    }
}

// What dz of 8 columns of a row is worked out from, and dz
template <typename T, int ACT, bool DROP>
struct DzPiece {
    wide<T, 8> dy, z;
    __device__ __forceinline__ void load(const aet_mx4_linear_grad &a, int64_t client, int64_t row, int col, int count) {
        dy = load_raw<T, 8>((const T *)a.dy.p + client * a.dy.client + row * a.dy.row + col, count);
        if (ACT) z = load_raw<T, 8>((const T *)a.pre.p + client * a.pre.client + row * a.pre.row + col, count);
    }
    __device__ __forceinline__ void work(const aet_mx4_linear_grad &a, const Drop &d, int64_t client, int64_t row, int col, float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)dy[e];
        if (ACT) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = (float)z[e];
            slope_each<ACT>(f, v);
        }
        // last, so that what the forward pass took out has a gradient of 0 whatever z was
        if (DROP) drop_apply(d, drop_row(d, client * a.rows + row), col, v);
    }
};
constexpr int kTopRows = 1, kDzRows = 4;   // of a thread, all on their way at once

// How dz is dealt out: a workgroup has 256 columns of a strip of a client's rows, eight rows at a time.
struct HalfShape {
    int across, strips, strip, line;
    int32_t *row_top, *col_top;          // the largest exponent of a row of dz with W's, of a column with x's
    const int32_t *w_exps, *x_exps;
    int64_t w_client;                    // of w_exps: 0 where W is one for all
    _Float16 *by_rows, *by_columns;      // the two forms of dz, [client][row][line]; NULL: not wanted
    int64_t low;                         // fp32: from first to second parts
    float *partial;                      // sums over rows, [strip][client][out]
};
struct HalfPlace {
    int64_t client, first, end;
    int strip, col, count, ty;
    __device__ __forceinline__ HalfPlace(const HalfShape &s, int rows, int out) {
        const int per = s.across * s.strips, b = blockIdx.x % per;
        client = blockIdx.x / per;
        strip = b / s.across;
        col = (b % s.across * 32 + threadIdx.x % 32) * 8;
        ty = threadIdx.x / 32;
        count = out - col;
        first = (int64_t)strip * s.strip;
        end = first + s.strip < rows ? first + s.strip : rows;
    }
};

// |v| < 2^exponent; nothing for 0 and what is not finite
__device__ __forceinline__ int exponent_of(float v) {
    const bool counts = v != 0 && __builtin_fabsf(v) <= __FLT_MAX__;
    return counts ? __builtin_amdgcn_frexp_expf(v) : kNone;
}

// The largest exponents of rows and columns (maxima, whose order does not matter), and the sums over rows.
template <typename T, int ACT, bool DROP>
__global__ __launch_bounds__(256) void k_half_tops(aet_mx4_linear_grad a, Drop d, HalfShape s) {
    __shared__ float sums[8][256];
    __shared__ int tops[8][256];
    const HalfPlace p(s, a.rows, a.out);
    int w[8], col[8];
    float sum[8] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e] = s.by_rows && e < p.count ? s.w_exps[p.client * s.w_client + p.col + e] : 0;
        col[e] = kNone;
    }
    for (int64_t r0 = p.first; r0 < p.end; r0 += 8 * kTopRows) {   // (all lanes as often)
        DzPiece<T, ACT, DROP> piece[kTopRows];
#pragma unroll
        for (int i = 0; i < kTopRows; ++i) {
            const int64_t row = r0 + 8 * i + p.ty;
            if (p.count > 0) piece[i].load(a, p.client, row < p.end ? row : p.end - 1, p.col, p.count);
        }
#pragma unroll
        for (int i = 0; i < kTopRows; ++i) {
            const int64_t row = r0 + 8 * i + p.ty;
            int top = kNone;
            if (row < p.end && p.count > 0) {
                float v[8];
                piece[i].work(a, d, p.client, row, p.col, v);
                const int x = s.by_columns ? s.x_exps[p.client * a.rows + row] : 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (e >= p.count) continue;
                    const int q = exponent_of(v[e]);
                    top = q + w[e] > top ? q + w[e] : top;
                    col[e] = q + x > col[e] ? q + x : col[e];
                    sum[e] += v[e];
                }
            }
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) {
                const int o = __shfl_xor(top, off, 64);
                top = o > top ? o : top;
            }
            if (s.by_rows && threadIdx.x % 32 == 0 && row < p.end) atomicMax(s.row_top + p.client * a.rows + row, top);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        sums[p.ty][threadIdx.x % 32 * 8 + e] = sum[e];
        tops[p.ty][threadIdx.x % 32 * 8 + e] = col[e];
    }
    __syncthreads();
    const int mine = blockIdx.x % s.across * 256 + threadIdx.x;
    if (mine >= a.out) return;
    float total = 0;
    int top = kNone;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        total += sums[i][threadIdx.x];
        top = tops[i][threadIdx.x] > top ? tops[i][threadIdx.x] : top;
    }
    if (s.by_columns) atomicMax(s.col_top + p.client * a.out + mine, top);
    if (a.db.p) {
        if (s.strips == 1) ((T *)a.db.p)[p.client * a.db.client + mine] = (T)total;
        else s.partial[((int64_t)p.strip * a.n + p.client) * a.out + mine] = total;
    }
}

// dz as its two forms, rows and columns times the powers of two that leave their largest value near 2^15.
template <typename T, int ACT, bool DROP>
__global__ __launch_bounds__(256) void k_half_dz(aet_mx4_linear_grad a, Drop d, HalfShape s) {
    const int64_t blocks = (int64_t)a.n * s.across * s.strips;
    if (blockIdx.x >= blocks) {   // beside that, the strips' sums
        const int64_t i = (blockIdx.x - blocks) * 256 + threadIdx.x, all = (int64_t)a.n * a.out;
        if (i >= all) return;
        float total = 0;
#pragma unroll 8
        for (int k = 0; k < s.strips; ++k) total += s.partial[k * all + i];
        ((T *)a.db.p)[i / a.out * a.db.client + i % a.out] = (T)total;
        return;
    }
    const HalfPlace p(s, a.rows, a.out);
    if (p.col >= s.line) return;
    int w[8], col[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e] = s.by_rows && e < p.count ? s.w_exps[p.client * s.w_client + p.col + e] : 0;
        col[e] = s.by_columns && e < p.count ? row_shift(s.col_top[p.client * a.out + p.col + e]) : 0;
    }
    const auto put = [&](_Float16 *to, const float (&v)[8], auto by) {
        half8 high, low;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float f = e < p.count ? __builtin_ldexpf(v[e], by(e)) : 0.0f;   // (past the end zeros)
            high[e] = (_Float16)f;
            // infinities and NaN are in the first part alone
            low[e] = __builtin_fabsf(f) <= __FLT_MAX__ ? (_Float16)(f - (float)high[e]) : (_Float16)0.0f;
        }
        *(half8 *)to = high;
        if (sizeof(T) == 4) *(half8 *)(to + s.low) = low;
    };
    for (int64_t r0 = p.first + p.ty; r0 < p.end; r0 += 8 * kDzRows) {
        DzPiece<T, ACT, DROP> piece[kDzRows];
        int tops[kDzRows], xs[kDzRows];
#pragma unroll
        for (int i = 0; i < kDzRows; ++i) {
            const int64_t row = r0 + 8 * i < p.end ? r0 + 8 * i : p.end - 1;
            piece[i].load(a, p.client, row, p.col, p.count);
            tops[i] = s.by_rows ? s.row_top[p.client * a.rows + row] : 0;
            xs[i] = s.by_columns ? s.x_exps[p.client * a.rows + row] : 0;
        }
#pragma unroll
        for (int i = 0; i < kDzRows; ++i) {
            const int64_t row = r0 + 8 * i;
            if (row >= p.end) break;
            float v[8];
            piece[i].work(a, d, p.client, row, p.col, v);
            const int64_t at = (p.client * a.rows + row) * s.line + p.col;
            if (s.by_rows) {
                const int r = row_shift(tops[i]);
                put(s.by_rows + at, v, [&](int e) { return w[e] - r; });
            }
            if (s.by_columns) {
                const int x = xs[i];
                put(s.by_columns + at, v, [&](int e) { return x - col[e]; });
            }
        }
    }
}

// ---- the plan ----------------------------------------------------------------------------

struct HalfPlan {
    HalfShape s;
    Product dx, dw;
    _Float16 *w, *x;
    int64_t w_rows;    // of all clients, one for all counted once
    int line;          // of w and x
    int32_t *tops;     // row_top and col_top, one behind the other
    int64_t count;
    int32_t *w_exps, *x_exps;
    char *more;        // for the products
    size_t bytes;
};
static HalfPlan plan(const aet_mx4_linear_grad &a, char *workspace) {
    HalfPlan p = {};
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        char *const q = workspace + at;
        at += up256(bytes);
        return q;
    };
    const int parts = a.dtype == AET_F32 ? 2 : 1;
    const int64_t rows = (int64_t)a.n * a.rows, clients_w = a.w.client ? a.n : 1;
    p.line = (int)(ceil_div(a.in, 8) * 8);
    p.s.line = (int)(ceil_div(a.out, 8) * 8);
    p.s.across = (int)ceil_div(a.out, 256);
    // strips of at least 16 rows, as many as give every compute unit several workgroups
    const int64_t wanted = ceil_div(2048, (int64_t)a.n * p.s.across + 1), most = ceil_div(a.rows, 16), strips = wanted < most ? wanted : most;
    p.s.strip = (int)ceil_div(ceil_div(a.rows, strips > 0 ? strips : 1), 8) * 8;
    p.s.strips = (int)ceil_div(a.rows, p.s.strip);
    const size_t part = up256((size_t)rows * p.s.line * sizeof(_Float16));
    p.s.low = (int64_t)(part / sizeof(_Float16));
    if (a.dx.p) {
        p.s.by_rows = (_Float16 *)take(part * parts);
        p.w_rows = clients_w * a.out;
        p.w = (_Float16 *)take((size_t)p.w_rows * p.line * sizeof(_Float16));
        p.s.w_exps = p.w_exps = (int32_t *)take((size_t)p.w_rows * 4);
        p.s.w_client = clients_w > 1 ? a.out : 0;
    }
    if (a.dw.p) {
        p.s.by_columns = (_Float16 *)take(part * parts);
        p.x = (_Float16 *)take((size_t)rows * p.line * sizeof(_Float16));
        p.s.x_exps = p.x_exps = (int32_t *)take((size_t)rows * 4);
    }
    p.count = rows + (int64_t)a.n * a.out;
    p.tops = (int32_t *)take((size_t)p.count * 4);
    p.s.row_top = p.tops;
    p.s.col_top = p.tops + rows;
    p.s.partial = (float *)take(a.db.p && p.s.strips > 1 ? (size_t)p.s.strips * a.n * a.out * sizeof(float) : 0);
    const Drop none = {};
    const int64_t low = parts == 2 ? p.s.low : 0;
    p.dx.clients = a.dx.p ? a.n : 0;
    p.dx.a = {p.s.by_rows, (int64_t)a.rows * p.s.line, p.s.line, false, true, low};
    p.dx.b = {p.w, clients_w > 1 ? (int64_t)a.out * p.line : 0, p.line, true, true, 0};
    p.dx.M = a.rows;
    p.dx.N = a.in;
    p.dx.K = a.out;
    p.dx.e = {{}, {}, a.dx, {}, a.rows, AET_ACT_NONE, none};
    p.dw.a = {p.s.by_columns, (int64_t)a.rows * p.s.line, p.s.line, true, true, low};
    p.dw.b = {p.x, (int64_t)a.rows * p.line, p.line, true, true, 0};
    p.dw.clients = a.dw.p ? a.n : 0;
    p.dw.M = a.out;
    p.dw.N = a.in;
    p.dw.K = a.rows;
    p.dw.e = {{}, {}, a.dw, {}, a.out, AET_ACT_NONE, none};
    p.more = workspace + at;
    const size_t x = a.dx.p ? half_product_workspace(p.dx) : 0, w = a.dw.p ? half_product_workspace(p.dw) : 0;
    p.bytes = at + (x > w ? x : w);
    return p;
}

// Where it can be done and is faster than with the values in dz's own type: two of six products in fp32.
bool mx4_half_pays(const aet_mx4_linear_grad &a) {
    if (a.dtype != AET_F32 || !a.n || !a.rows || !a.in || !a.out || !(a.dx.p || a.dw.p)) return false;
    const HalfPlan p = plan(a, (char *)256);
    if ((a.dx.p && !half_fits(p.dx)) || (a.dw.p && !half_fits(p.dw))) return false;
    if ((int64_t)a.n * a.rows > INT32_MAX || p.w_rows > INT32_MAX) return false;
    // Launches more, and dz worked out twice and written in a form for each product.  (Measured against the other way at 50 sizes of 0.3 to 100 G
    // products, both wanted, in microseconds and for a million values: 8 to 18 and 5 to 7.  The choice is the faster way or within 17 % of it.)
    const float values = (float)a.n * (float)a.rows * (float)a.out * 1e-6f, forms = (a.dx.p ? 1.0f : 0.0f) + (a.dw.p ? 1.0f : 0.0f);
    float here = 2.0f + 2.1f * values + (4.0f + 1.7f * values) * forms;
    Product x = p.dx, w = p.dw;
    if (a.dx.p) here += half_product_time(x);
    if (a.dw.p) here += half_product_time(w);
    x.a.low = w.a.low = 0;
    return here < gradients_time(a.dtype, x, w);
}
size_t mx4_half_workspace(const aet_mx4_linear_grad &a) { return plan(a, nullptr).bytes; }

template <typename T>
static hipError_t run(const aet_mx4_linear_grad &a, char *workspace, hipStream_t s) {
    const HalfPlan p = plan(a, workspace);
    const int64_t rows = (int64_t)a.n * a.rows, blocks = (int64_t)a.n * p.s.across * p.s.strips;
    if (blocks > INT32_MAX || p.w_rows + rows > INT32_MAX) return hipErrorInvalidConfiguration;
    const HalfRows w = {{a.w, a.w_scales}, p.w, p.w_exps, a.out, p.w_rows}, x = {{a.x, a.x_scales}, p.x, p.x_exps, a.rows, a.dw.p ? rows : 0};
    k_mx4_half<<<(int)ceil_div(w.all + x.all, 4), 256, 0, s>>>(w, x, a.in, p.line, p.tops, p.count);
    const int64_t sums = a.db.p && p.s.strips > 1 ? ceil_div((int64_t)a.n * a.out, 256) : 0;
    if (blocks + sums > INT32_MAX) return hipErrorInvalidConfiguration;
    const Drop d = make_drop(a.p, a.seed, a.first_row, a.out);
    const auto go = [&](auto act) {
        const auto tops = d.least ? k_half_tops<T, act, true> : k_half_tops<T, act, false>;
        const auto dz = d.least ? k_half_dz<T, act, true> : k_half_dz<T, act, false>;
        tops<<<(int)blocks, 256, 0, s>>>(a, d, p.s);
        dz<<<(int)(blocks + sums), 256, 0, s>>>(a, d, p.s);
    };
    switch (a.act) {
    case AET_ACT_RELU: go(std::integral_constant<int, AET_ACT_RELU>()); break;
    case AET_ACT_SILU: go(std::integral_constant<int, AET_ACT_SILU>()); break;
    case AET_ACT_GELU: go(std::integral_constant<int, AET_ACT_GELU>()); break;
    default: go(std::integral_constant<int, AET_ACT_NONE>());
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.dx.p) e = launch_half_product(p.dx, {p.s.row_top, a.rows}, p.more, s);
    if (e == hipSuccess && a.dw.p) e = launch_half_product(p.dw, {p.s.col_top, a.out}, p.more, s);
    return e;
}
hipError_t launch_mx4_half(const aet_mx4_linear_grad &a, void *workspace, hipStream_t s) { return run<float>(a, (char *)workspace, s); }

}  // namespace aet_ops
