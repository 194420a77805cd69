// The gradient of the linear layer of values held in 4 bits.
//
// dx = dz W and dw = dz^T x, dz = dropout'(dy) act'(z).  A quarter of every value that codes stand for is one of bf16 (2 bits of it), so the products
// are of the matrix unit's bf16 instructions with W and x in one part, and with dz in as many as it takes: two for results in bf16 (to
// within 2^-16 of it), as in the linear layer's gradient, three for results in fp32 (24 bits, where that layer's fp32 products, whose
// operands both have 24, are six).  Without activation and dropout a dz in bf16 is dy as it is.
//
// Bound by the products: 8192 x 4096 x 4096 behind SiLU in bf16 976 to 1050 us, of which dz takes 55 (268 MB: 4.8 TB/s), W and x 32, dx and dw 519
// and 510 (1060 TF/s; the matrix unit is busy for 55 % of the cycles); in fp32 1.50 to 1.59 ms, of which dz takes 85 (5.5 TB/s), dx and dw 786 and 766.
// With dy as it is in bf16 482 to 515.  16 x 32 x 784 x 128 17 in bf16 and 19 in fp32: three launches of 5, 5 and 8 to 10.
#include "ops_internal.h"
#include "ops_mx4.h"
#include "ops_stage.h"

#include <type_traits>

namespace aet_ops {

typedef float f2 __attribute__((ext_vector_type(2)));

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// ---- dz ----------------------------------------------------------------------------------

// What dz of 8 columns of a row is worked out from, and dz
template <typename T, int ACT, bool DROP>
struct DzPiece {
    wide<T, 8> dy, z;
    __device__ __forceinline__ void load(const aet_mx4_linear_grad &a, int64_t client, int64_t row, int col, int count) {
        dy = load_raw<T, 8>((const T *)a.dy.p + client * a.dy.client + row * a.dy.row + col, count);
        if (ACT) z = load_raw<T, 8>((const T *)a.pre.p + client * a.pre.client + row * a.pre.row + col, count);
    }
    // (past the end 0)
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
constexpr int kDzRows = 4;   // of a thread, all on their way at once

// How dz is dealt out: a workgroup has 256 columns of a strip of a client's rows, eight rows at a time.
struct HeldDz {
    int across, strips, strip, line;
    bf16 *to;        // [part][client][row][line], zeros up to a multiple of 8; NULL: not wanted
    int64_t low;     // from part to part; 0: one
    float *partial;  // sums over rows, [strip][client][out]
};

// dz in parts, and its sums over rows.  Bound by memory.
template <typename T, int ACT, bool DROP>
__global__ __launch_bounds__(256) void k_held_dz(aet_mx4_linear_grad a, Drop d, HeldDz s) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 2;
    __shared__ float sums[8][256];
    const int per = s.across * s.strips, b = blockIdx.x % per, strip = b / s.across, ty = threadIdx.x / 32;
    const int64_t client = blockIdx.x / per;
    const int col = (b % s.across * 32 + threadIdx.x % 32) * 8, count = a.out - col;
    const int64_t first = (int64_t)strip * s.strip, end = first + s.strip < a.rows ? first + s.strip : a.rows;
    float sum[8] = {};
    for (int64_t r0 = first + ty; r0 < end && count > 0; r0 += 8 * kDzRows) {
        DzPiece<T, ACT, DROP> piece[kDzRows];
#pragma unroll
        for (int i = 0; i < kDzRows; ++i) piece[i].load(a, client, r0 + 8 * i < end ? r0 + 8 * i : end - 1, col, count);
#pragma unroll
        for (int i = 0; i < kDzRows; ++i) {
            const int64_t row = r0 + 8 * i;
            if (row >= end) break;
            float v[8];
            piece[i].work(a, d, client, row, col, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
            if (!s.to) continue;
            bf16 *const to = s.to + (client * a.rows + row) * s.line + col;
#pragma unroll
            for (int q = 0; q < PARTS; ++q) {
                if (q && !s.low) break;
                bf8 part;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float high = (float)(bf16)v[e];
                    // what would round to infinity has the largest value; infinities and NaN are in the first part alone
                    const bool finite = __builtin_fabsf(v[e]) <= __FLT_MAX__;
                    if (finite && __builtin_fabsf(high) > __FLT_MAX__) high = __builtin_copysignf(0x1.fep127f, v[e]);
                    part[e] = (bf16)high;
                    v[e] = finite ? v[e] - high : 0.0f;
                }
                *(bf8 *)(to + q * s.low) = part;
            }
        }
    }
    if (!a.db.p) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[ty][threadIdx.x % 32 * 8 + e] = sum[e];
    __syncthreads();
    const int mine = b % s.across * 256 + threadIdx.x;
    if (mine >= a.out) return;
    float total = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) total += sums[i][threadIdx.x];
    if (s.strips == 1) ((T *)a.db.p)[client * a.db.client + mine] = (T)total;
    else s.partial[((int64_t)strip * a.n + client) * a.out + mine] = total;
}

// ---- W and x -----------------------------------------------------------------------------

// Rows of held values as bf16, with zeros up to a multiple of 8.  They are a quarter of what they stand for, which the products make up for:
// 6 x 2^127, the largest, is beyond bf16's (and fp32's) largest value, while the smallest, 2^-128, leaves it room below.
struct HeldRows16 {
    Held from;
    bf16 *to;
    int64_t rows, all;   // of a client, and of all
};
// W's rows and x's, 2^lanes threads each, a piece of 8 columns at a time; and beside that, the strips' sums of dz.  Bound by memory.
template <typename T>
__global__ __launch_bounds__(256) void k_held_values(HeldRows16 w, HeldRows16 x, int cols, int line, int lanes, int64_t blocks, aet_mx4_linear_grad a, HeldDz s) {
    if (blockIdx.x >= blocks) {
        const int64_t i = (blockIdx.x - blocks) * 256 + threadIdx.x, all = (int64_t)a.n * a.out;
        if (i >= all) return;
        float total = 0;
#pragma unroll 8
        for (int k = 0; k < s.strips; ++k) total += s.partial[k * all + i];
        ((T *)a.db.p)[i / a.out * a.db.client + i % a.out] = (T)total;
        return;
    }
    int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> lanes;
    const HeldRows16 &r = at < w.all ? w : x;
    if (at >= w.all) at -= w.all;
    if (at >= r.all) return;
    const int64_t client = at / r.rows, row = at - client * r.rows;
    const uint8_t *codes = (const uint8_t *)r.from.codes.p + client * r.from.codes.client + row * r.from.codes.row;
    const uint8_t *scales = (const uint8_t *)r.from.scales.p + client * r.from.scales.client + row * r.from.scales.row;
    const int pieces = line / 8;
#pragma unroll 4
    for (int i = threadIdx.x & ((1 << lanes) - 1); i < pieces; i += 1 << lanes) {
        const int left = cols - 8 * i, bytes = (left + 1) / 2, scale = scales[i / 4];
        const uint8_t *p = codes + (int64_t)i * 4;
        uint32_t code = 0;
        if (left >= 8) {
            code = __builtin_bit_cast(uint32_t, (uint8_t __attribute__((ext_vector_type(4))))(*(const wide<uint8_t, 4> *)p));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) code |= e < bytes ? (uint32_t)p[e] << (8 * e) : 0;
        }
        bf8 v;
        const auto two = [&](f2 q, int e) {
#pragma unroll
            for (int y = 0; y < 2; ++y) v[e + y] = e + y < left ? (bf16)(scale == 255 ? __builtin_nanf("") : __builtin_ldexpf(q[y], scale - 129)) : (bf16)0.0f;
        };
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0), 0);
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 1), 2);
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 2), 4);
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 3), 6);
        *(bf8 *)(r.to + at * line + (int64_t)i * 8) = v;
    }
}

// ---- the plan ----------------------------------------------------------------------------

struct HeldPlan {
    HeldDz dz;
    Product dx, dw;
    HeldRows16 w, x;
    int line;       // of w and x
    char *more;     // for the products
    size_t bytes;
};
// a: with the clients as one where W is one for all; given: as the caller has it.
static HeldPlan plan(const aet_mx4_linear_grad &a, const aet_mx4_linear_grad &given, char *workspace) {
    HeldPlan p = {};
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        char *const q = workspace + at;
        at += up256(bytes);
        return q;
    };
    const bool products = a.dx.p || a.dw.p;
    const int64_t rows = (int64_t)a.n * a.rows, held_w = given.w.client && given.n > 1 ? given.n : 1;
    p.line = (int)(ceil_div(a.in, 8) * 8);
    p.dz.line = (int)(ceil_div(a.out, 8) * 8);
    p.dz.across = (int)ceil_div(a.out, 256);
    // strips of at least 16 rows, as many as give every compute unit several workgroups, and no more than 256, since one thread adds them
    const int64_t some = ceil_div(2048, (int64_t)a.n * p.dz.across + 1), wanted = some < 256 ? some : 256, most = ceil_div(a.rows, 16), strips = wanted < most ? wanted : most;
    p.dz.strip = (int)ceil_div(ceil_div(a.rows, strips), 8) * 8;
    p.dz.strips = (int)ceil_div(a.rows, p.dz.strip);
    // room for dz in any case, so that it does not depend on where dy lies
    const int parts = a.dtype == AET_F32 ? 3 : a.act != AET_ACT_NONE || a.p > 0 ? 2 : 1;
    const size_t part = products ? up256((size_t)rows * p.dz.line * sizeof(bf16)) : 0;
    p.dz.to = (bf16 *)take(part * parts);
    p.dz.low = parts > 1 ? (int64_t)(part / sizeof(bf16)) : 0;
    p.dz.partial = (float *)take(a.db.p && p.dz.strips > 1 ? (size_t)p.dz.strips * a.n * a.out * sizeof(float) : 0);
    const auto held = [&](const aet_in &codes, const aet_in &scales, int64_t of_client, int64_t all) {
        return HeldRows16{{codes, scales}, (bf16 *)take((size_t)all * p.line * sizeof(bf16)), of_client, all};
    };
    p.w = held(given.w, given.w_scales, a.out, a.dx.p ? held_w * a.out : 0);
    p.x = held(given.x, given.x_scales, given.rows, a.dw.p ? rows : 0);
    Operand dz = {p.dz.to, a.rows * (int64_t)p.dz.line, p.dz.line, false, true, p.dz.low, parts == 3};
    const Operand dy = {a.dy.p, a.dy.client, a.dy.row};
    if (!products) {
        p.dz.to = nullptr;
    } else if (parts == 1 && held_straight(dy, a.rows, a.out)) {
        p.dz.to = nullptr;
        dz = dy;
    }
    const Drop none = {};
    p.dx.a = dz;
    p.dx.b = {p.w.to, held_w > 1 ? (int64_t)a.out * p.line : 0, p.line, true, true};
    p.dx.M = a.rows;
    p.dx.N = a.in;
    p.dx.K = a.out;
    p.dx.e = {{}, {}, a.dx, {}, a.rows, AET_ACT_NONE, none};
    p.dw.a = dz;
    p.dw.a.by_columns = true;
    p.dw.b = {p.x.to, (int64_t)a.rows * p.line, p.line, true, true};
    p.dw.M = a.out;
    p.dw.N = a.in;
    p.dw.K = a.rows;
    p.dw.e = {{}, {}, a.dw, {}, a.out, AET_ACT_NONE, none};
    p.dx.clients = p.dw.clients = a.n;
    p.more = workspace + at;
    p.bytes = at + held_products_workspace(p.dx, p.dw);
    return p;
}
size_t mx4_gradient_workspace(const aet_mx4_linear_grad &a, const aet_mx4_linear_grad &given) { return plan(a, given, nullptr).bytes; }

template <typename T>
static hipError_t run(const aet_mx4_linear_grad &a, const aet_mx4_linear_grad &given, char *workspace, hipStream_t s) {
    const HeldPlan p = plan(a, given, workspace);
    const int64_t blocks = (int64_t)a.n * p.dz.across * p.dz.strips;
    int lanes = 0;
    while (lanes < 6 && 8 << lanes < p.line) ++lanes;
    const int64_t values = ceil_div((p.w.all + p.x.all) << lanes, 256), sums = a.db.p && p.dz.strips > 1 ? ceil_div((int64_t)a.n * a.out, 256) : 0;
    if (!grid_fits(blocks, 256) || !grid_fits(values + sums, 256)) return hipErrorInvalidConfiguration;
    if (p.dz.to || a.db.p) {
        const Drop d = make_drop(a.p, a.seed, a.first_row, a.out);
        const auto go = [&](auto act) {
            const auto dz = d.least ? k_held_dz<T, act, true> : k_held_dz<T, act, false>;
            dz<<<(int)blocks, 256, 0, s>>>(a, d, p.dz);
        };
        switch (a.act) {
        case AET_ACT_RELU: go(std::integral_constant<int, AET_ACT_RELU>()); break;
        case AET_ACT_SILU: go(std::integral_constant<int, AET_ACT_SILU>()); break;
        case AET_ACT_GELU: go(std::integral_constant<int, AET_ACT_GELU>()); break;
        default: go(std::integral_constant<int, AET_ACT_NONE>());
        }
    }
    if (values + sums) k_held_values<T><<<(int)(values + sums), 256, 0, s>>>(p.w, p.x, a.in, p.line, lanes, values, a, p.dz);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess && (a.dx.p || a.dw.p) ? launch_held_products(a.dtype, p.dx, p.dw, p.more, s) : e;
}
hipError_t launch_mx4_gradient(const aet_mx4_linear_grad &a, const aet_mx4_linear_grad &given, void *workspace, hipStream_t s) {
    return a.dtype == AET_F32 ? run<float>(a, given, (char *)workspace, s) : run<bf16>(a, given, (char *)workspace, s);
}

}  // namespace aet_ops
