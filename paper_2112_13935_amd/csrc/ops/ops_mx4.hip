// Microscaled 4-bit floating point: values to codes and scales, and back.
//
// Bound by memory.  To codes four lanes have a block of 32 values, 8 each: their largest magnitude's exponent by two exchanges
// between neighbours, then the hardware's conversions, which divide by the scale (given by its exponent alone; 0 is 2^-127,
// 255 NaN), round to the nearest of the 16 values, ties to the even code, and end at 6.
//   16384 x 4096 of bf16 to codes and scales 31 us (5.5 TB/s); 16384 x 8192 there and back 139 us, at a large copy's rate
//   (5.0 TB/s) 136; 128 x 784 of fp32 there and back 9.8 us, the two calls.
#include "ops_internal.h"
#include "ops_mx4.h"

#include <type_traits>

namespace aet_ops {

typedef bf16 bf2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

// Rows of a thread, all on their way at once, and its columns.  16384 x 8192, microseconds for 1, 2, 4 rows: 8 columns of bf16 to codes 81, 67, 67 (of
// half as many 36, 31, 33) and back 87, 71, 66; of fp32, where that is 32 bytes, 105, 111, 115 and 140, 153, 159; 4 columns of fp32
// 145, 118, 121 and 156, 132, 125.
template <typename T>
constexpr int kToRows = sizeof(T) == 2 ? 2 : 1;
template <typename T>
constexpr int kBackPiece = 16 / sizeof(T);

struct Mx4Shape {
    int pieces, wide;         // pieces of V columns in a row, whole blocks; threads side by side (a power of two, a block's and more)
    int64_t across, down;     // workgroups: of a row of pieces, of a client
};

struct Mx4Place {
    int64_t client, row0;
    int col, high;
};
template <int V, int ROWS>
__device__ __forceinline__ bool place_of(const Mx4Shape &s, Mx4Place &p) {
    const int64_t per = s.across * s.down, b = blockIdx.x % per;
    p.client = blockIdx.x / per;
    const int piece = (int)(b % s.across) * s.wide + (threadIdx.x & (s.wide - 1));
    p.high = 256 / s.wide;
    p.row0 = b / s.across * (p.high * ROWS) + threadIdx.x / s.wide;
    p.col = piece * V;
    return piece < s.pieces;   // (the same for the lanes of a block)
}

// 8 values to codes; the block's scale
template <typename T>
__device__ __forceinline__ uint32_t quantise8(const wide<T, 8> &v, uint32_t &scale) {
    uint32_t top = 0;   // the largest magnitude's bits: NaN is above infinity, which is above all others
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t m = __builtin_bit_cast(uint32_t, (float)v[e]) & 0x7fffffffu;
        top = m > top ? m : top;
    }
#pragma unroll
    for (int off = 1; off < 4; off *= 2) {
        const uint32_t m = __shfl_xor(top, off, 64);
        top = m > top ? m : top;
    }
    // floor(log2(top)) - 2 + 127 where that is 0 or more; subnormal values and 0 have 0 too
    const uint32_t x = top >> 23;
    scale = x == 255 ? 255 : x > 2 ? x - 2 : 0;
    const float by = __builtin_bit_cast(float, scale << 23);
    uint32_t code = 0;
    if constexpr (sizeof(T) == 2) {
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, bf2{v[0], v[1]}, by, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, bf2{v[2], v[3]}, by, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, bf2{v[4], v[5]}, by, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, bf2{v[6], v[7]}, by, 3);
    } else {
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], by, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], by, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], by, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], by, 3);
    }
    return scale == 255 ? 0 : code;
}

template <typename T>
__global__ __launch_bounds__(256) void k_mx4_quantise(aet_mx4_values a, Mx4Shape s) {
    constexpr int ROWS = kToRows<T>;
    Mx4Place p;
    if (!place_of<8, ROWS>(s, p)) return;
    const T *x = (const T *)a.x.p + p.client * a.x.client + p.col;
    uint8_t *codes = (uint8_t *)a.codes.p + p.client * a.codes.client + p.col / 2;
    uint8_t *scales = (uint8_t *)a.scales.p + p.client * a.scales.client + p.col / 32;
    const int count = a.cols - p.col, bytes = (count + 1) / 2;
    wide<T, 8> v[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t row = p.row0 + i * p.high;
        if (row < a.rows) v[i] = load_raw<T, 8>(x + row * a.x.row, count);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t row = p.row0 + i * p.high;
        if (row >= a.rows) continue;
        uint32_t scale;
        const wide<uint8_t, 4> code = __builtin_bit_cast(uint8_t __attribute__((ext_vector_type(4))), quantise8<T>(v[i], scale));
        uint8_t *const to = codes + row * a.codes.row;
        if (bytes >= 4) *(wide<uint8_t, 4> *)to = code;
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < bytes) to[e] = code[e];
        if (p.col % 32 == 0) scales[row * a.scales.row] = (uint8_t)scale;
    }
}

template <typename T>
__device__ __forceinline__ wide<T, kBackPiece<T>> expand_piece(uint32_t code, uint32_t scale) {
    const float by = __builtin_bit_cast(float, scale << 23);
    if constexpr (sizeof(T) == 2) {
        const bf2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, by, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, by, 1),
                  c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, by, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, by, 3);
        return wide<T, 8>{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, by, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, by, 1);
        return wide<T, 4>{a[0], a[1], b[0], b[1]};
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_mx4_dequantise(aet_mx4_codes a, Mx4Shape s) {
    constexpr int ROWS = 4, V = kBackPiece<T>;
    Mx4Place p;
    if (!place_of<V, ROWS>(s, p) || p.col >= a.cols) return;
    const uint8_t *codes = (const uint8_t *)a.codes.p + p.client * a.codes.client + p.col / 2;
    const uint8_t *scales = (const uint8_t *)a.scales.p + p.client * a.scales.client + p.col / 32;
    T *y = (T *)a.y.p + p.client * a.y.client + p.col;
    const int count = a.cols - p.col, bytes = (count + 1) / 2;
    uint32_t code[ROWS], scale[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t row = p.row0 + i * p.high;
        if (row >= a.rows) continue;
        const uint8_t *from = codes + row * a.codes.row;
        code[i] = 0;
        if (bytes >= V / 2) {
            const wide<uint8_t, V / 2> all = *(const wide<uint8_t, V / 2> *)from;
#pragma unroll
            for (int e = 0; e < V / 2; ++e) code[i] |= (uint32_t)all[e] << (8 * e);
        } else {
#pragma unroll
            for (int e = 0; e < V / 2; ++e) code[i] |= (uint32_t)from[e < bytes ? e : bytes - 1] << (8 * e);
        }
        scale[i] = scales[row * a.scales.row];
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t row = p.row0 + i * p.high;
        if (row >= a.rows) continue;
        const wide<T, V> v = expand_piece<T>(code[i], scale[i]);
        T *const to = y + row * a.y.row;
        if (count >= V) *(wide<T, V> *)to = v;
        else
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < count) to[e] = v[e];
    }
}

static bool shape_of(int64_t n, int64_t rows, int64_t cols, int piece, int each, Mx4Shape *s, int64_t *blocks) {
    *s = {(int)ceil_div(cols, 32) * (32 / piece), 32 / piece, 0, 0};
    while (s->wide < s->pieces && s->wide < 256) s->wide *= 2;
    s->across = ceil_div(s->pieces, s->wide);
    s->down = ceil_div(rows, 256 / s->wide * each);
    *blocks = n * s->across * s->down;
    return grid_fits(*blocks, 256);
}
template <typename T>
static hipError_t quantise(const aet_mx4_values &a, hipStream_t s) {
    Mx4Shape d;
    int64_t blocks;
    if (!shape_of(a.n, a.rows, a.cols, 8, kToRows<T>, &d, &blocks)) return hipErrorInvalidConfiguration;
    k_mx4_quantise<T><<<(int)blocks, 256, 0, s>>>(a, d);
    return hipGetLastError();
}
template <typename T>
static hipError_t dequantise(const aet_mx4_codes &a, hipStream_t s) {
    Mx4Shape d;
    int64_t blocks;
    if (!shape_of(a.n, a.rows, a.cols, kBackPiece<T>, 4, &d, &blocks)) return hipErrorInvalidConfiguration;
    k_mx4_dequantise<T><<<(int)blocks, 256, 0, s>>>(a, d);
    return hipGetLastError();
}
hipError_t launch_mx4_quantise(const aet_mx4_values &a, hipStream_t s) { return a.dtype == AET_F32 ? quantise<float>(a, s) : quantise<bf16>(a, s); }
hipError_t launch_mx4_dequantise(const aet_mx4_codes &a, hipStream_t s) { return a.dtype == AET_F32 ? dequantise<float>(a, s) : dequantise<bf16>(a, s); }

// ---- the linear layer --------------------------------------------------------------------

static HeldProduct forward_product(const aet_mx4_linear &a) {
    HeldProduct p = {{a.x, a.x_scales}, {a.w, a.w_scales}, a.n, a.rows, a.out, a.in};
    p.e = {a.bias, a.residual, a.y, a.pre, a.rows, a.act, make_drop(a.p, a.seed, a.first_row, a.out)};
    return p;
}
size_t mx4_linear_forward_workspace(const aet_mx4_linear &a) { return mx4_product_workspace(forward_product(a)); }
hipError_t launch_mx4_linear_forward(const aet_mx4_linear &a, void *workspace, hipStream_t s) {
    return launch_mx4_product(a.dtype, forward_product(a), workspace, s);
}

}  // namespace aet_ops
