// Dropout: y = residual + mask * x / (1 - p), the mask from the counter generator.
//
// Bound by memory: a value is read (with the residual, two) and written once.  A thread has 16 bytes of kRows rows, all
// of them on their way before the first is worked on; a hash decides two columns, which is 3 of the unit's slow 32-bit
// multiplications a value.  16384 x 4096 in bf16 with a residual: 75 us, 5.3 TB/s (a copy of as much: 80).
#include "ops_internal.h"

namespace aet_ops {

constexpr int kRows = 4;

struct DropShape {
    int pieces, wide;         // pieces of V columns in a row; threads side by side (a power of two)
    int64_t across, down;     // workgroups: of a row of pieces, of a client
};

template <typename T, int V>
__global__ __launch_bounds__(256) void k_dropout(aet_dropout a, Drop d, DropShape s) {
    const int64_t per = s.across * s.down;
    const int64_t client = blockIdx.x / per, b = blockIdx.x % per;
    const int piece = (int)(b % s.across) * s.wide + (threadIdx.x & (s.wide - 1));
    const int high = 256 / s.wide;   // rows side by side
    const int64_t row0 = b / s.across * (high * kRows) + threadIdx.x / s.wide;
    if (piece >= s.pieces) return;
    const int col = piece * V, count = a.cols - col;
    const T *x = (const T *)a.x.p + client * a.x.client + col;
    const T *res = a.residual.p ? (const T *)a.residual.p + client * a.residual.client + col : nullptr;
    T *y = (T *)a.y.p + client * a.y.client + col;
    wide<T, V> v[kRows], r[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t row = row0 + i * high;
        if (row >= a.rows) continue;
        v[i] = load_raw<T, V>(x + row * a.x.row, count);
        if (res) r[i] = load_raw<T, V>(res + row * a.residual.row, count);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t row = row0 + i * high;
        if (row >= a.rows) continue;
        float f[V];
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = (float)v[i][e];
        if (d.least) drop_apply(d, drop_row(d, client * a.rows + row), col, f);
        if (res) {
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] += (float)r[i][e];
        }
        store_some(y + row * a.y.row, count, f);
    }
}

template <typename T>
static hipError_t run(const aet_dropout &a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    DropShape d = {(int)ceil_div(a.cols, V), 1, 0, 0};
    while (d.wide < d.pieces && d.wide < 256) d.wide *= 2;
    d.across = ceil_div(d.pieces, d.wide);
    d.down = ceil_div(a.rows, 256 / d.wide * kRows);
    const int64_t blocks = a.n * d.across * d.down;
    if (blocks > INT32_MAX) return hipErrorInvalidConfiguration;
    k_dropout<T, V><<<(int)blocks, 256, 0, s>>>(a, make_drop(a.p, a.seed, a.first_row, a.cols), d);
    return hipGetLastError();
}

hipError_t launch_dropout(const aet_dropout &a, hipStream_t s) {
    return a.dtype == AET_F32 ? run<float>(a, s) : run<bf16>(a, s);
}

}  // namespace aet_ops
