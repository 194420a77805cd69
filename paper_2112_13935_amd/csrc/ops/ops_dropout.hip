// Dropout: y = residual + mask * x / (1 - p), the mask from the counter generator.
#include "ops_internal.h"

namespace aet_ops {

// One value a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_dropout(aet_dropout a, Drop d) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = i / a.cols;
    if (row >= (int64_t)a.n * a.rows) return;
    const int col = (int)(i - row * a.cols);
    const int64_t c = row / a.rows, r = row - c * a.rows;
    float v[1] = {(float)((const T *)a.x.p)[c * a.x.client + r * a.x.row + col]};
    if (d.least) drop_apply(d, drop_row(d, row), col, v);
    if (a.residual.p) v[0] += (float)((const T *)a.residual.p)[c * a.residual.client + r * a.residual.row + col];
    ((T *)a.y.p)[c * a.y.client + r * a.y.row + col] = (T)v[0];
}

hipError_t launch_dropout(const aet_dropout &a, hipStream_t s) {
    const Drop d = make_drop(a.p, a.seed, a.first_row, a.cols);
    const int64_t blocks = ceil_div((int64_t)a.n * a.rows * a.cols, 256);
    if (blocks > INT32_MAX) return hipErrorInvalidConfiguration;
    if (a.dtype == AET_F32) k_dropout<float><<<(int)blocks, 256, 0, s>>>(a, d);
    else k_dropout<bf16><<<(int)blocks, 256, 0, s>>>(a, d);
    return hipGetLastError();
}

}  // namespace aet_ops
