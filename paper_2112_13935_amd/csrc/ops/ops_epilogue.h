// What becomes of a sum of products of the linear layer: bias, activation, dropout, residual, and the stores.
#pragma once
#include "ops_device.h"

namespace aet_ops {

// Also the gradients' products, which have none of them (act none, pointers NULL).
struct Epilogue {
    aet_in bias, residual;
    aet_out y, pre;
    int64_t rows;   // of a client, for the dropout's row numbers
    int act;
    Drop d;
};

// Columns col .. col + count - 1 (col a multiple of V, count 1 to V) of a client's row; v: the sums plus bias.
template <typename T, int V>
__device__ __forceinline__ void finish(const Epilogue &e, int64_t client, int64_t row, int col, int count, float (&v)[V]) {
    if (e.pre.p) store_some((T *)e.pre.p + client * e.pre.client + row * e.pre.row + col, count, v);
    act_each(e.act, v);
    if (e.d.least) drop_apply(e.d, drop_row(e.d, client * e.rows + row), col, v);
    if (e.residual.p) {
        float r[V];
        load_some((const T *)e.residual.p + client * e.residual.client + row * e.residual.row + col, count, r);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += r[i];
    }
    store_some((T *)e.y.p + client * e.y.client + row * e.y.row + col, count, v);
}
template <typename T, int V>
__device__ __forceinline__ void bias_of(const Epilogue &e, int64_t client, int col, int count, float (&b)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = 0.0f;
    if (e.bias.p && count > 0) load_some((const T *)e.bias.p + client * e.bias.client + col, count, b);
}

}  // namespace aet_ops
