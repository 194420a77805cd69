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

// Values from memory that is aligned to their type only: one wide access all the same.
template <typename T>
struct Wide {
    typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
    const auto raw = *(const typename Wide<T>::type *)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)raw[i];
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    typename Wide<T>::type raw;
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = (T)v[i];
    *(typename Wide<T>::type *)p = raw;
}
// The first count (1 to 8) of 8 values; the rest are 0.
template <typename T>
__device__ __forceinline__ void load_some(const T *p, int count, float (&v)[8]) {
    if (count >= 8) {
        load8(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? (float)p[i] : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store_some(T *p, int count, const float (&v)[8]) {
    if (count >= 8) {
        store8(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = (T)v[i];
    }
}

template <int ACT>
__device__ __forceinline__ void act8(float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_value<ACT>(v[i]);
}
__device__ __forceinline__ void act8(int act, float (&v)[8]) {
    switch (act) {
    case AET_ACT_RELU: act8<AET_ACT_RELU>(v); break;
    case AET_ACT_SILU: act8<AET_ACT_SILU>(v); break;
    case AET_ACT_GELU: act8<AET_ACT_GELU>(v); break;
    default: break;
    }
}
template <int ACT>
__device__ __forceinline__ void slope8(const float (&z)[8], float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= act_slope<ACT>(z[i]);
}
__device__ __forceinline__ void slope8(int act, const float (&z)[8], float (&v)[8]) {
    switch (act) {
    case AET_ACT_RELU: slope8<AET_ACT_RELU>(z, v); break;
    case AET_ACT_SILU: slope8<AET_ACT_SILU>(z, v); break;
    case AET_ACT_GELU: slope8<AET_ACT_GELU>(z, v); break;
    default: break;
    }
}

// Columns col .. col + count - 1 (col a multiple of 8, count 1 to 8) of a client's row; v: the sums plus bias.
template <typename T>
__device__ __forceinline__ void finish8(const Epilogue &e, int64_t client, int64_t row, int col, int count, float (&v)[8]) {
    if (e.pre.p) store_some((T *)e.pre.p + client * e.pre.client + row * e.pre.row + col, count, v);
    act8(e.act, v);
    if (e.d.least) drop_apply<8>(e.d, drop_row(e.d, client * e.rows + row), col, v);
    if (e.residual.p) {
        float r[8];
        load_some((const T *)e.residual.p + client * e.residual.client + row * e.residual.row + col, count, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    store_some((T *)e.y.p + client * e.y.client + row * e.y.row + col, count, v);
}
template <typename T>
__device__ __forceinline__ void bias8(const Epilogue &e, int64_t client, int col, int count, float (&b)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = 0.0f;
    if (e.bias.p && count > 0) load_some((const T *)e.bias.p + client * e.bias.client + col, count, b);
}

}  // namespace aet_ops
