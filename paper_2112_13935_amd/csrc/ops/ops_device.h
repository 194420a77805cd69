// Device-side helpers of the operators: values in fp32 and bf16, activations, the dropout's mask.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../aet_device.h"
#include "aet_ops.h"

namespace aet_ops {

typedef __bf16 bf16;
typedef bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));

// V values in memory, in one wide access whatever their alignment beyond the type's own.
template <typename T, int V>
struct Wide {
    typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <typename T, int V>
using wide = typename Wide<T, V>::type;

// The first count (may be below 0, or V and more) of V values; the rest are 0.
template <typename T, int V>
__device__ __forceinline__ wide<T, V> load_raw(const T *p, int count) {
    if (count >= V) return *(const wide<T, V> *)p;
    wide<T, V> v = {};
    if (count > 0) {   // all loads at once: what is past the end is the last one again, and then 0
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = p[i < count ? i : count - 1];
#pragma unroll
        for (int i = 1; i < V; ++i) v[i] = i < count ? v[i] : (T)0.0f;
    }
    return v;
}
template <typename T, int V>
__device__ __forceinline__ void load_some(const T *p, int count, float (&v)[V]) {
    const wide<T, V> raw = load_raw<T, V>(p, count);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)raw[i];
}
// One rounding, to nearest even.
template <typename T, int V>
__device__ __forceinline__ void store_some(T *p, int count, const float (&v)[V]) {
    if (count >= V) {
        wide<T, V> raw;
#pragma unroll
        for (int i = 0; i < V; ++i) raw[i] = (T)v[i];
        *(wide<T, V> *)p = raw;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < count) p[i] = (T)v[i];
    }
}

// Workgroups go to the XCDs in turn: the order that gives each XCD consecutive ones, so that what they share meets in its L2.
__device__ __forceinline__ int xcd_order(int id, int blocks) {
    const int q = blocks / 8, r = blocks % 8, x = id % 8;
    return x * q + (x < r ? x : r) + id / 8;
}

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// Phi(z) and exp(-z^2 / 2).  With u = |z| / sqrt(2) the tail is erfc(u) / 2 = (b1 t + ... + b8 t^8) exp(-u^2), t = 1 / (1 + 0.6 u),
// which is the form of Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26, three terms longer; the b are a
// least-squares fit to exp(u^2) erfc(u) / 2 over u = 0 to 10, weighted towards an even error.  It is within 1e-8, and 8e-6
// of itself down to z = -5.  GELU of N(0, 1) in fp32: relative 2-norm 3.6e-8, its slope 5.0e-8; with an exact erf in fp32 3.8e-8 and 3.9e-8,
// with that formula's five terms 8.5e-8 and 1.0e-7.
__device__ __forceinline__ float normal_cdf(float z, float &e) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.42426407f, __builtin_fabsf(z), 1.0f));
    float s = __builtin_fmaf(t, -0.0266033318f, 0.115691967f);
    s = __builtin_fmaf(t, s, -0.146613598f);
    s = __builtin_fmaf(t, s, -0.0431476533f);
    s = __builtin_fmaf(t, s, 0.150449857f);
    s = __builtin_fmaf(t, s, 0.105136529f);
    s = __builtin_fmaf(t, s, 0.17642127f);
    s = __builtin_fmaf(t, s, 0.168664962f);
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
    const float tail = t * s * e;
    return z < 0 ? tail : 1.0f - tail;
}

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == AET_ACT_RELU) return z <= 0 ? 0.0f : z;
    if constexpr (ACT == AET_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + exp_fast(-z));
    if constexpr (ACT == AET_ACT_GELU) {
        float e;
        return z * normal_cdf(z, e);
    }
    return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == AET_ACT_RELU) return z > 0 ? 1.0f : 0.0f;
    if constexpr (ACT == AET_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + exp_fast(-z));
        return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
    }
    if constexpr (ACT == AET_ACT_GELU) {
        float e;
        const float c = normal_cdf(z, e);
        return __builtin_fmaf(z * 0.39894228f, e, c);
    }
    return 1.0f;
}

template <int ACT, int V>
__device__ __forceinline__ void act_each(float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = act_value<ACT>(v[i]);
}
template <int V>
__device__ __forceinline__ void act_each(int act, float (&v)[V]) {
    switch (act) {
    case AET_ACT_RELU: act_each<AET_ACT_RELU>(v); break;
    case AET_ACT_SILU: act_each<AET_ACT_SILU>(v); break;
    case AET_ACT_GELU: act_each<AET_ACT_GELU>(v); break;
    default: break;
    }
}
// v times the slope at z
template <int ACT, int V>
__device__ __forceinline__ void slope_each(const float (&z)[V], float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= act_slope<ACT>(z[i]);
}
template <int V>
__device__ __forceinline__ void slope_each(int act, const float (&z)[V], float (&v)[V]) {
    switch (act) {
    case AET_ACT_RELU: slope_each<AET_ACT_RELU>(z, v); break;
    case AET_ACT_SILU: slope_each<AET_ACT_SILU>(z, v); break;
    case AET_ACT_GELU: slope_each<AET_ACT_GELU>(z, v); break;
    default: break;
    }
}

// The dropout of a call: rows of `half` counters.
struct Drop {
    uint64_t key;      // of the stream
    uint64_t first;    // counter of the first row's first pair
    uint64_t half;     // ceil(cols / 2)
    uint32_t least;    // a value stays where its half of the hash is no less; 0: everything stays
    float scale;
};
__device__ __forceinline__ uint64_t drop_row(const Drop &d, int64_t row) { return d.first + (uint64_t)row * d.half; }
// The hash of columns 2 j (lower half) and 2 j + 1 (upper half) of the row whose counters begin at q.
__device__ __forceinline__ uint64_t drop_hash(const Drop &d, uint64_t q, int j) {
    return aet::splitmix_at(d.key, q + (uint32_t)j);
}
// v[i]: columns col .. col + V - 1, col even
template <int V>
__device__ __forceinline__ void drop_apply(const Drop &d, uint64_t q, int col, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        const uint64_t h = drop_hash(d, q, (col + i) >> 1);
        v[i] = (uint32_t)h >= d.least ? v[i] * d.scale : 0.0f;
        v[i + 1] = (uint32_t)(h >> 32) >= d.least ? v[i + 1] * d.scale : 0.0f;
    }
}

// The same, col odd or even: a hash more.
template <int V>
__device__ __forceinline__ void drop_apply_any(const Drop &d, uint64_t q, int col, float (&v)[V]) {
    const uint32_t odd = -(uint32_t)(col & 1);
    uint32_t half[V + 2];
#pragma unroll
    for (int i = 0; i < V + 2; i += 2) {
        const uint64_t h = drop_hash(d, q, (col + i) >> 1);
        half[i] = (uint32_t)h;
        half[i + 1] = (uint32_t)(h >> 32);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t u = (odd & half[i + 1]) | (~odd & half[i]);   // (a choice of an array's element would put it in memory)
        v[i] = u >= d.least ? v[i] * d.scale : 0.0f;
    }
}

}  // namespace aet_ops
