// Group normalisation with an activation, channels last, and its gradient.
#include "ops_internal.h"

namespace aet_ops {

__device__ __forceinline__ float block_sum(float v, float *lds) {   // 256 threads
    v = aet::wave_sum(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

// One workgroup per sample and group.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_norm(aet_group_norm a) {
    __shared__ float lds[4];
    const int64_t sample = blockIdx.x / a.groups;
    const int g = blockIdx.x % a.groups;
    const int64_t c = sample / a.batch, b = sample % a.batch;
    const T *x = (const T *)a.x.p + c * a.x.client + b * a.x.sample + g * a.width;
    T *y = (T *)a.y.p + c * a.y.client + b * a.y.sample + g * a.width;
    const int64_t count = (int64_t)a.positions * a.width;
    float s = 0;
    for (int64_t i = threadIdx.x; i < count; i += 256) s += (float)x[i / a.width * a.x.row + i % a.width];
    const float mean = count ? block_sum(s, lds) / (float)count : 0.0f;
    s = 0;
    for (int64_t i = threadIdx.x; i < count; i += 256) {
        const float d = (float)x[i / a.width * a.x.row + i % a.width] - mean;
        s += d * d;
    }
    const float rstd = 1.0f / __builtin_sqrtf((count ? block_sum(s, lds) / (float)count : 0.0f) + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[blockIdx.x] = mean;
        if (a.rstd) a.rstd[blockIdx.x] = rstd;
    }
    for (int64_t i = threadIdx.x; i < count; i += 256) {
        const int k = (int)(i % a.width), ch = g * a.width + k;
        const float gamma = a.gamma.p ? (float)((const T *)a.gamma.p)[c * a.gamma.client + ch] : 1.0f;
        const float beta = a.beta.p ? (float)((const T *)a.beta.p)[c * a.beta.client + ch] : 0.0f;
        const float t = ((float)x[i / a.width * a.x.row + k] - mean) * rstd * gamma + beta;
        y[i / a.width * a.y.row + k] = (T)act_value<ACT>(t);
    }
}

// One workgroup per sample and group; sums: A and B of each sample and channel.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_norm_back(aet_group_norm_grad a, float *sums) {
    __shared__ float lds[4];
    const int64_t sample = blockIdx.x / a.groups;
    const int g = blockIdx.x % a.groups;
    const int64_t c = sample / a.batch, b = sample % a.batch;
    const int64_t C = (int64_t)a.groups * a.width;
    const T *x = (const T *)a.x.p + c * a.x.client + b * a.x.sample + g * a.width;
    const T *dy = (const T *)a.dy.p + c * a.dy.client + b * a.dy.sample + g * a.width;
    const float mean = a.mean[blockIdx.x], rstd = a.rstd[blockIdx.x];
    float s1 = 0, s2 = 0;
    for (int k = 0; k < a.width; ++k) {
        const int ch = g * a.width + k;
        const float gamma = a.gamma.p ? (float)((const T *)a.gamma.p)[c * a.gamma.client + ch] : 1.0f;
        const float beta = a.beta.p ? (float)((const T *)a.beta.p)[c * a.beta.client + ch] : 0.0f;
        float A = 0, B = 0;
        for (int i = threadIdx.x; i < a.positions; i += 256) {
            const float xh = ((float)x[i * a.x.row + k] - mean) * rstd;
            const float d = (float)dy[i * a.dy.row + k] * act_slope<ACT>(xh * gamma + beta);
            A += d;
            B += d * xh;
        }
        A = block_sum(A, lds);
        B = block_sum(B, lds);
        s1 += gamma * A;
        s2 += gamma * B;
        if (threadIdx.x == 0) {
            sums[(sample * 2 + 0) * C + ch] = A;
            sums[(sample * 2 + 1) * C + ch] = B;
        }
    }
    if (!a.dx.p) return;
    T *dx = (T *)a.dx.p + c * a.dx.client + b * a.dx.sample + g * a.width;
    const int64_t count = (int64_t)a.positions * a.width;
    s1 /= (float)count;
    s2 /= (float)count;
    for (int64_t i = threadIdx.x; i < count; i += 256) {
        const int k = (int)(i % a.width), ch = g * a.width + k;
        const int64_t pos = i / a.width;
        const float gamma = a.gamma.p ? (float)((const T *)a.gamma.p)[c * a.gamma.client + ch] : 1.0f;
        const float beta = a.beta.p ? (float)((const T *)a.beta.p)[c * a.beta.client + ch] : 0.0f;
        const float xh = ((float)x[pos * a.x.row + k] - mean) * rstd;
        const float d = (float)dy[pos * a.dy.row + k] * act_slope<ACT>(xh * gamma + beta) * gamma;
        dx[pos * a.dx.row + k] = (T)((d - s1 - xh * s2) * rstd);
    }
}

// One thread per client and channel.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_params(aet_group_norm_grad a, const float *sums, int clients, int64_t samples) {
    const int64_t C = (int64_t)a.groups * a.width, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= clients * C) return;
    const int64_t c = i / C, ch = i % C;
    float A = 0, B = 0;
    for (int64_t k = c * samples; k < (c + 1) * samples; ++k) {
        A += sums[(k * 2 + 0) * C + ch];
        B += sums[(k * 2 + 1) * C + ch];
    }
    if (a.dbeta.p) ((T *)a.dbeta.p)[c * a.dbeta.client + ch] = (T)A;
    if (a.dgamma.p) ((T *)a.dgamma.p)[c * a.dgamma.client + ch] = (T)B;
}

size_t group_norm_forward_workspace(const aet_group_norm &) { return 0; }
size_t group_norm_backward_workspace(const aet_group_norm_grad &a) {
    return a.positions ? (size_t)a.n * a.batch * 2 * a.groups * a.width * sizeof(float) : 0;
}

template <typename T>
static void norm(const aet_group_norm &a, hipStream_t s, int blocks) {
    switch (a.act) {
    case AET_ACT_RELU: k_norm<T, AET_ACT_RELU><<<blocks, 256, 0, s>>>(a); break;
    case AET_ACT_SILU: k_norm<T, AET_ACT_SILU><<<blocks, 256, 0, s>>>(a); break;
    case AET_ACT_GELU: k_norm<T, AET_ACT_GELU><<<blocks, 256, 0, s>>>(a); break;
    default: k_norm<T, AET_ACT_NONE><<<blocks, 256, 0, s>>>(a);
    }
}
hipError_t launch_group_norm_forward(const aet_group_norm &a, void *, hipStream_t s) {
    const int64_t blocks = (int64_t)a.n * a.batch * a.groups;
    if (blocks > INT32_MAX) return hipErrorInvalidConfiguration;
    a.dtype == AET_F32 ? norm<float>(a, s, (int)blocks) : norm<bf16>(a, s, (int)blocks);
    return hipGetLastError();
}

template <typename T>
static void norm_back(const aet_group_norm_grad &a, float *sums, hipStream_t s, int blocks) {
    if (blocks) switch (a.act) {
    case AET_ACT_RELU: k_norm_back<T, AET_ACT_RELU><<<blocks, 256, 0, s>>>(a, sums); break;
    case AET_ACT_SILU: k_norm_back<T, AET_ACT_SILU><<<blocks, 256, 0, s>>>(a, sums); break;
    case AET_ACT_GELU: k_norm_back<T, AET_ACT_GELU><<<blocks, 256, 0, s>>>(a, sums); break;
    default: k_norm_back<T, AET_ACT_NONE><<<blocks, 256, 0, s>>>(a, sums);
    }
    if (!a.dgamma.p && !a.dbeta.p) return;
    const bool shared = (a.dgamma.p && !a.dgamma.client) || (a.dbeta.p && !a.dbeta.client);
    const int clients = shared ? 1 : a.n;
    const int64_t samples = blocks ? (int64_t)a.batch * (shared ? a.n : 1) : 0;
    k_norm_params<T><<<(int)ceil_div((int64_t)clients * a.groups * a.width, 256), 256, 0, s>>>(a, sums, clients, samples);
}
hipError_t launch_group_norm_backward(const aet_group_norm_grad &a, void *workspace, hipStream_t s) {
    const int64_t blocks = a.positions ? (int64_t)a.n * a.batch * a.groups : 0;
    if (blocks > INT32_MAX) return hipErrorInvalidConfiguration;
    a.dtype == AET_F32 ? norm_back<float>(a, (float *)workspace, s, (int)blocks) : norm_back<bf16>(a, (float *)workspace, s, (int)blocks);
    return hipGetLastError();
}

}  // namespace aet_ops
