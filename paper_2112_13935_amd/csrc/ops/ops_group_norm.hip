// Group normalisation with an activation, channels last, and its gradient.
//
// Bound by memory.  A thread has V neighbouring channels (16 bytes) of several positions, whatever groups they belong to;
// sums are kept by channel and come together by group in the end, so that memory is read in whole lines also where
// a group has few channels.  Where a sample's groups fit the registers of a workgroup, one kernel reads every value once
// (k_norm_whole, k_norm_back_whole): mean first, then the squares of the differences from it.  Larger samples take
// three: sums of strips of positions, their union by group, and a second pass over the values.
//   2048 samples of 1024 x 32 in fp32, groups of 4 channels, silu: 122 us (537 MB, 4.4 TB/s; a copy of as much 107)
//   gradient of 128 samples of 4096 x 320 in bf16, groups of 10: 328 us: sums 156 (671 MB read, 4.3 TB/s), union 9, second
//   pass 175 (1.0 GB, 5.8 TB/s); reading the values once would be 201, but four groups, the least of whole 64 bytes, are 655 KB of x
//   and dy, and a compute unit's registers 512
#include "ops_internal.h"

#include <type_traits>

namespace aet_ops {

constexpr int kThreads = 512;

// How a sample is dealt out.  A workgroup has `span` channels (the last of a sample: what is left), in `pieces` of V.
struct NormShape {
    int channels, span, spans, span_groups;
    int pieces, lanes;      // threads side by side; positions at a time
    int threads;            // pieces * lanes, in whole waves
    int strips, strip;      // positions' parts: for the sums (three kernels only)
    int parts, part;        // and for the second pass
    float *sums;            // whole: [sample][2][channels]; else [sample][strips][2][channels]
    float *stats;           // [sample][2][groups], three kernels only: mean and rstd; or s1 rstd and s2 rstd^2, s1 and s2 over the number of values
};

struct Where {
    int64_t sample, client, in_batch;
    int ch0, chans, piece, lane, count;   // count: how many channels the thread has
    // A thread reads V values from channel `ch` on, of which [lo, lo + count) are its own: where fewer are left it reads
    // neighbours' too, or begins earlier, so that nobody has to look where pieces end.  (Samples of fewer channels than V
    // have count values from ch on.)
    int ch, lo;
    int group[8];                         // of the channels read
};
// ODD: some pieces are not whole.  (Compiled apart: 2 to 3 % where all are.)
template <int V, bool ODD>
__device__ __forceinline__ Where where(const NormShape &s, int batch, int width, uint32_t block) {
    Where w;
    const uint32_t sample = block / (uint32_t)s.spans, client = sample / (uint32_t)batch;
    w.sample = sample;
    w.ch0 = (int)(block - sample * (uint32_t)s.spans) * s.span;
    w.chans = s.channels - w.ch0 < s.span ? s.channels - w.ch0 : s.span;
    w.client = client;
    w.in_batch = sample - client * (uint32_t)batch;
    w.lane = threadIdx.x / (uint32_t)s.pieces;
    w.piece = threadIdx.x - w.lane * s.pieces;
    const int own = w.ch0 + w.piece * V;
    w.count = w.lane < s.lanes ? w.chans - w.piece * V : 0;
    if (w.count > V) w.count = V;
    w.ch = !ODD || s.channels < V || own + V <= s.channels ? own : s.channels - V;
    w.lo = own - w.ch;
    // (channels of other workgroups have the group of one that is here, so that nothing has to be tested to read what it has)
    int g = w.ch / width, k = w.ch - g * width;
    const int first = w.ch0 / width, last = (w.ch0 + w.chans - 1) / width;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        w.group[e] = g < first ? first : g < last ? g : last;
        if (++k == width) {
            k = 0;
            ++g;
        }
    }
    return w;
}

// Sums by channel over the workgroup's threads, of N arrays at a time: tot[n * span + k], k < chans.  lds: N * threads * V
// floats.  First within waves where a wave has whole rows of pieces, then by halving the rows until two are left.
template <bool ODD, int V, int N>
__device__ __forceinline__ void channel_sums(const NormShape &s, const Where &w, float (&v)[N][V], float *lds, float *tot) {
    const int line = s.pieces * V, all = s.threads * V;
    int rows = s.lanes, row = w.lane;
    if (ODD && w.count < V) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < w.lo || e >= w.lo + w.count) v[n][e] = 0.0f;
    }
    bool mine = w.lane < s.lanes;
    if (s.pieces < 64 && !(s.pieces & (s.pieces - 1))) {   // (threads without a position have zeros)
        for (int off = 32; off >= s.pieces; off >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < V; ++e) v[n][e] += __shfl_xor(v[n][e], off, 64);
        rows = s.threads / 64;
        row = threadIdx.x / 64;
        mine = threadIdx.x % 64 < s.pieces;
    }
    __syncthreads();
    if (mine && (!ODD || w.lo == 0)) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < V; e += 4)
                *(f4 *)(lds + n * all + row * line + w.piece * V + e) = f4{v[n][e], v[n][e + 1], v[n][e + 2], v[n][e + 3]};
    } else if (ODD && mine) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e >= w.lo) lds[n * all + row * line + w.piece * V + e - w.lo] = v[n][e];
    }
    __syncthreads();
    while (rows > 2) {
        const int half = (rows + 1) / 2, count = (rows - half) * line;
        for (int i = threadIdx.x; i < count; i += blockDim.x)
#pragma unroll
            for (int n = 0; n < N; ++n) lds[n * all + i] += lds[n * all + half * line + i];
        __syncthreads();
        rows = half;
    }
    for (int k = threadIdx.x; k < w.chans; k += blockDim.x)
#pragma unroll
        for (int n = 0; n < N; ++n) tot[n * s.span + k] = lds[n * all + k] + (rows > 1 ? lds[n * all + line + k] : 0.0f);
    __syncthreads();
}
// Sums of a group's channels, a wave per group: out[g] = scale * sum of tot[k] (* by[k])
__device__ __forceinline__ void group_sums(const float *tot, const float *by, int groups, int width, float scale, float *out) {
    const int waves = blockDim.x / 64, lane = threadIdx.x % 64;
    for (int g = threadIdx.x / 64; g < groups; g += waves) {
        float sum = 0;
        for (int k = lane; k < width; k += 64) sum += by ? tot[g * width + k] * by[g * width + k] : tot[g * width + k];
        sum = aet::wave_sum(sum);
        if (lane == 0) out[g] = sum * scale;
    }
    __syncthreads();
}

// The thread's V values of a row (count: V, or fewer in samples of fewer channels), and its own of them to their places.
template <int V, bool ODD>
__device__ __forceinline__ int to_read(const NormShape &s, const Where &w) { return w.count <= 0 ? 0 : ODD && s.channels < V ? w.count : V; }
template <bool ODD, typename T, int V>
__device__ __forceinline__ void store_own(T *p, const Where &w, const float (&v)[V]) {
    if (!ODD || w.count == V) {
        store_some(p, V, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e >= w.lo && e < w.lo + w.count) p[e] = (T)v[e];
    }
}

template <typename T, int V>
__device__ __forceinline__ void params(const aet_in &p, int64_t client, int ch, int count, float none, float (&v)[V]) {
    if (p.p && count > 0) {
        load_some((const T *)p.p + client * p.client + ch, count, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = none;
    }
}
// from[group of the thread's channel - first]
template <int V>
__device__ __forceinline__ void by_channel(const Where &w, int first, const float *from, float (&v)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = from[w.group[e] - first];
}

// ---- a sample's groups in registers ------------------------------------------------------

template <typename T, int V, int N, bool ODD>
__global__ __launch_bounds__(kThreads) void k_norm_whole(aet_group_norm a, NormShape s) {
    extern __shared__ float lds[];   // threads * V, then by channel, then by group
    float *const tot = lds + s.threads * V, *const stat = tot + s.span;
    const Where w = where<V, ODD>(s, a.batch, a.width, xcd_order(blockIdx.x, gridDim.x));
    const T *x = (const T *)a.x.p + w.client * a.x.client + w.in_batch * a.x.sample + w.ch;
    T *y = (T *)a.y.p + w.client * a.y.client + w.in_batch * a.y.sample + w.ch;
    wide<T, V> raw[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int pos = w.lane + i * s.lanes;
        raw[i] = load_raw<T, V>(x + pos * a.x.row, pos < a.positions ? to_read<V, ODD>(s, w) : 0);
    }
    float gamma[V], beta[V];
    params<T>(a.gamma, w.client, w.ch, to_read<V, ODD>(s, w), 1.0f, gamma);
    params<T>(a.beta, w.client, w.ch, to_read<V, ODD>(s, w), 0.0f, beta);
    float acc[1][V] = {};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[0][e] += (float)raw[i][e];
    const int groups = w.chans / a.width, g0 = w.ch0 / a.width;
    const float inv = 1.0f / ((float)a.positions * (float)a.width);
    channel_sums<ODD>(s, w, acc, lds, tot);
    group_sums(tot, nullptr, groups, a.width, inv, stat);
    float mean[V], scale[V];
    by_channel(w, g0, stat, mean);
#pragma unroll
    for (int e = 0; e < V; ++e) acc[0][e] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (w.lane + i * s.lanes < a.positions) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = (float)raw[i][e] - mean[e];
                acc[0][e] += d * d;
            }
        }
    channel_sums<ODD>(s, w, acc, lds, tot);
    if (a.mean)
        for (int g = threadIdx.x; g < groups; g += blockDim.x) a.mean[w.sample * a.groups + g0 + g] = stat[g];
    __syncthreads();
    group_sums(tot, nullptr, groups, a.width, inv, stat);
    for (int g = threadIdx.x; g < groups; g += blockDim.x) {
        stat[g] = 1.0f / __builtin_sqrtf(stat[g] + a.eps);
        if (a.rstd) a.rstd[w.sample * a.groups + g0 + g] = stat[g];
    }
    __syncthreads();
    by_channel(w, g0, stat, scale);
#pragma unroll
    for (int e = 0; e < V; ++e) scale[e] *= gamma[e];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int pos = w.lane + i * s.lanes;
        if (pos >= a.positions || w.count <= 0) continue;
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = __builtin_fmaf((float)raw[i][e] - mean[e], scale[e], beta[e]);
        act_each(a.act, v);
        store_own<ODD>(y + pos * a.y.row, w, v);
    }
}

// d = dy * act'(t) and xm = x - mean at one position; scale: rstd * gamma
template <typename T, int V>
__device__ __forceinline__ void slopes(int act, const wide<T, V> &x, const wide<T, V> &dy, const float (&mean)[V], const float (&scale)[V],
                                       const float (&beta)[V], float (&d)[V], float (&xm)[V]) {
    float t[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        xm[e] = (float)x[e] - mean[e];
        t[e] = __builtin_fmaf(xm[e], scale[e], beta[e]);
        d[e] = (float)dy[e];
    }
    slope_each(act, t, d);
}
// What a thread's channels need for it.
template <bool ODD, typename T, int V>
__device__ __forceinline__ void slope_params(const aet_group_norm_grad &a, const NormShape &s, const Where &w, float (&mean)[V], float (&scale)[V], float (&beta)[V]) {
    float rstd[V];
    by_channel(w, 0, a.mean + w.sample * a.groups, mean);
    by_channel(w, 0, a.rstd + w.sample * a.groups, rstd);
    params<T>(a.gamma, w.client, w.ch, to_read<V, ODD>(s, w), 1.0f, scale);
    params<T>(a.beta, w.client, w.ch, to_read<V, ODD>(s, w), 0.0f, beta);
#pragma unroll
    for (int e = 0; e < V; ++e) scale[e] *= rstd[e];
}
// dx = (d gamma - s1 - x^ s2) rstd = d scale - (x - mean) (rstd^2 s2) - rstd s1
template <int V>
__device__ __forceinline__ void to_dx(const float (&scale)[V], const float (&c1)[V], const float (&c2)[V], const float (&xm)[V], float (&d)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) d[e] = __builtin_fmaf(d[e], scale[e], -__builtin_fmaf(xm[e], c2[e], c1[e]));
}

template <typename T, int V, int N, bool ODD>
__global__ __launch_bounds__(kThreads) void k_norm_back_whole(aet_group_norm_grad a, NormShape s) {
    extern __shared__ float lds[];
    float *const totA = lds + 2 * s.threads * V, *const totB = totA + s.span, *const gam = totB + s.span, *const stat = gam + s.span;
    const Where w = where<V, ODD>(s, a.batch, a.width, xcd_order(blockIdx.x, gridDim.x));
    const T *x = (const T *)a.x.p + w.client * a.x.client + w.in_batch * a.x.sample + w.ch;
    const T *dy = (const T *)a.dy.p + w.client * a.dy.client + w.in_batch * a.dy.sample + w.ch;
    wide<T, V> rx[N], rd[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int pos = w.lane + i * s.lanes, count = pos < a.positions ? to_read<V, ODD>(s, w) : 0;
        rx[i] = load_raw<T, V>(x + pos * a.x.row, count);
        rd[i] = load_raw<T, V>(dy + pos * a.dy.row, count);
    }
    const int groups = w.chans / a.width, g0 = w.ch0 / a.width;
    float mean[V], scale[V], beta[V];
    slope_params<ODD, T>(a, s, w, mean, scale, beta);
    float AB[2][V] = {};
    float d[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float xm[V];
        slopes<T, V>(a.act, rx[i], rd[i], mean, scale, beta, d[i], xm);   // dy is 0 where there is no position
#pragma unroll
        for (int e = 0; e < V; ++e) {
            AB[0][e] += d[i][e];
            AB[1][e] += d[i][e] * xm[e];
        }
    }
    channel_sums<ODD>(s, w, AB, lds, totA);
    const float *const rstd_of = a.rstd + w.sample * a.groups + g0;
    for (int k = threadIdx.x; k < w.chans; k += blockDim.x) {
        float *to = s.sums + w.sample * 2 * s.channels + w.ch0 + k;
        totB[k] *= rstd_of[k / a.width];
        to[0] = totA[k];
        to[s.channels] = totB[k];
        gam[k] = a.gamma.p ? (float)((const T *)a.gamma.p)[w.client * a.gamma.client + w.ch0 + k] : 1.0f;
    }
    __syncthreads();
    if (!a.dx.p) return;
    const float inv = 1.0f / ((float)a.positions * (float)a.width);
    group_sums(totA, gam, groups, a.width, inv, stat);
    group_sums(totB, gam, groups, a.width, inv, stat + groups);
    for (int g = threadIdx.x; g < groups; g += blockDim.x) {
        stat[g] *= rstd_of[g];
        stat[groups + g] *= rstd_of[g] * rstd_of[g];
    }
    __syncthreads();
    T *dx = (T *)a.dx.p + w.client * a.dx.client + w.in_batch * a.dx.sample + w.ch;
    float c1[V], c2[V];
    by_channel(w, g0, stat, c1);
    by_channel(w, g0, stat + groups, c2);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int pos = w.lane + i * s.lanes;
        if (pos >= a.positions || w.count <= 0) continue;
        float xm[V];
#pragma unroll
        for (int e = 0; e < V; ++e) xm[e] = (float)rx[i][e] - mean[e];
        to_dx(scale, c1, c2, xm, d[i]);
        store_own<ODD>(dx + pos * a.dx.row, w, d[i]);
    }
}

// ---- larger samples ----------------------------------------------------------------------

// load(position, slot, count) and then use(position, slot, count) for a thread's positions, four of them at a time: their
// loads are on their way together.  With whole pieces the count is a constant there.
template <class L, class U>
__device__ __forceinline__ void each_position(int pos, int end, int step, int count, int V, L load, U use) {
    const auto some = [&](int have) {
        for (; pos < end; pos += 4 * step) {
#pragma unroll
            for (int i = 0; i < 4; ++i) load(pos + i * step < end ? pos + i * step : end - 1, i, have);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (pos + i * step < end) use(pos + i * step, i, have);
        }
    };
    if (count >= V) some(V);
    else if (count > 0) some(count);
}

// Of a strip's values of a channel: their mean, and the sum of squares of the differences from it.  No value is more than
// any other: a thread takes its positions by four, their mean and then the squares of the differences from it in registers,
// and joins them to what it has (Chan, Golub and LeVeque 1983); the threads' are joined about the strip's mean.  (Squares
// about the first value cancel where that is unlike the others, a corner or a border of zeros: rstd of 4096 values was 2^-13 off.)
template <typename T, int V, bool ODD>
__global__ __launch_bounds__(kThreads) void k_norm_strips(aet_group_norm a, NormShape s) {
    extern __shared__ float lds[];
    float *const tot = lds + 2 * s.threads * V;
    const int strip = blockIdx.x % (uint32_t)s.strips;
    const Where w = where<V, ODD>(s, a.batch, a.width, blockIdx.x / (uint32_t)s.strips);
    const int first = strip * s.strip, end = a.positions - first < s.strip ? a.positions : first + s.strip;
    const int start = first + w.lane, count = start < end ? to_read<V, ODD>(s, w) : 0;
    const T *x = (const T *)a.x.p + w.client * a.x.client + w.in_batch * a.x.sample + w.ch;
    // All differences are from the thread's first value, and in the end from the strip's, so that means far from 0 lose no bits.
    const wide<T, V> own = load_raw<T, V>(x + (start < end ? start : first) * a.x.row, count);
    const wide<T, V> about = load_raw<T, V>(x + first * a.x.row, count);
    float n = 0, mean[V] = {}, m2[V] = {};
    wide<T, V> raw[4];
    // FOUR: all four have a value, not the first `here` of them only
    const auto join = [&](auto four, int here) {
        constexpr bool FOUR = four;
        const float k = (float)here, share = k / (n + k), inv = FOUR ? 0.25f : 1.0f / k;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float d[4], q = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = FOUR || i < here ? (float)raw[i][e] - (float)own[e] : 0.0f;
            const float m = (d[0] + d[1] + (d[2] + d[3])) * inv, off = m - mean[e];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float r = FOUR || i < here ? d[i] - m : 0.0f;
                q = __builtin_fmaf(r, r, q);
            }
            m2[e] += __builtin_fmaf(off * share, off * n, q);
            mean[e] = __builtin_fmaf(off, share, mean[e]);
        }
        n += k;
    };
    const auto some = [&](int have) {
        for (int pos = start; pos < end; pos += 4 * s.lanes) {
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[i] = load_raw<T, V>(x + (pos + i * s.lanes < end ? pos + i * s.lanes : end - 1) * a.x.row, have);
            if (pos + 3 * s.lanes < end) join(std::true_type(), 4);
            else join(std::false_type(), (end - pos + s.lanes - 1) / s.lanes);
        }
    };
    if (count >= V) some(V);
    else if (count > 0) some(count);
    float sum[1][V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        mean[e] += (float)own[e] - (float)about[e];
        sum[0][e] = n * mean[e];
    }
    float *to = s.sums + (w.sample * s.strips + strip) * 2 * s.channels + w.ch0;
    const float inv = 1.0f / (float)(end - first);
    channel_sums<ODD>(s, w, sum, lds, tot);
    // what the sum's roundings have left of the mean, and the squares about it
    float DQ[2][V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int k = w.ch + e - w.ch0;   // (one of another workgroup's channels, or none: not counted)
        const float off = mean[e] - tot[k < 0 ? 0 : k < w.chans ? k : w.chans - 1] * inv;
        DQ[0][e] = n * off;
        DQ[1][e] = __builtin_fmaf(n * off, off, m2[e]);
    }
    const T *about0 = (const T *)a.x.p + w.client * a.x.client + w.in_batch * a.x.sample + first * a.x.row + w.ch0;
    for (int k = threadIdx.x; k < w.chans; k += blockDim.x) to[k] = (float)about0[k] + tot[k] * inv;
    channel_sums<ODD>(s, w, DQ, lds, tot);
    for (int k = threadIdx.x; k < w.chans; k += blockDim.x) {
        const float more = tot[k] * inv, squares = tot[s.span + k] - tot[k] * more;
        to[k] += more;
        to[s.channels + k] = squares < 0 ? 0.0f : squares;
    }
}

// The union of a group's strips and channels (Chan, Golub and LeVeque 1983): one workgroup per sample and group.
__device__ __forceinline__ float block_sum(float v, float *lds) {
    v = aet::wave_sum(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}
__global__ __launch_bounds__(256) void k_norm_union(aet_group_norm a, NormShape s) {
    __shared__ float lds[4];
    const int64_t sample = blockIdx.x / (uint32_t)a.groups;
    const int ch = (int)(blockIdx.x % (uint32_t)a.groups) * a.width;
    const float *from = s.sums + sample * s.strips * 2 * s.channels + ch;
    const int64_t entries = (int64_t)s.strips * a.width;
    const float inv = 1.0f / ((float)a.positions * (float)a.width);
    const float first = from[0];
    float sum = 0;
    for (int64_t i = threadIdx.x; i < entries; i += 256) {
        const int strip = (int)(i / a.width), k = (int)(i % a.width), left = a.positions - strip * s.strip;
        sum += (float)(left < s.strip ? left : s.strip) * (from[(int64_t)strip * 2 * s.channels + k] - first);
    }
    const float mean = first + block_sum(sum, lds) * inv;
    sum = 0;
    for (int64_t i = threadIdx.x; i < entries; i += 256) {
        const int strip = (int)(i / a.width), k = (int)(i % a.width), left = a.positions - strip * s.strip;
        const float *at = from + (int64_t)strip * 2 * s.channels + k;
        const float d = at[0] - mean;
        sum += at[s.channels] + (float)(left < s.strip ? left : s.strip) * d * d;
    }
    const float rstd = 1.0f / __builtin_sqrtf(block_sum(sum, lds) * inv + a.eps);
    if (threadIdx.x) return;
    const int64_t at = sample * 2 * a.groups + ch / a.width;
    s.stats[at] = mean;
    s.stats[at + a.groups] = rstd;
    if (a.mean) a.mean[blockIdx.x] = mean;
    if (a.rstd) a.rstd[blockIdx.x] = rstd;
}

template <typename T, int V, bool ODD>
__global__ __launch_bounds__(kThreads) void k_norm_apply(aet_group_norm a, NormShape s) {
    const int part = blockIdx.x % (uint32_t)s.parts;
    const Where w = where<V, ODD>(s, a.batch, a.width, blockIdx.x / (uint32_t)s.parts);
    if (w.count <= 0) return;
    const int first = part * s.part, end = a.positions - first < s.part ? a.positions : first + s.part;
    const T *x = (const T *)a.x.p + w.client * a.x.client + w.in_batch * a.x.sample + w.ch;
    T *y = (T *)a.y.p + w.client * a.y.client + w.in_batch * a.y.sample + w.ch;
    float mean[V], scale[V], gamma[V], beta[V];
    const float *stat = s.stats + w.sample * 2 * a.groups;
    by_channel(w, 0, stat, mean);
    by_channel(w, 0, stat + a.groups, scale);
    params<T>(a.gamma, w.client, w.ch, to_read<V, ODD>(s, w), 1.0f, gamma);
    params<T>(a.beta, w.client, w.ch, to_read<V, ODD>(s, w), 0.0f, beta);
#pragma unroll
    for (int e = 0; e < V; ++e) scale[e] *= gamma[e];
    wide<T, V> raw[4];
    each_position(first + w.lane, end, s.lanes, to_read<V, ODD>(s, w), V, [&](int pos, int i, int count) { raw[i] = load_raw<T, V>(x + pos * a.x.row, count); },
                  [&](int pos, int i, int count) {
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = __builtin_fmaf((float)raw[i][e] - mean[e], scale[e], beta[e]);
        act_each(a.act, v);
        store_own<ODD>(y + pos * a.y.row, w, v);
    });
}

template <typename T, int V, bool ODD>
__global__ __launch_bounds__(kThreads) void k_norm_back_strips(aet_group_norm_grad a, NormShape s) {
    extern __shared__ float lds[];
    float *const tot = lds + 2 * s.threads * V;
    const int strip = blockIdx.x % (uint32_t)s.strips;
    const Where w = where<V, ODD>(s, a.batch, a.width, blockIdx.x / (uint32_t)s.strips);
    const int first = strip * s.strip, end = a.positions - first < s.strip ? a.positions : first + s.strip;
    const T *x = (const T *)a.x.p + w.client * a.x.client + w.in_batch * a.x.sample + w.ch;
    const T *dy = (const T *)a.dy.p + w.client * a.dy.client + w.in_batch * a.dy.sample + w.ch;
    float mean[V], scale[V], beta[V], AB[2][V] = {};
    slope_params<ODD, T>(a, s, w, mean, scale, beta);
    wide<T, V> rx[4], rd[4];
    const auto load = [&](int pos, int i, int count) {
        rx[i] = load_raw<T, V>(x + pos * a.x.row, count);
        rd[i] = load_raw<T, V>(dy + pos * a.dy.row, count);
    };
    each_position(first + w.lane, end, s.lanes, to_read<V, ODD>(s, w), V, load, [&](int, int i, int) {
        float d[V], xm[V];
        slopes<T, V>(a.act, rx[i], rd[i], mean, scale, beta, d, xm);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            AB[0][e] += d[e];
            AB[1][e] += d[e] * xm[e];
        }
    });
    float *to = s.sums + (w.sample * s.strips + strip) * 2 * s.channels + w.ch0;
    channel_sums<ODD>(s, w, AB, lds, tot);
    for (int k = threadIdx.x; k < w.chans; k += blockDim.x) {
        to[k] = tot[k];
        to[s.channels + k] = tot[s.span + k] * a.rstd[w.sample * a.groups + (w.ch0 + k) / a.width];
    }
}

// The strips' sums by channel go to the first strip's place; what to_dx wants, s1 rstd and s2 rstd^2, to the group's.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_back_union(aet_group_norm_grad a, NormShape s) {
    __shared__ float lds[4];
    const int64_t sample = blockIdx.x / (uint32_t)a.groups, client = (uint32_t)sample / (uint32_t)a.batch;
    const int ch = (int)(blockIdx.x % (uint32_t)a.groups) * a.width;
    float *from = s.sums + sample * s.strips * 2 * s.channels + ch;
    const float inv = 1.0f / ((float)a.positions * (float)a.width);
    float s1 = 0, s2 = 0;
    for (int k = threadIdx.x; k < a.width; k += 256) {
        float A = 0, B = 0;
#pragma unroll 8
        for (int i = 0; i < s.strips; ++i) {
            A += from[(int64_t)i * 2 * s.channels + k];
            B += from[((int64_t)i * 2 + 1) * s.channels + k];
        }
        from[k] = A;
        from[s.channels + k] = B;
        const float gamma = a.gamma.p ? (float)((const T *)a.gamma.p)[client * a.gamma.client + ch + k] : 1.0f;
        s1 += A * gamma;
        s2 += B * gamma;
    }
    s1 = block_sum(s1, lds) * inv;
    s2 = block_sum(s2, lds) * inv;
    if (threadIdx.x) return;
    const int64_t at = sample * 2 * a.groups + ch / a.width;
    const float rstd = a.rstd[blockIdx.x];
    s.stats[at] = s1 * rstd;
    s.stats[at + a.groups] = s2 * rstd * rstd;
}

template <typename T, int V, bool ODD>
__global__ __launch_bounds__(kThreads) void k_norm_back_apply(aet_group_norm_grad a, NormShape s) {
    const int part = blockIdx.x % (uint32_t)s.parts;
    const Where w = where<V, ODD>(s, a.batch, a.width, blockIdx.x / (uint32_t)s.parts);
    if (w.count <= 0) return;
    const int first = part * s.part, end = a.positions - first < s.part ? a.positions : first + s.part;
    const T *x = (const T *)a.x.p + w.client * a.x.client + w.in_batch * a.x.sample + w.ch;
    const T *dy = (const T *)a.dy.p + w.client * a.dy.client + w.in_batch * a.dy.sample + w.ch;
    T *dx = (T *)a.dx.p + w.client * a.dx.client + w.in_batch * a.dx.sample + w.ch;
    float mean[V], scale[V], beta[V], c1[V], c2[V];
    slope_params<ODD, T>(a, s, w, mean, scale, beta);
    by_channel(w, 0, s.stats + w.sample * 2 * a.groups, c1);
    by_channel(w, 0, s.stats + (w.sample * 2 + 1) * a.groups, c2);
    wide<T, V> rx[4], rd[4];
    const auto load = [&](int pos, int i, int count) {
        rx[i] = load_raw<T, V>(x + pos * a.x.row, count);
        rd[i] = load_raw<T, V>(dy + pos * a.dy.row, count);
    };
    each_position(first + w.lane, end, s.lanes, to_read<V, ODD>(s, w), V, load, [&](int pos, int i, int count) {
        float d[V], xm[V];
        slopes<T, V>(a.act, rx[i], rd[i], mean, scale, beta, d, xm);
        to_dx(scale, c1, c2, xm, d);
        store_own<ODD>(dx + pos * a.dx.row, w, d);
    });
}

// dgamma and dbeta: samples' sums, 64 channels a workgroup, four samples at a time.  apart: between samples, in floats.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_params(aet_group_norm_grad a, const float *sums, int64_t apart, int channels, int across, int64_t samples) {
    __shared__ float lds[2][4][64];
    const int64_t client = blockIdx.x / (uint32_t)across;
    const int k = threadIdx.x % 64, part = threadIdx.x / 64, ch = (int)(blockIdx.x % (uint32_t)across) * 64 + k;
    float A = 0, B = 0;
    if (ch < channels) {
#pragma unroll 8
        for (int64_t i = client * samples + part; i < (client + 1) * samples; i += 4) {
            A += sums[i * apart + ch];
            B += sums[i * apart + channels + ch];
        }
    }
    lds[0][part][k] = A;
    lds[1][part][k] = B;
    __syncthreads();
    if (part || ch >= channels) return;
    if (a.dbeta.p) ((T *)a.dbeta.p)[client * a.dbeta.client + ch] = (T)(lds[0][0][k] + lds[0][1][k] + lds[0][2][k] + lds[0][3][k]);
    if (a.dgamma.p) ((T *)a.dgamma.p)[client * a.dgamma.client + ch] = (T)(lds[1][0][k] + lds[1][1][k] + lds[1][2][k] + lds[1][3][k]);
}

// No positions: the statistics of nothing.
__global__ __launch_bounds__(256) void k_norm_nothing(float *mean, float *rstd, float eps, int64_t count) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    if (mean) mean[i] = 0.0f;
    if (rstd) rstd[i] = 1.0f / __builtin_sqrtf(eps);
}

// ---- the choice --------------------------------------------------------------------------

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

struct NormPlan {
    bool whole;
    int n;             // positions a thread has (whole)
    NormShape s;
    size_t lds, sums_bytes, bytes;
};

static void deal(NormShape &s, int V, int span) {
    s.span = span;
    s.spans = (int)ceil_div(s.channels, span);
    s.pieces = (int)ceil_div(span, V);
}

static NormPlan make_plan(int64_t samples, int positions, int groups, int width, int V, bool back) {
    NormPlan p = {};
    NormShape &s = p.s;
    s.channels = groups * width;
    // Whole groups: as many as fit the registers, of those as give 512 workgroups, but 64 bytes of neighbouring channels
    // unless that leaves fewer than 128.  A sample's workgroups share lines of memory and run on one XCD (128 samples of
    // 4096 x 128 in bf16, 16 channels each: 75 us, dealt over the XCDs 139).  Less than 64 bytes: three kernels (the same
    // samples 72 us; 256 samples of 1024 x 320 in fp32, the gradient in groups of 10 channels: 340 us, in one kernel 500),
    // unless the launches are what counts.
    const int most = back ? 8 : 16;
    const int64_t lanes = ceil_div(positions, most), fit_pieces = lanes > kThreads ? 0 : kThreads / lanes;
    int64_t fit = (fit_pieces < 256 ? fit_pieces : 256) * V / width;
    if (fit > 1024) fit = 1024;   // their statistics and their channels' sums have 64 KB of LDS with the threads' sums
    if (fit > groups) fit = groups;
    if (fit > 0) {
        const auto at_least_1 = [](int64_t v) { return v < 1 ? 1 : v; };
        int64_t best = at_least_1(samples * groups / 512);
        if (best < ceil_div(4 * V, width)) best = ceil_div(4 * V, width);
        if (best > at_least_1(samples * groups / 128)) best = at_least_1(samples * groups / 128);
        if (best > fit) best = fit;
        best = ceil_div(groups, ceil_div(groups, best));
        s.span_groups = (int)best;
    }
    const int best = s.span_groups;
    p.whole = best && (best == groups || best * width >= 4 * V || samples * positions * s.channels < (1 << 22));
    if (p.whole) {
        deal(s, V, best * width);
        s.lanes = kThreads / s.pieces;
        if (s.lanes > positions) s.lanes = positions;
        p.n = (int)ceil_div(positions, s.lanes);
        s.threads = (int)ceil_div(s.pieces * s.lanes, 64) * 64;
        s.strips = 1;
        s.strip = positions;
        p.lds = sizeof(float) * ((size_t)(back ? 2 : 1) * s.threads * V + (back ? 3 : 1) * s.span + 2 * best);
        p.sums_bytes = back ? up256((size_t)samples * 2 * s.channels * sizeof(float)) : 0;
        p.bytes = p.sums_bytes;
        return p;
    }
    deal(s, V, s.channels < 256 * V ? s.channels : 256 * V);
    s.lanes = kThreads / s.pieces;
    // Sums: as many strips as give every compute unit four workgroups, of 8 positions a thread or more (a workgroup's
    // own sums and their union cost as much as some 10 positions: gradient of 128 samples of 4096 x 320 in bf16, 1024 workgroups
    // 156 us; forward, all three, 209).  Second pass: short parts, 4 positions a thread (with 1024 workgroups 8 % more).
    const int64_t wanted = ceil_div(1024, samples * s.spans), most_strips = ceil_div(positions, (int64_t)s.lanes * 8);
    s.strip = (int)ceil_div(ceil_div(positions, wanted < most_strips ? wanted : most_strips), s.lanes) * s.lanes;
    s.strips = (int)ceil_div(positions, s.strip);
    s.part = 4 * s.lanes;
    while (s.part < positions && samples * s.spans * ceil_div(positions, s.part) > 8192) s.part *= 2;
    s.parts = (int)ceil_div(positions, s.part);
    s.threads = (int)ceil_div(s.pieces * s.lanes, 64) * 64;
    p.lds = sizeof(float) * 2 * ((size_t)s.threads * V + s.span);
    p.sums_bytes = up256((size_t)samples * s.strips * 2 * s.channels * sizeof(float));
    p.bytes = p.sums_bytes + up256((size_t)samples * 2 * groups * sizeof(float));
    return p;
}
static int vec(int dtype) { return dtype == AET_F32 ? 4 : 8; }
static NormPlan plan(const aet_group_norm &a) {
    return make_plan((int64_t)a.n * a.batch, a.positions, a.groups, a.width, vec(a.dtype), false);
}
static NormPlan plan(const aet_group_norm_grad &a) {
    return make_plan((int64_t)a.n * a.batch, a.positions, a.groups, a.width, vec(a.dtype), true);
}

size_t group_norm_forward_workspace(const aet_group_norm &a) { return a.n && a.batch && a.positions ? plan(a).bytes : 0; }
size_t group_norm_backward_workspace(const aet_group_norm_grad &a) { return a.n && a.batch && a.positions ? plan(a).bytes : 0; }

// Whether a workgroup's channels are not whole pieces.
template <typename T>
static bool odd_pieces(const NormShape &s) {
    constexpr int V = 16 / sizeof(T);
    return s.channels % V || (s.spans > 1 && s.span % V);
}

template <typename T, bool ODD>
static hipError_t forward(const aet_group_norm &a, char *workspace, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const int64_t samples = (int64_t)a.n * a.batch;
    if (!a.positions) {
        if (a.mean || a.rstd) k_norm_nothing<<<(int)ceil_div(samples * a.groups, 256), 256, 0, s>>>(a.mean, a.rstd, a.eps, samples * a.groups);
        return hipGetLastError();
    }
    NormPlan p = plan(a);
    p.s.sums = (float *)workspace;
    p.s.stats = (float *)(workspace + p.sums_bytes);
    const int64_t blocks = samples * p.s.spans * p.s.strips;
    if (blocks > INT32_MAX || samples * p.s.spans * p.s.parts > INT32_MAX || samples * a.groups > INT32_MAX) return hipErrorInvalidConfiguration;
    if (p.whole) {
        if (p.n <= 4) k_norm_whole<T, V, 4, ODD><<<(int)blocks, p.s.threads, p.lds, s>>>(a, p.s);
        else if (p.n <= 8) k_norm_whole<T, V, 8, ODD><<<(int)blocks, p.s.threads, p.lds, s>>>(a, p.s);
        else k_norm_whole<T, V, 16, ODD><<<(int)blocks, p.s.threads, p.lds, s>>>(a, p.s);
    } else {
        k_norm_strips<T, V, ODD><<<(int)blocks, p.s.threads, p.lds, s>>>(a, p.s);
        k_norm_union<<<(int)(samples * a.groups), 256, 0, s>>>(a, p.s);
        k_norm_apply<T, V, ODD><<<(int)(samples * p.s.spans * p.s.parts), p.s.threads, 0, s>>>(a, p.s);
    }
    return hipGetLastError();
}
template <typename T>
static hipError_t forward(const aet_group_norm &a, char *workspace, hipStream_t s) {
    return odd_pieces<T>(a.positions ? plan(a).s : NormShape()) ? forward<T, true>(a, workspace, s) : forward<T, false>(a, workspace, s);
}
hipError_t launch_group_norm_forward(const aet_group_norm &a, void *workspace, hipStream_t s) {
    return a.dtype == AET_F32 ? forward<float>(a, (char *)workspace, s) : forward<bf16>(a, (char *)workspace, s);
}

template <typename T, bool ODD>
static hipError_t backward(const aet_group_norm_grad &a, char *workspace, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const int64_t samples = a.positions ? (int64_t)a.n * a.batch : 0, channels = (int64_t)a.groups * a.width;
    NormPlan p = {};
    if (samples) {
        p = plan(a);
        p.s.sums = (float *)workspace;
        p.s.stats = (float *)(workspace + p.sums_bytes);
        const int64_t blocks = samples * p.s.spans * p.s.strips;
        if (blocks > INT32_MAX || samples * p.s.spans * p.s.parts > INT32_MAX || samples * a.groups > INT32_MAX) return hipErrorInvalidConfiguration;
        if (p.whole) {
            if (p.n <= 4) k_norm_back_whole<T, V, 4, ODD><<<(int)blocks, p.s.threads, p.lds, s>>>(a, p.s);
            else k_norm_back_whole<T, V, 8, ODD><<<(int)blocks, p.s.threads, p.lds, s>>>(a, p.s);
        } else {
            k_norm_back_strips<T, V, ODD><<<(int)blocks, p.s.threads, p.lds, s>>>(a, p.s);
            k_norm_back_union<T><<<(int)(samples * a.groups), 256, 0, s>>>(a, p.s);
            if (a.dx.p) k_norm_back_apply<T, V, ODD><<<(int)(samples * p.s.spans * p.s.parts), p.s.threads, 0, s>>>(a, p.s);
        }
    }
    if (a.dgamma.p || a.dbeta.p) {
        const bool shared = (a.dgamma.p && !a.dgamma.client) || (a.dbeta.p && !a.dbeta.client);
        const int clients = shared ? 1 : a.n, across = (int)ceil_div(channels, 64);
        if (!clients) return hipSuccess;
        if ((int64_t)clients * across > INT32_MAX) return hipErrorInvalidConfiguration;
        k_norm_params<T><<<clients * across, 256, 0, s>>>(a, p.s.sums, (int64_t)p.s.strips * 2 * channels, (int)channels, across, samples / clients);
    }
    return hipGetLastError();
}
template <typename T>
static hipError_t backward(const aet_group_norm_grad &a, char *workspace, hipStream_t s) {
    const bool some = a.n && a.batch && a.positions;
    return odd_pieces<T>(some ? plan(a).s : NormShape()) ? backward<T, true>(a, workspace, s) : backward<T, false>(a, workspace, s);
}
hipError_t launch_group_norm_backward(const aet_group_norm_grad &a, void *workspace, hipStream_t s) {
    return a.dtype == AET_F32 ? backward<float>(a, (char *)workspace, s) : backward<bf16>(a, (char *)workspace, s);
}

}  // namespace aet_ops
