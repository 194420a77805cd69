// The linear layer for few rows a client (single requests, small mini-batches).
//
// Bound by reading W once.  A workgroup has 16 outputs of a client and all its rows, its waves parts of the sum; operands
// go from memory straight into the lanes that want them (v_mfma_f32_16x16x32_bf16; v_mfma_f32_16x16x4_f32, whose four
// k of a step are taken from places 4 apart so that a lane reads 16 bytes), several steps ahead of their use.  The waves'
// sums meet in LDS.  One row of 4096 x 4096 in bf16: 9.9 us (34 MB: 6.7 at a copy's rate); 16 clients' 32 x 784 x 128 in
// fp32: 6.0 us.  Up to 32 rows; with 1, 16 and 32 in a graph, this way and in tiles (ops_tiles.hip), us:
//   fp32  4096 x 4096  17.6, 19.8, 26.6 and 27, 27, 28;   16 x (784 x 128)  4.2, 4.9, 6.0 and 10, 11, 12
//   bf16  4096 x 4096  7.6, 10.2, 13.9 and 12.2, 12.7, 13.3;   1000 x 100  3.0, 3.3, 4.2 and 10, 10, 10
#include "ops_internal.h"
#include "ops_tiles.h"

#include <type_traits>

namespace aet_ops {

template <typename T>
struct Step;
template <>
struct Step<bf16> {
    static constexpr int kDepth = 32, kLane = 8;   // k of a step, and of a lane
    static __device__ __forceinline__ f4 product(const wide<bf16, 8> &a, const wide<bf16, 8> &b, f4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16((bf8)a, (bf8)b, c, 0, 0, 0);
    }
};
template <>
struct Step<float> {
    static constexpr int kDepth = 16, kLane = 4;
    static __device__ __forceinline__ f4 product(const wide<float, 4> &a, const wide<float, 4> &b, f4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

struct RowsShape {
    int M, N, K;
    int tiles_n;    // workgroups of a client
};

// bf16 whose rows do not all begin at multiples of 4 bytes: 16 bytes from another address take 3.6 times as long (9 TB/s
// from the L2, not 33), so they are loaded from the multiple below.  What is missing is the first 4 bytes of the lane with
// the next 8 k, 16 lanes on or in the next step; of the last step of those in a row it is loaded.
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
template <int N>
struct OddRow {
    const char *p;   // the multiple of 4 at or below the lane's first value
    int shift;       // in bits: 0 or 16
    wide<uint32_t, 4> v[N];
    uint32_t after;
    __device__ __forceinline__ void begin(const bf16 *at) {
        p = (const char *)((uintptr_t)at & ~(uintptr_t)3);
        shift = (int)((uintptr_t)at & 2) * 8;
    }
    __device__ __forceinline__ void load(int i, int64_t k) { v[i] = *(const wide<uint32_t, 4> *)(p + 2 * k); }
    // k: of the last step
    __device__ __forceinline__ void load_after(int64_t k) {
        if (shift && threadIdx.x % 64 >= 48) after = *(const uint32_t *)(p + 2 * k + 16);
    }
    __device__ __forceinline__ bf8 step(int i, bool last) const {
        const int lane = threadIdx.x % 64;
        const uint32_t mine = lane < 16 && i + 1 < N ? v[i + 1 < N ? i + 1 : i][0] : v[i][0];
        uint32_t next = __shfl(mine, (lane + 16) & 63, 64);
        if (last && lane >= 48) next = after;
        u4 r;
#pragma unroll
        for (int e = 0; e < 3; ++e) r[e] = __builtin_amdgcn_alignbit(v[i][e + 1], v[i][e], shift);
        r[3] = __builtin_amdgcn_alignbit(next, v[i][3], shift);
        return __builtin_bit_cast(bf8, r);
    }
};

// G: groups of 16 rows.  AHEAD steps of a wave are on their way at a time.
template <typename T, int G, int WAVES, bool ODD>
__global__ __launch_bounds__(64 * WAVES) void k_rows(Operand ox, Operand ow, RowsShape s, Epilogue e) {
    using S = Step<T>;
    constexpr int AHEAD = G == 1 ? 8 : 4;
    __shared__ float lds[WAVES][G * 16][20];
    const int64_t client = blockIdx.x / s.tiles_n;
    const int n0 = (int)(blockIdx.x % s.tiles_n) * 16;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int line = lane % 16, kl = lane / 16 * S::kLane;
    // lines past the last are read from the last again, and not stored
    const T *w = (const T *)ow.p + client * ow.client + (int64_t)(n0 + line < s.N ? n0 + line : s.N - 1) * ow.row + kl;
    const T *x[G];
#pragma unroll
    for (int g = 0; g < G; ++g)
        x[g] = (const T *)ox.p + client * ox.client + (int64_t)(16 * g + line < s.M ? 16 * g + line : s.M - 1) * ox.row + kl;
    f4 acc[G] = {};
    const int whole = s.K / S::kDepth;   // steps
    // a wave's steps: AHEAD in a row, then those of the others
    if constexpr (ODD) {
        OddRow<AHEAD> a, b[G];
        a.begin(w);
#pragma unroll
        for (int g = 0; g < G; ++g) b[g].begin(x[g]);
        for (int i0 = wave * AHEAD; i0 < whole; i0 += WAVES * AHEAD) {
            const int last = i0 + AHEAD < whole ? i0 + AHEAD - 1 : whole - 1;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int64_t k = (int64_t)(i0 + i < last ? i0 + i : last) * S::kDepth;
                a.load(i, k);
#pragma unroll
                for (int g = 0; g < G; ++g) b[g].load(i, k);
            }
            a.load_after((int64_t)last * S::kDepth);
#pragma unroll
            for (int g = 0; g < G; ++g) b[g].load_after((int64_t)last * S::kDepth);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (i0 + i <= last) {
                    const bf8 va = a.step(i, i0 + i == last);
#pragma unroll
                    for (int g = 0; g < G; ++g) acc[g] = S::product(va, b[g].step(i, i0 + i == last), acc[g]);
                }
        }
    } else {
        for (int i0 = wave * AHEAD; i0 < whole; i0 += WAVES * AHEAD) {
            wide<T, S::kLane> a[AHEAD], b[AHEAD][G];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int64_t k = (int64_t)(i0 + i < whole ? i0 + i : whole - 1) * S::kDepth;
                a[i] = *(const wide<T, S::kLane> *)(w + k);
#pragma unroll
                for (int g = 0; g < G; ++g) b[i][g] = *(const wide<T, S::kLane> *)(x[g] + k);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (i0 + i < whole)
#pragma unroll
                    for (int g = 0; g < G; ++g) acc[g] = S::product(a[i], b[i][g], acc[g]);
        }
    }
    const int rest = s.K - whole * S::kDepth;   // the sum's end, less than a step
    if (rest && wave == WAVES - 1) {
        const int64_t k = (int64_t)whole * S::kDepth;
        const wide<T, S::kLane> a = load_raw<T, S::kLane>(w + k, rest - kl);
#pragma unroll
        for (int g = 0; g < G; ++g) acc[g] = S::product(a, load_raw<T, S::kLane>(x[g] + k, rest - kl), acc[g]);
    }
    // lane: row lane % 16, outputs 4 (lane / 16) ..
#pragma unroll
    for (int g = 0; g < G; ++g) *(f4 *)&lds[wave][16 * g + line][lane / 16 * 4] = acc[g];
    __syncthreads();
    const int row = threadIdx.x / 2, half = threadIdx.x % 2 * 8, count = s.N - n0 - half;
    if (row >= G * 16 || row >= s.M || count <= 0) return;
    float v[8];
    bias_of<T>(e, client, n0 + half, count, v);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const f4 lo = *(const f4 *)&lds[i][row][half], hi = *(const f4 *)&lds[i][row][half + 4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            v[y] += lo[y];
            v[4 + y] += hi[y];
        }
    }
    finish<T>(e, client, row, n0 + half, count, v);
}

bool rows_fit(const Product &p) { return !p.a.by_columns && !p.b.by_columns && p.M <= 32; }

template <typename T>
static hipError_t run(const Product &p, hipStream_t stream) {
    const RowsShape s = {p.M, p.N, p.K, (int)ceil_div(p.N, 16)};
    const int64_t blocks = (int64_t)p.clients * s.tiles_n;
    if (!blocks || !p.M) return hipSuccess;
    if (blocks > INT32_MAX) return hipErrorInvalidConfiguration;
    // waves: 16 where each has 4 steps or more (32 rows of 4096 x 4096 in bf16 14 us, with 4 waves 16; 64 x (256 x 256) in
    // fp32 with 16 waves 8.2, with 4 5.0)
    const bool deep = p.K >= 16 * 4 * Step<T>::kDepth;
    const auto go = [&](auto odd) {
        if (p.M <= 16) {
            if (deep) k_rows<T, 1, 16, odd><<<(int)blocks, 1024, 0, stream>>>(p.a, p.b, s, p.e);
            else k_rows<T, 1, 4, odd><<<(int)blocks, 256, 0, stream>>>(p.a, p.b, s, p.e);
        } else {
            if (deep) k_rows<T, 2, 16, odd><<<(int)blocks, 1024, 0, stream>>>(p.a, p.b, s, p.e);
            else k_rows<T, 2, 4, odd><<<(int)blocks, 256, 0, stream>>>(p.a, p.b, s, p.e);
        }
    };
    const auto odd = [](const Operand &o) { return ((o.row | o.client) & 1) || (uintptr_t)o.p % 4; };
    if (sizeof(T) == 2 && (odd(p.a) || odd(p.b))) go(std::bool_constant<sizeof(T) == 2>());
    else go(std::false_type());
    return hipGetLastError();
}

hipError_t launch_rows(int dtype, const Product &p, hipStream_t s) { return dtype == AET_F32 ? run<float>(p, s) : run<bf16>(p, s); }

}  // namespace aet_ops
