// Products of values held in microscaled 4-bit floating point, on the matrix unit's own instructions for them.
//
// C[m][n] = sum over k of A(m, k) B(n, k), both as codes by rows with a scale for each 32 k.  A lane of
// v_mfma_scale_f32_32x32x64_f8f6f4 has the 16 bytes and the scale of one block of a row: the codes go as they lie in
// memory from there to LDS and to the unit, four times the values a byte of bf16 products.
//
// Bound by the parts of a tile one after the other; no unit is full.  Over the whole of 16384 x 4096 x 4096 with bias and GELU the matrix unit is
// busy for 30 % of the cycles, LDS for 26 %, and waves are at a wait for 35 % of their time.  A tile of 256 x 256 takes 2.0 us for 256 k, and some 10
// from its first load to its last store beside that, a quarter of 16 stages' time; two tiles at once, which would hide that, do not fit
// into LDS.  That size takes 181 to 225 us to bf16 (2.4 to 3.0 PF/s) and 195 to fp32, 8192^3 299 to 317 (3.5 to 3.7).  (A loop of the unit's instructions
// alone runs at 5.0 to 5.8 PF/s with random codes and at 8.7 with zeros: the clock gives way.)
#include "ops_internal.h"
#include "ops_mx4.h"
#include "ops_stage.h"

#include <type_traits>

namespace aet_ops {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));

constexpr int kFp4 = 4;   // the format's number in the instructions
__device__ __forceinline__ i8v widen(i4 v) { return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1); }

// ---- tiles -------------------------------------------------------------------------------

// k of a stage, 128 bytes of codes a row (64 bytes a row, half the k: all kinds of tiles at 2.2 PF/s); stages whose scales come
// together, 32 bytes a row
constexpr int kDeep = 256, kGroup = 4;
constexpr int kUnit = 512;               // sums are whole ones of these: 16 bytes of scales a row

// Scales of BM rows of A and BN of B, a group of stages at a time.  (8 bytes a row and stage would be a line of memory for each.)
template <int BM, int BN, int THREADS>
struct ScaleGroup {
    static constexpr int kBytes = (BM + BN) * 32, kCount = (BM + BN) * 2 / THREADS;
    static_assert(kCount * THREADS == (BM + BN) * 2 && THREADS % 32 == 0, "whole pieces a thread");
    const uint8_t *p[kCount];
    int piece, last;   // of 16 bytes, from the row's first on
    // Where a row's piece lies in its 32 bytes: of eight rows the other way round than of the next eight, so that a wave's lanes
    // read from twice the banks.  (8192 x 8192 x 8192: 334 -> 317 us.)
    static __device__ __forceinline__ int turn(int row) { return row >> 3 & 1; }
    __device__ __forceinline__ void begin(const Held &a, const Held &b, int64_t client, int m0, int M, int n0, int N, int k0, int K) {
        piece = k0 / kUnit + (threadIdx.x % 2 ^ turn(threadIdx.x / 2));   // (the same for all of a thread's rows)
        last = K / kUnit - 1;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int r = (threadIdx.x + i * THREADS) / 2, row = r < BM ? m0 + r : n0 + r - BM;
            const aet_in &o = r < BM ? a.scales : b.scales;
            const int most = (r < BM ? M : N) - 1;
            p[i] = (const uint8_t *)o.p + client * o.client + (int64_t)(row < most ? row : most) * o.row;
        }
    }
    // (behind the sum's end: the last piece again, which nobody reads)
    __device__ __forceinline__ void load(lds_ptr to) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const int at = (piece < last ? piece : last) * 16;
#pragma unroll
        for (int i = 0; i < kCount; ++i)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(p[i] + at),
                                             (__attribute__((address_space(3))) void *)(to + (i * THREADS + wave * 64) * 16), 16, 0, 0);
        piece += 2;
    }
};

// In LDS: two stages of codes of A and B, two groups of scales of A and B.  (Codes are moved as values of bf16, of 4 k each.)
template <int BM, int BN, int THREADS>
struct HeldTile {
    using SA = Stage<BM, kDeep / 4, false>;
    using SB = Stage<BN, kDeep / 4, false>;
    using Scales = ScaleGroup<BM, BN, THREADS>;
    static constexpr int kStage = SA::kBytes + SB::kBytes, kScales = 2 * kStage, kLds = kScales + 2 * Scales::kBytes;
};

template <typename T, int BM, int BN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC, BM == 64 ? 4 : 2) void k_mx4_tiles(Held oa, Held ob, Shape s, Epilogue e) {
    extern __shared__ __attribute__((aligned(1024))) char lds_[];
    const lds_ptr lds = (lds_ptr)lds_;
    constexpr int THREADS = 64 * WR * WC, FM = BM / WR / 32, FN = BN / WC / 32, KS = kDeep / 64;
    using L = HeldTile<BM, BN, THREADS>;
    using SA = typename L::SA;
    using SB = typename L::SB;
    int id = xcd_order(blockIdx.x, s.blocks);
    const int tile = id % s.tiles;
    id /= s.tiles;
    const int slice = id % s.slices;
    const int64_t client = id / s.slices;
    // eight rows of tiles at a time, column after column
    const int tiles_m = s.tiles / s.tiles_n, group = tile / (8 * s.tiles_n) * 8;
    const int high = tiles_m - group < 8 ? tiles_m - group : 8, in = tile - group * s.tiles_n;
    const int m0 = (group + in % high) * BM, n0 = in / high * BN;
    const int k0 = slice * s.slice_k, k1 = k0 + s.slice_k < s.K ? k0 + s.slice_k : s.K;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wr = wave / WC, wc = wave % WC;

    f16v acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = f16v{};

    struct Fragments {
        i4 a[FM], b[FN];
    };
    struct Scaled {   // of 128 k, shifted so that bytes 0 and 2 are the lane's
        uint32_t a[FM], b[FN];
    };
    const auto read = [&](Fragments &f, int stage, int ks) {
        const lds_ptr at = lds + stage % 2 * L::kStage;
#pragma unroll
        for (int i = 0; i < FN; ++i) f.b[i] = __builtin_bit_cast(i4, SB::fragment(at + SA::kBytes, wc * FN + i, ks, lane));
#pragma unroll
        for (int j = 0; j < FM; ++j) f.a[j] = __builtin_bit_cast(i4, SA::fragment(at, wr * FM + j, ks, lane));
    };
    const auto read_scales = [&](Scaled &f, int stage, int word) {
        const lds_ptr at = lds + L::kScales + stage / kGroup % 2 * L::Scales::kBytes + stage % 2 * 8 + word * 4 +
                           ((lane & 31) * 32 + (stage % kGroup / 2 ^ L::Scales::turn(lane)) * 16);
        const auto one = [&](lds_ptr at, int t) { return *(__attribute__((address_space(3))) uint32_t *)(at + t * 1024) >> (lane >> 5) * 8; };
#pragma unroll
        for (int i = 0; i < FN; ++i) f.b[i] = one(at + BM * 32, wc * FN + i);
#pragma unroll
        for (int j = 0; j < FM; ++j) f.a[j] = one(at, wr * FM + j);
    };
    const auto multiply = [&](const Fragments &f, const Scaled &c, auto ks) {
        constexpr int byte = ks % 2 * 2;
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(widen(f.b[i]), widen(f.a[j]), acc[i][j], kFp4, kFp4, byte, (int)c.b[i], byte, (int)c.a[j]);
    };

    DirectStage<BM, kDeep / 4, false, THREADS> la;
    DirectStage<BN, kDeep / 4, false, THREADS> lb;
    typename L::Scales sc;
    la.begin({oa.codes.p, oa.codes.client / 2, oa.codes.row / 2, false, false, 0}, client, m0, s.M, k0 / 4, k1 / 4);
    lb.begin({ob.codes.p, ob.codes.client / 2, ob.codes.row / 2, false, false, 0}, client, n0, s.N, k0 / 4, k1 / 4);
    sc.begin(oa, ob, client, m0, s.M, n0, s.N, k0, s.K);
    const int stages = k1 > k0 ? (k1 - k0) / kDeep : 0;
    const auto fetch = [&](int i) {
        const lds_ptr to = lds + i % 2 * L::kStage;
        la.load(to);
        lb.load(to + SA::kBytes);
    };
    const auto fetch_scales = [&](int g) { sc.load(lds + L::kScales + g % 2 * L::Scales::kBytes); };
    const auto arrived = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);   // all that is on its way to LDS, and what was read of it
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The fragments of the next 64 k are read while the matrix unit has the last ones, also across the barrier that says that the
    // next stage has arrived everywhere and that this one's place may be written again.
    Fragments f[2];
    Scaled c[2];
    if (stages > 0) {
        fetch_scales(0);
        fetch(0);
        if (stages > 1) fetch(1);
        if (stages > kGroup) fetch_scales(1);
        arrived();
        read(f[0], 0, 0);
        read_scales(c[0], 0, 0);
    }
    // Stage i; more: there is another behind it; get: sends for those that take its place.  (No branch inside: the unit's
    // instructions and the reads that they want stay mixed.)
    const auto stage = [&](int i, auto more, auto get) {
        const auto part = [&](auto ks) {
            if constexpr (ks + 1 == KS) {
                arrived();
                get(i);
                if constexpr (more) {
                    read(f[0], i + 1, 0);
                    read_scales(c[0], i + 1, 0);
                }
            } else {
                read(f[(ks + 1) % 2], i, ks + 1);
                if constexpr (ks == 1) read_scales(c[1], i, 1);
            }
            multiply(f[ks % 2], c[ks / 2], ks);
            interleave<FM * FN, FM + FN>();
        };
        part(std::integral_constant<int, 0>());
        part(std::integral_constant<int, 1>());
        part(std::integral_constant<int, 2>());
        part(std::integral_constant<int, 3>());
    };
    static_assert(kGroup == 4 && kUnit == 2 * kDeep, "stages come in twos, scales for four");
    const auto next = [&](int i) { fetch(i + 2); };
    const auto none = [](int) {};
    const int groups = stages > 0 ? (stages - 2) / kGroup : 0;   // with another group or half of one behind them
    for (int g = 0; g < groups; ++g) {
        const int i = g * kGroup;
        stage(i, std::true_type(), next);
        stage(i + 1, std::true_type(), next);
        stage(i + 2, std::true_type(), next);
        stage(i + 3, std::true_type(), [&](int i) {
            fetch(i + 2);
            fetch_scales(g);   // the one after the next takes this one's place
        });
    }
    if (stages - groups * kGroup == kGroup) {
        stage(groups * kGroup, std::true_type(), next);
        stage(groups * kGroup + 1, std::true_type(), next);
    }
    if (stages > 0) {
        stage(stages - 2, std::true_type(), none);
        stage(stages - 1, std::false_type(), none);
    }
    __syncthreads();

    // A lane has, of row m0 + lane % 32 of a fragment, four columns at a time: through LDS, a wave for itself, to lanes
    // with V columns (16 bytes) each, in whole lines of memory.
    constexpr int V = 16 / sizeof(T), W = FN * 32, LINE = W + 4, ACROSS = W / V, DOWN = 64 / ACROSS;
    __attribute__((address_space(3))) float *mine = (__attribute__((address_space(3))) float *)lds + wave * (32 * LINE);
    const auto settle = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    };
    const int col = n0 + wc * W + lane % ACROSS * V, count = s.N - col;
    float bias[V];
    bias_of<T>(e, client, col, s.slices > 1 ? 0 : count, bias);
#pragma unroll
    for (int j = 0; j < FM; ++j) {
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(__attribute__((address_space(3))) f4 *)(mine + (lane & 31) * LINE + i * 32 + 8 * q + 4 * (lane >> 5)) =
                    f4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        settle();
#pragma unroll 1
        for (int r = 0; r < 32; r += DOWN) {
            const int line = r + lane / ACROSS;
            const int64_t row = m0 + (wr * FM + j) * 32 + line;
            float v[V];
#pragma unroll
            for (int h = 0; h < V / 4; ++h) {
                const f4 x = *(__attribute__((address_space(3))) f4 *)(mine + line * LINE + lane % ACROSS * V + 4 * h);
#pragma unroll
                for (int y = 0; y < 4; ++y) v[4 * h + y] = x[y] + bias[4 * h + y];
            }
            if (row < s.M && count > 0) {
                if (s.slices > 1) store_some(s.partial + (((int64_t)slice * s.clients + client) * s.M + row) * s.N + col, count, v);
                else finish<T>(e, client, row, col, count, v);
            }
        }
        settle();
    }
}

// ---- few rows ----------------------------------------------------------------------------

// Up to 32 rows: bound by reading W once, and by latency.  One row by 4096 x 4096 5.3 us (8.9 MB: 1.7 TB/s; the call alone takes 5).
// 16 outputs a workgroup and all rows, its waves parts of the sum; operands go from memory straight into the lanes that want them
// (v_mfma_scale_f32_16x16x128_f8f6f4: a lane has a block of a row), several steps ahead of their use.  Any alignment, any end of a sum.
struct HeldRows {
    int M, N, K, tiles_n, tiles;   // tiles: of a client, of 16 FM rows by 16 outputs
};
constexpr int kRowWaves = 8, kAhead = 4;

template <typename T, int FM>
__global__ __launch_bounds__(64 * kRowWaves) void k_mx4_rows(Held oa, Held ob, HeldRows s, Epilogue e) {
    __shared__ float sums[kRowWaves][FM][16][17];
    const int64_t client = blockIdx.x / s.tiles;
    const int tile = blockIdx.x % s.tiles, n0 = tile % s.tiles_n * 16, m0 = tile / s.tiles_n * (16 * FM);
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, block = lane / 16;
    const int nr = n0 + r < s.N ? n0 + r : s.N - 1;   // (rows past the last: the last again, not stored)
    const uint8_t *bc = (const uint8_t *)ob.codes.p + client * ob.codes.client + nr * ob.codes.row;
    const uint8_t *bs = (const uint8_t *)ob.scales.p + client * ob.scales.client + nr * ob.scales.row;
    const uint8_t *ac[FM], *as[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int mr = m0 + j * 16 + r < s.M ? m0 + j * 16 + r : s.M - 1;
        ac[j] = (const uint8_t *)oa.codes.p + client * oa.codes.client + mr * oa.codes.row;
        as[j] = (const uint8_t *)oa.scales.p + client * oa.scales.client + mr * oa.scales.row;
    }
    const int blocks = (s.K + 31) / 32, steps = (blocks + 3) / 4, whole = s.K / 32;
    // 32 codes and their scale; past the end codes of 0, and a scale of 1
    const auto codes = [&](const uint8_t *p, int b) {
        if (b < whole) return __builtin_bit_cast(i4, (uint8_t __attribute__((ext_vector_type(16))))(*(const wide<uint8_t, 16> *)(p + b * 16)));
        i4 v = {0, 0, 0, 0};
        const int left = s.K - b * 32;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            uint32_t byte = 2 * i < left ? p[b * 16 + i] : 0;
            if (2 * i + 1 == left) byte &= 15;
            v[i / 4] |= (int)(byte << (i % 4 * 8));
        }
        return v;
    };
    const auto scale = [&](const uint8_t *p, int b) { return b < blocks ? (int)p[b] : 127; };
    f4 acc[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int t0 = wave; t0 < steps; t0 += kRowWaves * kAhead) {
        i4 cb[kAhead], ca[kAhead][FM];
        int sb[kAhead], sa[kAhead][FM];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int b = (t0 + q * kRowWaves) * 4 + block;
            cb[q] = codes(bc, b);
            sb[q] = scale(bs, b);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                ca[q][j] = codes(ac[j], b);
                sa[q][j] = scale(as[j], b);
            }
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
#pragma unroll
            for (int j = 0; j < FM; ++j)
                acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(widen(cb[q]), widen(ca[q][j]), acc[j], kFp4, kFp4, 0, sb[q], 0, sa[q][j]);
    }
    // register i of a lane: output 4 (lane / 16) + i of row lane % 16
#pragma unroll
    for (int j = 0; j < FM; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[wave][j][r][4 * block + i] = acc[j][i];
    __syncthreads();
    for (int i = threadIdx.x; i < FM * 16 * 8; i += 64 * kRowWaves) {   // two outputs each, whose dropout is one hash
        const int j = i / 128, row = i / 8 % 16, col = i % 8 * 2, count = s.N - n0 - col;
        if (m0 + j * 16 + row >= s.M || count <= 0) continue;
        float v[2];
        bias_of<T>(e, client, n0 + col, count, v);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int w = 0; w < kRowWaves; ++w) v[x] += sums[w][j][row][col + x];
        finish<T>(e, client, m0 + j * 16 + row, n0 + col, count, v);
    }
}

// ---- the choice --------------------------------------------------------------------------

// (the tiles' offsets between rows have 32 bits)
static bool rows_fit(const HeldProduct &p) { return p.M <= 32 || p.K >= 1 << 24; }

// Kinds of tiles, as in ops_tiles.hip: microseconds for a stage where a compute unit has one workgroup, for each further one
// up to the `fit` that it holds, and for each workgroup's epilogue.  (They rank the kinds, and are no forecast: with all units busy a stage of 256 x
// 256 takes 2.0, and a tile's beginning and end 10.)  Of 24 sizes between 64 x 512 x 512 and 8192 x 8192 x 4096 the choice is
// the fastest kind and split or within 8 % of it; e. g. in tiles of 256, 128, 64: 512 x 4096 x 4096 34, 17, 12.6 us; 2048 x 4096 x 4096 37,
// 27, 34; 4096^3 43, 49, 66; 512 x 512 x 16384 in 4 parts 37, 21, 15 (whole 111, 47, 31).
struct Kind {
    int bm, bn, fit;
    float alone, more, end;
};
static const Kind kKinds[] = {{256, 256, 1, 1.3f, 0.0f, 8.0f}, {128, 128, 2, 0.6f, 0.4f, 2.0f}, {64, 64, 4, 0.45f, 0.15f, 0.5f}};
struct Choice {
    const Kind *kind;
    int slices;
};
static Choice choose(const HeldProduct &p) {
    Choice best = {};
    float least = 0;
    for (const Kind &k : kKinds) {
        const int64_t tiles = p.clients * ceil_div(p.M, k.bm) * ceil_div(p.N, k.bn), stages = ceil_div(p.K, kUnit) * (kUnit / kDeep);
        const float sums = (float)p.clients * (float)p.M * (float)p.N * 4.0f;
        for (int64_t slices = 1; slices == 1 || (slices <= 16 && stages / slices >= 4); slices *= 2) {
            const float waves = (float)ceil_div(tiles * slices, 256);
            const float stage = waves <= k.fit ? k.alone + (waves - 1) * k.more : (k.alone + (k.fit - 1) * k.more) * waves / k.fit;
            float t = (float)ceil_div(stages, slices) * stage + waves * k.end;
            if (slices > 1) t += 4.0f + (float)(2 * slices + 1) * sums / 6e6f;
            if (!best.kind || t < least) {
                best = {&k, (int)slices};
                least = t;
            }
        }
    }
    return best;
}

// Whether the tiles can read an operand as it lies.
static bool aligned(const Held &o, int64_t K) {
    return K % kUnit == 0 && aligned16(o.codes.p, 1, o.codes.client, o.codes.row) && o.codes.row <= INT64_C(1) << 23 &&
           aligned16(o.scales.p, 1, o.scales.client, o.scales.row);
}

// Copies codes and scales into rows of whole units: zeros and scales of 1 behind the end.  A thread has 16 bytes of codes.
static __global__ __launch_bounds__(256) void k_mx4_lay(Held from, Held to, int64_t n, int rows, int K, int pieces) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, line = i / pieces, client = line / rows;
    if (client >= n) return;
    const int b = (int)(i - line * pieces), left = K - b * 32;
    const int64_t row = line - client * rows;
    const uint8_t *p = (const uint8_t *)from.codes.p + client * from.codes.client + row * from.codes.row + (int64_t)b * 16;
    uint8_t __attribute__((ext_vector_type(16))) v;
    if (left >= 32) {
        v = *(const wide<uint8_t, 16> *)p;
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint8_t byte = 2 * e < left ? p[e] : 0;
            v[e] = 2 * e + 1 == left ? byte & 15 : byte;
        }
    }
    *(uint8_t __attribute__((ext_vector_type(16))) *)((uint8_t *)to.codes.p + client * to.codes.client + row * to.codes.row + (int64_t)b * 16) = v;
    ((uint8_t *)to.scales.p)[client * to.scales.client + row * to.scales.row + b] =
        left > 0 ? ((const uint8_t *)from.scales.p)[client * from.scales.client + row * from.scales.row + b] : 127;
}
static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
static int64_t lines_of(const Held &o, int64_t clients, int64_t rows) { return (o.codes.client || o.scales.client ? clients : 1) * rows; }
static size_t lay_bytes(const Held &o, int64_t clients, int64_t rows, int64_t K) {
    const int64_t units = ceil_div(K, kUnit), lines = lines_of(o, clients, rows);
    return up256((size_t)lines * units * (kUnit / 2)) + up256((size_t)lines * units * (kUnit / 32));
}
static hipError_t lay(Held &o, int64_t clients, int64_t rows, int64_t K, char *to, hipStream_t s) {
    const int64_t units = ceil_div(K, kUnit), lines = lines_of(o, clients, rows), n = lines / rows, pieces = units * (kUnit / 32), blocks = ceil_div(lines * pieces, 256);
    if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
    Held d;
    d.codes = {to, n > 1 ? rows * units * (kUnit / 2) : 0, units * (kUnit / 2)};
    d.scales = {to + up256((size_t)lines * units * (kUnit / 2)), n > 1 ? rows * units * (kUnit / 32) : 0, units * (kUnit / 32)};
    k_mx4_lay<<<(int)blocks, 256, 0, s>>>(o, d, n, (int)rows, (int)K, (int)pieces);
    o = d;
    return hipGetLastError();
}

// Bytes of scratch, in this order: operands that have to be laid out, and partial sums.
size_t mx4_product_workspace(const HeldProduct &p) {
    if (rows_fit(p) || !p.K) return 0;
    const int slices = choose(p).slices;
    return (aligned(p.a, p.K) ? 0 : lay_bytes(p.a, p.clients, p.M, p.K)) + (aligned(p.b, p.K) ? 0 : lay_bytes(p.b, p.clients, p.N, p.K)) +
           (slices > 1 ? (size_t)slices * p.clients * p.M * p.N * sizeof(float) : 0);
}

template <typename T, int BM, int BN, int WR, int WC>
static hipError_t run_tiles(const HeldProduct &p, const Shape &s, hipStream_t stream) {
    const auto kernel = k_mx4_tiles<T, BM, BN, WR, WC>;
    constexpr int stages = HeldTile<BM, BN, 64 * WR * WC>::kLds, ends = WR * WC * 32 * (BN / WC + 4) * 4, lds = stages > ends ? stages : ends;
    if constexpr (lds > 64 * 1024) {
        static aet::PerDevice allowed;
        int dev = 0, ok = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        e = allowed.get(dev, &ok, [&](int *v) {
            *v = 1;
            return hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        });
        if (e != hipSuccess) return e;
    }
    kernel<<<s.blocks, 64 * WR * WC, lds, stream>>>(p.a, p.b, s, p.e);
    return hipGetLastError();
}

template <typename T>
static hipError_t run(HeldProduct p, char *workspace, hipStream_t stream) {
    if (rows_fit(p)) {
        const int64_t tiles_n = ceil_div(p.N, 16), tiles = tiles_n * ceil_div(p.M, p.M <= 16 ? 16 : 32), blocks = tiles * p.clients;
        if (!grid_fits(blocks, 64 * kRowWaves)) return hipErrorInvalidConfiguration;
        const HeldRows s = {p.M, p.N, p.K, (int)tiles_n, (int)tiles};
        if (p.M <= 16) k_mx4_rows<T, 1><<<(int)blocks, 64 * kRowWaves, 0, stream>>>(p.a, p.b, s, p.e);
        else k_mx4_rows<T, 2><<<(int)blocks, 64 * kRowWaves, 0, stream>>>(p.a, p.b, s, p.e);
        return hipGetLastError();
    }
    const Choice c = choose(p);
    const Kind &k = *c.kind;
    const int64_t tiles_n = ceil_div(p.N, k.bn), tiles = ceil_div(p.M, k.bm) * tiles_n, blocks = tiles * p.clients * c.slices;
    if (!grid_fits(blocks, k.bm == 256 ? 512 : 256)) return hipErrorInvalidConfiguration;
    hipError_t e = hipSuccess;
    if (p.K && !aligned(p.a, p.K)) {
        const size_t bytes = lay_bytes(p.a, p.clients, p.M, p.K);
        e = lay(p.a, p.clients, p.M, p.K, workspace, stream);
        workspace += bytes;
    }
    if (p.K && e == hipSuccess && !aligned(p.b, p.K)) {
        const size_t bytes = lay_bytes(p.b, p.clients, p.N, p.K);
        e = lay(p.b, p.clients, p.N, p.K, workspace, stream);
        workspace += bytes;
    }
    if (e != hipSuccess) return e;
    Shape s = {p.M, p.N, (int)(ceil_div(p.K, kUnit) * kUnit)};
    s.tiles_n = (int)tiles_n;
    s.tiles = (int)tiles;
    s.slices = c.slices;
    s.slice_k = (int)(ceil_div(ceil_div(p.K, kUnit), c.slices) * kUnit);
    s.blocks = (int)blocks;
    s.partial = (float *)workspace;
    s.clients = p.clients;
    if (k.bm == 256) e = run_tiles<T, 256, 256, 2, 4>(p, s, stream);
    else if (k.bm == 128) e = run_tiles<T, 128, 128, 2, 2>(p, s, stream);
    else e = run_tiles<T, 64, 64, 2, 2>(p, s, stream);
    if (e != hipSuccess || s.slices == 1) return e;
    return launch_join(sizeof(T) == 4 ? AET_F32 : AET_BF16, s, p.e, stream);
}
hipError_t launch_mx4_product(int dtype, const HeldProduct &p, void *workspace, hipStream_t s) {
    return dtype == AET_F32 ? run<float>(p, (char *)workspace, s) : run<bf16>(p, (char *)workspace, s);
}

}  // namespace aet_ops
