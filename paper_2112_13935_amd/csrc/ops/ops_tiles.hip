// Products on the matrix cores, for the linear layer and its gradient: a tile of C per workgroup, staged through LDS.
//
// bf16: v_mfma_f32_32x32x16_bf16.  fp32: the same unit, each value in three bf16 parts and six products (split_bf16.h),
// which holds 24 bits at 6/16 of the fp32 unit's time.
//
// A stage of BK along k of both operands lies in LDS in pieces of 16 bytes (8 values, in one part): by rows as [row][BK],
// by columns as [k][row], so that both are copied as they lie in memory and no transposition is made on the way.  A lane
// of the matrix unit wants 8 consecutive k of one row: by rows one ds_read_b128, by columns two ds_read_b64_tr_b16, which
// hand 16 lanes the transpose of 4 pieces of memory.  The pieces of a row are permuted by exclusive or with the row's number
// (by columns: in groups of 4 with k), so that the lanes that read together find different banks.
//
// Where there are tiles enough: 16384 x 4096 x 4096 in bf16 455 us (1210 TF/s; with zeros, at the full clock, 1376), 4 x
// (4096 x 2048 x 8192) with B by columns 530, with both 500, with A in two parts twice that; 4096 x 4096 x 4096 in fp32 690 us (199
// TF/s, which is as many bf16 products a second).  In the first the matrix unit is busy 54 % of the cycles; the waves, two a
// SIMD, are at a wait or barrier 27 % of their time and ready but not chosen 47 %; LDS is busy 22 % (by columns 47, 53, 35 and 18 %).  256 x 256 in bf16 is the tile whose operands the L2 brings in
// the time of its products (256 x 128, two workgroups a unit: 1037 TF/s).  fp32 has 128 x 128, whose parts and two
// accumulators fill registers and LDS, two workgroups a unit: one splits and stores while the other multiplies.  Deeper
// prefetch, more buffers and tiles that fetch the next tile's operands cost more than they gave.
#include "ops_internal.h"
#include "ops_tiles.h"

#include <type_traits>

#include "../split_bf16.h"

namespace aet_ops {

typedef short s4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char *lds_ptr;

struct Shape {
    int M, N, K;
    int tiles_n, tiles;       // tiles of C: in a row, of a client
    int slices, slice_k;      // parts of the sum (slice_k a multiple of BK); partial sums go to `partial` where there are several
    int blocks;
    float *partial;           // [slice][client][M][N]
    int clients;
};

// ---- staging -----------------------------------------------------------------------------

// Piece (r, c) of an operand's stage: by rows row r, values 8 c .. of the stage; by columns k = r, rows 8 c ..
template <int R, int BK, bool COLS>
struct Stage {
    static constexpr int kPieces = R * BK / 8;
    static constexpr int kWidth = COLS ? R / 8 : BK / 8;   // pieces side by side
    static constexpr int kBytes = R * BK * 2;              // of a part
    static __device__ __forceinline__ int slot(int r, int c) {
        if constexpr (COLS) return r * kWidth + (c ^ ((r & 3 & (R / 32 - 1)) << 2));
        else return r * kWidth + (c ^ (BK == 64 ? (r >> 1) & 7 : (r >> 2) & 3));
    }
    // Lane addresses of fragment t (rows 32 t ..): 8 k of row 32 t + lane % 32 from k = 16 ks + 8 (lane / 32) on
    static __device__ __forceinline__ bf8 fragment(lds_ptr part, int t, int ks, int lane) {
        if constexpr (COLS) {
            const int i = lane & 15, j = i >> 2, k = 16 * ks + 8 * (lane >> 5) + j;
            const int c = (4 * t + 2 * (lane >> 4 & 1) + (i >> 1 & 1)) ^ ((j & (R / 32 - 1)) << 2);
            const lds_ptr at = part + k * (R * 2) + c * 16 + (i & 1) * 8;
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)at);
            const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(at + 4 * R * 2));
            typedef short s8 __attribute__((ext_vector_type(8)));
            const s8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(bf8, both);
        } else {
            const int r = lane & 31, c = 2 * ks + (lane >> 5);
            return *(__attribute__((address_space(3))) bf8 *)(part + t * (32 * BK * 2) + slot(r, c) * 16);
        }
    }
};

// Through registers: any alignment, any end of rows and sums.
template <typename T, int R, int BK, bool COLS, int THREADS>
struct RegStage {
    using S = Stage<R, BK, COLS>;
    static constexpr int kCount = S::kPieces / THREADS;
    static_assert(kCount > 0 && S::kPieces % THREADS == 0 && THREADS % S::kWidth == 0, "whole pieces a thread");
    static constexpr int kStep = THREADS / S::kWidth;   // rows between a thread's pieces
    wide<T, 8> raw[kCount];
    const T *p;          // of the thread's piece column in the next stage
    int64_t row;
    int r, c, piece, left;   // left: of the sum
    int rows;            // of the operand, from the tile's first on

    __device__ __forceinline__ void begin(const Operand &o, int64_t client, int r0, int rows_all, int k0, int k1) {
        r = threadIdx.x / S::kWidth;
        c = piece = threadIdx.x % S::kWidth;
        row = o.row;
        rows = rows_all - r0;
        left = k1 - k0;
        if (COLS && 8 * c >= rows) c = (rows - 1) / 8;   // (the place in LDS is `piece`)
        p = (const T *)o.p + client * o.client + (COLS ? (int64_t)k0 * row + r0 + 8 * c : (int64_t)r0 * row + k0 + 8 * c);
    }
    // Stages from the first that can be read without looking where each piece ends.  Rows past the last are read from
    // the last again, and become rows of C that are not stored.  By columns so are pieces past the last; the last runs over
    // the end of its line, which is in the operand's memory where lines of 8 and more values follow.
    __device__ __forceinline__ int plain() const {
        if (!COLS || rows >= R || rows % 8 == 0) return left / BK;
        return row >= 8 ? (left - 1) / BK : 0;
    }
    template <bool PLAIN>
    __device__ __forceinline__ void load() {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int ri = r + i * kStep;
            if (PLAIN) {
                raw[i] = *(const wide<T, 8> *)(p + (int64_t)(COLS || ri < rows ? ri : rows - 1) * row);
            } else {
                const bool in = ri < (COLS ? left : rows);
                raw[i] = load_raw<T, 8>(p + (int64_t)ri * row, in ? (COLS ? rows : left) - 8 * c : 0);
            }
        }
        p += COLS ? BK * row : BK;
        left -= BK;
    }
    // parts: of kBytes each
    __device__ __forceinline__ void store(lds_ptr to) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const lds_ptr at = to + S::slot(r + i * kStep, piece) * 16;
            if constexpr (sizeof(T) == 2) {
                *(__attribute__((address_space(3))) bf8 *)at = raw[i];
            } else {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = raw[i][e];
                aet::Split8 s = aet::split8<false>(v);
                uint32_t seen = 0;
                aet::split_watch(seen, s);
                if (aet::split_over(seen)) s = aet::split8<true>(v);   // something infinite, NaN or next to it
#pragma unroll
                for (int q = 0; q < 3; ++q) *(__attribute__((address_space(3))) bf8 *)(at + q * S::kBytes) = s.p[q];
            }
        }
    }
};

// From memory into LDS, without registers: 16-byte aligned pieces, none of which an end of the rows or the sum parts.  Rows
// past the last are read from the last again: they become rows of C that are not stored.
template <int R, int BK, bool COLS, int THREADS>
struct DirectStage {
    using S = Stage<R, BK, COLS>;
    static constexpr int kCount = S::kPieces / THREADS;
    const char *p;              // the stage's first byte, the same for all threads
    uint32_t at[kCount];
    int64_t step;

    // The thread's piece i: its row and place in the row
    static __device__ __forceinline__ int row_of(int i) { return (threadIdx.x + i * THREADS) / S::kWidth; }
    static __device__ __forceinline__ int place_of(int i) {
        const int r = row_of(i);
        return S::slot(r, (threadIdx.x + i * THREADS) % S::kWidth) - r * S::kWidth;   // the permutation is its own inverse
    }
    __device__ __forceinline__ void begin(const Operand &o, int64_t client, int r0, int rows_all, int k0, int) {
        const int rows = rows_all - r0;
        p = (const char *)((const bf16 *)o.p + client * o.client + (COLS ? (int64_t)k0 * o.row + r0 : (int64_t)r0 * o.row + k0));
        step = (COLS ? BK * o.row : BK) * 2;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int r = row_of(i), c = place_of(i);
            if (COLS) {
                const int last = (o.padded ? (rows + 7) & ~7 : rows) - 8;
                at[i] = (uint32_t)r * (uint32_t)(o.row * 2) + (uint32_t)(8 * c < last ? 8 * c : last) * 2;
            } else {
                at[i] = (uint32_t)(r < rows ? r : rows - 1) * (uint32_t)(o.row * 2) + c * 16;
            }
        }
    }
    __device__ __forceinline__ void load(lds_ptr to) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
        for (int i = 0; i < kCount; ++i)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(p + at[i]),
                                             (__attribute__((address_space(3))) void *)(to + (i * THREADS + wave * 64) * 16), 16, 0, 0);
        p += step;
    }
    // The sum's last stage, of which `left` k are there: the rest are zeros.
    __device__ __forceinline__ void load_end(lds_ptr to, int left) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            if ((COLS ? row_of(i) : 8 * place_of(i)) < left)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(p + at[i]),
                                                 (__attribute__((address_space(3))) void *)(to + (i * THREADS + wave * 64) * 16), 16, 0, 0);
            else
                *(__attribute__((address_space(3))) bf8 *)(to + (i * THREADS + threadIdx.x) * 16) = bf8{};
        }
    }
};

// Asks the compiler to put READS of LDS behind the first of PRODUCTS of the matrix unit, so that they have the others' time.
template <int PRODUCTS, int READS>
__device__ __forceinline__ void interleave() {
    constexpr int first = PRODUCTS >= 8 ? 3 : 1, each = (READS + first - 1) / first;
#pragma unroll
    for (int i = 0; i < first; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, each, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS - first, 0);
}

// ---- the kernel --------------------------------------------------------------------------

template <typename T>
struct Parts {
    static constexpr int kParts = sizeof(T) == 2 ? 1 : 3;
};

// BM x BN of C, waves WR x WC; a wave has BM / WR x BN / WC in fragments of 32 x 32.
template <typename T, int BM, int BN, int BK, int WR, int WC, bool TA, bool TB, bool DIRECT>
struct Tile {
    static constexpr int kThreads = 64 * WR * WC;
    static constexpr int FM = BM / WR / 32, FN = BN / WC / 32;
    static constexpr int kParts = Parts<T>::kParts;
    using SA = Stage<BM, BK, TA>;
    using SB = Stage<BN, BK, TB>;
    static constexpr int kStage = kParts * (SA::kBytes + SB::kBytes);
    static constexpr int kBuffers = DIRECT ? 2 : 1;
    static constexpr int kEpilogue = WR * WC * 32 * (FN * 32 + 4) * 4;
    static constexpr int kLds = kStage * kBuffers > kEpilogue ? kStage * kBuffers : kEpilogue;
};

template <typename T, int BM, int BN, int BK, int WR, int WC, bool TA, bool TB, bool DIRECT>
__device__ __forceinline__ void tile_of(const Operand &oa, const Operand &ob, const Shape &s, const Epilogue &e, int block, lds_ptr lds) {
    using L = Tile<T, BM, BN, BK, WR, WC, TA, TB, DIRECT>;
    constexpr int FM = L::FM, FN = L::FN, P = L::kParts;
    using SA = typename L::SA;
    using SB = typename L::SB;
    int id = xcd_order(block, s.blocks);
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

    f16v acc[FN][FM], corr[P == 3 ? FN : 1][P == 3 ? FM : 1];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            acc[i][j] = f16v{};
            if constexpr (P == 3) corr[i][j] = f16v{};
        }

    struct Fragments {
        bf8 a[FM][P], b[FN][P];
    };
    const auto read = [&](Fragments &f, lds_ptr stage, int ks) {
#pragma unroll
        for (int q = 0; q < P; ++q) {
#pragma unroll
            for (int i = 0; i < FN; ++i) f.b[i][q] = SB::fragment(stage + (P * SA::kBytes + q * SB::kBytes), wc * FN + i, ks, lane);
#pragma unroll
            for (int j = 0; j < FM; ++j) f.a[j][q] = SA::fragment(stage + q * SA::kBytes, wr * FM + j, ks, lane);
        }
    };
    const auto multiply = [&](const Fragments &f) {
        if constexpr (P == 1) {
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int j = 0; j < FM; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.b[i][0], f.a[j][0], acc[i][j], 0, 0, 0);
        } else {
#pragma unroll
            for (int q = 0; q < 6; ++q)
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int j = 0; j < FM; ++j) aet::split_mfma(q, f.b[i], f.a[j], acc[i][j], corr[i][j]);
        }
    };

    const int stages = (k1 - k0 + BK - 1) / BK;
    constexpr int kPartA = P * SA::kBytes;
    const auto sum = [&](const Operand &oa) {
        if constexpr (DIRECT) {
            DirectStage<BM, BK, TA, L::kThreads> la;
            DirectStage<BN, BK, TB, L::kThreads> lb;
            la.begin(oa, client, m0, s.M, k0, k1);
            lb.begin(ob, client, n0, s.N, k0, k1);
            // The fragments of the next 16 k are read while the matrix unit has the last ones, also across the barrier that
            // says that the next stage has arrived everywhere and that this one's place may be written again: it comes
            // ahead of the stage's last products, and right behind it the stage after the next is sent for.
            constexpr int kBuffers = L::kBuffers, KS = BK / 16, kReads = (TA ? 2 : 1) * FM + (TB ? 2 : 1) * FN;
            constexpr int kLoads = decltype(la)::kCount + decltype(lb)::kCount;
            static_assert(kBuffers == 2, "every wait in the loop is for all that is on its way");
            const int whole = k1 > k0 ? (k1 - k0) / BK : 0;   // stages; there may be an end of another
            const auto fetch = [&](int i) {
                const lds_ptr to = lds + i % kBuffers * L::kStage;
                la.load(to);
                lb.load(to + kPartA);
            };
            const auto fetch_end = [&]() {
                const lds_ptr to = lds + whole % kBuffers * L::kStage;
                la.load_end(to, k1 - k0 - whole * BK);
                lb.load_end(to + kPartA, k1 - k0 - whole * BK);
            };
            // s_waitcnt by its encoding (vmcnt low and high bits, lgkmcnt 0), which the compiler takes into account
            const auto arrived = [&](auto still) {
                __builtin_amdgcn_s_waitcnt(0x0070 | (still & 15) | (still >> 4) << 14);
                __builtin_amdgcn_s_barrier();
            };
            typedef std::integral_constant<int, (kBuffers - 2) * kLoads> Others;
            typedef std::integral_constant<int, 0> None;
            Fragments f[2];
            for (int i = 0; i < kBuffers && i < whole; ++i) fetch(i);
            if (whole < stages && whole < kBuffers) fetch_end();   // (whose loads cannot be counted)
            if (whole >= kBuffers) arrived(std::integral_constant<int, (kBuffers - 1) * kLoads>());
            else arrived(None());
            if (stages > 0) read(f[0], lds, 0);
            int i = 0;
            const auto stage = [&](auto get) {
    #pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    if (ks + 1 == KS) {
                        arrived(Others());
                        get();
                    }
                    read(f[(ks + 1) % 2], lds + (i + (ks + 1) / KS) % kBuffers * L::kStage, (ks + 1) % KS);
                    multiply(f[ks % 2]);
                    interleave<FM * FN, kReads>();
                }
            };
            for (; i + kBuffers < whole; ++i) stage([&]() { fetch(i + kBuffers); });
            if (i + kBuffers < stages) {
                stage(fetch_end);
                ++i;
            }
            for (; i < stages; ++i) {
    #pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    if (ks + 1 == KS) arrived(None());
                    if (ks + 1 < KS || i + 1 < stages) read(f[(ks + 1) % 2], lds + (i + (ks + 1) / KS) % kBuffers * L::kStage, (ks + 1) % KS);
                    multiply(f[ks % 2]);
                }
            }
        } else {
            RegStage<T, BM, BK, TA, L::kThreads> la;
            RegStage<T, BN, BK, TB, L::kThreads> lb;
            la.begin(oa, client, m0, s.M, k0, k1);
            lb.begin(ob, client, n0, s.N, k0, k1);
            // A stage goes from memory to registers while the one before it is worked on.  One buffer: there is another
            // workgroup on the compute unit whose products go on while this one splits and stores.
            const auto work = [&]() {
    #pragma unroll
                for (int ks = 0; ks < BK / 16; ++ks) {
                    Fragments f;
                    read(f, lds, ks);
                    multiply(f);
                }
            };
            const auto put = [&]() {
                __syncthreads();
                la.store(lds);
                lb.store(lds + kPartA);
                __syncthreads();
            };
            const int whole = la.plain() < lb.plain() ? la.plain() : lb.plain();
            if (whole > 0) {
                la.template load<true>();
                lb.template load<true>();
            } else {
                la.template load<false>();
                lb.template load<false>();
            }
            int i = 0;
            for (; i + 1 < whole; ++i) {
                put();
                la.template load<true>();
                lb.template load<true>();
                work();
            }
            for (; i < stages; ++i) {
                put();
                la.template load<false>();
                lb.template load<false>();
                work();
            }
        }
    };
    sum(oa);
    if constexpr (TB && sizeof(T) == 2) {   // A in two parts: the sum over the second on top
        if (oa.low) {
            Operand low = oa;
            low.p = (const T *)oa.p + oa.low;
            __syncthreads();   // the last stage has been read
            sum(low);
        }
    }
    __syncthreads();

    // A lane has, of row m0 + lane % 32 of a fragment, four columns at a time: through LDS, a wave for itself, to lanes
    // with V columns (16 bytes) each, in whole lines of memory.
    constexpr int V = 16 / sizeof(T), W = FN * 32, LINE = W + 4, ACROSS = W / V, DOWN = 64 / ACROSS;
    __attribute__((address_space(3))) float *mine = (__attribute__((address_space(3))) float *)lds + wave * (32 * LINE);
    const int col = n0 + wc * W + lane % ACROSS * V;
    const int count = s.N - col;
    float bias[V];
    bias_of<T>(e, client, col, s.slices > 1 ? 0 : count, bias);
#pragma unroll
    for (int j = 0; j < FM; ++j) {
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f4 v;
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = P == 3 ? aet::split_sum(acc[i][j][4 * q + x], corr[P == 3 ? i : 0][P == 3 ? j : 0][4 * q + x]) : acc[i][j][4 * q + x];
                *(__attribute__((address_space(3))) f4 *)(mine + (lane & 31) * LINE + i * 32 + 8 * q + 4 * (lane >> 5)) = v;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
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
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T, int BM, int BN, int BK, int WR, int WC, bool TA, bool TB, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_tiles(Operand oa, Operand ob, Shape s, Epilogue e) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    tile_of<T, BM, BN, BK, WR, WC, TA, TB, DIRECT>(oa, ob, s, e, blockIdx.x, (lds_ptr)lds);
}

// Two small products in one launch: the gradients of a layer's inputs (B by columns) and of its weights (both by columns).
template <typename T, int BM, int BN, int BK, int WR, int WC, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_tiles_pair(Product x, Shape sx, Product w, Shape sw) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int block = blockIdx.x;
    if (block < sx.blocks) tile_of<T, BM, BN, BK, WR, WC, false, true, DIRECT>(x.a, x.b, sx, x.e, block, (lds_ptr)lds);
    else tile_of<T, BM, BN, BK, WR, WC, true, true, DIRECT>(w.a, w.b, sw, w.e, block - sx.blocks, (lds_ptr)lds);
}

// Adds the slices of a split sum, in their order, and ends it.  A thread has 16 bytes of C.  Bound by memory: two slices of
// 3 x (1001 x 771) in fp32 with a residual, 37 MB from the caches, 8 to 11 us.
template <typename T>
__global__ __launch_bounds__(256) void k_join(Shape s, Epilogue e) {
    constexpr int V = 16 / sizeof(T);
    const int wide = (s.N + V - 1) / V;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t line = i / wide;
    if (line >= (int64_t)s.clients * s.M) return;
    const int col = (int)(i - line * wide) * V, count = s.N - col;
    const int64_t client = line / s.M, row = line - client * s.M;
    float v[V];
    bias_of<T>(e, client, col, count, v);
    for (int k = 0; k < s.slices; ++k) {
        float x[V];
        load_some(s.partial + ((int64_t)k * s.clients * s.M + line) * s.N + col, count, x);
#pragma unroll
        for (int y = 0; y < V; ++y) v[y] += x[y];
    }
    finish<T>(e, client, row, col, count, v);
}

// ---- the choice --------------------------------------------------------------------------

// Whether the operand's stages of BK can go straight into LDS.
static bool direct(const Operand &o, int rows, int K, int BK) {
    const int64_t across = o.by_columns ? BK : 256;
    return aligned16(o.p, 2, o.client, o.row) && o.row * 2 * across < (INT64_C(1) << 31) && K > 0 &&
           (o.padded || (o.by_columns ? rows : K) % 8 == 0);
}

template <typename T, int BM, int BN, int BK, int WR, int WC, bool TA, bool TB, bool DIRECT>
static hipError_t run_tiles(const Product &p, Shape s, hipStream_t stream) {
    using L = Tile<T, BM, BN, BK, WR, WC, TA, TB, DIRECT>;
    const auto kernel = k_tiles<T, BM, BN, BK, WR, WC, TA, TB, DIRECT>;
    if constexpr (L::kLds > 64 * 1024) {
        static aet::PerDevice allowed;
        int dev = 0, ok = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        e = allowed.get(dev, &ok, [&](int *v) {
            *v = 1;
            return hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, L::kLds);
        });
        if (e != hipSuccess) return e;
    }
    kernel<<<s.blocks, L::kThreads, L::kLds, stream>>>(p.a, p.b, s, p.e);
    return hipGetLastError();
}

// Kinds of tiles, and what they take: `alone` microseconds for a stage where a compute unit has one workgroup, `more` for
// each further one up to the `fit` that it holds at a time (then it goes on as with all of them), `end` for each
// workgroup's epilogue.  Measured on products of 33 to 8192 rows, 100 to
// 4096 columns and sums of 32 to 8192; a few examples, in microseconds, with the kinds as they are listed here:
//   fp32  4096 x 4096 x 4096  690, 810, 900;   2048 x 2048 x 1024  72, 63, 67;   3 x (1001 x 771 x 1155)  85, 66, 58
//   bf16  4096 x 4096 x 4096  124, 140, 166, 199;   2048 x 2048 x 1024  28, 13.8, 13.6, 15.8;   512 x 4096 x 4096  83, 41, 36, 32
// A sum is split where its tiles leave compute units idle (fp32 512 x 4096 x 4096, 128 x 128: 238, two slices 138, four 109);
// partial sums are written and read at about 6 TB/s (they stay in the caches), and the launch that adds them takes 4.
struct Kind {
    int bm, bn, bk, fit;
    float alone, more, end;
};
static const Kind kKinds32[] = {{128, 128, 32, 2, 2.2f, 0.5f, 2.0f}, {64, 128, 32, 3, 1.35f, 0.60f, 1.0f}, {64, 64, 32, 5, 0.95f, 0.35f, 0.5f}};
static const Kind kKinds16[] = {{256, 256, 64, 1, 1.6f, 0.0f, 8.0f}, {128, 128, 64, 2, 0.65f, 0.45f, 2.0f}, {64, 128, 64, 3, 0.54f, 0.22f, 1.0f}, {64, 64, 64, 5, 0.46f, 0.13f, 0.5f}};

// bf16 through registers (256 x 256 by rows only: 4095 x 4097 x 4093 by rows 160, 128 x 128 209, by columns 281 and 217)
static const Kind kKinds16Any[] = {{256, 256, 64, 1, 2.6f, 0.0f, 8.0f}, {128, 128, 64, 2, 1.7f, 0.4f, 2.0f}, {64, 128, 64, 3, 0.95f, 0.42f, 1.0f}, {64, 64, 64, 5, 0.62f, 0.31f, 0.5f}};

struct Choice {
    const Kind *kind;
    int slices;
    float time;
};
static float time_of(const Kind &k, int64_t stages, int64_t blocks) {
    const float waves = (float)ceil_div(blocks, 256);
    const float stage = waves <= k.fit ? k.alone + (waves - 1) * k.more : (k.alone + (k.fit - 1) * k.more) * waves / k.fit;
    return (float)stages * stage + waves * k.end;
}
static Choice choose(int dtype, const Product &p, bool straight) {
    Choice best = {};
    const auto consider = [&](const Kind &k) {
        const int64_t tiles = p.clients * ceil_div(p.M, k.bm) * ceil_div(p.N, k.bn), stages = ceil_div(p.K, k.bk);
        const float sums = (float)p.clients * (float)p.M * (float)p.N * 4.0f;
        const int parts = p.a.low ? 2 : 1;
        for (int64_t slices = 1; slices == 1 || (slices <= 64 && stages / slices >= 2); slices *= 2) {
            float t = time_of(k, ceil_div(stages, slices) * parts, tiles * slices);
            if (slices > 1) t += 4.0f + (float)(2 * slices + 1) * sums / 6e6f;
            if (!best.kind || t < best.time) best = {&k, (int)slices, t};
        }
    };
    if (dtype == AET_F32) for (const Kind &k : kKinds32) consider(k);
    else if (straight) for (const Kind &k : kKinds16) consider(k);
    else for (const Kind &k : kKinds16Any) if (k.bm < 256 || !p.b.by_columns) consider(k);
    return best;
}

size_t product_workspace(int dtype, const Product &p) {
    if (rows_fit(p)) return 0;
    // enough for either way, so that it does not depend on where the tensors lie
    const int a = choose(dtype, p, true).slices, b = choose(dtype, p, false).slices, slices = a > b ? a : b;
    return slices > 1 ? (size_t)slices * p.clients * p.M * p.N * sizeof(float) : 0;
}

// The product's tiles of this kind.
static bool shape_of(const Product &p, const Choice &c, void *workspace, Shape *s) {
    const Kind &k = *c.kind;
    *s = {p.M, p.N, p.K};
    s->clients = p.clients;
    s->tiles_n = (int)ceil_div(p.N, k.bn);
    const int64_t tiles = ceil_div(p.M, k.bm) * s->tiles_n, blocks = tiles * p.clients * c.slices;
    s->tiles = (int)tiles;
    s->blocks = (int)blocks;
    s->slices = c.slices;
    s->slice_k = (int)ceil_div(ceil_div(p.K, k.bk), c.slices) * k.bk;
    s->partial = (float *)workspace;
    return blocks <= INT32_MAX;
}
template <typename T>
static bool straight(const Product &p) {
    return sizeof(T) == 2 && direct(p.a, p.M, p.K, 64) && direct(p.b, p.N, p.K, 64);
}

template <typename T, bool TA, bool TB>
static hipError_t run_product(const Product &p, void *workspace, hipStream_t stream) {
    const bool d = straight<T>(p);
    const Choice c = choose(sizeof(T) == 4 ? AET_F32 : AET_BF16, p, d);
    const Kind &k = *c.kind;
    Shape s;
    if (!shape_of(p, c, workspace, &s)) return hipErrorInvalidConfiguration;
    if (!s.blocks) return hipSuccess;
    hipError_t e;
    if constexpr (sizeof(T) == 4) {
        if (k.bm == 128) e = run_tiles<T, 128, 128, 32, 2, 2, TA, TB, false>(p, s, stream);
        else if (k.bn == 128) e = run_tiles<T, 64, 128, 32, 2, 2, TA, TB, false>(p, s, stream);
        else e = run_tiles<T, 64, 64, 32, 2, 2, TA, TB, false>(p, s, stream);
    } else {
        if (k.bm == 256) {
            if constexpr (TB) e = run_tiles<T, 256, 256, 64, 2, 4, TA, TB, true>(p, s, stream);
            else e = d ? run_tiles<T, 256, 256, 64, 2, 4, TA, TB, true>(p, s, stream) : run_tiles<T, 256, 256, 64, 2, 4, TA, TB, false>(p, s, stream);
        } else if (k.bm == 128) e = d ? run_tiles<T, 128, 128, 64, 2, 2, TA, TB, true>(p, s, stream) : run_tiles<T, 128, 128, 64, 2, 2, TA, TB, false>(p, s, stream);
        else if (k.bn == 128) e = d ? run_tiles<T, 64, 128, 64, 2, 2, TA, TB, true>(p, s, stream) : run_tiles<T, 64, 128, 64, 2, 2, TA, TB, false>(p, s, stream);
        else e = d ? run_tiles<T, 64, 64, 64, 2, 2, TA, TB, true>(p, s, stream) : run_tiles<T, 64, 64, 64, 2, 2, TA, TB, false>(p, s, stream);
    }
    if (e != hipSuccess || s.slices == 1) return e;
    k_join<T><<<(int)ceil_div((int64_t)p.clients * p.M * ceil_div(p.N, 16 / sizeof(T)), 256), 256, 0, stream>>>(s, p.e);
    return hipGetLastError();
}

hipError_t launch_product(int dtype, const Product &p, void *workspace, hipStream_t s) {
    if (rows_fit(p)) return launch_rows(dtype, p, s);
    const bool f32 = dtype == AET_F32;
    if (!p.a.by_columns && !p.b.by_columns) return f32 ? run_product<float, false, false>(p, workspace, s) : run_product<bf16, false, false>(p, workspace, s);
    if (!p.a.by_columns) return f32 ? run_product<float, false, true>(p, workspace, s) : run_product<bf16, false, true>(p, workspace, s);
    return f32 ? run_product<float, true, true>(p, workspace, s) : run_product<bf16, true, true>(p, workspace, s);
}

template <typename T>
static hipError_t run_pair(const Product &x, const Product &w, hipStream_t stream, bool *taken) {
    const int dtype = sizeof(T) == 4 ? AET_F32 : AET_BF16;
    // the smallest kind, sums in one piece; a launch less is worth 3
    const bool d = straight<T>(x);
    const Kind &k = dtype == AET_F32 ? kKinds32[2] : d ? kKinds16[3] : kKinds16Any[3];
    const Choice one = {&k, 1};
    *taken = false;
    Shape sx, sw;
    if (d != straight<T>(w) || !shape_of(x, one, nullptr, &sx) || !shape_of(w, one, nullptr, &sw) || !sx.blocks || !sw.blocks ||
        sx.blocks > INT32_MAX - sw.blocks)
        return hipSuccess;
    if (time_of(k, ceil_div(x.K > w.K ? x.K : w.K, k.bk) * (x.a.low ? 2 : 1), (int64_t)sx.blocks + sw.blocks) > choose(dtype, x, d).time + choose(dtype, w, d).time + 3.0f)
        return hipSuccess;
    *taken = true;
    constexpr int BK = sizeof(T) == 4 ? 32 : 64;
    const int blocks = sx.blocks + sw.blocks;
    if constexpr (sizeof(T) == 2) {
        if (d) {
            using L = Tile<T, 64, 64, BK, 2, 2, true, true, true>;
            k_tiles_pair<T, 64, 64, BK, 2, 2, true><<<blocks, L::kThreads, L::kLds, stream>>>(x, sx, w, sw);
            return hipGetLastError();
        }
    }
    using L = Tile<T, 64, 64, BK, 2, 2, true, true, false>;
    static_assert(L::kLds <= 64 * 1024, "no permission needed");
    k_tiles_pair<T, 64, 64, BK, 2, 2, false><<<blocks, L::kThreads, L::kLds, stream>>>(x, sx, w, sw);
    return hipGetLastError();
}
hipError_t launch_pair(int dtype, const Product &x, const Product &w, hipStream_t s, bool *taken) {
    return dtype == AET_F32 ? run_pair<float>(x, w, s, taken) : run_pair<bf16>(x, w, s, taken);
}

}  // namespace aet_ops
