// Stages of products on the matrix cores: operands in LDS, and the ways there.
#pragma once
#include "ops_tiles.h"

namespace aet_ops {

typedef short s4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char *lds_ptr;

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

}  // namespace aet_ops
