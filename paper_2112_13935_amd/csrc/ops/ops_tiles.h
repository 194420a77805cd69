// C[m][n] = sum over k of A(m, k) B(n, k) on the matrix cores, a tile of C per workgroup.
#pragma once
#include "ops_epilogue.h"

namespace aet_ops {

// By rows: element (r, k) is at p + client * c + row * r + k.  By columns: at p + client * c + row * k + r.  Padded: what
// lies side by side goes on with zeros up to a multiple of 8.  low: where not 0, the values are in two bf16 parts, whose second
// lies that many elements behind the first (A of a product with B by columns only).
struct Operand {
    const void *p;
    int64_t client, row;
    bool by_columns, padded;
    int64_t low;
};

struct Product {
    Operand a, b;
    int clients, M, N, K;
    Epilogue e;
};

// A product's tiles.
struct Shape {
    int M, N, K;
    int tiles_n, tiles;       // tiles of C: in a row, of a client
    int slices, slice_k;      // parts of the sum (slice_k a multiple of BK); partial sums go to `partial` where there are several
    int blocks;
    float *partial;           // [slice][client][M][N]
    int clients;
};

// Adds the slices of a split sum, in their order, and ends it.
hipError_t launch_join(int dtype, const Shape &s, const Epilogue &e, hipStream_t stream);

// Few rows (ops_rows.hip): both operands by rows, no scratch.
bool rows_fit(const Product &p);
hipError_t launch_rows(int dtype, const Product &p, hipStream_t s);

// Bytes of scratch that the product wants (for sums that are split along k).
size_t product_workspace(int dtype, const Product &p);
hipError_t launch_product(int dtype, const Product &p, void *workspace, hipStream_t s);
// C's rows times 2^row_shift(tops[client * .client + row]), tops being the exponent of the largest value of the row that A stands for,
// which was made to lie below 2^15 so (no more than kNoExponent: there is none).
struct RowExponents {
    const int32_t *tops;
    int64_t client;
};
constexpr int kNoExponent = -100000;
__device__ __forceinline__ int row_shift(int top) { return top < kNoExponent / 2 ? 0 : top - 15; }
// The same of fp16 operands (A in one part or two), B by columns, where both can go straight into LDS; C is fp32.
bool half_fits(const Product &p);
size_t half_product_workspace(const Product &p);
hipError_t launch_half_product(const Product &p, const RowExponents &half, void *workspace, hipStream_t s);
// Microseconds that products are expected to take; of a layer's gradients (the operands of launch_product in one piece, or by
// launch_pair), those that have clients.
float half_product_time(const Product &p);
float gradients_time(int dtype, const Product &x, const Product &w);
// Both gradients of a layer in one launch, where both are small (taken).
hipError_t launch_pair(int dtype, const Product &x, const Product &w, hipStream_t s, bool *taken);

}  // namespace aet_ops
