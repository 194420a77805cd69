// C[m][n] = sum over k of A(m, k) B(n, k) on the matrix cores, a tile of C per workgroup.
#pragma once
#include "ops_epilogue.h"

namespace aet_ops {

// By rows: element (r, k) is at p + client * c + row * r + k.  By columns: at p + client * c + row * k + r.  Padded: what
// lies side by side goes on with zeros up to a multiple of 8.  low: where not 0, the values are in two bf16 parts, whose second
// lies that many elements behind the first (A of a product with B by columns only); third: and a third one as far behind the second.
struct Operand {
    const void *p;
    int64_t client, row;
    bool by_columns, padded;
    int64_t low;
    bool third;
};
__host__ __device__ inline int parts_of(const Operand &o) { return o.low ? (o.third ? 3 : 2) : 1; }

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
// Both gradients of a layer in one launch, where both are small (taken).
hipError_t launch_pair(int dtype, const Product &x, const Product &w, hipStream_t s, bool *taken);

// Both gradients of a layer whose W and x lie expanded (bf16, a quarter of their values; B of w and x): A, which is dz, in up to three parts; those that have a
// place.  The results are of `dtype`.  In one launch where both are small.
bool held_straight(const Operand &dz, int rows, int out);   // whether dz can be read as it lies
size_t held_products_workspace(const Product &x, const Product &w);
hipError_t launch_held_products(int dtype, const Product &x, const Product &w, void *workspace, hipStream_t s);

}  // namespace aet_ops
