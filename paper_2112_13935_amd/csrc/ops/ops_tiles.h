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

// Few rows (ops_rows.hip): both operands by rows, no scratch.
bool rows_fit(const Product &p);
hipError_t launch_rows(int dtype, const Product &p, hipStream_t s);

// Bytes of scratch that the product wants (for sums that are split along k).
size_t product_workspace(int dtype, const Product &p);
hipError_t launch_product(int dtype, const Product &p, void *workspace, hipStream_t s);
// Both gradients of a layer in one launch, where both are small (taken).
hipError_t launch_pair(int dtype, const Product &x, const Product &w, hipStream_t s, bool *taken);

}  // namespace aet_ops
