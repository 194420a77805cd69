// C[m][n] = sum over k of A(m, k) B(n, k) of values held in microscaled 4-bit floating point.
#pragma once
#include "ops_tiles.h"

namespace aet_ops {

// Rows of codes and scales; strides in bytes.
struct Held {
    aet_in codes, scales;
};
struct HeldProduct {
    Held a, b;
    int clients, M, N, K;
    Epilogue e;
};
size_t mx4_product_workspace(const HeldProduct &p);
hipError_t launch_mx4_product(int dtype, const HeldProduct &p, void *workspace, hipStream_t s);

}  // namespace aet_ops
