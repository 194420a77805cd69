// Internal declarations shared by the operators' entry points and their kernel launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../per_device.h"
#include "ops_device.h"

namespace aet_ops {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Whether vectors of 16 bytes can be read at p + any multiples of the strides (elements of e bytes).
inline bool aligned16(const void *p, int64_t e, int64_t s1, int64_t s2, int64_t s3 = 0) {
    return ((uintptr_t)p | (uintptr_t)(s1 * e) | (uintptr_t)(s2 * e) | (uintptr_t)(s3 * e)) % 16 == 0;
}

Drop make_drop(double p, uint64_t seed, int64_t first_row, int64_t cols);

hipError_t launch_dropout(const aet_dropout &a, hipStream_t s);

size_t linear_forward_workspace(const aet_linear &a);
hipError_t launch_linear_forward(const aet_linear &a, void *workspace, hipStream_t s);
size_t linear_backward_workspace(const aet_linear_grad &a);
hipError_t launch_linear_backward(const aet_linear_grad &a, void *workspace, hipStream_t s);

size_t group_norm_forward_workspace(const aet_group_norm &a);
hipError_t launch_group_norm_forward(const aet_group_norm &a, void *workspace, hipStream_t s);
size_t group_norm_backward_workspace(const aet_group_norm_grad &a);
hipError_t launch_group_norm_backward(const aet_group_norm_grad &a, void *workspace, hipStream_t s);

}  // namespace aet_ops
