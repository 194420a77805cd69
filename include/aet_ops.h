/*
 * aet_ops.h -- C ABI of the operators that residual blocks of clients' models are composed
 * from, on MI355X (gfx950): a linear layer with bias, activation, dropout and residual in its
 * epilogue, group normalisation with an activation on channels-last maps, and dropout from
 * the counter generator, each with its gradient.  All of them take many clients' models side
 * by side in one call (`n`), each with parameters of its own or all with the same ones.
 *
 * Conventions
 *   - Every pointer is DEVICE memory owned by the caller.  The library allocates nothing;
 *     calls that need scratch memory take a workspace (size from aet_*_workspace_bytes,
 *     256-byte aligned; NULL where that is 0).  It keeps nothing between calls.
 *   - All tensors of a call have the call's dtype, but for the statistics of a normalisation
 *     (fp32).  Products, sums, statistics and everything between a call's inputs and its
 *     outputs are fp32 or wider; an output is rounded once, to its type.  Two exceptions: dz in
 *     the gradient of a linear layer in bf16 (named there); and fp32 products of more than 32
 *     rows, and all of fp32 gradients, take their operands to within 2^-134, which is less
 *     than 24 bits of one below 2^-110 (forward products of up to 32 rows take all of them).
 *   - Strides are in elements; the last axis has stride 1.  Inputs may have any strides that
 *     are not negative (0: the same values for every row or client).  Outputs must not
 *     overlap themselves, nor an input, except where a call says so.  Any alignment that
 *     the type itself has is taken; 16-byte aligned pointers and strides of whole 16 bytes
 *     are faster.  Memory between the rows of an input may be read; what it holds does not
 *     count.
 *   - Work is enqueued on the given stream of the current device and is asynchronous; nothing
 *     synchronises, so that calls can be captured into a graph.  (The numbers in the
 *     argument record, the dropout's seed among them, are then part of the graph.)
 *   - Every call returns an aet_status; on anything but AET_OK nothing has been enqueued, or
 *     (AET_EHIP) what was enqueued is not to be used.  aet_ops_last_error() describes the
 *     problem of the calling thread's last failed call.  Nothing aborts or throws across the
 *     boundary.  Calls are thread safe.
 *   - Sizes of 0 are legal: sums over nothing are 0.  The largest is 2^30.
 *   - The same call gives the same bits every time.
 */
#ifndef AET_OPS_H
#define AET_OPS_H

#include "aet_sgd.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AET_F32 0
#define AET_BF16 1

/* Activations: z; max(z, 0) (NaN stays); z / (1 + exp(-z)); z Phi(z), Phi the normal
 * distribution function.  The slope of AET_ACT_RELU is 1 for z > 0, else 0. */
#define AET_ACT_NONE 0
#define AET_ACT_RELU 1
#define AET_ACT_SILU 2
#define AET_ACT_GELU 3

/* Dropout, here and in the linear layer: of a tensor with `cols` columns, the value at
 * column j of row number r (first_row + its place among the call's rows, client after
 * client) stays, times 1 / (1 - p), where its half of
 *   h = value number r * ceil(cols / 2) + floor(j / 2)
 * of the SplitMix64 stream of key = value number 3 of the stream of `seed` is no less than
 * p * 2^32 (rounded, at most 2^32 - 1); the lower half for even j, the upper one for odd j.
 * Else it is 0, whatever it was.  A pure function of (seed, r, j, p, cols): nothing is
 * stored for the gradient, which draws the same mask.  0 <= p < 1; p = 0 leaves everything
 * as it is.  first_row >= 0 places a part of a larger tensor. */

/* Element (c, r, j) of a matrix per client is at p + c * client + r * row + j. */
typedef struct {
    const void *p;
    int64_t client, row;
} aet_in;
typedef struct {
    void *p;
    int64_t client, row;
} aet_out;

/* y = residual + dropout(act(z)),  z = x W^T + bias, for n clients.
 *   x         n x rows x in
 *   w         n x out x in (row: stride of an output's weights); client = 0: one W for all
 *   bias      n x out (row is ignored), or p = NULL
 *   residual  n x rows x out, or p = NULL
 *   y         n x rows x out; may be `residual` itself, with the same strides
 *   pre       n x rows x out: z, for the gradient; or p = NULL */
typedef struct {
    int32_t dtype, act;
    int32_t n, rows, in, out;
    double p;
    uint64_t seed;
    int64_t first_row;
    aet_in x, w, bias, residual;
    aet_out y, pre;
} aet_linear;
size_t aet_linear_workspace_bytes(const aet_linear *a);
aet_status aet_linear_forward(const aet_linear *a, void *workspace, size_t workspace_bytes, void *hip_stream);

/* The gradient:  dz = dropout'(dy) * act'(z),  dx = dz W,  dw = dz^T x,  db = sum of dz over
 * rows; that of the residual is dy itself.  Each output is left out where its p is NULL.
 *   pre       z as the forward call gave it; p = NULL where act is AET_ACT_NONE
 *   dw, db    client = 0 with n other than 1: one W (bias) for all clients, whose gradient is the sum
 *             over them; x, dy, pre and dx, those of them that the call wants, then lie row after
 *             row, client after client (client = rows * row; with one row a client, any), and
 *             w.client (for dx), dw.client and db.client are all 0
 * bf16: the matrix cores take bf16 only, so dz goes into the products as a sum of two bf16
 * values, to within 2^-16 of it (and 2^-134 where it is tiny), a product with each; without
 * activation and dropout it is dy as it is.  db sums dz in fp32. */
typedef struct {
    int32_t dtype, act;
    int32_t n, rows, in, out;
    double p;
    uint64_t seed;
    int64_t first_row;
    aet_in dy, x, w, pre;
    aet_out dx, dw, db;
} aet_linear_grad;
size_t aet_linear_backward_workspace_bytes(const aet_linear_grad *a);
aet_status aet_linear_backward(const aet_linear_grad *a, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Group normalisation, channels last.  A sample has `positions` rows of groups * width
 * channels; element (c, b, i, k) is at p + c * client + b * sample + i * row + k. */
typedef struct {
    const void *p;
    int64_t client, sample, row;
} aet_in_maps;
typedef struct {
    void *p;
    int64_t client, sample, row;
} aet_out_maps;

/* Over the positions * width values of a sample's group: mean m and variance v (divided by
 * their number), rstd = 1 / sqrt(v + eps);  y = act((x - m) rstd gamma + beta).
 *   gamma, beta  n x channels (row is ignored; client = 0: the same for all), or p = NULL: 1, 0
 *   y            may be x itself, with the same strides
 *   mean, rstd   fp32, n x batch x groups without gaps, for the gradient; NULL: not wanted.
 *                With no positions: 0 and 1 / sqrt(eps). */
typedef struct {
    int32_t dtype, act;
    int32_t n, batch, positions, groups, width;
    float eps;
    aet_in_maps x;
    aet_in gamma, beta;
    aet_out_maps y;
    float *mean, *rstd;
} aet_group_norm;
size_t aet_group_norm_workspace_bytes(const aet_group_norm *a);
aet_status aet_group_norm_forward(const aet_group_norm *a, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Its gradient, from the inputs and the statistics that the forward call gave.
 *   dx            may be dy itself, with the same strides; or p = NULL
 *   dgamma, dbeta n x channels; client = 0 with n other than 1: the sum over the clients
 *                 (then of both); or p = NULL */
typedef struct {
    int32_t dtype, act;
    int32_t n, batch, positions, groups, width;
    aet_in_maps dy, x;
    const float *mean, *rstd;
    aet_in gamma, beta;
    aet_out_maps dx;
    aet_out dgamma, dbeta;
} aet_group_norm_grad;
size_t aet_group_norm_backward_workspace_bytes(const aet_group_norm_grad *a);
aet_status aet_group_norm_backward(const aet_group_norm_grad *a, void *workspace, size_t workspace_bytes,
                                   void *hip_stream);

/* y = residual + dropout(x): n x rows x cols each; residual may have p = NULL, y may be x or
 * residual itself, with the same strides.  The gradient of x is the same mask and scale on
 * dy: aet_dropout_backward takes the forward call's record with dy as x and dx as y, and no
 * residual (whose gradient is dy itself). */
typedef struct {
    int32_t dtype;
    int32_t n, rows, cols;
    double p;
    uint64_t seed;
    int64_t first_row;
    aet_in x, residual;
    aet_out y;
} aet_dropout;
aet_status aet_dropout_forward(const aet_dropout *a, void *hip_stream);
aet_status aet_dropout_backward(const aet_dropout *a, void *hip_stream);

/* Text of the calling thread's last failed call of this header, "" if there was none. */
const char *aet_ops_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* AET_OPS_H */
