/*
 * aet_ops.h -- C ABI of the operators that residual blocks of clients' models are composed
 * from, on MI355X (gfx950): a linear layer with bias, activation, dropout and residual in its
 * epilogue, group normalisation with an activation on channels-last maps, layer normalisation
 * of rows, and dropout from the counter generator, each with its gradient; values held in
 * microscaled 4-bit floating point, and the linear layer of such values; and the orthogonalised
 * update of weight matrices.  All of them take many clients' models side
 * by side in one call (`n`), each with parameters of its own or all with the same ones.
 *
 * Conventions
 *   - Every pointer is DEVICE memory owned by the caller.  The library allocates nothing;
 *     calls that need scratch memory take a workspace (size from aet_*_workspace_bytes,
 *     256-byte aligned; NULL where that is 0).  It keeps nothing between calls.
 *   - All tensors of a call have the call's dtype, but for the statistics of a normalisation
 *     (fp32), and held values (bytes).  Products, sums, statistics and everything between a
 *     call's inputs and its outputs are fp32 or wider; an output is rounded once, to its type.
 *     Exceptions: dz in the gradient of a linear layer in bf16, of held values or not, and the
 *     matrices between the steps of an orthogonalised update (named there);
 *     and fp32 products of more than 32 rows, and all of fp32 gradients, take their operands
 *     to within 2^-134, which is less than 24 bits of one below 2^-110 (forward products of up
 *     to 32 rows take all of them).
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
 *   - Sizes of 0 are legal: sums over nothing are 0.  The largest is 2^30; and a call of which a launch would have 2^32
 *     threads is refused (AET_EHIP): that takes 2^22 clients or rows, or more.
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

/* Layer normalisation of rows, the residual stream joined in:  h = x + residual; over the cols
 * values of a row of h: mean m and variance v (divided by their number), rstd = 1 / sqrt(v + eps);
 * y = (h - m) rstd gamma + beta, of h before it is rounded to its type.
 *   x, residual  n x rows x cols; residual: or p = NULL
 *   gamma, beta  n x cols (row is ignored; client = 0: the same for all), or p = NULL: 1, 0
 *   y, h         n x rows x cols; h, the stream as it goes on: or p = NULL.  Either may be x or
 *                residual itself, with the same strides (not both the same one).
 *   mean, rstd   fp32, n x rows without gaps, for the gradient; NULL: not wanted.  With no
 *                columns: 0 and 1 / sqrt(eps). */
typedef struct {
    int32_t dtype;
    int32_t n, rows, cols;
    float eps;
    aet_in x, residual, gamma, beta;
    aet_out y, h;
    float *mean, *rstd;
} aet_layer_norm;
aet_status aet_layer_norm_forward(const aet_layer_norm *a, void *hip_stream);

/* Its gradient.  x is what was normalised (the forward call's h, or its x where there was no
 * residual), mean and rstd as that call gave them, dh what comes to h along the stream:
 * dx = (gradient through the normalisation) + dh, which is that of x and of residual.
 *   dh            n x rows x cols, or p = NULL
 *   dx            n x rows x cols; may be dy or dh itself, with the same strides; or p = NULL
 *   dgamma, dbeta n x cols; client = 0 with n other than 1: the sum over the clients (then of
 *                 both); or p = NULL */
typedef struct {
    int32_t dtype;
    int32_t n, rows, cols;
    aet_in dy, x, dh, gamma;
    const float *mean, *rstd;
    aet_out dx, dgamma, dbeta;
} aet_layer_norm_grad;
size_t aet_layer_norm_backward_workspace_bytes(const aet_layer_norm_grad *a);
aet_status aet_layer_norm_backward(const aet_layer_norm_grad *a, void *workspace, size_t workspace_bytes, void *hip_stream);

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

/* The orthogonalised update of weight matrices (Newton-Schulz products, as the Muon optimiser makes them):
 *   X = g / (|g| + eps), |g| the root of the sum of g's squares (0 where both are 0);
 *   `steps` times  X = a X + (b A + c A A) X, A = X X^T, which takes a singular value s to a s + b s^3 + c s^5
 *   and leaves the singular vectors;
 *   y = keep w + scale X.
 *   g   n x rows x cols: a gradient, a sum of them, or a momentum of each client
 *   w   n x rows x cols, or p = NULL: y = scale X
 *   y   n x rows x cols; may be w or g itself, with the same strides
 * The sides are at most 2^20, the polynomial one under which singular values up to 1 stay below 2^30.  Everything
 * between is to within 2^-22 of each value and 2^-39 of what the norm and the polynomial bound all values of that step by; products'
 * sums are fp32, the norm's 64 bits.  In AET_BF16 several steps may go by A alone, without X between them (where that is faster, which n, rows
 * and cols decide), as long as the square of what they make of small singular values stays below 200, by which A's errors grow.  Before it
 * is rounded y is then about as far off as with products in fp32, in the 2-norm 3e-6 to 1e-4 of X after five steps of the polynomial (3.4445,
 * -4.775, 2.0315), and within 4 times that.  A client whose g has an infinity or NaN has a y of NaN. */
typedef struct {
    int32_t dtype;
    int32_t n, rows, cols, steps;
    double a, b, c, eps, keep, scale;
    aet_in g, w;
    aet_out y;
} aet_orthogonal;
size_t aet_orthogonalise_workspace_bytes(const aet_orthogonal *a);
aet_status aet_orthogonalise(const aet_orthogonal *a, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Microscaled 4-bit floating point, as messages and weights are held in.  The 32 neighbouring values
 * of a row (the last ones of it may be fewer) that make up a block share an exponent x; a value is held
 * as one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, times 2^x: the nearest to it, of two that are
 * as near the one with the even code, and 6 for all beyond.  x = floor(log2(the largest magnitude)) - 2, at
 * least -127, which is also that of a block of zeros.  A block with an infinity or NaN is NaN.
 *   codes   a byte for two columns, the even one in its lower half: the sign's bit, and the place of the
 *           magnitude in the list above.  ceil(cols / 2) bytes a row; a half that is left is 0, and not read.
 *   scales  a byte for a block: x + 127, or 255 for NaN.  ceil(cols / 32) bytes a row.
 * (The OCP Microscaling Formats specification's MXFP4.)  Their strides are in bytes, of any alignment;
 * products of more than 32 rows are faster where the columns are a multiple of 512, and rows of codes and of scales begin
 * at multiples of 16 bytes: else they are first copied so, into the workspace.  Any bytes are legal codes and scales. */

/* x, n x rows x cols, to codes and scales. */
typedef struct {
    int32_t dtype;
    int32_t n, rows, cols;
    aet_in x;
    aet_out codes, scales;
} aet_mx4_values;
aet_status aet_mx4_quantise(const aet_mx4_values *a, void *hip_stream);

/* What codes and scales stand for: y, n x rows x cols.  (Exact, but for magnitudes of 2^128 and more, which the
 * first call does not make.) */
typedef struct {
    int32_t dtype;
    int32_t n, rows, cols;
    aet_in codes, scales;
    aet_out y;
} aet_mx4_codes;
aet_status aet_mx4_dequantise(const aet_mx4_codes *a, void *hip_stream);

/* aet_linear_forward of held inputs and weights: y = residual + dropout(act(z)), z = x W^T + bias.
 *   x, x_scales   n x rows x in, as codes and scales
 *   w, w_scales   n x out x in; client = 0 (of both): one W for all
 * dtype is that of bias, residual, y and pre; all else as in aet_linear.  Products are exact and sums fp32
 * (a block's products that are below 2^-126 may be 0). */
typedef struct {
    int32_t dtype, act;
    int32_t n, rows, in, out;
    double p;
    uint64_t seed;
    int64_t first_row;
    aet_in x, x_scales, w, w_scales, bias, residual;
    aet_out y, pre;
} aet_mx4_linear;
size_t aet_mx4_linear_workspace_bytes(const aet_mx4_linear *a);
aet_status aet_mx4_linear_forward(const aet_mx4_linear *a, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Its gradient with regard to what the codes stand for, from the codes: dx = dz W, dw = dz^T x, db = sum of dz over
 * rows.  (That of the values that were quantised is the same where rounding is taken to have a slope of 1.)  dtype is that
 * of dy, pre, dx, dw and db; all else as in aet_linear_grad, but x may lie anyhow also where one W is for all.  The products
 * take dz whole where dtype is AET_F32 (to within 2^-134), else as those of aet_linear_grad do, and what codes stand for as it
 * is; sums below 2^-124 may be 0. */
typedef struct {
    int32_t dtype, act;
    int32_t n, rows, in, out;
    double p;
    uint64_t seed;
    int64_t first_row;
    aet_in dy, x, x_scales, w, w_scales, pre;
    aet_out dx, dw, db;
} aet_mx4_linear_grad;
size_t aet_mx4_linear_backward_workspace_bytes(const aet_mx4_linear_grad *a);
aet_status aet_mx4_linear_backward(const aet_mx4_linear_grad *a, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Text of the calling thread's last failed call of this header, "" if there was none. */
const char *aet_ops_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* AET_OPS_H */
