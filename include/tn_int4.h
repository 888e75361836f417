/*
 * tn_int4: projections with frozen 4-bit weights on one MI355X (gfx950): products of weights that are whole numbers of 4 bits under group
 * scales with bf16 activations, silu(gate) * up of two such products, and the input gradient. They stand beside the 8-bit projections of
 * tn_fp8.h in the same library and share its conventions: status codes and types of tn_linear.h; every pointer is memory of the device that is
 * current; strides are in elements, from row to row, and elements of a row are contiguous; all functions enqueue kernels on `stream`
 * (hipStream_t) and return without waiting, without allocating (tn_int4_linear_create apart) and without any HIP call but launches, so that they
 * can be captured into a graph; tokens == 0 is a no-op; no function throws, and nothing is launched after an error in the arguments; results are
 * the same from call to call, bit for bit, for the same inputs and sizes.
 *
 * Format. A weight W [M, N] (outputs, inputs) is
 *     W[f][k] = (code[f][k] - zero[f][k / group]) * scale[f][k / group],   code, zero in 0 .. 15,   group 32, 64 or 128
 * with scales in bf16 or fp16; without zeros they are 8. The last group of a row may be shorter. A weight that the library quantises itself has,
 * in fp32, for lo and hi the least and largest of a group's values and 0:
 *     scale = (hi / 15 - lo / 15), rounded to bf16;  zero = -lo / scale and code = v / scale + zero, each quotient rounded to the nearest whole
 *     number (ties to even), limited to 0 .. 15;  a group of scale 0 has zero = code = 8
 * A group that holds an infinity or a NaN gets the scale NaN, zero = code = 8, so that the fault shows wherever the group is used.
 *
 * Tokens: up to 2^30 a call; features up to TN_INT4_MAX_FEATURES per tensor and side, TN_INT4_MAX_WEIGHTS together. More is TN_ERR_UNSUPPORTED.
 */
#ifndef TN_INT4_H
#define TN_INT4_H

#include "tn_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TN_INT4_MAX_FEATURES (1 << 21)
#define TN_INT4_MAX_WEIGHTS (INT64_C(1) << 32)      /* of a tensor, with its sides rounded up to multiples of 64 (features) and 128 (the side that is summed over) */

/* tn_int4_linear_desc.dtype, beside TN_DTYPE_F32 and TN_DTYPE_BF16: tensors that are in 4 bits already */
#define TN_DTYPE_INT4 3
/* tn_int4_linear_desc.scale_dtype, beside TN_DTYPE_BF16 */
#define TN_DTYPE_F16 4

typedef struct tn_int4_linear_s* tn_int4_linear_t;

/*
 *  dtype        F32 or BF16: contiguous [M, N] tensors, quantised by create. TN_DTYPE_INT4: codes, contiguous [M, ceil(N / 2)] bytes with the
 *               even k in the low half of a byte (the spare half of an odd N is ignored)
 *  n_tensors    1, or 2: two weights of the same size that read the same activations (gate and up of an MLP block)
 *  out_features, in_features   M and N of each tensor
 *  group        32, 64 or 128 inputs to a scale
 *  scale_dtype  BF16 or F16 (TN_DTYPE_INT4 only)
 *  tensors      n_tensors device pointers (the arrays of pointers are host memory)
 *  scales       TN_DTYPE_INT4: device pointers to contiguous [M, ceil(N / group)] scales; else ignored
 *  zeros        TN_DTYPE_INT4: NULL, or device pointers to contiguous [M, ceil(N / group)] bytes, of which the low four bits count; else ignored
 *  flags        0 or TN_FLAG_TRANSPOSE: the products take gradients of the outputs and give that of the inputs
 *  stream       on which create enqueues its work; it waits for it before it returns
 */
typedef struct tn_int4_linear_desc {
    int32_t dtype;
    int32_t n_tensors;
    int64_t out_features;
    int64_t in_features;
    int32_t group;
    int32_t scale_dtype;
    const void* const* tensors;
    const void* const* scales;
    const void* const* zeros;
    int32_t flags;
    void* stream;
} tn_int4_linear_desc;

/* On success *out receives the handle, which holds one 4-bit copy of the weights in an order of its own; the caller may free its tensors.
 * On failure *out is untouched. */
int tn_int4_linear_create(tn_int4_linear_t* out, const tn_int4_linear_desc* desc);

/*
 * Bytes of workspace that a call with `tokens` tokens needs (host only; negative: an error): for partial sums of products whose inputs are
 * split, and for rows that are laid out anew - in fp16 for tiles; where the weight is streamed, if their length is no multiple of 128, x is not
 * 16-byte aligned, or x_stride is no multiple of 8, or 2^22 or more. gated: 1 for tn_int4_linear_gated. The rows of the call itself must be no
 * less aligned than the x that was asked for, with its x_stride.
 */
int64_t tn_int4_linear_workspace(tn_int4_linear_t h, const void* x, int64_t x_stride, int64_t tokens, int32_t gated);

/*
 * y = X W^T in bf16, summed in fp32: x bf16 [tokens, N], y bf16 [tokens, n_tensors * M], the tensors' outputs beside each other. With TN_FLAG_TRANSPOSE: x
 * is [tokens, n_tensors * M], y is [tokens, N], the sum over the tensors of X_i W_i. y may not overlap x (TN_ERR_INVALID_ARG): no
 * element is of both; columns of the same rows, with one stride, lie beside each other. Of two different strides all between the first element and the last counts.
 * workspace: what the function above says, 256-byte aligned, for this call alone until its work is done: calls with workspaces of their own may be in
 * flight together. Nothing in it has to start at zero.
 * Rounding. Up to 64 tokens (where tn_int4_linear_plan_query says that the weight is streamed) products are taken with the codes as they are, which is exact,
 * and fp32 sums of a group are multiplied with its scale. In tiles, weights are rounded to fp16 under a power of two for each feature (with TN_FLAG_TRANSPOSE for each
 * group of features): off by 2^-11 of themselves, and where their scale is below 2^-24 of the largest scale of the feature (group) by up to 2^-31 of that largest on top (the scale is off by
 * 2^-35 of it, the weight by up to 15 times that); and tokens are in fp16 under a power of two for
 * each row (each range of a row, where the inputs are split), which is exact, or off by 2^-39 of the row's largest finite magnitude. Sums are fp32's (in the matrix cores). Infinities and NaN of a token show in its row alone, and as
 * sums of W[f][k] * x[k] have them.
 */
int tn_int4_linear_forward(tn_int4_linear_t h, const void* x, int64_t x_stride, void* y, int64_t y_stride, int64_t tokens,
                           void* workspace, int64_t workspace_bytes, void* stream);

/* silu(X Wg^T) * (X Wu^T) in bf16 [tokens, M], for a handle of two tensors (Wg, Wu) without TN_FLAG_TRANSPOSE: gate and up are not rounded on the way. */
int tn_int4_linear_gated(tn_int4_linear_t h, const void* x, int64_t x_stride, void* y, int64_t y_stride, int64_t tokens,
                         void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Host only, no GPU call, no tensor read (desc->tensors may be NULL): how a call with `tokens` tokens would run. For the library's own tests and
 * measurements.
 */
#define TN_INT4_PLAN_TILE_TOKENS 0      /* tokens of a tile; 0: the weight is streamed */
#define TN_INT4_PLAN_RANGES 1           /* ranges that the inputs are split into, partial sums in the workspace */
#define TN_INT4_PLAN_STREAM_TOKENS 2    /* streamed: tokens that a workgroup multiplies a piece of the weight with, else 0 */
#define TN_INT4_PLAN_STREAM_PIECES 3    /* streamed: runs of 16 features to a workgroup, else 0 */
int tn_int4_linear_plan_query(const tn_int4_linear_desc* desc, int64_t tokens, int32_t gated, int32_t what, int64_t* value);

/* Tensor `slot` as the description takes it: codes [M, ceil(N / 2)] bytes, scales fp32 [M, ceil(N / group)] (which hold those in 16 bits exactly), zeros
 * [M, ceil(N / group)] bytes, also from a handle made with TN_FLAG_TRANSPOSE. Each pointer may be NULL. */
int tn_int4_linear_tensor(tn_int4_linear_t h, int32_t slot, void* codes, void* scales, void* zeros, void* stream);

/* what: TN_QUERY_OUT_FEATURES and TN_QUERY_IN_FEATURES (columns of y and of x, all segments), TN_QUERY_PACKED_BYTES, TN_QUERY_PARAM_COUNT */
int tn_int4_linear_query(tn_int4_linear_t h, int32_t what, int64_t* value);

/* No call may be in flight, and no graph that captured one may be replayed afterwards. NULL is accepted. */
int tn_int4_linear_destroy(tn_int4_linear_t h);

#ifdef __cplusplus
}
#endif
#endif /* TN_INT4_H */
