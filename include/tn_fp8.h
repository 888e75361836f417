/*
 * tn_fp8: the operators around 8-bit projections of a decoder on one MI355X (gfx950): root-mean-square norm with the
 * residual's addition, silu(gate) * up, the products of 8-bit weights with 8-bit activations, and the gradients of all
 * three. They stand beside the factorised layers of tn_linear.h in the same library and share its status codes and types.
 *
 * 8-bit format. Values are e4m3 codes (OCP FP8: largest 448, one NaN per sign, no infinity) under power-of-two scales in
 * blocks: 128 consecutive elements of a row of activations, or 128 x 128 elements of a weight (blocks counted from the
 * first element; the last of a row or column may be shorter). With a the largest finite |v| of a block, its scale is
 *
 *     2^e,  e = the least integer >= -127 with a <= 448 * 2^e      (a = 0: e = -127), stored as the byte e + 127 (E8M0)
 *
 * and v is stored as the e4m3 value nearest to v / 2^e, ties to the even code. Nothing overflows, and the division is
 * exact. Infinities and NaN are stored as NaN and do not take part in a.
 *
 * Rows in 8 bits. [rows, segments * cols] values are held as
 *     codes   [rows][segments * P] bytes,  P = cols rounded up to a multiple of 128: each segment starts a block
 *     scales  [rows][S] bytes,  S = segments * P / 128 rounded up to a multiple of 4
 * with zero codes and zero scale bytes where there is no value (all functions here write them, and the products read them:
 * a caller that makes such rows itself writes them too). One segment is what most rows have; the gradients of a gate / up
 * pair have two. codes must be 16-byte and scales 4-byte aligned.
 *
 * Every pointer is memory of the device that is current, unless it says otherwise, and a handle is used while the device that it was
 * made on is current. Strides are in elements, from row to row; elements of a row are
 * contiguous. Values of type F32 / BF16 need no more than their own alignment. All functions enqueue kernels on `stream`
 * (hipStream_t) and return without waiting, without allocating (tn_fp8_linear_create apart) and without any HIP call but
 * launches, so that they can be captured into a graph. rows == 0 is a no-op where nothing is left to compute. No function
 * throws; all return TN_OK or an error of tn_linear.h, and nothing is launched after an error in the arguments. Results are
 * the same from call to call, bit for bit, for the same inputs and sizes.
 * Rows (tokens): up to 2^30; columns: up to 2^24 where no other limit is given. More is TN_ERR_UNSUPPORTED.
 */
#ifndef TN_FP8_H
#define TN_FP8_H

#include "tn_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TN_FP8_BLOCK      128
#define TN_FP8_MAX_NORM_COLS 16384      /* widest row of tn_rms_norm and its gradients */
#define TN_FP8_MAX_FEATURES (1 << 21)   /* of tn_fp8_linear, per tensor and side */

/* tn_fp8_linear_desc.dtype, beside TN_DTYPE_F32 and TN_DTYPE_BF16: tensors that are quantised already */
#define TN_DTYPE_FP8 2

/* Strides of rows in 8 bits (host only): bytes from row to row of codes and of scales. Either pointer may be NULL. */
int tn_fp8_row_strides(int64_t cols, int32_t segments, int64_t* code_stride, int64_t* scale_stride);

/* x [rows, segments * cols] of `dtype` (F32 or BF16) in 8 bits. */
int tn_fp8_quantize(int32_t dtype, int64_t rows, int64_t cols, int32_t segments, const void* x, int64_t x_stride,
                    void* codes, void* scales, void* stream);

/*
 * s = x + residual (added in fp32, rounded to `dtype`; residual NULL: s = x), y = s / sqrt(mean(s^2) + eps) * weight.
 *  weight [cols] of `dtype`, or NULL for ones
 *  sum    NULL, or where s goes; it may be x or residual itself (same stride), but not overlap them otherwise
 *  y      NULL, or y rounded to `dtype`; it may be x or residual itself (same stride), but not sum
 *  codes, scales  NULL both, or y in 8 bits, quantised from fp32 (one segment)
 * One of sum, y and codes is needed at the least. The mean and y are computed in fp32 from s as it is rounded, which is what
 * the gradients below are given. cols <= TN_FP8_MAX_NORM_COLS.
 */
int tn_rms_norm(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride, const void* residual,
                int64_t residual_stride, const void* weight, float eps, void* sum, int64_t sum_stride, void* y,
                int64_t y_stride, void* codes, void* scales, void* stream);

/*
 * For L with dL/dy = dy, and dL/ds = dsum by way of whatever else reads s (NULL: none), the whole
 *     dx = dL/ds = r * (g - u * mean(g * u)) + dsum,   u = s * r,  g = dy * weight,  r = 1 / sqrt(mean(s^2) + eps)
 * rounded to `dtype` (it is the gradient of x and of residual), and, where dweight is not NULL, fp32
 *     dweight[j] = sum over rows of dy * u             (zeros for no rows; partial sums over rows added in a fixed order).
 * dx may be dy, s or dsum itself (same stride). `workspace`: tn_rms_norm_gradients_workspace(rows, cols) bytes, 16-byte aligned, needed with
 * dweight only; nothing in it has to start at zero, and it may be used for anything else once the call's work is done.
 */
int tn_rms_norm_gradients(int32_t dtype, int64_t rows, int64_t cols, const void* dy, int64_t dy_stride, const void* s,
                          int64_t s_stride, const void* weight, float eps, const void* dsum, int64_t dsum_stride, void* dx,
                          int64_t dx_stride, float* dweight, void* workspace, int64_t workspace_bytes, void* stream);
int64_t tn_rms_norm_gradients_workspace(int64_t rows, int64_t cols);   /* host only; negative: an error */

/*
 * h = silu(gate) * up with gate = gate_up[:, :cols], up = gate_up[:, cols:2 * cols] and silu(v) = v / (1 + exp(-v)), in fp32.
 *  y  NULL, or h rounded to `dtype`;  codes, scales  NULL both, or h in 8 bits (one segment). One of the two at the least.
 */
int tn_silu_gate(int32_t dtype, int64_t rows, int64_t cols, const void* gate_up, int64_t gate_up_stride, void* y,
                 int64_t y_stride, void* codes, void* scales, void* stream);

/*
 * The gradients of gate and up for dL/dh = dh [rows, cols], beside each other like gate and up themselves:
 *     dgate = dh * up * sig * (1 + gate * (1 - sig)),   dup = dh * gate * sig,   sig = 1 / (1 + exp(-gate))
 *  d_gate_up  NULL, or [rows, 2 * cols] of `dtype` (it may be gate_up itself);  codes, scales  NULL both, or the same in 8 bits
 *  (two segments: what a handle of the pair made with TN_FLAG_TRANSPOSE takes). One of the two at the least.
 */
int tn_silu_gate_gradients(int32_t dtype, int64_t rows, int64_t cols, const void* gate_up, int64_t gate_up_stride,
                           const void* dh, int64_t dh_stride, void* d_gate_up, int64_t d_gate_up_stride, void* codes,
                           void* scales, void* stream);

typedef struct tn_fp8_linear_s* tn_fp8_linear_t;

/*
 *  dtype        F32 or BF16: the tensors are quantised by create. TN_DTYPE_FP8: they are codes already.
 *  n_tensors    1, or 2: two weights of the same size that read the same activations (gate and up of an MLP block)
 *  out_features, in_features   M and N of each tensor, up to TN_FP8_MAX_FEATURES
 *  tensors      n_tensors device pointers to contiguous [M, N] arrays (the array of pointers is host memory)
 *  scales       TN_DTYPE_FP8 only: device pointers to contiguous [ceil(M / 128), ceil(N / 128)] scale bytes; else ignored
 *  max_tokens   the handle's own workspace (partial sums of products whose inputs are split) is sized for calls of up to
 *               this many tokens, 64 MB at the most; larger calls work too, and may take a slower form
 *  flags        0 or TN_FLAG_TRANSPOSE: the products take gradients of the outputs and give that of the inputs
 *  stream       on which create enqueues its work; it waits for it before it returns
 *  workspace, workspace_bytes
 *               optional device block of the caller, 256-byte aligned, instead of one of the handle's own (NULL, 0): it must outlive the
 *               handle, and several handles may share it as long as their calls never overlap in time. Any size works; less than
 *               64 MB may mean a slower form.
 */
typedef struct tn_fp8_linear_desc {
    int32_t dtype;
    int32_t n_tensors;
    int64_t out_features;
    int64_t in_features;
    const void* const* tensors;
    const void* const* scales;
    int64_t max_tokens;
    int32_t flags;
    void* stream;
    void* workspace;
    int64_t workspace_bytes;
} tn_fp8_linear_desc;

/* On success *out receives the handle, which holds one 8-bit copy of the weights in an order of its own; the caller may
 * free its tensors. On failure *out is untouched. */
int tn_fp8_linear_create(tn_fp8_linear_t* out, const tn_fp8_linear_desc* desc);

/*
 * y = X W^T in bf16, accumulated in the matrix cores' fp32. X: `tokens` rows in 8 bits, N columns, one segment; y [tokens, n_tensors * M],
 * the tensors' outputs beside each other. With TN_FLAG_TRANSPOSE: X has M columns and n_tensors segments, y is [tokens, N], the sum over the
 * tensors of X_i W_i. y overlaps nothing. One call per handle may be in flight at a time (they share its workspace).
 * Accumulation is the matrix cores': products of 8 consecutive k are aligned to the largest of them and cut off (towards zero) at 2^-13 of it, all
 * further sums are fp32's. Before it is rounded to bf16 (half a unit, 2^-8 of it at most), a sum is off by less than
 *     (7 * 2^-13 + 2^-18) * sum over the groups of 8 k of (largest |x| in the group) * (largest |w| in the group)
 * with x and w the values of the codes: where a channel towers over its seven neighbours, it is theirs that are cut. On independent terms of one
 * size it is 1.5e-5 of the result. In the 8-bit outputs below three to four codes in a thousand become their neighbours for it.
 */
int tn_fp8_linear_forward(tn_fp8_linear_t h, const void* codes, const void* scales, void* y, int64_t y_stride, int64_t tokens,
                          void* stream);

/* silu(X Wg^T) * (X Wu^T) in 8 bits ([tokens, M], one segment), for a handle of two tensors (Wg, Wu) without TN_FLAG_TRANSPOSE:
 * gate and up are not rounded on the way. The output overlaps nothing; on X it is TN_ERR_INVALID_ARG. */
int tn_fp8_linear_gated(tn_fp8_linear_t h, const void* codes, const void* scales, void* out_codes, void* out_scales, int64_t tokens,
                        void* stream);

/*
 * Host only, no GPU call, no tensor read (desc->tensors may be NULL): how a call of tn_fp8_linear_forward (gated = 0) or tn_fp8_linear_gated (1) with
 * `tokens` tokens would run. For the library's own tests and measurements.
 */
#define TN_FP8_PLAN_TILE_TOKENS   0   /* tokens of a tile; 0: the weight is streamed, 16 tokens at a time */
#define TN_FP8_PLAN_TILE_FEATURES 1   /* features of a tile; 0 likewise */
#define TN_FP8_PLAN_RANGES        2   /* ranges that the inputs are split into, partial sums in the workspace */
#define TN_FP8_PLAN_FUSED         3   /* gated: silu(gate) * up within the product's launch */
#define TN_FP8_PLAN_STREAM_PIECES 4   /* streamed: runs of 16 features to a workgroup, else 0 */
int tn_fp8_linear_plan_query(const tn_fp8_linear_desc* desc, int64_t tokens, int32_t gated, int32_t what, int64_t* value);

/* Codes [M, N] and scale bytes [ceil(M / 128), ceil(N / 128)] of tensor `slot`, as the description takes them (also from a
 * handle made with TN_FLAG_TRANSPOSE). Either pointer may be NULL. */
int tn_fp8_linear_tensor(tn_fp8_linear_t h, int32_t slot, void* codes, void* scales, void* stream);

/* what: TN_QUERY_OUT_FEATURES and TN_QUERY_IN_FEATURES (columns of y and of X, all segments), TN_QUERY_PACKED_BYTES,
 * TN_QUERY_WORKSPACE_BYTES, TN_QUERY_PARAM_COUNT */
int tn_fp8_linear_query(tn_fp8_linear_t h, int32_t what, int64_t* value);

/* No call may be in flight. NULL is accepted. */
int tn_fp8_linear_destroy(tn_fp8_linear_t h);

#ifdef __cplusplus
}
#endif
#endif /* TN_FP8_H */
