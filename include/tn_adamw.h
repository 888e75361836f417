/*
 * tn_adamw: the update of many parameter tensors at once on one MI355X (gfx950) - the norm of all their gradients, and the AdamW step with states in
 * 32 bits or in 8. It stands beside the gradients of tn_linear.h and tn_fp8.h in the same library and shares their conventions: status codes and types
 * of tn_linear.h; every pointer is memory of the device that is current, unless it says otherwise; all functions enqueue kernels on `stream` (hipStream_t) and
 * return without waiting, without allocating (tn_adamw_create apart) and without any HIP call but launches, so that they can be captured into a graph; no
 * function throws, and nothing is launched after an error in the arguments; results are the same from call to call, bit for bit, for the same inputs.
 *
 * Step t, the count before it and one, for the gradients g of all tensors and n = sqrt(sum of all g^2):
 *     g <- g * max_norm / n             where there is a max_norm and n > max_norm
 *     m <- beta1 * m + (1 - beta1) * g,  v <- beta2 * v + (1 - beta2) * g^2
 *     p <- p * (1 - lr * decay) - lr * (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * all in fp32 (the powers, and what is made of them once a step, and n in 64 bits). lr * decay * p and the move are added up and taken off p in one subtraction, whose rounding, 2^-24 of p, is
 * the only one at p's size: a decay below that is right on average over moves of different sizes (with no move beside it, it is lost). With a max_norm and an n that is not finite nothing changes, the count
 * neither. A parameter in bf16 is the rounding of an fp32 master, which is what the step reads and writes: a step of 1e-4 of a parameter's size would be
 * lost in its 8 bits.
 *
 * State. One buffer of L values over all tensors, each tensor starting at a multiple of 128 (tn_adamw_state_values gives L; nothing between tensors is
 * read or written but with zeros). 32 bits: m and v in fp32. 8 bits: m and r = sqrt(v) as e4m3 codes with a power-of-two scale byte (E8M0) for each 128, as
 * tn_fp8.h has them for rows: 2^e with the least e >= -127 for which nothing finite of the block exceeds 448 * 2^e. The root because e4m3 spans 2^18 and
 * v the square of what g spans. Values between two codes are rounded to either of them at random, with the probability that makes the result right on
 * average: r moves by about (1 - beta2) / 2 of itself in a step, 0.05 %, and a step between codes is 6 to 12 %, so that the nearest code would hold it in place for
 * good (from zero it would stop at a tenth of its value). The random numbers are a hash: for place i of the state and step t
 *     h = mix(low 32 bits of i ^ mix(mix(mix(seed) ^ low 32 bits of t) ^ high 32 bits of i))
 *     mix(x): x = (x ^ x >> 16) * 0x9E3779B1;  x = (x ^ x >> 15) * 0xB7E15163;  x ^ x >> 16        (modulo 2^32; the factors are from the golden ratio and e)
 * |value| / 2^e between neighbouring e4m3 values a < b goes to b where the part of the way (|value| / 2^e - a) / (b - a) + (h16 + 1/2) / 2^16 >= 1, with
 * h16 the low half of h for m and the high half for r. (Below the least normal code, 2^-6, the part is computed after 2^-6 is added, so that it is
 * rounded to 2^-20.) What is not finite becomes a NaN code and stays out of its block's scale.
 * Where beta1^2 < beta2, |m| <= B sqrt(v) with B = (1 - beta1) / sqrt((1 - beta2) (1 - beta1^2 / beta2)), 7.3 for 0.9 and 0.999, whatever the gradients were; a root that is
 * less than |m| / B is one that was rounded (to zero, beside values 2^18 times larger in its block), and in 8 bits the step divides by |m| / B in its place: without that one
 * such value moves by m / eps. That holds for states that began at zero with these betas. One loaded from a run with others, or made elsewhere, may have such roots without any
 * rounding: the steps of those values are shorter than the formula's, until m has forgotten (states in 32 bits are taken as they are).
 */
#ifndef TN_ADAMW_H
#define TN_ADAMW_H

#include "tn_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TN_ADAMW_BLOCK 128
#define TN_ADAMW_MAX_TENSORS (1 << 20)

typedef struct tn_adamw_s* tn_adamw_t;

/*
 *  n_tensors, sizes   values of each tensor (host array; 0 is allowed), 2^40 together at the most
 *  dtypes             TN_DTYPE_F32 or TN_DTYPE_BF16 of each parameter (host array)
 *  params             device pointers of contiguous parameters, no two of which overlap (host array of pointers)
 *  decays             weight decay of each tensor (host array)
 *  state_bits         32 or 8
 *  first, second      m, and v or r: fp32 or code bytes [L], 256-byte aligned, device
 *  first_scales, second_scales   8 bits: scale bytes [L / 128], device; else ignored
 *  master             fp32 [L], laid out like the state, 256-byte aligned; needed where a parameter is in bf16, and not read or written for others
 *  count              steps so far, on the device (8-byte aligned)
 *  beta1, beta2       0 <= beta < 1;  eps >= 0
 * The arrays on the host are read by create alone; everything on the device has to outlive the handle. create copies parameters in bf16 to their masters where
 * init_master is not 0, on `stream`, and waits for it; it neither reads nor writes the rest of the state.
 */
typedef struct tn_adamw_desc {
    int32_t n_tensors;
    int32_t state_bits;
    const int64_t* sizes;
    const int32_t* dtypes;
    void* const* params;
    const float* decays;
    void* first;
    void* second;
    void* first_scales;
    void* second_scales;
    float* master;
    int64_t* count;
    double beta1;
    double beta2;
    double eps;
    uint32_t seed;
    int32_t init_master;
    void* stream;
} tn_adamw_desc;

/* L for these tensors (host only; negative: an error) */
int64_t tn_adamw_state_values(int32_t n_tensors, const int64_t* sizes);

int tn_adamw_create(tn_adamw_t* out, const tn_adamw_desc* desc);

/* Bytes of workspace of the two functions below (host only): 256-byte aligned, for the call alone until its work is done */
int64_t tn_adamw_workspace(tn_adamw_t h);

/*
 * *norm = sqrt(sum of the squares of all gradients), summed in 64 bits in a fixed order and rounded to fp32 once.
 *  grads        n_tensors device pointers of contiguous gradients with the parameters' sizes, aligned to their type (host array of pointers; not NULL where
 *               the size is not 0)
 *  grad_dtypes  TN_DTYPE_F32 or TN_DTYPE_BF16 of each (host array)
 * Both arrays are read before the function returns.
 */
int tn_adamw_gradient_norm(tn_adamw_t h, const void* const* grads, const int32_t* grad_dtypes, float* norm, void* workspace, int64_t workspace_bytes,
                           void* stream);

/*
 * One step. grads as above; none of them is written.
 *  lr         the learning rate, rounded to fp32; lr_device, where it is not NULL, is where an fp32 one is read from instead (a captured step may be replayed with other rates)
 *  max_norm   0 or less: no clipping
 *  norm       with clipping: where the norm of the gradients goes (NULL: nowhere), or, with norm_given, is read from instead of being computed - the norm
 *             over the ranks that share a model, or that of gradient_norm
 * A handle's steps must not overlap in time.
 */
int tn_adamw_step(tn_adamw_t h, const void* const* grads, const int32_t* grad_dtypes, double lr, const float* lr_device, double max_norm, float* norm,
                  int32_t norm_given, void* workspace, int64_t workspace_bytes, void* stream);

/* Masters of the parameters in bf16 from the parameters as they are: for whoever sets a parameter from outside. The handle stays as it is, so that captured steps
 * are replayed as before; where no parameter is in bf16 there is nothing to do. It is one of the handle's steps: none of them may overlap it in time. */
int tn_adamw_reset_master(tn_adamw_t h, void* stream);

/* No call may be in flight, and no graph that captured one may be replayed afterwards: its kernels read the handle's memory. NULL is accepted. */
int tn_adamw_destroy(tn_adamw_t h);

#ifdef __cplusplus
}
#endif
#endif /* TN_ADAMW_H */
