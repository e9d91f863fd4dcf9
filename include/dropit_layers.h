/*
 * dropit_layers.h -- C ABI of the operators that stand beside the dropped cache in a training step:
 *
 *   the gated projection of a feed-forward block and its backward pass   -> dropit_gated_forward, dropit_gated_backward
 *   the AdamW step over many tensors, states in 32 or in 8 bits          -> dropit_adamw, dropit_adamw_unpack
 *   the global gradient norm and the factor that clips it                -> dropit_grad_norm
 *
 * The conventions of dropit.h hold: device pointers owned by the caller, nothing allocated or kept, all work
 * enqueued on `hip_stream`, no host synchronisation, arguments validated before any HIP call, status codes
 * instead of aborts, results bit-reproducible run to run, distinct workspaces for concurrent calls.  Every call
 * uses ordinary kernel launches only and can be captured into a HIP graph.
 */
#ifndef DROPIT_LAYERS_H
#define DROPIT_LAYERS_H

#include "dropit.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Gated projection of a feed-forward block: the gate and the up projection of every token, the activation and
 * the product, in one pass.  With W [2 * hidden, c_in] (gate rows first), bias [2 * hidden] or NULL:
 *     pre = x W^T + bias                                          [tokens, 2 * hidden], sums in fp32
 *     h   = act(pre[:, :hidden]) * pre[:, hidden:]                [tokens, hidden]
 * h is computed from the unrounded fp32 pre and rounded once; pre, where it is asked for, is rounded once too.
 *     DROPIT_ACT_SILU z / (1 + e^-z), DROPIT_ACT_GELU z * Phi(z), DROPIT_ACT_GELU_TANH its tanh form
 *     z / 2 * (1 + tanh(sqrt(2 / pi) * (z + 0.044715 z^3))), DROPIT_ACT_RELU max(z, 0), DROPIT_ACT_SIGMOID 1 / (1 + e^-z)
 * bf16 evaluates them with the hardware's exponential and reciprocal (a relative 2^-20 or so, times the exponent; the forward
 * pass's Phi(z) by a fitted polynomial whose smaller tail Phi(-|z|) is off by 8e-6 of itself up to |z| = 4, 2.2e-5 up to 8 and
 * 1e-4 up to 12.9, where it leaves fp32's range), fp32 with the fp32 math library.
 *
 * x [tokens, c_in], w, bias, h, pre: device, row-major, type dt, 16-byte aligned; pre may be NULL (inference).
 * 0 <= tokens < 2^31, 1 <= c_in <= 2^28, 1 <= hidden <= 2^27, and ceil(tokens / 64) times the larger of ceil(hidden / 32) and
 * ceil(c_in / 64) at most 2^24 - 8.  Row offsets are 64-bit: none of the tensors is limited to 2^31 elements.
 */
typedef DROPIT_ENUM(dropit_act) {
    DROPIT_ACT_SILU = 0,
    DROPIT_ACT_GELU = 1,
    DROPIT_ACT_GELU_TANH = 2,
    DROPIT_ACT_RELU = 3,
    DROPIT_ACT_SIGMOID = 4
} dropit_act;

size_t dropit_gated_forward_workspace_bytes(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt);
dropit_status dropit_gated_forward(const void *x, int64_t tokens, int64_t c_in, dropit_dtype dt, const void *w, const void *bias,
                                   int64_t hidden, dropit_act act, void *h, void *pre, void *workspace,
                                   size_t workspace_bytes, void *hip_stream);

/*
 * Its backward pass.  With g = pre[:, :hidden], u = pre[:, hidden:]:
 *     dpre  = [ dh * u * act'(g) | dh * act(g) ]                  [tokens, 2 * hidden], type dt
 *     dx    = dpre W                                              [tokens, c_in], type dt, sums in fp32; may be NULL
 *     dbias = sum of dpre over the tokens, before its rounding    [2 * hidden], fp32; may be NULL
 * dx is computed from the rounded dpre.  The weight gradient dpre^T R(a^) is dropit_weight_grad's, with dY = dpre and
 * c_out = 2 * hidden.  act'(0) of ReLU is 0.  The workspace query takes need_dx and need_dbias as 0 or 1.
 * dh [tokens, hidden]; sizes, alignment and types as above.  dpre must not overlap pre.
 */
size_t dropit_gated_backward_workspace_bytes(int64_t tokens, int64_t c_in, int64_t hidden, dropit_dtype dt, int need_dx,
                                             int need_dbias);
dropit_status dropit_gated_backward(const void *dh, const void *pre, int64_t tokens, int64_t c_in, dropit_dtype dt,
                                    const void *w, int64_t hidden, dropit_act act, void *dpre, void *dx, float *dbias,
                                    void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * AdamW over many tensors at once.  For every element, with t the step (1 for the first) and s the value at
 * `grad_scale` (1 if NULL), in fp32, each operation rounded by itself (no fused multiply-adds):
 *     g = s * grad
 *     m = beta1 * m + (1 - beta1) * g
 *     v = beta2 * v + (1 - beta2) * (g * g)
 *     p = p * (1 - lr * weight_decay) - m / (sqrt(v) * (1 / sqrt(1 - beta2^t)) + eps) * (lr / (1 - beta1^t))
 * The scalars are evaluated in double and rounded once.
 *
 * Parameters: fp32; bf16 (rounded to nearest even); or bf16 with a residual, 16 more bits that make it an exact
 * fp32 master: pattern(master) = (pattern(p) << 16) + residual (a signed sum), p being master rounded to nearest,
 * ties away from zero.  A residual of zeros starts from the bf16 values as they are.
 *
 * States of 32 bits are fp32.  States of 8 bits are codes in blocks of DROPIT_ADAMW_BLOCK consecutive elements
 * of a tensor that share an int16 offset: with b the fp32 pattern of |value| and B the block's largest,
 *     offset = max(min((B + 0xfffff) >> 20, 0x7f7) - top, 0)          top = 127 for m, 255 for v
 *     code   = clamp(min((b + d) >> 20, 0x7f7) - offset, 0, top)      m: plus 128 where the value is negative
 * and a code c > 0 (its low seven bits for m) stands for the fp32 pattern (c + offset) << 20, 0 for zero: three
 * bits of mantissa, 15.9 octaves below the block's largest for m, 31.75 for v.  A v below that takes code 1, not
 * 0, unless it is zero, so a small v never turns into a division by eps.  d is a dither in [0, 2^20): the upper 20
 * bits of i * 0x6a09e667 + t * 0x9e3779b9 (mod 2^32) for element i of its tensor, complemented for v.  Over the
 * steps it takes every value equally often, so the rounding is right on average; rounding to nearest would hold
 * an average of 1 - beta2 = 0.001 where it is.  A block with an infinity or a NaN decodes to NaN throughout.
 * Codes and offsets of zeros are states of zeros.
 */
#define DROPIT_ADAMW_BLOCK 256
typedef struct {
    void *p;                   /* numel parameters, updated */
    const void *g;             /* numel gradients */
    void *m, *v;               /* numel states each, fp32 or 8-bit codes, updated */
    int16_t *m_offset;         /* 8-bit states: ceil(numel / DROPIT_ADAMW_BLOCK) offsets each, updated; else NULL */
    int16_t *v_offset;
    int16_t *residual;         /* numel residuals of bf16 parameters, updated, or NULL; NULL for all tensors of a call or none */
    int64_t numel;             /* 0 .. 2^34 */
} dropit_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps, weight_decay;   /* finite; betas in [0, 1), eps >= 0 */
    int64_t step;                                 /* t >= 1, unless step_device is given */
    const int32_t *step_device;                   /* device, or NULL: t is read there when the kernels run (>= 1), so that a
                                                     captured graph can be replayed with another t */
    const float *grad_scale;                      /* device, or NULL */
} dropit_adamw_hyper;

/*
 * tensors    host array of `count` entries (count >= 0), read during the call only.  Pointers need the alignment of
 *            their element type; where all of a tensor's are 16-byte aligned (8 for codes) it moves in wide accesses.
 *            A tensor's storage appears once in a call.
 * p_dtype, g_dtype  of all tensors; state_bits 32 or 8
 */
dropit_status dropit_adamw(const dropit_adamw_tensor *tensors, int64_t count, dropit_dtype p_dtype, dropit_dtype g_dtype,
                           int state_bits, const dropit_adamw_hyper *hyper, void *hip_stream);

/* The values that 8-bit states stand for, as bf16 (which holds them exactly): codes [numel], offsets
 * [ceil(numel / DROPIT_ADAMW_BLOCK)], is_signed 1 for m and 0 for v, values [numel] out; numel 0 .. 2^34. */
dropit_status dropit_adamw_unpack(const uint8_t *codes, const int16_t *offsets, int64_t numel, int is_signed,
                                  void *values, void *hip_stream);

/*
 * The 2-norm over all elements of `count` tensors, and the factor that brings it to at most max_norm:
 *     out[0] = sqrt(sum of squares),  out[1] = min(1, max_norm / (out[0] + 1e-6))         (device fp32)
 * Squares and a thread's sum of 64 of them in fp32, everything above in fp64, in a fixed order.  A NaN norm gives a
 * NaN factor, an infinite one the factor 0.  max_norm > 0, infinity for a factor of 1.
 * grads [count] device pointers with the alignment of their type, numels [count] 0 .. 2^34, dtypes [count] dropit_dtype: host
 * arrays.  workspace: device, 256-byte aligned, >= dropit_grad_norm_workspace_bytes of the same numels and count
 * (0 on invalid arguments or where none is needed).
 */
size_t dropit_grad_norm_workspace_bytes(const int64_t *numels, int64_t count);
dropit_status dropit_grad_norm(const void *const *grads, const int64_t *numels, const int32_t *dtypes, int64_t count,
                               double max_norm, float *out, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DROPIT_LAYERS_H */
