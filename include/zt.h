/*
 * zt.h -- C ABI of libzc, training-step operators: what a rank does with its messages once
 * they are decoded (MI355X, gfx950).
 *
 * Two kinds of messages carry most of the traffic that include/zc.h compresses: the
 * tensor-parallel all-reduce of a block's output and the data-parallel reduction of the
 * gradients, with ZeRO stage 1 sharding the optimizer (Sec. II-A, Table I).  Behind the first comes the
 * residual join with the norms around a block; behind the second the global norm over all
 * gradient tensors, clipping, and the optimizer's step on this rank's shard, which writes the
 * parameters that the all-gather sends.
 *
 * Conventions
 *   - d_* are DEVICE pointers owned by the caller, aligned to their elements (no more: a
 *     tensor may be a slice of a bucket that starts anywhere).  The library neither allocates,
 *     frees nor keeps them; arrays of pointers are HOST arrays, read before the call returns.
 *   - `stream` is a hipStream_t as void*; calls enqueue kernels on it and return without
 *     synchronising.  They only launch kernels, so sequences of them can be captured in a HIP
 *     graph; its replays repeat the numbers that the calls were given (zt_adamw: see d_state).
 *     Calls on different streams may run concurrently where they share no output and no workspace.
 *   - Return value: ZC_OK or a negative code of include/zc.h; on error nothing is launched.
 *   - dtype: enum zc_dtype.  Sums, statistics and products are held in fp32 (sums of squares
 *     in 64 bits); a value is rounded once, to the nearest with ties to even, where it is
 *     stored.  Results do not depend on the order in which workgroups run.
 *   - Infinities and NaN give what the formulas give, within their own row (norms) or tensor
 *     element (clip), unless said otherwise.
 */
#ifndef ZT_H
#define ZT_H

#include <stddef.h>

#include "zc.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Residual join with the norms around a block.  For each of `rows` rows of `cols` values
 *
 *     y = residual_scale * x + gate * post(b)        h = pre(y)
 *
 * x is the residual stream, b the output of a block (decoded from its message), y the new
 * residual stream and h the next block's input.  pre and post are norms of the given kind,
 *
 *     ZT_RMS:    v r w,              r = 1 / sqrt(mean(v^2) + eps)
 *     ZT_LAYER:  (v - mean) r w + c, r = 1 / sqrt(mean((v - mean)^2) + eps)
 *
 * with weights w and biases c (ZT_LAYER's alone) of `cols` values; w = NULL stands for ones, c = NULL for zeros.
 * Without `post` (0) the block's output joins as it is.  The gate is absent, one value per channel, or
 * one per element.  h is made of y before y is rounded.
 *
 * x, b, gate, weights, biases, y and h are of type `dtype`.  A stride is the number of
 * elements from one row to the next, 0 for `cols`; an input's may be smaller than cols (rows
 * that overlap), an output's may not.  cols is at most ZT_MAX_COLS.
 */
enum zt_norm_kind { ZT_RMS = 0, ZT_LAYER = 1 };
enum zt_gate { ZT_GATE_NONE = 0, ZT_GATE_CHANNEL = 1, ZT_GATE_FULL = 2 };
enum { ZT_MAX_COLS = 32768, ZT_MAX_ROWS = 1 << 30 };

struct zt_residual {
  size_t rows, cols;
  int dtype;            /* enum zc_dtype */
  int kind;             /* enum zt_norm_kind */
  int post;             /* 1: the block's output is normed before it joins */
  int gate;             /* enum zt_gate */
  float residual_scale; /* finite */
  float eps;            /* >= 0; the forward call's alone */
  size_t stride_x, stride_b, stride_gate, stride_y, stride_h;   /* gate: with ZT_GATE_FULL */
  size_t stride_dy, stride_dh, stride_dx, stride_db, stride_dgate;   /* the backward call's */
};

/* d_b may be NULL (with post = 0 and no gate): y = residual_scale * x.  d_y may be NULL if the
 * residual stream ends here.  d_stats (aligned to 16), if not NULL, gets what the backward call needs, four
 * floats a row: mean and r of post, mean and r of pre (0 for means of ZT_RMS and for a norm
 * that is absent).  d_y may be d_x and d_h may be d_b or d_x, with the same strides; no other overlap of
 * an output with an input or another output. */
int zt_residual_norm(const struct zt_residual* form, const void* d_x, const void* d_b, const void* d_gate,
                     const void* d_pre_weight, const void* d_pre_bias, const void* d_post_weight, const void* d_post_bias,
                     void* d_y, void* d_h, float* d_stats, void* stream);

/* The gradients of all of it, from those of y (d_dy; NULL for zero) and of h (d_dh):
 * d_dx, d_db of type dtype, d_dgate of type dtype with ZT_GATE_FULL and fp32 with
 * ZT_GATE_CHANNEL (the sum over the rows), and the sums over the rows for weights and biases
 * in fp32, the type of a gradient bucket.  d_y, d_b, d_gate, weights and d_stats are those of
 * the forward call (d_y as it was stored).  Any output may be NULL if it is not wanted; so may d_b, as in the forward call.
 * d_dx may be d_dy, and d_db or d_dx may be d_dh, with the same strides; no other overlap.
 * d_work holds work_bytes >= zt_residual_work_bytes(form) bytes, aligned to 16; its contents
 * before and after do not matter. */
size_t zt_residual_work_bytes(const struct zt_residual* form);
int zt_residual_norm_backward(const struct zt_residual* form, const void* d_dy, const void* d_dh, const void* d_y,
                              const void* d_b, const void* d_gate, const void* d_pre_weight, const void* d_post_weight,
                              const void* d_post_bias, const float* d_stats, void* d_dx, void* d_db, void* d_dgate,
                              float* d_dpre_weight, float* d_dpre_bias, float* d_dpost_weight, float* d_dpost_bias,
                              void* d_work, size_t work_bytes, void* stream);

/*
 * The global norm over many gradient tensors.  The sum of squares is kept as ZT_SLOTS doubles
 * whose total it is: calls add to them, and ranks add theirs up (an all-reduce of 4 KiB)
 * before the norm is taken.
 */
enum { ZT_SLOTS = 512 };

/* d_slots[0..ZT_SLOTS) (aligned to 16 bytes) = the sums of squares of `count` tensors, tensor i of n[i] values
 * of type dtype[i]; added to what d_slots holds if `accumulate` is not 0.  Squares are exact
 * and added in 64 bits, so neither overflows nor vanishes what fp32 holds.  n[i] = 0 (d_in[i]
 * may then be NULL) and count = 0 are valid. */
int zt_sum_squares(const void* const* d_in, const size_t* n, const int* dtype, int count, int accumulate,
                   double* d_slots, void* stream);

/* d_norm[0] = scale * sqrt(total of d_slots): the norm of gradients that still have to be
 * multiplied by scale (1 / ranks for sums over ranks, 1 / loss scale).  scale > 0, finite. */
int zt_norm(const double* d_slots, float scale, float* d_norm, void* stream);

/* Clipping: d_out[i] = c * d_in[i] for every tensor, with zt_norm's formula and
 *     c = scale                      if norm <= max_norm
 *     c = scale * max_norm / norm    otherwise (NaN if the norm is NaN).
 * c is made in 64 bits, of the norm before it is rounded, and rounded to fp32: a norm that 64 bits
 * hold and fp32 does not is clipped by as it is, although d_norm gets infinity.
 * max_norm > 0; infinity asks for no clipping.  In place with c = 1 nothing is written.  Tensor i is read as dtype_in[i] and written as
 * dtype_out[i]; d_out[i] may be d_in[i] if the types are the same, no other overlap.  d_norm
 * may be NULL. */
int zt_clip(const void* const* d_in, const size_t* n, const int* dtype_in, void* const* d_out, const int* dtype_out,
            int count, const double* d_slots, float scale, float max_norm, float* d_norm, void* stream);

/*
 * One AdamW step on n parameters of this rank's shard, the gradients multiplied by zt_clip's c as
 * they are read:
 *
 *     g = c * grad      m = beta1 m + (1 - beta1) g      v = beta2 v + (1 - beta2) g^2
 *     param -= lr * ((m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps) + weight_decay * param)
 *
 * param, m and v are fp32, grad of type grad_dtype; d_half, if not NULL, gets the new
 * parameters rounded to half_dtype (ZC_BF16 or ZC_F16): the message of the parameter
 * all-gather.  If the norm that d_norm gets (fp32) is not finite nothing is changed, and d_half gets the
 * old parameters.  d_slots may be NULL: c = scale.  d_norm may be NULL.  No overlap.
 *
 * step and lr are numbers of the call: one that is captured in a graph repeats that one step in each
 * replay, and whether a step was left out is known to the GPU alone.  With d_state (device, 4 values,
 * aligned to 16) the call counts for itself: d_state[0] is the number of steps taken before it (>= 0),
 * to which it adds one unless it leaves the step out, d_state[1] the learning rate (>= 0), and it writes
 * what it needs into the other two.  step and lr of the form are then not read.  Each shard has a
 * state of its own.  One more small kernel is launched.
 */
struct zt_adamw_form {
  size_t n;
  int grad_dtype, half_dtype;   /* half_dtype is read if d_half is not NULL */
  long long step;               /* >= 1, counting this one */
  double lr, beta1, beta2, eps, weight_decay;   /* lr, eps, weight_decay >= 0; 0 <= beta < 1 */
  float scale, max_norm;        /* as in zt_clip; max_norm is read if d_slots is not NULL */
  double* d_state;              /* NULL, or in place of step and lr */
};
int zt_adamw(const struct zt_adamw_form* form, const void* d_grad, const double* d_slots, float* d_param, float* d_m,
             float* d_v, void* d_half, float* d_norm, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ZT_H */
