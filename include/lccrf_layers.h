/*
 * lccrf_layers.h - what a smaller tagger adds to the encoder (lccrf_encoder.h): a gated linear recurrence with one state a
 * channel, group norm with an activation over channels that lie last, and distillation from a teacher's top logits, with their
 * gradients and, for the recurrence, its single-token form.
 *
 * Conventions are those of lccrf_encoder.h: device pointers of the caller's, work enqueued on `stream`, no allocation, no
 * synchronisation, errors found before anything is enqueued, results bit-identical from run to run; `dtype` (LCCRF_F32 or
 * LCCRF_BF16) is the type of activations and their gradients, weights and their gradients, states and statistics are float, and
 * everything is computed in float and rounded once, on its way out.  Rows of inputs may lie anywhere (lccrf_rows); outputs are dense and
 * may not overlap inputs, except where stated.  lengths: int32 [B] or NULL (= all N), clamped to [0, N]; inputs at and past the
 * length are never read, outputs and gradients there are 0.
 * LCCRF_EINVAL where a size is below 1 or above its limit (B * N at most 2^31 - 1024; D, V and K below), LCCRF_EALIGN where a
 * pointer is not aligned to its element (workspaces and `saved`: 256 bytes).  A workspace of 256 bytes is one that nothing is kept in: it may
 * be NULL.
 */
#ifndef LCCRF_LAYERS_H
#define LCCRF_LAYERS_H

#include "lccrf_encoder.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Gated linear recurrence.  With s(v) = 1 / (1 + exp(-v)), for every channel by itself:
 *     u[l]   = -rate * log(1 + exp(decay)) * s(f[l] + f_bias)
 *     h[l]   = exp(u[l]) * h[l-1] + sqrt(1 - exp(2 u[l])) * s(g[l] + g_bias) * x[l],     h[-1] = state or 0
 *     out[l] = h[l] * z[l] * s(z[l])                                                     (z.data NULL: h[l])
 *   x, f, g, z [B][N][D] rows; decay [D], f_bias and g_bias [D] or NULL (= 0); state and final [B][D] float (state NULL: 0;
 *   final NULL: not wanted; final may be state itself).  rate is positive and finite, and so has to be its product
 *   with log(1 + exp(decay)) in float; D at most 2^22.
 * saved: NULL, or lccrf_recurrence_saved_bytes of device memory that takes what the gradient would otherwise compute again (the
 * states in front of every eighth position; its layout is the library's own).
 */
typedef struct {
    lccrf_rows x, f, g, z;
    const float *decay, *f_bias, *g_bias;
} lccrf_recurrence_inputs;

size_t lccrf_recurrence_saved_bytes(int B, int N, int D);
size_t lccrf_recurrence_workspace_bytes(int B, int N, int D);
int lccrf_recurrence(const lccrf_recurrence_inputs* in, lccrf_dtype dtype, float rate, const int32_t* lengths, int B, int N, int D,
                     const float* state, void* out, float* final_state, void* saved, void* workspace, size_t workspace_bytes,
                     void* stream);

/*
 * Gradients of a loss given its gradient by out (what follows through `final` is not part of it).  dx, df, dg, dz [B][N][D]; ddecay,
 * df_bias, dg_bias [D]; dstate [B][D].  dz is wanted exactly where z is given; df_bias, dg_bias and dstate (needs state) may be
 * NULL.  saved: of a lccrf_recurrence with the same inputs, or NULL (then the workspace holds it: workspace_bytes with with_saved = 0).
 */
typedef struct {
    void *dx, *df, *dg, *dz;
    float *ddecay, *df_bias, *dg_bias, *dstate;
} lccrf_recurrence_grads;

size_t lccrf_recurrence_grad_workspace_bytes(int B, int N, int D, int with_saved);
int lccrf_recurrence_grad(const lccrf_rows* dout, const lccrf_recurrence_inputs* in, lccrf_dtype dtype, float rate,
                          const int32_t* lengths, int B, int N, int D, const float* state, const void* saved,
                          const lccrf_recurrence_grads* grads, void* workspace, size_t workspace_bytes, void* stream);

/* One position for B streams: the inputs' rows are [B][D] (`batch` strides; `row` is not looked at), state [B][D] is
 * updated in place, out [B][D]. */
int lccrf_recurrence_step(const lccrf_recurrence_inputs* in, lccrf_dtype dtype, float rate, int B, int D, float* state, void* out,
                          void* stream);

/*
 * Group norm with an activation.  The D channels are G groups of D / G; a set of values normalised together is a group's channels at
 * all positions of a sequence (per_position 0) or at one position (per_position 1: what streams can run), of n values in all:
 *     mean = sum x / n,   var = sum (x - mean)^2 / n,   rstd = 1 / sqrt(var + eps)
 *     y    = (x - mean) * rstd * weight + bias,         out = y * s(y)   (silu 0: y)
 *   x [B][N][D] rows, weight [D] or NULL (= 1), bias [D] or NULL (= 0), out [B][N][D]; eps is finite and at least 2^-126.
 * stats: NULL, or [B][G][2] ([B][N][G][2] per position) floats that take (mean, rstd), 0 where there is nothing to normalise:
 * what the gradient would otherwise compute again.
 */
size_t lccrf_group_norm_workspace_bytes(lccrf_dtype dtype, int B, int N, int D, int G, int per_position);
int lccrf_group_norm(const lccrf_rows* x, lccrf_dtype dtype, const float* weight, const float* bias, const int32_t* lengths, int B,
                     int N, int D, int G, int per_position, float eps, int silu, void* out, float* stats, void* workspace,
                     size_t workspace_bytes, void* stream);

/* Gradients of a loss given its gradient by out: dx [B][N][D], dweight and dbias [D] or NULL.  stats: of a lccrf_group_norm with the
 * same inputs, or NULL (computed again). */
size_t lccrf_group_norm_grad_workspace_bytes(lccrf_dtype dtype, int B, int N, int D, int G, int per_position);
int lccrf_group_norm_grad(const lccrf_rows* dout, const lccrf_rows* x, lccrf_dtype dtype, const float* weight, const float* bias,
                          const int32_t* lengths, int B, int N, int D, int G, int per_position, float eps, int silu,
                          const float* stats, void* dx, float* dweight, float* dbias, void* workspace, size_t workspace_bytes,
                          void* stream);

/*
 * Distillation from a teacher's top logits, position by position (n of them, V classes).  The teacher names up to K classes with
 * their logits: ids int32 [n][K], teacher float [n][K]; an entry whose id is outside [0, V) or whose logit is -inf is not there, and a
 * class may be named twice (its probabilities add up).  With temperature t, q = softmax(teacher / t) over the entries there and
 * p = softmax(logits / t) over all classes:
 *     lse  = log sum_v exp(logits[v] / t)
 *     loss = t^2 * sum_k q_k * (log q_k - (logits[ids_k] / t - lse))
 *   logits [n][V], rows logits_row elements apart; loss and lse float [n].  A position without an entry (padding) has loss 0 and lse 0, and
 *   its logits are not read.  t is finite and at least 2^-126, K at most LCCRF_MAX_TOP, V at most 2^30; n = 0 is allowed, n at most 2^31 - 1.
 *   (The loss is a difference of logarithms: what their rounding leaves in it grows as t^2.)
 */
#define LCCRF_MAX_TOP 256
int lccrf_distill(const void* logits, int64_t logits_row, lccrf_dtype dtype, const int32_t* ids, const float* teacher, int64_t n, int V,
                  int K, float temperature, float* loss, float* lse, void* stream);

/*
 * Its gradient: dlogits[v] = dloss * t * (p[v] - sum of q_k with ids_k = v), [n][V] dense, 0 for positions without an entry; dloss
 * float [n].  lse: of lccrf_distill, or NULL (computed again, with exponentials of differences from the largest logit).  A given lse is looked
 * at in rows past 256 pieces of 16 bytes, where p is exp(logits / t - lse): what both have lost at their own size, some
 * 2^-22 (|lse| + |logits| / t), is in p as a relative error.  loss: NULL, or [n] that takes the loss as well: where dloss is known ahead
 * (weights of positions), this one call is all of a training step's loss.  dlogits may be logits itself (logits_row = V then).
 */
int lccrf_distill_grad(const float* dloss, const void* logits, int64_t logits_row, lccrf_dtype dtype, const int32_t* ids,
                       const float* teacher, int64_t n, int V, int K, float temperature, const float* lse, float* loss, void* dlogits,
                       void* stream);

#ifdef __cplusplus
}
#endif
#endif
