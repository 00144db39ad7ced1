/*
 * lccrf_encoder.h - the encoder in front of a tagger's chain: embedding lookup, short causal
 * convolution and selective state space scan, with their gradients and their single-token forms.
 *
 * Conventions are those of lccrf.h (device pointers of the caller's, work enqueued on `stream`, no
 * allocation, no synchronisation, errors found before anything is enqueued, results bit-identical from
 * run to run), and:
 *  - dtype (LCCRF_F32 or LCCRF_BF16) is the type of activations: table, x, dt, Bm, Cm, z, out, dout and
 *    the gradients of those, and the convolution's state.  Weights (weight, bias, A, D, dt_bias), their
 *    gradients and the scan's state are float.  Everything is computed in float and rounded once,
 *    on its way out.
 *  - lccrf_rows names an input whose rows are dense but may lie anywhere (half of a projection's output,
 *    say): element strides between sequences and between positions; a stride of 0 repeats a row.
 *    Addresses need no more than the element's alignment.  Outputs are dense.
 *  - lengths: int32 [B] or NULL (= all N), clamped to [0, N].  Inputs at and past the length are never
 *    read; outputs and gradients there are 0.
 *  - outputs may not overlap inputs, except where stated.
 *  - LCCRF_EINVAL where a size is below 1 or above its limit (LCCRF_MAX_TAPS, LCCRF_MAX_STATES;
 *    B * N at most 2^31 - 1024, so that positions and what a kernel goes beyond them fit 32 bits; D below 2^31, the
 *    scan's D at most 2^22 and a multiple of G, G * S below 2^27), LCCRF_EALIGN where a pointer is not aligned to its
 *    element (workspaces and `saved`: 256 bytes).
 */
#ifndef LCCRF_ENCODER_H
#define LCCRF_ENCODER_H

#include "lccrf.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LCCRF_MIN_TAPS 2
#define LCCRF_MAX_TAPS 8
#define LCCRF_MAX_STATES 64

typedef struct {
    const void* data;
    int64_t batch; /* elements from a sequence to the next */
    int64_t row;   /* elements from a position to the next */
} lccrf_rows;

/*
 * Embedding: out[p] = scale * table[ids[p]] for n positions; an id outside [0, V) (padding) gives a row of 0.
 *   table [V][D], rows table_row elements apart; ids int32 [n]; out [n][D].  n = 0 is allowed.
 */
int lccrf_embed(const void* table, lccrf_dtype dt, int V, int D, int64_t table_row, const int32_t* ids, int64_t n,
                float scale, void* out, void* stream);

/*
 * Its gradient: grad[v] = scale * sum of dout[p] over the positions with ids[p] = v, [V][D], every row
 * written (0 where no position has it).  The positions are sorted by token first, so that every row is
 * summed in a fixed order.  dout: [B][N][D] rows; ids int32 [B * N], B * N <= 2^30.
 * The sums are held in float and rounded once, to dt: a table and its gradient are one type, half of the bytes written
 * in LCCRF_BF16 (a float gradient of the same positions takes float dout).  B or N may be 0.
 */
size_t lccrf_embed_grad_workspace_bytes(int64_t n, int V, int D);
int lccrf_embed_grad(const lccrf_rows* dout, lccrf_dtype dt, const int32_t* ids, int B, int N, int V, int D,
                     float scale, void* grad, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Short causal convolution with the gate x * sigmoid(x), K taps a channel (2 .. 8):
 *     r        = the K - 1 inputs before the sequence (state, or 0), then x
 *     pre[l]   = bias + sum_k weight[.][k] * r[l + k],      out[l] = pre[l] * sigmoid(pre[l])
 *     final    = r[length .. length + K - 2]: the state from which a later call continues
 *   weight [D][K], bias [D] or NULL, state [B][K-1][D] or NULL, out [B][N][D], final [B][K-1][D] or NULL.
 */
int lccrf_conv(const lccrf_rows* x, lccrf_dtype dt, const float* weight, const float* bias, const void* state,
               const int32_t* lengths, int B, int N, int D, int K, void* out, void* final_state, void* stream);

/*
 * Gradient of a loss by x, weight, bias and state, given its gradient by out (what follows through `final` is
 * not part of it).  dx [B][N][D], dweight [D][K], dbias [D] or NULL, dstate [B][K-1][D] or NULL (needs state).
 */
size_t lccrf_conv_grad_workspace_bytes(int B, int N, int D, int K);
int lccrf_conv_grad(const lccrf_rows* dout, const lccrf_rows* x, lccrf_dtype dt, const float* weight,
                    const float* bias, const void* state, const int32_t* lengths, int B, int N, int D, int K,
                    void* dx, float* dweight, float* dbias, void* dstate, void* workspace, size_t workspace_bytes,
                    void* stream);

/* One position for B streams: x [B][D] (rows x_row elements apart), state [B][K-1][D] read, shifted and
 * completed by x in place, out [B][D]. */
int lccrf_conv_step(const void* x, int64_t x_row, lccrf_dtype dt, const float* weight, const float* bias,
                    void* state, int B, int D, int K, void* out, void* stream);

/*
 * Selective state space scan, S states a channel (1 .. 64), G groups of D / G channels that share Bm and Cm:
 *     step[l]  = log(1 + exp(dt[l] + dt_bias))
 *     h[l]     = exp(step[l] * A) * h[l-1] + step[l] * x[l] * Bm[l],    h[-1] = state or 0
 *     y[l]     = sum_s Cm[l][s] * h[l][s] + D * x[l],                   out[l] = y[l] * z[l] * sigmoid(z[l])
 *   x, dt, z [B][N][D] rows (z.data NULL: out = y), Bm, Cm [B][N][G][S] rows (b_group, c_group elements from a
 *   group to the next), A [D][S], D and dt_bias [D] or NULL (= 0), state and final [B][D][S] float (state NULL:
 *   0; final NULL: not wanted).  final may be state itself.
 */
typedef struct {
    lccrf_rows x, dt, Bm, Cm, z;
    int64_t b_group, c_group;
    const float *A, *D, *dt_bias;
} lccrf_scan_inputs;

/* saved: NULL, or lccrf_state_scan_saved_bytes of device memory that takes what the gradient would otherwise
 * compute again (the states in front of every eighth position; its layout is the library's own). */
size_t lccrf_state_scan_saved_bytes(int B, int N, int D, int S);
size_t lccrf_state_scan_workspace_bytes(int B, int N, int D, int S, int G);
int lccrf_state_scan(const lccrf_scan_inputs* in, lccrf_dtype dtype, const int32_t* lengths, int B, int N, int D,
                     int S, int G, const float* state, void* out, float* final_state, void* saved, void* workspace,
                     size_t workspace_bytes, void* stream);

/*
 * Gradients of a loss given its gradient by out (what follows through `final` is not part of it).  dx, ddt, dz [B][N][D],
 * dBm, dCm [B][N][G][S], dA [D][S], dD, ddt_bias [D], dstate [B][D][S]; dz is wanted exactly where z is given,
 * dD, ddt_bias and dstate may be NULL.  saved: of a lccrf_state_scan with the same inputs, or NULL (then the
 * workspace holds it: workspace_bytes with with_saved = 0).
 */
typedef struct {
    void *dx, *ddt, *dBm, *dCm, *dz;
    float *dA, *dD, *ddt_bias, *dstate;
} lccrf_scan_grads;

size_t lccrf_state_scan_grad_workspace_bytes(int B, int N, int D, int S, int G, int with_saved);
int lccrf_state_scan_grad(const lccrf_rows* dout, const lccrf_scan_inputs* in, lccrf_dtype dtype,
                          const int32_t* lengths, int B, int N, int D, int S, int G, const float* state,
                          const void* saved, const lccrf_scan_grads* grads, void* workspace, size_t workspace_bytes,
                          void* stream);

/* One position for B streams: the inputs' rows are [B][...] (`batch` strides; `row` is not looked at), state
 * [B][D][S] is updated in place, out [B][D]. */
int lccrf_state_step(const lccrf_scan_inputs* in, lccrf_dtype dtype, int B, int D, int S, int G, float* state,
                     void* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif
