/*
 * lstm_dyn_layer.h -- C ABI of the operators of a layer around the MI355X
 * (gfx950) time loop, of its training and of its answers.
 *
 *   lstm_dyn_attend_*  linear attention with a decay for each head: a recurrence
 *                      whose state is a matrix, over whole sequences (in chunks, as
 *                      products), its backward pass, and one step
 *   lstm_dyn_norm_*    layer norm over the last axis, and its backward pass
 *   lstm_dyn_clip_*    the norm of all gradients of a model, and clipping to it;
 *                      lstm_dyn_adamw_step_clipped takes the clipping along
 *   lstm_dyn_sample_*  one token a row from its logits and a given random number
 *
 * As in lstm_dyn_ops.h: buffers are caller-owned DEVICE memory, row-major and
 * contiguous; a handle is used from one host thread at a time with one call in
 * flight; calls only enqueue work on `stream` (a hipStream_t; NULL = the default
 * stream), never wait for the host and allocate nothing, so they can be captured
 * in a graph; the handle owns its workspace, made at create for the current
 * device, and is used with that device current (else ERR_INVALID).  Host
 * argument problems are returned synchronously; lengths outside [0, T_max] are
 * clamped and reported by the operator's query (the selectors of lstm_dyn_ops.h).
 * "dtype" is LSTM_DYN_F32 or LSTM_DYN_BF16; all sums, statistics and states are
 * formed and held in fp32 or more (what enters some products with fewer bits stands
 * at the operator).
 */
#ifndef LSTM_DYN_LAYER_H
#define LSTM_DYN_LAYER_H

#include "lstm_dyn_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* --- layer norm ------------------------------------------------------------- *
 *
 * For every (b, t), t < L[b], over its D elements:
 *     n = (x - mean x) / sqrt(mean (x - mean x)^2 + eps),  y = n weight + bias
 * and y = 0 for t >= L[b].  Backward, with g = dy weight:
 *     dx = (g - mean g - n mean (g n)) / sqrt(...),  0 for t >= L[b]
 *     d_weight = sum over (b, t), t < L[b], of dy n,   d_bias = the same of dy
 * Nothing at t >= L[b] is read.  The statistics are formed again in the backward,
 * so it needs no forward before it.
 *     x        [B][T_max][D]   dtype, 16-byte aligned
 *     lengths  [B]             int32 in [0, T_max], or NULL: all T_max
 *     weight   [D]             fp32, or NULL: ones;  bias [D] fp32, or NULL: zeros
 *     out_y    [B][T_max][D]   dtype (written in full), 16-byte aligned; may be x itself
 *     dy       [B][T_max][D]   dy_dtype (lstm_dyn_backward gives fp32), 16-byte aligned
 *     out_dx   [B][T_max][D]   dy_dtype (written in full), 16-byte aligned; may be dy itself
 *     d_weight, d_bias [D]     fp32 (written)
 * Sums over rows go in an order that the sizes alone decide: the same call gives the same bits. */
typedef struct lstm_dyn_norm lstm_dyn_norm_t;

/* B, T_max, D >= 1, D <= 32768, B * T_max < 2^31, eps >= 0 (finite). */
int lstm_dyn_norm_create(lstm_dyn_norm_t** out, int B, int T_max, int D, int dtype, float eps);
int lstm_dyn_norm_forward(lstm_dyn_norm_t* h, const void* x, const int32_t* lengths,
                          const float* weight, const float* bias, void* out_y, void* stream);
int lstm_dyn_norm_backward(lstm_dyn_norm_t* h, const void* x, const int32_t* lengths,
                           const float* weight, const void* dy, int dy_dtype, void* out_dx,
                           float* d_weight, float* d_bias, void* stream);
int lstm_dyn_norm_query(lstm_dyn_norm_t* h, int what, long long* value);
int lstm_dyn_norm_destroy(lstm_dyn_norm_t* h);

/* The checks of the forward (dy, out_dx, d_weight, d_bias NULL) or the backward (bias, out_y NULL). */
int lstm_dyn_check_norm_args(int B, int T_max, int D, int dtype, float eps, const void* x,
                             const int32_t* lengths, const float* weight, const float* bias,
                             const void* out_y, const void* dy, int dy_dtype, const void* out_dx,
                             const float* d_weight, const float* d_bias);

/* --- gradient norm and clipping ------------------------------------------------ *
 *
 *     result[0] = |grad_scale| sqrt(sum over all tensors and elements of g^2)
 *     result[1] = grad_scale min(1, max_norm / result[0])   (grad_scale where result[0] is 0)
 * The sum is formed in 64 bits: it neither overflows nor underflows where the
 * norm is an fp32 number.  A norm that is infinite gives a factor of zero (but for an infinite
 * max_norm, which clips nothing), one that is not a number gives such a factor.  Clipping writes out = g result[1], rounded once
 * (an infinite g times zero is not a number). */
typedef struct lstm_dyn_clip lstm_dyn_clip_t;

/* n: the tensors' elements (host array, copied), each 0 <= n[i] < 2^40, together under 2^36. */
int lstm_dyn_clip_create(lstm_dyn_clip_t** out, const long long* n, int count);

/* grads: `count` device pointers (host array), grad_dtype F32 (4-byte aligned) or BF16 (2-byte); result
 * [2] fp32 (written).  max_norm >= 0 and grad_scale finite. */
int lstm_dyn_clip_norm(lstm_dyn_clip_t* h, const void* const* grads, int grad_dtype,
                       double grad_scale, double max_norm, float* result, void* stream);

/* out[i] = grads[i] result[1] in the gradients' type; out[i] may be grads[i] itself, and overlaps no
 * other gradient or output.  result: as lstm_dyn_clip_norm wrote it, or any fp32 [2]. */
int lstm_dyn_clip_apply(lstm_dyn_clip_t* h, const void* const* grads, int grad_dtype,
                        const float* result, void* const* out, void* stream);
int lstm_dyn_clip_query(lstm_dyn_clip_t* h, int what, long long* value);
int lstm_dyn_clip_destroy(lstm_dyn_clip_t* h);

/* The checks of lstm_dyn_clip_create; with grads and result of the norm; with out too of clipping. */
int lstm_dyn_check_clip_args(const long long* n, int count, const void* const* grads,
                             int grad_dtype, const float* result, void* const* out);

/* lstm_dyn_adamw_step whose gradients are each times result[1] (read on the device when the
 * step runs) in place of grad_scale. */
int lstm_dyn_adamw_step_clipped(lstm_dyn_adamw_t* h, const void* const* grads, int grad_dtype,
                                double lr, double beta1, double beta2, double eps,
                                const float* result, long long step, void* stream);

/* --- sampling ---------------------------------------------------------------- *
 *
 * For each row, its tokens in order: by logit from the largest, equal ones by the lowest index
 * (a NaN logit counts as -inf); p = exp((logit - largest) / temperature).  Kept are
 *     of all tokens the first top_k (0 < top_k < V),
 *     of those the shortest start whose p sum to top_p of theirs or more (top_p < 1; at least one token),
 *     of those the ones with p >= min_p (0 < min_p; 1 at most)
 * and the token is the lowest index j for which the p of the kept tokens up to j sum to more than
 * u of all the kept ones'.  out_logp = log(p[token] / sum of the kept p).
 * A temperature that is not above zero (or so small that 1 / it is infinite) takes the first token,
 * logp 0.  Where the largest logit is +inf, such tokens have p = 1, all others 0.  A row whose logits
 * are all -inf has no token: -1, with logp -inf.  top_k <= 0 and top_p or min_p that are NaN are as if
 * not given, top_p <= 0 keeps the first token.
 * p are fp32 exponentials, off by up to 2^-22 of themselves, held as multiples of 2^-46 (of 2^-(62 - n) if
 * V > 2^16, for the n with 2^(n-1) < V <= 2^n), rounded down: the sums of these p are exact, so the order of summation
 * changes nothing, and a token whose p is below one of them is not chosen.  Where u or top_p comes nearer than about 2^-22 of
 * the whole to a sum that it is compared with, or min_p to a p, the token may be that of its other side.
 *     logits  [N][V]  dtype, aligned to its elements
 *     u       [N]     fp32 in [0, 1) (clamped; NaN is 0)
 *     out_token int32 [N], out_logp fp32 [N]; they overlap nothing else */
typedef struct lstm_dyn_sample lstm_dyn_sample_t;

/* A value for all rows, or one a row: an array [N] of device memory, if not NULL, takes its place. */
typedef struct {
    float temperature;
    float top_p;
    float min_p;
    int32_t top_k;
    const float* temperatures;
    const float* top_ps;
    const float* min_ps;
    const int32_t* top_ks;
} lstm_dyn_sample_filter_t;

/* N, V >= 1, N < 2^22, V < 2^27. */
int lstm_dyn_sample_create(lstm_dyn_sample_t** out, int N, int V, int dtype);

/* filter: host memory, read before the call returns; NULL: temperature 1 and no filter. */
int lstm_dyn_sample_step(lstm_dyn_sample_t* h, const void* logits, const float* u,
                         const lstm_dyn_sample_filter_t* filter, int32_t* out_token,
                         float* out_logp, void* stream);
int lstm_dyn_sample_query(lstm_dyn_sample_t* h, int what, long long* value);
int lstm_dyn_sample_destroy(lstm_dyn_sample_t* h);
int lstm_dyn_check_sample_args(int N, int V, int dtype, const void* logits, const float* u,
                               const lstm_dyn_sample_filter_t* filter, const int32_t* out_token,
                               const float* out_logp);

/* --- linear attention ------------------------------------------------------------ *
 *
 * For every row b and head, with the head's decay a, over t < L[b]:
 *     S_t = a S_{t-1} + k_t v_t^T,   y_t = S_t^T q_t,   S_{-1} = S0
 * a row's state stays from its length on, and y_t = 0 there.  Backward, with
 * R_t = q_t dy_t^T + a R_{t+1} (at t = L[b] - 1: + d_out_S in its place):
 *     dq_t = S_t dy_t,   dk_t = R_t v_t,   dv_t = R_t^T k_t,   dS0 = a R_0 (L[b] = 0: d_out_S)
 * Nothing of z or dy at t >= L[b] reaches a result.
 *     z        [B][T_max][heads (2 Dk + Dv)]  dtype: q of all heads, k of all heads, v of all
 *                                             heads; aligned to its elements
 *     lengths  [B]                            int32 in [0, T_max], or NULL: all T_max
 *     S0       [B][heads][Dk][Dv]             fp32
 *     out_S    [B][heads][Dk][Dv]             fp32 (written): the state after L[b] steps; may be S0 itself
 *     out_y    [B][T_max][heads Dv]           dtype (written in full)
 *     dy       [B][T_max][heads Dv]           dtype
 *     d_out_S  [B][heads][Dk][Dv]             fp32, or NULL (zero)
 *     dz       as z                           dtype (written; zero at t >= L[b])
 *     dS0      [B][heads][Dk][Dv]             fp32 (written)
 * Inside a chunk of 64 steps (32 with fp32 data) an infinity or a NaN in z or dy makes what comes before it in the
 * chunk no number as well; with bf16 data a state beyond 3.39e38 makes y in its column no number.
 * With bf16 data a state and a product q k, v dy, ... of two steps enter the products that give y and dz as 16 bits (two
 * bf16 parts): beside their rounding to bf16, y and dz are off by up to 2^-17 of the magnitudes that they are the sum of.
 * States themselves and dS0 are fp32 sums of unrounded products.
 * No scale is put on q k: it belongs into the weights that q or k come from.
 * The backward needs no forward before it.  Sums go in an order that the sizes alone decide. */
typedef struct lstm_dyn_attend lstm_dyn_attend_t;

/* decay: [heads] host memory (copied), each in [0, 1].  B, heads, T_max >= 1, 1 <= Dk, Dv <= 128,
 * heads <= 16384, B * heads < 2^20, B * T_max < 2^31, T_max < 2^30. */
int lstm_dyn_attend_create(lstm_dyn_attend_t** out, int B, int heads, int Dk, int Dv, int T_max,
                           int dtype, const float* decay);
int lstm_dyn_attend_forward(lstm_dyn_attend_t* h, const void* z, const int32_t* lengths,
                            const float* S0, float* out_S, void* out_y, void* stream);
int lstm_dyn_attend_backward(lstm_dyn_attend_t* h, const void* z, const int32_t* lengths,
                             const float* S0, const void* dy, const float* d_out_S, void* dz,
                             float* dS0, void* stream);

/* One step of `rows` independent rows (a decoder's; any number, not the handle's B): z [rows][heads (2 Dk
 * + Dv)], S and out_S [rows][heads][Dk][Dv] (out_S may be S itself), out_y [rows][heads Dv].
 * rows * heads < 2^24. */
int lstm_dyn_attend_step(lstm_dyn_attend_t* h, int rows, const void* z, const float* S,
                         float* out_S, void* out_y, void* stream);
int lstm_dyn_attend_query(lstm_dyn_attend_t* h, int what, long long* value);
int lstm_dyn_attend_destroy(lstm_dyn_attend_t* h);

/* The checks of create (z NULL), of the forward (dy, dz, dS0 NULL) or the backward (out_S, out_y NULL). */
int lstm_dyn_check_attend_args(int B, int heads, int Dk, int Dv, int T_max, int dtype,
                               const float* decay, const void* z, const int32_t* lengths,
                               const float* S0, const float* out_S, const void* out_y,
                               const void* dy, const float* d_out_S, const void* dz,
                               const float* dS0);

#ifdef __cplusplus
}
#endif

#endif /* LSTM_DYN_LAYER_H */
