/*
 * lstm_dyn_ops.h -- C ABI of the operators around the MI355X (gfx950) time
 * loop of lstm_dyn.h: what a model over tokens needs next to the loop to be
 * trained and to answer.
 *
 *   lstm_dyn_embed_*  rows of a token table as the loop's input x, and the
 *                     gradient of that table from dx
 *   lstm_dyn_scan_*   a gated linear recurrence, whose steps need no product
 *                     with the state, over whole sequences (the time axis is
 *                     split over the device), its backward pass, and one step
 *   lstm_dyn_adamw_*  one AdamW step over all tensors of a model, with states
 *                     in 32 bits or in 8
 *   lstm_dyn_beam_*   one selection of a beam search (the paper's Appendix D
 *                     decoder) over beams and vocabulary, and the reordering
 *                     of the beams' states
 *
 * As in lstm_dyn.h: buffers are caller-owned DEVICE memory, row-major and
 * contiguous; a handle is used from one host thread at a time with one call in
 * flight; calls only enqueue work on `stream` (a hipStream_t; NULL = the default
 * stream), never wait for the host and allocate nothing (the first
 * lstm_dyn_scan_forward_train of a handle apart), so they can be captured
 * in a graph; the handle owns its workspace, made at create for the current
 * device, and is used with that device current (else ERR_INVALID).  Host
 * argument problems are returned synchronously; problems in device data
 * (lengths, tokens) are made harmless as each operator says and reported by its
 * query.  "dtype" is LSTM_DYN_F32 or LSTM_DYN_BF16; all sums, statistics and
 * states are formed in fp32.
 */
#ifndef LSTM_DYN_OPS_H
#define LSTM_DYN_OPS_H

#include "lstm_dyn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A device status beside those of lstm_dyn.h: a token outside [0, V). */
enum { LSTM_DYN_ERR_BAD_TOKENS = 8 };

/* Selectors of the operators' queries. */
enum {
    LSTM_DYN_OPS_Q_STATUS = 0,           /* the device status of the calls since the last such query,
                                            which clears it (synchronises the handle's last stream) */
    LSTM_DYN_OPS_Q_WORKSPACE_BYTES = 1,  /* device workspace owned by the handle */
    LSTM_DYN_OPS_Q_LAUNCHES = 2          /* kernel launches of the last call */
};

/* --- gated linear recurrence ---------------------------------------------- *
 *
 *     a_t = sigmoid(zf_t),  h_t = a_t h_{t-1} + (1 - a_t) zv_t,  y_t = sigmoid(zo_t) h_t
 *
 * for t < L[b], h_{-1} = h0; a row's state stays from its length on, and
 * y_t = 0 there.  Nothing of z at t >= L[b] reaches a result.
 *     z        [B][T_max][3H]   dtype; gate blocks (f, v, o) along 3H; 16-byte aligned
 *     lengths  [B]              int32 in [0, T_max] (clamped, ERR_BAD_LENGTHS)
 *     h0       [B][H]           fp32
 *     out_h    [B][H]           fp32 (written): the state after L[b] steps; may be h0 itself
 *     out_y    [B][T_max][H]    dtype (written in full); 16-byte aligned
 * An infinite state times a gate product that underflows is a NaN here even
 * where it is infinite step by step. */
typedef struct lstm_dyn_scan lstm_dyn_scan_t;

/* B, H, T_max >= 1, B * T_max < 2^31, H < 2^18, T_max < 2^31 - 256, and a launch of less than
 * 2^32 threads: for a row and each 64 of its channels (32 of odd H) about two a step with bf16
 * data, four with fp32, at least 64 a row.  Beyond these ERR_UNSUPPORTED. */
int lstm_dyn_scan_create(lstm_dyn_scan_t** out, int B, int H, int T_max, int dtype);

int lstm_dyn_scan_forward(lstm_dyn_scan_t* h, const void* z, const int32_t* lengths,
                          const float* h0, float* out_h, void* out_y, void* stream);

/* lstm_dyn_scan_forward, also keeping in the handle what lstm_dyn_scan_backward
 * needs (a state every few steps; the first call allocates room for them:
 * about B * T_max * H / 4 bytes with bf16 data, twice that with fp32; under a
 * capture it is refused with ERR_INVALID, later calls are not).  out_h may
 * not be h0.  Any other forward on the handle discards what was kept. */
int lstm_dyn_scan_forward_train(lstm_dyn_scan_t* h, const void* z, const int32_t* lengths,
                                const float* h0, float* out_h, void* out_y, void* stream);

/* Gradients after lstm_dyn_scan_forward_train with the same z, lengths and h0,
 * which it consumes.
 *     dy       [B][T_max][H]    dtype: gradient of out_y (no effect at t >= L[b]); 16-byte aligned
 *     d_out_h  [B][H]           fp32: gradient of out_h, or NULL (zero)
 *     dz       [B][T_max][3H]   dtype (written; zero at t >= L[b]); 16-byte aligned
 *     dh0      [B][H]           fp32 (written)
 * dz has the data's type, unlike the loop's fp32 dx: its reader is a product
 * with operands of that type, which would round it so in any case. */
int lstm_dyn_scan_backward(lstm_dyn_scan_t* h, const void* z, const int32_t* lengths,
                           const float* h0, const void* dy, const float* d_out_h, void* dz,
                           float* dh0, void* stream);

/* One step of `rows` independent rows (a decoder's): z [rows][3H], h and out_h
 * [rows][H] fp32 (out_h may be h itself), out_y [rows][H] dtype; z and out_y
 * aligned to their elements; rows, H >= 1, H < 2^18, less than about 2^32 elements, four times as
 * many where H is a multiple of four and z and out_y are aligned to four elements (else
 * ERR_UNSUPPORTED).  No handle. */
int lstm_dyn_scan_step(int rows, int H, int dtype, const void* z, const float* h, float* out_h,
                       void* out_y, void* stream);

int lstm_dyn_scan_query(lstm_dyn_scan_t* h, int what, long long* value);
int lstm_dyn_scan_destroy(lstm_dyn_scan_t* h);

/* The argument checks of the forwards (dy, dz, dh0 NULL) or of the backward
 * (out_h, out_y NULL), without touching the memory. */
int lstm_dyn_check_scan_args(int B, int H, int T_max, int dtype, const void* z,
                             const int32_t* lengths, const float* h0, const float* out_h,
                             const void* out_y, const void* dy, const float* d_out_h,
                             const void* dz, const float* dh0);

/* --- token table ------------------------------------------------------------ *
 *
 *     x[b][t] = scale * table[tokens[b][t]]                        for t < L[b], else 0
 *     d_table[v] = scale * sum over (b, t), t < L[b], tokens[b][t] = v, of dx[b][t]
 *
 *     tokens   [B][T_max]       int32; one outside [0, V) gives a zero row and no
 *                               gradient (ERR_BAD_TOKENS); not looked at for t >= L[b]
 *     lengths  [B]              int32 in [0, T_max] (clamped), or NULL: all T_max
 *     table    [V][D]           dtype, 16-byte aligned
 *     out_x    [B][T_max][D]    dtype (written in full), 16-byte aligned
 *     dx       [B][T_max][D]    dx_dtype (lstm_dyn_backward gives fp32), 16-byte aligned
 *     d_table  [V][D]           fp32 (written in full), 16-byte aligned
 * A row of d_table is summed in the order of its tokens' places, in pieces that
 * depend on the sizes alone: the same call gives the same bits. */
typedef struct lstm_dyn_embed lstm_dyn_embed_t;

/* All sizes >= 1; B * T_max < 2^30, V < 2^27, D < 2^21; for the gradient also B * T_max / 32 times
 * the tiles of 256 columns (128 where D is no multiple of four, 64 of odd D) under
 * 2^26 - 2^16.  Beyond these ERR_UNSUPPORTED. */
int lstm_dyn_embed_create(lstm_dyn_embed_t** out, int B, int T_max, int V, int D, int dtype);
int lstm_dyn_embed_forward(lstm_dyn_embed_t* h, const int32_t* tokens, const int32_t* lengths,
                           const void* table, float scale, void* out_x, void* stream);
int lstm_dyn_embed_backward(lstm_dyn_embed_t* h, const int32_t* tokens, const int32_t* lengths,
                            const void* dx, int dx_dtype, float scale, float* d_table,
                            void* stream);
int lstm_dyn_embed_query(lstm_dyn_embed_t* h, int what, long long* value);
int lstm_dyn_embed_destroy(lstm_dyn_embed_t* h);

/* The checks of the forward (dx, d_table NULL) or the backward (table, out_x NULL). */
int lstm_dyn_check_embed_args(int B, int T_max, int V, int D, int dtype, const int32_t* tokens,
                              const int32_t* lengths, const void* table, const void* out_x,
                              const void* dx, int dx_dtype, const float* d_table);

/* --- AdamW -------------------------------------------------------------------- *
 *
 * For every element, with the gradient g times grad_scale, at step t = 1, 2, ...:
 *     m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *     p = p - lr ((m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay p)
 * p is fp32; a tensor may have a bf16 copy, written with p rounded.
 *
 * State in 32 bits: m, v fp32.  State in 8 bits: m and r = sqrt(v) as e4m3 codes
 * (4 exponent bits, 3 mantissa bits, largest 448, no infinity), each 256 elements
 * in a row with one power of two 2^(exp - 127), exp a byte: the smallest for which
 * the block's largest finite magnitude is at most 448, and at least 2^-100.  Codes are rounded
 * to nearest even, except that an r that is not zero never becomes zero (a zero
 * there would divide what is left of m by eps).  The update itself uses the m and v
 * of this step in fp32, before they are rounded.  What is not finite becomes a NaN code. */
typedef struct lstm_dyn_adamw lstm_dyn_adamw_t;

typedef struct {
    float* p;            /* [n] parameters (read and written) */
    void* p_bf16;        /* [n] bf16 copy (written), or NULL */
    void* m;             /* [n] fp32, or e4m3 codes */
    void* v;             /* [n] fp32 v, or e4m3 codes of sqrt(v) */
    uint8_t* m_exp;      /* [ceil(n / 256)] exponents (8 bits; else NULL) */
    uint8_t* v_exp;
    long long n;         /* may be 0 */
    float weight_decay;
} lstm_dyn_adamw_tensor_t;

/* The handle copies `tensors` (host memory); p, m, v, p_bf16 lie where the caller keeps
 * them: fp32 4-byte aligned, bf16 2-byte, codes any. */
int lstm_dyn_adamw_create(lstm_dyn_adamw_t** out, const lstm_dyn_adamw_tensor_t* tensors, int count,
                          int state_bits);

/* grads: `count` device pointers (host array), grad_dtype F32 (4-byte aligned) or BF16;
 * read before the call returns only as pointers.  step >= 1. */
int lstm_dyn_adamw_step(lstm_dyn_adamw_t* h, const void* const* grads, int grad_dtype,
                        double lr, double beta1, double beta2, double eps, double grad_scale,
                        long long step, void* stream);

/* 8 bits: the values the codes stand for, m and r = sqrt(v), as bf16 (exact: three
 * mantissa bits and a power of two) into out_m[i], out_v[i] [n_i] each.  32 bits: ERR_UNSUPPORTED. */
int lstm_dyn_adamw_states(lstm_dyn_adamw_t* h, void* const* out_m, void* const* out_v, void* stream);
int lstm_dyn_adamw_query(lstm_dyn_adamw_t* h, int what, long long* value);
int lstm_dyn_adamw_destroy(lstm_dyn_adamw_t* h);

/* The checks of lstm_dyn_adamw_create, and with grads of the step. */
int lstm_dyn_check_adamw_args(const lstm_dyn_adamw_tensor_t* tensors, int count, int state_bits,
                              const void* const* grads, int grad_dtype);

/* --- beam selection -------------------------------------------------------------- *
 *
 * For each of B sequences, with K beams over a vocabulary of V:
 *     candidate (k, j) = scores[k] + (logits[k][j] - log sum_j' exp(logits[k][j']))
 * and for a finished beam the one candidate (k, end) = scores[k], all others -inf.
 * A NaN logit counts as -inf; a candidate that is not a number is -inf (a beam whose logits
 * are all -inf has no other).  The K largest candidates are taken, equal ones by the
 * lowest k V + j, in that order.  Of a beam only the K largest logits are candidates
 * (equal ones by the lowest token), so that sums that differ before they are rounded
 * are not cut off in the wrong order:
 *     out_scores[k'], out_parent[k'] = k, out_token[k'] = j,
 *     out_finished[k'] = finished[k] or j = end,
 * and every state's rows follow their parents, dst[b][k'] = src[b][out_parent[k']].
 *     logits [B][K][V] dtype, 16-byte aligned; scores [B][K] fp32; finished [B][K] uint8
 *     (not zero: finished); out_scores fp32, out_parent and out_token int32,
 *     out_finished uint8, all [B][K]; no output may overlap an input or another output.
 * end: the end token, or any value outside [0, V) for none (a finished beam then has no
 * candidate but -inf). */
typedef struct lstm_dyn_beam lstm_dyn_beam_t;

#define LSTM_DYN_BEAM_MAX_K 32
#define LSTM_DYN_BEAM_MAX_STATES 8
typedef struct {
    const void* src;     /* [B][K] rows */
    void* dst;           /* [B][K] rows (written), apart from every src */
    long long row_bytes; /* >= 1 */
} lstm_dyn_beam_state_t;

/* B, V >= 1, 1 <= K <= 32, B * K < 2^22, V < 2^27. */
int lstm_dyn_beam_create(lstm_dyn_beam_t** out, int B, int K, int V, int dtype);
int lstm_dyn_beam_step(lstm_dyn_beam_t* h, const void* logits, const float* scores,
                       const uint8_t* finished, int end, float* out_scores, int32_t* out_parent,
                       int32_t* out_token, uint8_t* out_finished,
                       const lstm_dyn_beam_state_t* states, int n_states, void* stream);
int lstm_dyn_beam_query(lstm_dyn_beam_t* h, int what, long long* value);
int lstm_dyn_beam_destroy(lstm_dyn_beam_t* h);
int lstm_dyn_check_beam_args(int B, int K, int V, int dtype, const void* logits,
                             const float* scores, const uint8_t* finished,
                             const float* out_scores, const int32_t* out_parent,
                             const int32_t* out_token, const uint8_t* out_finished,
                             const lstm_dyn_beam_state_t* states, int n_states);

#ifdef __cplusplus
}
#endif

#endif /* LSTM_DYN_OPS_H */
