// beam.hip -- one selection of a beam search: the K best of K V candidates of
// every sequence, and the reordering of the beams' states.
//
// Within a beam the candidates' order is the logits' (ties to the lowest
// token), so a beam's K best need its logits alone; its log-sum-exp enters
// where beams are compared.  A candidate is a 64-bit key, the value's bits in
// an order-preserving form above the complement of its index: keys are
// distinct, and the larger key is the earlier candidate.
//
// The simple form: one workgroup per beam takes the largest key below the
// last one K times over; one per sequence ranks its K K candidates; one per
// row and state copies.
#include "ops.h"

namespace ldyn {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

__device__ inline uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);  // -0 and 0 are equal
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ inline float unordered(uint32_t u) {
    return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu));
}
// The key of value x at index i; a NaN counts as -inf.
__device__ inline uint64_t key_of(float x, uint32_t i) {
    return (uint64_t)ordered(x == x ? x : -__builtin_inff()) << 32 | (uint32_t)~i;
}

struct BeamParams {
    const void* logits;
    const float* scores;
    const uint8_t* finished;
    float* out_scores;
    int32_t* out_parent;
    int32_t* out_token;
    uint8_t* out_finished;
    uint64_t* best;  // [B K][K] each beam's best keys, in order
    float* lse;      // [B K]
    int B, K, V, end;
};

// m, s of exp(x - m): joined with those of another part.
__device__ inline void join_sum(float& m, float& s, float m2, float s2) {
    const float t = fmaxf(m, m2);
    if (t > -__builtin_inff()) s = s * __expf(m - t) + s2 * __expf(m2 - t);
    m = t;
}

template <class E>
__global__ void __launch_bounds__(THREADS) beam_rows_simple(BeamParams p) {
    __shared__ float wm[WAVES], wsum[WAVES];
    __shared__ uint64_t wk[WAVES];
    const int row = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const E* x = static_cast<const E*>(p.logits) + (long)row * p.V;
    float m = -__builtin_inff(), s = 0.0f;
    for (int j = threadIdx.x; j < p.V; j += THREADS) {
        const float q = (float)x[j];
        if (q == q && q > -__builtin_inff()) join_sum(m, s, q, 1.0f);
    }
    for (int o = 32; o > 0; o >>= 1) {
        const float m2 = __shfl_xor(m, o), s2 = __shfl_xor(s, o);
        join_sum(m, s, m2, s2);
    }
    if (lane == 0) wm[w] = m, wsum[w] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < WAVES; ++i) join_sum(m, s, wm[i], wsum[i]);
        p.lse[row] = m + __logf(s);
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < p.K; ++k) {
        uint64_t best = 0;
        for (int j = threadIdx.x; j < p.V; j += THREADS) {
            const uint64_t q = key_of((float)x[j], (uint32_t)j);
            if (q < last && q > best) best = q;
        }
        for (int o = 32; o > 0; o >>= 1) {
            const uint64_t q = __shfl_xor((unsigned long long)best, o);
            best = q > best ? q : best;
        }
        __syncthreads();
        if (lane == 0) wk[w] = best;
        __syncthreads();
        for (int i = 0; i < WAVES; ++i) best = wk[i] > best ? wk[i] : best;
        last = best;
        if (threadIdx.x == 0) p.best[(long)row * p.K + k] = best;  // 0: fewer than K tokens
        if (best == 0) last = 0;
    }
}

// The k-th entry of a beam whose only candidate is `end` (or none): that one,
// then the other tokens in order.  Returns the token, or V past the last one.
__device__ inline int plain_token(int k, int end, int V) {
    if ((unsigned)end >= (unsigned)V) return k;
    return k == 0 ? end : (k <= end ? k - 1 : k);
}

__global__ void __launch_bounds__(THREADS) beam_select_simple(BeamParams p) {
    __shared__ uint64_t key[LSTM_DYN_BEAM_MAX_K * LSTM_DYN_BEAM_MAX_K];
    __shared__ int token[LSTM_DYN_BEAM_MAX_K * LSTM_DYN_BEAM_MAX_K];
    const int b = blockIdx.x, K = p.K, KK = K * K;
    for (int i = threadIdx.x; i < KK; i += THREADS) {
        const int k = i / K, r = i - k * K, row = b * K + k;
        const float score = p.scores[row], lse = p.lse[row];
        const bool done = p.finished[row] != 0;
        const bool dead = !(score > -__builtin_inff()) || !(lse < __builtin_inff());
        float c = -__builtin_inff();
        int t;
        if (done || dead) {
            t = plain_token(r, done && !dead ? p.end : -1, p.V);
            if (done && !dead && r == 0 && t == p.end) c = score;
        } else {
            const uint64_t q = p.best[(long)row * K + r];
            t = q ? (int)~(uint32_t)q : p.V;
            c = score + (unordered((uint32_t)(q >> 32)) - lse);
        }
        token[i] = t;
        // nothing is taken past a beam's last token
        key[i] = t < p.V ? key_of(c, (uint32_t)i) : 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < KK; i += THREADS) {
        const uint64_t q = key[i];
        if (!q) continue;
        int rank = 0;
        for (int j = 0; j < KK; ++j) rank += key[j] > q;
        if (rank < K) {
            const int k = i / K, o = b * K + rank;
            p.out_scores[o] = unordered((uint32_t)(q >> 32));
            p.out_parent[o] = k;
            p.out_token[o] = token[i];
            p.out_finished[o] = p.finished[b * K + k] != 0 || token[i] == p.end;
        }
    }
}

struct States {
    const char* src[LSTM_DYN_BEAM_MAX_STATES];
    char* dst[LSTM_DYN_BEAM_MAX_STATES];
    long long bytes[LSTM_DYN_BEAM_MAX_STATES];
    int unit[LSTM_DYN_BEAM_MAX_STATES];  // 16, 4 or 1 bytes at once
};

template <class U>
__device__ inline void copy_row(const char* src, char* dst, long long bytes) {
    const long long n = bytes / (long long)sizeof(U);
    for (long long i = threadIdx.x; i < n; i += THREADS)
        reinterpret_cast<U*>(dst)[i] = reinterpret_cast<const U*>(src)[i];
}

__global__ void __launch_bounds__(THREADS) beam_reorder_kernel(BeamParams p, States s) {
    const long row = blockIdx.x;
    const int q = blockIdx.y;
    const long from = row / p.K * p.K + p.out_parent[row];
    const char* src = s.src[q] + from * s.bytes[q];
    char* dst = s.dst[q] + row * s.bytes[q];
    if (s.unit[q] == 16) copy_row<uint4>(src, dst, s.bytes[q]);
    else if (s.unit[q] == 4) copy_row<uint32_t>(src, dst, s.bytes[q]);
    else copy_row<uint8_t>(src, dst, s.bytes[q]);
}

int check_beam_sizes(int B, int K, int V, int dtype) {
    if (B < 1 || K < 1 || V < 1 || !valid_dtype(dtype)) return LSTM_DYN_ERR_INVALID;
    if (K > LSTM_DYN_BEAM_MAX_K || (long long)B * K >= 1 << 24 || V >= 1 << 27) return LSTM_DYN_ERR_UNSUPPORTED;
    return LSTM_DYN_OK;
}

int check_beam_call(int B, int K, int V, int dtype, const void* logits, const float* scores,
                    const uint8_t* finished, const float* os, const int32_t* op, const int32_t* ot,
                    const uint8_t* of, const lstm_dyn_beam_state_t* st, int ns) {
    const int rc = check_beam_sizes(B, K, V, dtype);
    if (rc != LSTM_DYN_OK) return rc;
    if (ns < 0 || ns > LSTM_DYN_BEAM_MAX_STATES || (ns && !st)) return LSTM_DYN_ERR_INVALID;
    const long long n = (long long)B * K;
    Span s[7 + 2 * LSTM_DYN_BEAM_MAX_STATES] = {
        {logits, n * V * dtype_bytes(dtype), 16, false}, {scores, 4 * n, 4, false}, {finished, n, 1, false},
        {os, 4 * n, 4, true}, {op, 4 * n, 4, true}, {ot, 4 * n, 4, true}, {of, n, 1, true}};
    int c = 7;
    for (int i = 0; i < ns; ++i) {
        if (st[i].row_bytes < 1 || st[i].row_bytes >= 1LL << 36) return LSTM_DYN_ERR_INVALID;
        s[c++] = Span{st[i].src, n * st[i].row_bytes, 1, false};
        s[c++] = Span{st[i].dst, n * st[i].row_bytes, 1, true};
    }
    return check_spans(s, c);
}

}  // namespace
}  // namespace ldyn

using namespace ldyn;

struct lstm_dyn_beam : OpsHandle {
    int B, K, V, dtype;
    uint64_t* best;
    float* lse;
};

extern "C" int lstm_dyn_check_beam_args(int B, int K, int V, int dtype, const void* logits,
                                        const float* scores, const uint8_t* finished,
                                        const float* out_scores, const int32_t* out_parent,
                                        const int32_t* out_token, const uint8_t* out_finished,
                                        const lstm_dyn_beam_state_t* states, int n_states) {
    return check_beam_call(B, K, V, dtype, logits, scores, finished, out_scores, out_parent,
                           out_token, out_finished, states, n_states);
}

extern "C" int lstm_dyn_beam_create(lstm_dyn_beam_t** out, int B, int K, int V, int dtype) {
    if (!out) return LSTM_DYN_ERR_INVALID;
    *out = nullptr;
    int rc = check_beam_sizes(B, K, V, dtype);
    if (rc != LSTM_DYN_OK) return rc;
    lstm_dyn_beam* h = new (std::nothrow) lstm_dyn_beam();
    if (!h) return LSTM_DYN_ERR_NOMEM;
    h->B = B; h->K = K; h->V = V; h->dtype = dtype;
    const long long nb = 8LL * B * K * K;
    if ((rc = ops_init(h, 256 + nb + 4LL * B * K)) != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    h->best = reinterpret_cast<uint64_t*>(h->block + 256);
    h->lse = reinterpret_cast<float*>(h->block + 256 + nb);
    *out = h;
    return LSTM_DYN_OK;
}

extern "C" int lstm_dyn_beam_step(lstm_dyn_beam_t* h, const void* logits, const float* scores,
                                  const uint8_t* finished, int end, float* out_scores,
                                  int32_t* out_parent, int32_t* out_token, uint8_t* out_finished,
                                  const lstm_dyn_beam_state_t* states, int n_states, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc = check_beam_call(h->B, h->K, h->V, h->dtype, logits, scores, finished, out_scores,
                             out_parent, out_token, out_finished, states, n_states);
    if (rc != LSTM_DYN_OK) return rc;
    if ((rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const BeamParams p{logits, scores, finished, out_scores, out_parent, out_token, out_finished,
                       h->best, h->lse, h->B, h->K, h->V, end};
    const unsigned rows = (unsigned)(h->B * h->K);
    if (h->dtype == LSTM_DYN_BF16)
        hipLaunchKernelGGL((beam_rows_simple<__bf16>), dim3(rows), dim3(THREADS), 0, h->last_stream, p);
    else
        hipLaunchKernelGGL((beam_rows_simple<float>), dim3(rows), dim3(THREADS), 0, h->last_stream, p);
    if ((rc = ops_launched(h)) != LSTM_DYN_OK) return rc;
    hipLaunchKernelGGL(beam_select_simple, dim3((unsigned)h->B), dim3(THREADS), 0, h->last_stream, p);
    if ((rc = ops_launched(h)) != LSTM_DYN_OK || !n_states) return rc;
    States s{};
    for (int i = 0; i < n_states; ++i) {
        s.src[i] = static_cast<const char*>(states[i].src);
        s.dst[i] = static_cast<char*>(states[i].dst);
        s.bytes[i] = states[i].row_bytes;
        const uintptr_t a = reinterpret_cast<uintptr_t>(s.src[i]) | reinterpret_cast<uintptr_t>(s.dst[i]) |
                            (uintptr_t)s.bytes[i];
        s.unit[i] = a % 16 == 0 ? 16 : a % 4 == 0 ? 4 : 1;
    }
    hipLaunchKernelGGL(beam_reorder_kernel, dim3(rows, (unsigned)n_states), dim3(THREADS), 0,
                       h->last_stream, p, s);
    return ops_launched(h);
}

extern "C" int lstm_dyn_beam_query(lstm_dyn_beam_t* h, int what, long long* value) {
    return ops_query(h, what, value);
}

extern "C" int lstm_dyn_beam_destroy(lstm_dyn_beam_t* h) {
    if (!h) return LSTM_DYN_OK;
    const int rc = ops_free(h);
    delete h;
    return rc;
}
