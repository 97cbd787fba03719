// beam.hip -- one selection of a beam search: the K best of K V candidates of
// every sequence, and the reordering of the beams' states.
//
// Within a beam the candidates' order is the logits' (ties to the lowest
// token), so a beam's K best need its logits alone; its log-sum-exp enters
// where beams are compared.  A candidate is a 64-bit key, the value's bits in
// an order-preserving form above the complement of its index: keys are
// distinct, and the larger key is the earlier candidate.
//
// One launch reads the logits once: a workgroup holds a slice of a beam in
// registers, sums its exps and finds its K best keys:
//   the K-th largest of 64 lanes' own maxima, found bit by bit with ballots, is
//   a bound that K keys reach; of the four waves' bounds the largest is taken;
//   sixteen-byte pieces that hold something as large (about 4 K of them) go to LDS,
//   and their keys are ranked by counting.
// The last workgroup of a sequence to end joins the slices: the beams'
// log-sum-exps, then the K best of the slices' keys in the same way.  It moves small
// states too; large ones take a launch of their own.
//
// 64 x 16 beams over 65536 tokens in bf16: 43 us, 3.1 TB/s of logits.  About half of the
// time the vector units are busy (11.5 instructions per 64 tokens: widening, maximum,
// exp, sum; and the bounds), and the slices' ends wait for each other; the states (2 x 2048 floats a
// beam) 8 us more.  16 x 8 beams over 32768: 15 us, and one sequence with four
// beams over 1000: 10 us, both a chain of loads, barriers and the join.
#include "ops.h"

namespace ldyn {
namespace {

// States of a sequence up to this size are moved by its last workgroup (8
// beams of 8 KB: 20.6 us for the step so, 24.4 with a launch of its own; 64 x 16 beams of
// 16 KB: 75 and 54).
constexpr long long FUSED_STATE_BYTES = 64 << 10;

constexpr int THREADS = 256, WAVES = THREADS / 64, ARRIVED_WORDS = 16;
constexpr int GATHER = 512;  // keys ranked at once

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
    uint64_t* best;    // [B K][slices][K] each slice's best keys, in order; 0 past the last
    uint64_t* sums;    // [B K][slices] {m, s}
    unsigned* arrived; // [B] workgroups of the sequence that have ended, 64 bytes apart
    int B, K, V, end, slices;
};

// m, s of exp(x - m): joined with those of another part.
__device__ inline void join_sum(float& m, float& s, float m2, float s2) {
    const float t = fmaxf(m, m2);
    if (t > -__builtin_inff()) s = s * __expf(m - t) + s2 * __expf(m2 - t);
    m = t;
}

// Over the wave, in every lane (row shifts, then broadcasts of rows' last lanes).
template <int CTRL>
__device__ inline float dpp(float old, float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(x), CTRL, 0xf, 0xf, false));
}
__device__ inline float lane63(float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63)); }
__device__ inline float wave_max(float x) {
    const float ninf = -__builtin_inff();
    x = fmaxf(x, dpp<0x111>(ninf, x));
    x = fmaxf(x, dpp<0x112>(ninf, x));
    x = fmaxf(x, dpp<0x114>(ninf, x));
    x = fmaxf(x, dpp<0x118>(ninf, x));
    x = fmaxf(x, dpp<0x142>(ninf, x));
    x = fmaxf(x, dpp<0x143>(ninf, x));
    return lane63(x);
}
__device__ inline float wave_sum(float x) {
    x += dpp<0x111>(0.0f, x);
    x += dpp<0x112>(0.0f, x);
    x += dpp<0x114>(0.0f, x);
    x += dpp<0x118>(0.0f, x);
    x += dpp<0x142>(0.0f, x);
    x += dpp<0x143>(0.0f, x);
    return lane63(x);
}

// A bound that the keys of at least K lanes reach (0 if fewer have a key): the
// K-th largest, bit by bit from the top (LAST: below it all bits are the
// same), ended as soon as the bits so far tell exactly K lanes apart.  From the
// high words alone, where equal ones may let more than K lanes reach it; with
// `exact` also from low(), the lanes' low words.
template <int LAST, class Low>
__device__ inline uint64_t wave_bound(uint32_t high, int K, bool exact, Low low) {
    uint64_t alive = __ballot(high != 0);
    if (__popcll(alive) < K) return 0;
    int need = K;
    auto narrow = [&](uint32_t word, int last) {
        uint32_t bits = 0;
        for (int bit = 31; bit >= last && __popcll(alive) != need; --bit) {
            const uint64_t m = __ballot((word >> bit) & 1) & alive;
            const int c = __popcll(m);
            if (c >= need) {
                alive = m;
                bits |= 1u << bit;
            } else {
                need -= c;
                alive &= ~m;
            }
        }
        return bits;
    };
    const uint64_t hi = (uint64_t)narrow(high, LAST) << 32;
    if (!exact || __popcll(alive) == need) return hi;
    return hi | narrow(low(), 0);
}

struct Shared {
    uint64_t bound[WAVES];
    uint64_t best[LSTM_DYN_BEAM_MAX_K];  // the K largest keys so far, in order; 0: none
    uint64_t cand[GATHER + LSTM_DYN_BEAM_MAX_K];
    float m[WAVES], s[WAVES];
    float top[LSTM_DYN_BEAM_MAX_K], lse[LSTM_DYN_BEAM_MAX_K];  // a beam's largest logit; log sum exp(x - top)
    int parent[LSTM_DYN_BEAM_MAX_K];
    unsigned n, quads;
    int last;
};

__device__ inline void gather(uint64_t key, Shared* sh) { sh->cand[atomicAdd(&sh->n, 1u)] = key; }

// The K best of the gathered keys (at most GATHER) and of sh->best, into sh->best.
// Called by the whole workgroup after the gathering.
__device__ inline void rank_keys(int K, Shared* sh) {
    if (threadIdx.x < (unsigned)K && sh->best[threadIdx.x]) gather(sh->best[threadIdx.x], sh);
    __syncthreads();
    const unsigned n = sh->n;
    if (threadIdx.x < (unsigned)K) sh->best[threadIdx.x] = 0;
    __syncthreads();
    for (unsigned i = threadIdx.x; i < n; i += THREADS) {
        const uint64_t q = sh->cand[i];
        int rank = 0;
#pragma unroll 8
        for (unsigned j = 0; j < n; ++j) rank += sh->cand[j] > q;
        if (rank < K) sh->best[rank] = q;
    }
    if (threadIdx.x == 0) sh->n = sh->quads = 0;
    __syncthreads();
}

// Sixteen bytes of logits.
template <class E>
struct Quad {
    static constexpr int N = 16 / (int)sizeof(E);
    uint32_t w[4];

    __device__ float operator[](int i) const {
        if constexpr (sizeof(E) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
    __device__ void set_nan(int i) {
        if constexpr (sizeof(E) == 4) w[i] = 0x7fc00000u;
        else w[i >> 1] = i & 1 ? (w[i >> 1] & 0xffffu) | 0x7fc00000u : (w[i >> 1] & 0xffff0000u) | 0x7fc0u;
    }
};

// The compiler may not keep what it formed of these before here (bf16 pairs
// widened once and kept take twice their registers).
template <class E, int N>
__device__ inline void hold(Quad<E>* v) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(v[i].w[j]));
}

// The k-th entry of a beam whose only candidate is `end` (or none): that one,
// then the other tokens in order.
__device__ inline int plain_token(int k, int end, int V) {
    if ((unsigned)end >= (unsigned)V) return k;
    return k == 0 ? end : (k <= end ? k - 1 : k);
}

struct States {
    const char* src[LSTM_DYN_BEAM_MAX_STATES];
    char* dst[LSTM_DYN_BEAM_MAX_STATES];
    long long bytes[LSTM_DYN_BEAM_MAX_STATES];
    int unit[LSTM_DYN_BEAM_MAX_STATES];  // 16, 4 or 1 bytes at once
    int n;                               // how many the selection's launch reorders itself
};

template <class U>
__device__ inline void copy_rows(const char* src, char* dst, unsigned row_units, int K, const int* parent) {
    for (unsigned i = threadIdx.x; i < K * row_units; i += THREADS) {
        const unsigned k = i / row_units, u = i - k * row_units;
        reinterpret_cast<U*>(dst)[i] = reinterpret_cast<const U*>(src)[parent[k] * row_units + u];
    }
}

// Joins the slices of sequence b; its last workgroup does this.
__device__ void join_slices(const BeamParams& p, const States& st, int b, Shared* sh) {
    constexpr int HOLD = GATHER / THREADS;  // keys a thread holds at once
    const int K = p.K, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const float ninf = -__builtin_inff();
    if (threadIdx.x < (unsigned)K) {
        const int row = b * K + threadIdx.x;
        float m = ninf, s = 0.0f;
        for (int i = 0; i < p.slices; ++i) {
            const uint64_t q = __hip_atomic_load(p.sums + (long)row * p.slices + i, __ATOMIC_RELAXED,
                                                 __HIP_MEMORY_SCOPE_AGENT);
            join_sum(m, s, __uint_as_float((uint32_t)(q >> 32)), __uint_as_float((uint32_t)q));
        }
        // m and the log apart: their sum would be rounded at the size of m, which candidates of
        // other beams, with another m, are compared with
        const float lse = logf(s);
        const bool live = p.scores[row] > ninf && lse < __builtin_inff();
        // a beam that is not live has no number among its candidates
        sh->top[threadIdx.x] = m;
        sh->lse[threadIdx.x] = live || p.finished[row] ? lse : __builtin_nanf("");
        sh->best[threadIdx.x] = 0;
    }
    __syncthreads();
    const unsigned per = (unsigned)p.slices * K, total = per * K;
    for (unsigned base = 0; base < total; base += THREADS * HOLD) {
        uint64_t key[HOLD];
#pragma unroll
        for (int i = 0; i < HOLD; ++i) {
            const unsigned at = base + i * THREADS + threadIdx.x;
            key[i] = 0;
            if (at >= total) continue;
            const unsigned k = at / per, r = at - k * per;
            const int row = b * K + (int)k;
            const bool done = p.finished[row] != 0;
            const float score = p.scores[row], top = sh->top[k], lse = sh->lse[k];
            if (done || lse != lse) {
                const int end = done && score > ninf ? p.end : -1;
                const int t = r < (unsigned)K ? plain_token((int)r, end, p.V) : p.V;
                if (t < p.V) key[i] = key_of(t == end ? score : ninf, k * (unsigned)p.V + (unsigned)t);
            } else {
                const uint64_t q = __hip_atomic_load(p.best + (long)row * per + r, __ATOMIC_RELAXED,
                                                     __HIP_MEMORY_SCOPE_AGENT);
                if (q) key[i] = key_of(score + ((unordered((uint32_t)(q >> 32)) - top) - lse), k * (unsigned)p.V + ~(uint32_t)q);
            }
        }
        // no worse than the K-th so far, and than what K lanes of a wave have
        uint64_t most = key[0];
#pragma unroll
        for (int i = 1; i < HOLD; ++i) most = key[i] > most ? key[i] : most;
        const uint64_t bound = wave_bound<0>((uint32_t)(most >> 32), K, false, [] { return 0u; });
        if (lane == 0) sh->bound[w] = bound;
        __syncthreads();
        uint64_t least = sh->best[K - 1] | 1;
        for (int i = 0; i < WAVES; ++i) least = sh->bound[i] > least ? sh->bound[i] : least;
#pragma unroll
        for (int i = 0; i < HOLD; ++i)
            if (key[i] >= least) gather(key[i], sh);
        rank_keys(K, sh);
    }
    if (threadIdx.x < (unsigned)K) {
        const uint64_t q = sh->best[threadIdx.x];
        const uint32_t flat = ~(uint32_t)q;
        const int k = (int)(flat / (unsigned)p.V), t = (int)(flat - (unsigned)k * (unsigned)p.V);
        const int o = b * K + threadIdx.x;
        p.out_scores[o] = unordered((uint32_t)(q >> 32));
        p.out_parent[o] = k;
        p.out_token[o] = t;
        p.out_finished[o] = p.finished[b * K + k] != 0 || t == p.end;
        sh->parent[threadIdx.x] = k;
    }
    if (!st.n) return;
    __syncthreads();
    for (int q = 0; q < st.n; ++q) {
        const char* src = st.src[q] + (long)b * K * st.bytes[q];
        char* dst = st.dst[q] + (long)b * K * st.bytes[q];
        const unsigned units = (unsigned)(st.bytes[q] / st.unit[q]);
        if (st.unit[q] == 16) copy_rows<uint4>(src, dst, units, K, sh->parent);
        else if (st.unit[q] == 4) copy_rows<uint32_t>(src, dst, units, K, sh->parent);
        else copy_rows<uint8_t>(src, dst, units, K, sh->parent);
    }
}

// A lane's largest key.  Read again, element by element: only rows with more
// equal logits than a workgroup can put aside come here.
template <class E, int N>
__device__ __attribute__((noinline)) uint64_t largest_key(const E* row, int mine, int end, int off, int V) {
    uint64_t top = 0;
#pragma unroll 1
    for (int i = 0; i < N * Quad<E>::N; ++i) {
        const int quad = mine + i / Quad<E>::N * THREADS, t = quad * Quad<E>::N + i % Quad<E>::N - off;
        if (quad >= end || t < 0 || t >= V) continue;
        const uint64_t key = key_of((float)row[t], (uint32_t)t);
        top = key > top ? key : top;
    }
    return top;
}

// N: sixteen-byte loads a thread holds at once.  Six waves a SIMD: at eight loads 80 registers (64 x 16
// beams over 65536 tokens in bf16: 53 us for the step, with 82 and five waves 57).
template <class E, int N>
__global__ void __launch_bounds__(THREADS, 6) beam_kernel(BeamParams p, States st, unsigned room) {
    extern __shared__ uint4 held[];  // `room` quads, then their numbers
    __shared__ Shared sh;
    int* number = reinterpret_cast<int*>(held + room);
    constexpr int Q = Quad<E>::N;
    const float ninf = -__builtin_inff();
    const int K = p.K, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int row = (int)(blockIdx.x / (unsigned)p.slices), slice = (int)(blockIdx.x - (unsigned)row * p.slices);
    const int b = row / K;
    if (threadIdx.x < (unsigned)K) sh.best[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.n = sh.quads = 0;
    float m = ninf, s = 0.0f;  // of this wave
    if (!p.finished[row] && p.scores[row] > ninf) {
        // the quads of the buffer that hold the row's tokens; token j is element off + j of them
        const long first = (long)row * p.V, whole = ((long)p.B * K * p.V) / Q;
        const long quad0 = first / Q;
        const int off = (int)(first - quad0 * Q);
        const int quads = (int)(((long)off + p.V + Q - 1) / Q);
        const int per = (quads + p.slices - 1) / p.slices;
        const int end = min(quads, (slice + 1) * per);
        const Quad<E>* x = static_cast<const Quad<E>*>(p.logits) + quad0;
        const bool ragged = p.V % Q != 0;
        for (int from = slice * per; from < end; from += THREADS * N) {
            Quad<E> v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int at = from + i * THREADS + threadIdx.x;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].w[j] = sizeof(E) == 4 ? 0x7fc00000u : 0x7fc07fc0u;
                if (at < end && quad0 + at < whole) {
                    const uint4 u = *reinterpret_cast<const uint4*>(x + at);
                    v[i].w[0] = u.x;
                    v[i].w[1] = u.y;
                    v[i].w[2] = u.z;
                    v[i].w[3] = u.w;
                } else if (at < end) {  // the buffer ends inside this one
                    const E* e = static_cast<const E*>(p.logits) + (quad0 + at) * Q;
                    const int n = (int)((long)p.B * K * p.V - (quad0 + at) * Q);
#pragma unroll
                    for (int j = 0; j < Q - 1; ++j) {
                        if (j >= n) continue;
                        if constexpr (sizeof(E) == 4) v[i].w[j] = __float_as_uint(e[j]);
                        else v[i].w[j >> 1] = j & 1 ? (v[i].w[j >> 1] & 0xffffu) | (uint32_t)reinterpret_cast<const uint16_t*>(e)[j] << 16
                                                    : (v[i].w[j >> 1] & 0xffff0000u) | reinterpret_cast<const uint16_t*>(e)[j];
                    }
                }
                if (ragged && at < end && (at == 0 || at == quads - 1)) {  // other rows' tokens
#pragma unroll
                    for (int j = 0; j < Q; ++j) {
                        const int t = at * Q + j - off;
                        if (t < 0 || t >= p.V) v[i].set_nan(j);
                    }
                }
            }
            // a NaN is passed over by the maximum
            float most[N], top = ninf;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                most[i] = ninf;
#pragma unroll
                for (int j = 0; j < Q; ++j) most[i] = fmaxf(most[i], v[i][j]);
                top = fmaxf(top, most[i]);
            }
            const float wm = wave_max(top);
            hold<E, N>(v);
            if (wm > ninf) {
                // exp(x - wm) as 2^(x log2 e - c), an instruction less than from x - wm.  c is wm log2 e
                // rounded, at x = wm the exponent is that rounding: common to all terms, and taken out
                // of the sum (the fused product gives it whole).  It grows with wm: a strip whose
                // largest logit is large, masked tokens' mostly, forms x - wm, and so does one with NaN
                // logits, which add nothing.
                const float log2e = 1.44269504f, c = wm * log2e;
                float sum = 0.0f;
                bool apart = fabsf(wm) > 0x1p16f;
                if (!apart) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int j = 0; j < Q; ++j) sum += __builtin_amdgcn_exp2f(fmaf(v[i][j], log2e, -c));
                    sum = wave_sum(sum) * __builtin_amdgcn_exp2f(fmaf(-wm, log2e, c));
                    apart = sum != sum;
                }
                if (apart) {
                    hold<E, N>(v);
                    sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int j = 0; j < Q; ++j) sum += __builtin_amdgcn_exp2f((fmaxf(v[i][j], ninf) - wm) * log2e);
                    sum = wave_sum(sum);
                }
                join_sum(m, s, wm, sum);
            }
            const int mine = from + (int)threadIdx.x;  // this thread's first quad
            // Quads that hold a key as large as the bound go to LDS.  First by the maxima
            // alone; where equal logits make those too many, by the tokens too, which leaves
            // at most K lanes of a wave.
            bool exact = false;
            uint64_t least;
            for (;;) {
                const uint64_t own = exact ? largest_key<E, N>(static_cast<const E*>(p.logits) + first, mine, end, off, p.V)
                                           : (uint64_t)(mine < end ? ordered(top) : 0u) << 32;
                const uint64_t bound = exact ? wave_bound<0>((uint32_t)(own >> 32), K, true, [&] { return (uint32_t)own; })
                                             : wave_bound<sizeof(E) == 2 ? 16 : 0>((uint32_t)(own >> 32), K, false, [] { return 0u; });
                if (lane == 0) sh.bound[w] = bound;
                __syncthreads();
                least = sh.best[K - 1] | 1;
                for (int i = 0; i < WAVES; ++i) least = sh.bound[i] > least ? sh.bound[i] : least;
                const uint32_t low = (uint32_t)(least >> 32);
                // a lane whose own largest key does not reach the bound holds none that does
                const bool in = exact ? own >= least : (uint32_t)(own >> 32) >= low && mine < end;
                if (in) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (mine + i * THREADS < end && ordered(most[i]) >= low) {
                            const unsigned at = atomicAdd(&sh.quads, 1u);
                            if (at < room) {
                                held[at] = uint4{v[i].w[0], v[i].w[1], v[i].w[2], v[i].w[3]};
                                number[at] = mine + i * THREADS;
                            }
                        }
                }
                __syncthreads();
                if (sh.quads <= room || exact) break;
                exact = true;
                __syncthreads();
                if (threadIdx.x == 0) sh.quads = 0;
                __syncthreads();
            }
            // their keys, GATHER at a time
            const unsigned elems = min(sh.quads, room) * Q;
            for (unsigned base = 0; base < elems; base += GATHER) {
                least = sh.best[K - 1] > least ? sh.best[K - 1] : least;
                for (unsigned at = base + threadIdx.x; at < min(elems, base + GATHER); at += THREADS) {
                    const unsigned q = at / Q, j = at % Q;
                    const float x = sizeof(E) == 4 ? reinterpret_cast<const float*>(held)[at]
                                                   : __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(held)[at] << 16);
                    const int t = number[q] * Q + (int)j - off;
                    const uint64_t key = key_of(x, (uint32_t)t);
                    if (t >= 0 && t < p.V && key >= least) gather(key, &sh);
                }
                rank_keys(K, &sh);
            }
        }
    }
    if (lane == 0) sh.m[w] = m, sh.s[w] = s;
    __syncthreads();
    // Written past the caches of this XCD, and counted once they are there.
    if (threadIdx.x < (unsigned)K)
        __hip_atomic_store(p.best + ((long)row * p.slices + slice) * K + threadIdx.x, sh.best[threadIdx.x],
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (threadIdx.x == 64) {
        for (int i = 0; i < WAVES; ++i)
            if (i != w) join_sum(m, s, sh.m[i], sh.s[i]);
        __hip_atomic_store(p.sums + (long)row * p.slices + slice, (uint64_t)__float_as_uint(m) << 32 | __float_as_uint(s),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned* count = p.arrived + (long)b * ARRIVED_WORDS;
        const unsigned all = (unsigned)(K * p.slices);
        sh.last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == all - 1;
        if (sh.last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next launch
    }
    __syncthreads();
    if (sh.last) join_slices(p, st, b, &sh);
}

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
    if (K > LSTM_DYN_BEAM_MAX_K || (long long)B * K >= 1 << 22 || V >= 1 << 27) return LSTM_DYN_ERR_UNSUPPORTED;
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
    int hold, slices;  // sixteen-byte loads a thread holds; slices of a beam
    unsigned room;     // quads a workgroup puts aside at most
    uint64_t *best, *sums;
    unsigned* arrived;
};

// How a beam's logits are cut: eight loads a thread (64 x 16 beams over 65536
// tokens 53 us; four 71, two 85, sixteen 54), fewer where that would leave
// fewer workgroups than CUs (8 x 10 beams over 30000 tokens in fp32: 20.8 us so,
// 26 for four a CU); and no more slices than can be joined in a few rounds (a
// workgroup takes its slice in pieces then).
static void beam_shape(lstm_dyn_beam* h) {
    const int quad = 16 / dtype_bytes(h->dtype);
    const long quads = ((long)h->V + quad - 1) / quad + (h->V % quad ? 1 : 0), rows = (long)h->B * h->K;
    auto slices = [&](int n) { return (quads + THREADS * n - 1) / (THREADS * n); };
    int n = 8;
    while (n > 1 && rows * slices(n) < h->num_cus) n /= 2;
    long most = 2048 / (h->K * h->K);
    if (most < 8) most = 8;
    h->hold = n;
    h->slices = (int)(slices(n) < most ? slices(n) : most);
    h->room = (unsigned)(WAVES * h->K * n);  // all quads of K lanes of each wave
}

template <class E>
static void beam_launch(const lstm_dyn_beam* h, const BeamParams& p, const States& st) {
    auto* k = h->hold == 8   ? beam_kernel<E, 8>
              : h->hold == 4 ? beam_kernel<E, 4>
              : h->hold == 2 ? beam_kernel<E, 2>
                             : beam_kernel<E, 1>;
    hipLaunchKernelGGL(k, dim3((unsigned)(h->B * h->K) * (unsigned)h->slices), dim3(THREADS), 20 * h->room,
                       h->last_stream, p, st, h->room);
}

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
    if ((rc = ops_device(h)) != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    beam_shape(h);
    const long long na = 4LL * ARRIVED_WORDS * B, ns = 8LL * B * K * h->slices;
    if ((rc = ops_init(h, 256 + na + ns + ns * K)) != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    h->arrived = reinterpret_cast<unsigned*>(h->block + 256);
    h->sums = reinterpret_cast<uint64_t*>(h->block + 256 + na);
    h->best = h->sums + (long)B * K * h->slices;
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
                       h->best, h->sums, h->arrived, h->B, h->K, h->V, end, h->slices};
    States s{};
    long long bytes = 0;
    for (int i = 0; i < n_states; ++i) {
        s.src[i] = static_cast<const char*>(states[i].src);
        s.dst[i] = static_cast<char*>(states[i].dst);
        s.bytes[i] = states[i].row_bytes;
        bytes += states[i].row_bytes;
        const uintptr_t a = reinterpret_cast<uintptr_t>(s.src[i]) | reinterpret_cast<uintptr_t>(s.dst[i]) |
                            (uintptr_t)s.bytes[i];
        s.unit[i] = a % 16 == 0 ? 16 : a % 4 == 0 ? 4 : 1;
    }
    // up to this much of a sequence's states its last workgroup copies itself
    const bool own = bytes * h->K <= FUSED_STATE_BYTES;
    if (own) s.n = n_states;
    if (h->dtype == LSTM_DYN_BF16) beam_launch<__bf16>(h, p, s);
    else beam_launch<float>(h, p, s);
    if ((rc = ops_launched(h)) != LSTM_DYN_OK || own) return rc;
    hipLaunchKernelGGL(beam_reorder_kernel, dim3((unsigned)(h->B * h->K), (unsigned)n_states), dim3(THREADS), 0,
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
