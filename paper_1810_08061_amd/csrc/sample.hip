// sample.hip -- one token a row from its logits and a given random number:
// temperature, top-k, top-p, min-p, and the inverse of the running sum.
//
// A token's weight is exp((x - largest) / T) in fixed point, so sums of weights are
// integers: the order in which they are formed changes nothing, and no sort is needed.
// The kept tokens are a start of the tokens in order (largest first, equal ones by index),
// that is all whose 64-bit key, the logit's bits in an order-preserving form above the
// complement of the index, reaches a cut.  The cut for a count (top-k) or a sum of weights (top-p) is
// found by a histogram over 2048 ranges of the exponent, which leaves one range with the cut
// in it; its few tokens are listed, cut once more by key if they are many, and ranked by counting.  Where
// they are more than LIST (many equal logits), the row is cut again by key until they are not.  Then the kept weights of each
// segment of the row are summed, and one wave walks the segment that u falls into.
// Where the first histogram shows that FEW tokens at most can be taken (a small k, or weights
// that few tokens have), they are gathered once, and every cut and the running sum are formed by
// comparing each with each, without more passes.
//
// A workgroup holds a row: its passes, three to six, come from the L2 after the first.  While a long row is
// worked at, the vector units of its CU are busy for three quarters of the time (256 rows of 65536: 48 vector instructions a
// token, 20 us of an average row's 28; the waves wait for reads, LDS and joins for 56% of theirs, side by side), so where most tokens
// do not count a pass looks at them with as few instructions as
// decide that (two comparisons), and forms keys and weights of the rest
// alone; where most of them count it does the same for all, under no condition.  The call ends with its slowest row.
//
// Measured, bf16: 256 rows of 65536 with top-p and min-p 43 to 46 us (21 without filters, where the row is
// read and every weight formed once); 16 rows of 32768 with top-k to 1000 and top-p 27 to 31 us, each row on one CU:
// passes of about 3 us with the joins between them.  One row in fp32, T 0.8, with all filters at once (k 50, p 0.9, min-p 0.02) and with
// p 0.9 alone: of 1000 7.0 and 7.5 us, of 32768 12.5 and 24, of 131072 26 and 74.  With k 50 and p 0.9, few tokens: 16 rows of 32768
// 12.9 us (23.9 with the passes), 256 of 65536 19 (38), in fp32 one of 131072 27 (66).  FEW: comparing 256 with each
// other took 6 us and more, as much as it saves.  Tried: the far ranges of the histogram summed in
// registers instead (a branch an element: 74 us where one addition in LDS an element takes 62).
#include "ops.h"
#include "../../include/lstm_dyn_layer.h"

#include <cfloat>
#include <cmath>

namespace ldyn {
namespace {

typedef unsigned long long u64;

constexpr int BINS = 2048, LIST = 512, SEGMENTS = 1024, FEW = 128;
static_assert(BINS == 1 << 11, "a key's range is found by a shift");
constexpr int BITS = 46;         // of the largest weight
constexpr float REACH = 48.0f;   // powers of two that the histogram spans: below 2^-46 there is no weight
static_assert(BITS * (BINS / REACH) <= BINS - 64, "a range each for lanes whose tokens have no weight");

struct SampleParams {
    const void* logits;
    const float* u;
    lstm_dyn_sample_filter_t filter;
    int32_t* token;
    float* logp;
    int V, bits;       // weights are multiples of 2^-bits
};

struct RowLds {
    u64 hist[BINS];
    u64 key[LIST], weight[LIST];
    u64 segment[SEGMENTS];
    u64 part[16];
    float fpart[16];
    u64 found, rest;
    int range, count, first;
};

// A larger logit, then a lower index, is a larger key.  x is no NaN; -0 is 0.
__device__ inline u64 key_of(float x, int i) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (u64)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~i;
}
__device__ inline float logit_of(u64 key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}

// exp((x - largest) / T): 1 / (T ln 2) is held in two parts, so its rounding does not
// tilt the weights of tokens far from the largest.
// A token's weight is formed once for a sum and again where the token in which that sum's target lies is looked for. A
// target that no token reached would leave a cut or the row's token unwritten, so every compiled copy of these functions has to give
// the same bits: each rounding is written out, and no product is joined with a sum at the compiler's choice.
struct Weigh {
    float largest, hi, lo, unit, none, per_range;
    // How far below the largest x is, in ranges of the histogram.  From `none` on there is no weight.  (-inf at an
    // infinite T: the last range.)
    __device__ float depth(float x) const {
#pragma clang fp contract(off)
        return fminf((x - largest) * per_range, (float)(BINS - 1));
    }
    __device__ float power(float x) const {
#pragma clang fp contract(off)
        const float d = x - largest, t = d * hi, e = __builtin_amdgcn_exp2f(t);
        return __builtin_fmaf(e, __builtin_fmaf(d, lo, __builtin_fmaf(d, hi, -t)) * 0.69314718f, e);
    }
    // p in multiples of 1 / (2^32 unit), rounded down.
    __device__ u64 weight(float p) const {
#pragma clang fp contract(off)
        const float x = p * unit;
        const uint32_t high = (uint32_t)x;
        return (u64)high << 32 | (uint32_t)((x - (float)high) * 0x1p32f);
    }
};

// The tokens of the order's start: all of some weight whose keys are `key` or more.
struct Start {
    u64 key = 0;
    float logit = -__builtin_inff();   // of `key`: a smaller one is out
    bool done = false;                 // the row has its token
    __device__ bool has(float x, int i) const { return x > logit || (x == logit && key_of(x, i) >= key); }
};

// A row in pieces of 16 bytes, the first and the last perhaps in part.
template <class E>
struct Row {
    static constexpr int N = 16 / (int)sizeof(E);
    const E* p;
    int V, off, pieces;

    __device__ Row(const E* row, int V_) : p(row), V(V_) {
        off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(E));
        pieces = (V + off + N - 1) / N;
    }
    __device__ typename Vec<E, N>::type piece(int k) const {
        const int i0 = k * N - off;
        typename Vec<E, N>::type x;
        if (i0 >= 0 && i0 + N <= V) {
            x = *reinterpret_cast<const typename Vec<E, N>::type*>(p + i0);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = i0 + j >= 0 && i0 + j < V ? p[i0 + j] : (E)-__builtin_inff();
        }
        return x;
    }
    // f(x, index) of every element of pieces begin, begin + step, ... below end, in no order that counts (x may be NaN:
    // every f leaves it out by a comparison). Whole pieces
    // are read without a condition, so the next two are on their way while one is worked at; the row's first and last
    // piece come by themselves where they are in part.
    template <class F>
    __device__ void each(int begin, int end, int step, F f) const {
        using P = typename Vec<E, N>::type;
        const int low = off ? 1 : 0, high = (V + off) / N;  // the whole pieces
        const int stop = min(end, high);
        int k = begin;
        const auto work = [&](const P& x, int k) {
#pragma unroll
            for (int j = 0; j < N; ++j) f((float)x[j], k * N - off + j);
        };
        bool part = k < low && k < end;
        if (k < low) k += step;
        if (k < stop) {
            const P* from = reinterpret_cast<const P*>(p - off);
            P next = from[k], after = from[min(k + step, stop - 1)];
#pragma unroll 1
            for (; k < stop; k += step) {
                const P x = next;
                next = after;
                after = from[min(k + 2 * step, stop - 1)];
                work(x, k);
            }
        }
        // The last piece, if it is in part and this thread's, and the first.
        const int last = pieces - 1;
        const bool tail = last >= high && last >= low && last >= begin && last < end && (last - begin) % step == 0;
#pragma unroll 1
        for (int e = part ? 0 : 1; e < (tail ? 2 : 1); ++e) {
            const int at = e ? last : 0;
            work(piece(at), at);
        }
    }
};

// v of the lane that a row_shr or row_bcast names, zero where there is none.
template <int CTRL, int ROWS>
__device__ inline u64 moved(u64 v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
    return (u64)hi << 32 | lo;
}
// The sum over the lanes up to this one.
__device__ inline u64 wave_scan(u64 v) {
    v += moved<0x111, 0xf>(v);   // row_shr 1, 2, 4, 8: within 16 lanes
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);   // row_bcast 15 into rows 1 and 3, then 31 into rows 2 and 3
    v += moved<0x143, 0xc>(v);
    return v;
}
__device__ inline u64 last_lane(u64 v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), 63);
    return (u64)hi << 32 | lo;
}
__device__ inline u64 wave_sum(u64 v) { return last_lane(wave_scan(v)); }

// The first of n sums (a power of two, at least the workgroup's threads) at which their running sum reaches
// aim(the sum of all): writes its index and what is left of the target before it.  Returns the sum of all.
template <int THREADS, class A, class G>
__device__ inline u64 crossing(RowLds& s, int n, A aim, G value) {
    const int w = threadIdx.x >> 6, per = n / THREADS;
    u64 mine = 0;
    for (int i = 0; i < per; ++i) mine += value((int)threadIdx.x * per + i);
    const u64 up = wave_scan(mine);
    if ((threadIdx.x & 63) == 63) s.part[w] = up;
    __syncthreads();
    u64 before = up - mine, all = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
        const u64 p = s.part[i];
        before += i < w ? p : 0;
        all += p;
    }
    const u64 target = aim(all);
    if (before < target && before + mine >= target) {
        for (int i = 0; i < per; ++i) {
            const u64 v = value((int)threadIdx.x * per + i);
            if (before + v >= target) {
                s.range = (int)threadIdx.x * per + i;
                s.rest = target - before;
                break;
            }
            before += v;
        }
    }
    __syncthreads();
    return all;
}

// A logit that no token less deep than `upto` is below: 2^-20 of both terms further, where roundings are 2^-23.
__device__ inline float below(const Weigh& weigh, float upto) {
    const float far = upto / weigh.per_range;   // (-inf where no range has an end)
    return weigh.largest + far - 0x1p-20f * (fabsf(far) + fabsf(weigh.largest));
}

// What is left of the row where few tokens can be taken: those less deep than `upto`, the start of the order.  Of them the
// first k, of those the first whose weights reach goal(the sum of theirs), of those the ones that keep(x) leaves.  Each
// token's place and the sums before it are formed by comparing it with every other one: no more passes over the row.
// False, and nothing done, if they are more than FEW.
template <int THREADS, class E, class G, class K, class A, class F>
__device__ inline bool among_few(RowLds& s, const Row<E>& row, const Weigh& weigh, float upto, u64 k, G goal, K keep, A aim, F found) {
    const int tid = threadIdx.x;
    if (tid == 0) s.count = 0;
    for (int i = tid; i < 3 * FEW; i += THREADS) s.segment[i] = 0;
    __syncthreads();
    const float low = below(weigh, upto);
    row.each(tid, row.pieces, THREADS, [&](float x, int i) {
        if (x < low || !(weigh.depth(x) < upto)) return;
        const int to = atomicAdd(&s.count, 1);
        if (to < FEW) {
            s.key[to] = key_of(x, i);
            s.weight[to] = weigh.weight(weigh.power(x));
        }
    });
    __syncthreads();
    const int n = s.count;
    if (n > FEW) {
        __syncthreads();   // all have read s.count
        return false;
    }
    // several waves compare the same tokens, each with some of the others
    const int wide = n > 64 ? 128 : 64, token = tid & (wide - 1), part = tid / wide, parts = THREADS / wide;
    u64 *sums = s.segment, *places = sums + FEW, *sums_by_index = places + FEW;
    {
        const u64 key = s.key[token];
        u64 before = 0, place = 0;
#pragma unroll 4
        for (int e = part; e < n; e += parts) {
            const bool first = s.key[e] > key;
            before += first ? s.weight[e] : 0ull;
            place += first;
        }
        atomicAdd(sums + token, before);
        atomicAdd(places + token, place);
    }
    __syncthreads();
    // (a wave's tokens are a lane each: two waves)
    u64 key = 0, kept = 0, before = 0;
    if (tid < n) {
        key = s.key[tid];
        before = sums[tid];
        kept = places[tid] < k ? s.weight[tid] : 0;
    }
    u64 all = wave_sum(kept);
    if (tid < FEW && (tid & 63) == 0) s.part[tid >> 6] = all;
    __syncthreads();
    if (!(before < goal(s.part[0] + s.part[1])) || !keep(logit_of(key))) kept = 0;
    if (tid < n) s.weight[tid] = kept;
    all = wave_sum(kept);
    if (tid < FEW && (tid & 63) == 0) s.part[2 + (tid >> 6)] = all;
    __syncthreads();
    {
        const uint32_t index = ~(uint32_t)s.key[token];
        u64 before = 0;
#pragma unroll 4
        for (int e = part; e < n; e += parts) before += ~(uint32_t)s.key[e] < index ? s.weight[e] : 0ull;
        atomicAdd(sums_by_index + token, before);
    }
    __syncthreads();
    if (!kept) return true;
    before = sums_by_index[tid];
    all = s.part[2] + s.part[3];
    const u64 target = aim(all);
    if (before < target && before + kept >= target) found(logit_of(key), (int)~(uint32_t)key, all);
    return true;
}

// The shortest start, within `within` (ALL: it is all tokens), whose measure (the tokens' number, or with MASS
// their weight) reaches the target.  aim(all): the target, given the sum of all measures; if it is no less than
// all there is, `within` itself.  few(upto, measure, all): told that tokens of this measure are less deep than upto, among them the
// start's, may end the row.
template <int THREADS, bool MASS, bool ALL, class E, class A, class W>
__device__ inline Start find_start(RowLds& s, const Row<E>& row, const Weigh& weigh, const Start within, A aim, W few) {
    const int tid = threadIdx.x;
    auto clear = [&] {
        for (int i = tid; i < BINS; i += THREADS) s.hist[i] = 0;
        __syncthreads();
    };
    // the least a and the largest b of all threads
    auto ends = [&](u64& a, u64& b, u64* room) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const u64 a2 = __shfl_xor(a, o), b2 = __shfl_xor(b, o);
            a = a2 < a ? a2 : a;
            b = b2 > b ? b2 : b;
        }
        if ((tid & 63) == 0) {
            s.part[tid >> 6] = a;
            room[tid >> 6] = b;
        }
        __syncthreads();
#pragma unroll 2   // (all at once they would take 64 registers)
        for (int i = 0; i < THREADS / 64; ++i) {
            a = s.part[i] < a ? s.part[i] : a;
            b = room[i] > b ? room[i] : b;
        }
    };
    auto measure = [&](float x) { return MASS ? weigh.weight(weigh.power(x)) : 1ull; };
    clear();
    row.each(tid, row.pieces, THREADS, [&](float x, int i) {
        const float q = weigh.depth(x);
        const bool on = q < weigh.none;
        if constexpr (ALL) {
            // tokens of no weight add nothing, each lane's in a range of its own behind the others: in one range they
            // would wait for each other (16 rows of 32768 of which most have none, top-p 0.9: 29 us and 19)
            // (the weight of -inf at an infinite T is that of no number: not taken)
            const u64 m = measure(x);
            const int range = on ? (int)q : BINS - 64 + (tid & 63);
            if constexpr (MASS) atomicAdd(&s.hist[range], on ? m : 0ull);
            else atomicAdd(reinterpret_cast<uint32_t*>(&s.hist[range]), on ? 1u : 0u);
        } else {
            if (on && x >= within.logit && within.has(x, i)) atomicAdd(&s.hist[(int)q], measure(x));
        }
    });
    __syncthreads();
    u64 target = 0;
    const u64 all = crossing<THREADS>(s, BINS, [&](u64 sum) { return target = aim(sum); }, [&](int i) { return s.hist[i]; });
    Start done;
    done.done = true;
    if (target >= all) return few(weigh.none, all, all) ? done : within;
    const float from = (float)s.range, upto = fminf(from + 1.0f, weigh.none);
    u64 rest = s.rest, lo = 0, hi = ~0ull;
    if (few(upto, target - rest + s.hist[s.range], all)) return done;
    // f(x, key) of the range's tokens: bounds that hold more than the range (by 2^-20, roundings are 2^-23; all, where no
    // range has an end) leave most tokens out by two comparisons
    const float near = from / weigh.per_range;
    const float low = below(weigh, upto);
    const float high = weigh.largest + near + 0x1p-20f * (fabsf(near) + fabsf(weigh.largest));
    auto each = [&](auto f) {
        row.each(tid, row.pieces, THREADS, [&](float x, int i) {
            if (x < low || x > high) return;
            const float q = weigh.depth(x);
            if (q >= from && q < upto && (ALL || within.has(x, i))) f(x, key_of(x, i));
        });
    };
    for (bool by_key = false;; by_key = true) {
        // the tokens of the range, if they are few
        if (tid == 0) s.count = 0;
        __syncthreads();
        each([&](float x, u64 key) {
            if (key < lo || key > hi) return;
            const int to = atomicAdd(&s.count, 1);
            if (to < LIST) {
                s.key[to] = key;
                s.weight[to] = measure(x);
            }
        });
        __syncthreads();
        const int n = s.count;
        if (n <= LIST) {
            // the token of the first `number` in which the target is, by comparing each with each
            auto rank = [&](const u64* keys, const u64* weights, int number) {
                for (int e = tid; e < number; e += THREADS) {
                    const u64 key = keys[e];
                    u64 before = 0;
#pragma unroll 4
                    for (int f = 0; f < number; ++f) before += keys[f] > key ? weights[f] : 0ull;
                    if (before < rest && before + weights[e] >= rest) s.found = key;
                }
            };
            if (n <= 64) {
                rank(s.key, s.weight, n);
            } else {
                // cut by key among themselves: comparing each with each would take up to 6 us, this takes 2
                u64 a = ~0ull, b = 0;
                for (int e = tid; e < n; e += THREADS) {
                    a = s.key[e] < a ? s.key[e] : a;
                    b = s.key[e] > b ? s.key[e] : b;
                }
                ends(a, b, s.segment);
                const int shift = max(53 - __builtin_clzll((b - a) | 1), 0);   // (of 2^11 ranges)
                if (tid == 0) s.count = 0;
                clear();
                for (int e = tid; e < n; e += THREADS) atomicAdd(&s.hist[(b - s.key[e]) >> shift], s.weight[e]);
                __syncthreads();
                crossing<THREADS>(s, BINS, [&](u64) { return rest; }, [&](int i) { return s.hist[i]; });
                rest = s.rest;
                for (int e = tid; e < n; e += THREADS) {
                    if ((int)((b - s.key[e]) >> shift) != s.range) continue;
                    const int to = atomicAdd(&s.count, 1);
                    s.segment[to] = s.key[e];
                    s.segment[LIST + to] = s.weight[e];
                }
                __syncthreads();
                rank(s.segment, s.segment + LIST, s.count);
            }
            __syncthreads();
            const u64 key = s.found;
            return Start{key, logit_of(key)};
        }
        // cut [lo, hi] again: at first by the keys that are in it
        if (!by_key) {
            u64 a = ~0ull, b = 0;
            each([&](float x, u64 key) {
                a = key < a ? key : a;
                b = key > b ? key : b;
            });
            ends(a, b, s.weight);
            lo = a;
            hi = b;
            __syncthreads();
        }
        const int shift = max(53 - __builtin_clzll((hi - lo) | 1), 0);
        clear();
        each([&](float x, u64 key) {
            if (key >= lo && key <= hi) atomicAdd(&s.hist[(hi - key) >> shift], measure(x));
        });
        __syncthreads();
        crossing<THREADS>(s, BINS, [&](u64) { return rest; }, [&](int i) { return s.hist[i]; });
        rest = s.rest;
        const u64 top = hi - ((u64)s.range << shift), width = (1ull << shift) - 1;
        lo = top - lo > width ? top - width : lo;
        hi = top;
    }
}

// weight(x, index) of all tokens is summed by index; found(x, index, all) is called by one thread, for the first token at which
// the running sum reaches aim(all).
template <int THREADS, class E, class W, class A, class F>
__device__ inline void walk(RowLds& s, const Row<E>& row, W weight, A aim, F found) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // segments of 64 `rounds` pieces, each the work of one wave
    const int rounds = (row.pieces + 64 * SEGMENTS - 1) / (64 * SEGMENTS);
    __syncthreads();
    for (int i = tid; i < SEGMENTS; i += THREADS) s.segment[i] = 0;
    __syncthreads();
    const int segments = (row.pieces + 64 * rounds - 1) / (64 * rounds);
    for (int g = wave; g < segments; g += THREADS / 64) {
        u64 sum = 0;
        const int k0 = g * 64 * rounds;
        row.each(k0 + lane, min(row.pieces, k0 + 64 * rounds), 64, [&](float x, int i) { sum += weight(x, i); });
        sum = wave_sum(sum);
        if (lane == 0) s.segment[g] = sum;
    }
    __syncthreads();
    const u64 all = crossing<THREADS>(s, SEGMENTS, aim, [&](int i) { return s.segment[i]; });
    if (wave != 0) return;
    u64 rest = s.rest;
    const int k0 = s.range * 64 * rounds;
    for (int r = 0; r < rounds; ++r) {
        const int k = k0 + r * 64 + lane;
        constexpr int M = Row<E>::N;
        float x[M];
        u64 w[M], sum = 0;
        if (k < row.pieces) {
            const auto raw = row.piece(k);
#pragma unroll
            for (int j = 0; j < M; ++j) x[j] = (float)raw[j];
        }
#pragma unroll
        for (int j = 0; j < M; ++j) {
            w[j] = k < row.pieces ? weight(x[j], k * M - row.off + j) : 0;
            sum += w[j];
        }
        const u64 up = wave_scan(sum);
        if (up >= rest && up - sum < rest) {
            u64 before = up - sum;
#pragma unroll
            for (int j = 0; j < M; ++j) {
                if (before < rest && before + w[j] >= rest) found(x[j], k * M - row.off + j, all);
                before += w[j];
            }
        }
        const u64 whole = last_lane(up);
        if (whole >= rest) break;
        rest -= whole;
    }
}

// The first running sum above u of all.
__device__ inline u64 above(float u, u64 all) {
    u = fminf(fmaxf(u, 0.0f), 1.0f);   // (a NaN is 0)
    const u64 t = (u64)((double)u * (double)all) + 1;
    return t < all ? t : all;
}
__device__ inline u64 top_p_of(float top_p, u64 all) {
    const u64 t = (u64)ceil((double)top_p * (double)all);
    return t ? t : 1ull;
}

template <class E, int THREADS>
__global__ void __launch_bounds__(THREADS) sample_kernel(SampleParams a) {
    __shared__ RowLds s;
    const int n = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Row<E> row(static_cast<const E*>(a.logits) + (size_t)n * a.V, a.V);

    float mx = -__builtin_inff();
    row.each(tid, row.pieces, THREADS, [&](float x, int) { mx = fmaxf(mx, x); });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    if (lane == 0) s.fpart[wave] = mx;
    if (tid == 0) s.first = a.V;
    __syncthreads();
    for (int i = 0; i < THREADS / 64; ++i) mx = fmaxf(mx, s.fpart[i]);
    if (mx == -__builtin_inff()) {
        if (tid == 0) {
            a.token[n] = -1;
            a.logp[n] = mx;
        }
        return;
    }

    const lstm_dyn_sample_filter_t& f = a.filter;
    const float T = f.temperatures ? f.temperatures[n] : f.temperature;
    float top_p = f.top_ps ? f.top_ps[n] : f.top_p;
    const float min_p = fminf(f.min_ps ? f.min_ps[n] : f.min_p, 1.0f);
    int top_k = f.top_ks ? f.top_ks[n] : f.top_k;
    if (top_k <= 0 || top_k >= a.V) top_k = 0;
    const double per = 1.0 / (double)T * 1.4426950408889634;
    const bool least_p = f.min_ps ? f.min_ps[n] > 0.0f : f.min_p > 0.0f;   // a NaN is no filter
    if (!(T > 0.0f) || !((float)per < __builtin_inff()) || top_k == 1 || top_p <= 0.0f) {
        // the first token of the order
        int first = a.V;
        row.each(tid, row.pieces, THREADS, [&](float x, int i) { first = x == mx && i < first ? i : first; });
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o));
        if (lane == 0) atomicMin(&s.first, first);
        __syncthreads();
        if (tid == 0) {
            a.token[n] = s.first;
            a.logp[n] = 0.0f;
        }
        return;
    }

    const float u = a.u[n];
    if (mx == __builtin_inff()) {
        // such tokens are alike: their number is cut, not their sum
        walk<THREADS>(
            s, row, [&](float x, int) { return x == mx ? 1ull : 0ull; },
            [&](u64 all) {
                u64 kept = top_k && (u64)top_k < all ? (u64)top_k : all;
                if (top_p < 1.0f) kept = top_p_of(top_p, kept);
                if (tid == 0) s.found = kept;
                return above(u, kept);
            },
            [&](float, int i, u64) {
                a.token[n] = i;
                a.logp[n] = (float)-log((double)s.found);
            });
        return;
    }

    Weigh weigh;
    weigh.largest = mx;
    weigh.hi = (float)per;
    weigh.lo = (float)(per - (double)weigh.hi);
    weigh.unit = __uint_as_float((uint32_t)(a.bits - 32 + 127) << 23);
    weigh.per_range = fmaxf(weigh.hi * (-BINS / REACH), -FLT_MAX);   // (finite: the largest is at depth zero at any T)
    weigh.none = (float)a.bits * (BINS / REACH);
    auto token = [&](float x, int i, u64 all) {
        a.token[n] = i;
        a.logp[n] = (float)(((double)x - (double)mx) / (double)T - log((double)all * exp2(-(double)a.bits)));
    };
    auto aim = [&](u64 all) { return above(u, all); };
    auto goal = [&](u64 all) { return top_p < 1.0f ? top_p_of(top_p, all) : ~0ull; };
    auto keep = [&](float x) { return !(least_p && weigh.power(x) < min_p); };
    // depths from which on tokens are smaller than min_p
    const float min_p_depth = least_p ? fminf((1e-3f - __builtin_amdgcn_logf(min_p)) * (BINS / REACH), weigh.none) : weigh.none;
    auto none = [](float, u64, u64) { return false; };
    Start start;
    if (top_k) {
        start = find_start<THREADS, false, true>(s, row, weigh, start, [&](u64) { return (u64)top_k; }, [&](float upto, u64 tokens, u64) {
            return tokens <= FEW && among_few<THREADS>(s, row, weigh, upto, (u64)top_k, goal, keep, aim, token);
        });
        if (start.done) return;
        if (top_p < 1.0f)
            start = find_start<THREADS, true, false>(s, row, weigh, start, [&](u64 all) { return top_p_of(top_p, all); }, none);
    } else if (top_p < 1.0f) {
        start = find_start<THREADS, true, true>(s, row, weigh, start, [&](u64 all) { return top_p_of(top_p, all); },
                                                [&](float upto, u64 weights, u64 all) {
            // each of them has this weight at least (the last of them a rounding less)
            upto = fminf(upto, min_p_depth);
            const float least = __builtin_amdgcn_exp2f((float)a.bits - upto * (REACH / BINS));
            return (float)weights <= 0.98f * FEW * least &&
                   among_few<THREADS>(s, row, weigh, upto, ~0ull, [&](u64) { return top_p_of(top_p, all); }, keep, aim, token);
        });
        if (start.done) return;
    }
    // the least logit that may be left: for most tokens the only test
    const float least = fmaxf(fmaxf(below(weigh, min_p_depth), -FLT_MAX), start.logit);
    if (!top_k && !(top_p < 1.0f) && !least_p) {
        walk<THREADS>(
            s, row,
            [&](float x, int) {
                const u64 w = weigh.weight(weigh.power(x));
                return x >= least ? w : 0;
            },
            aim, token);
        return;
    }
    walk<THREADS>(
        s, row,
        [&](float x, int i) -> u64 {
            if (!(x >= least && start.has(x, i))) return 0;
            const float p = weigh.power(x);
            return least_p && p < min_p ? 0 : weigh.weight(p);
        },
        aim, token);
}

int check_sizes(int N, int V, int dtype) {
    if (N < 1 || V < 1 || !valid_dtype(dtype)) return LSTM_DYN_ERR_INVALID;
    return V >= 1 << 27 || N >= 1 << 22 ? LSTM_DYN_ERR_UNSUPPORTED : LSTM_DYN_OK;
}

int check_buffers(int N, int V, int dtype, const void* logits, const float* u, const lstm_dyn_sample_filter_t* f,
                  const int32_t* token, const float* logp) {
    Span s[8];
    int k = 0;
    const long long n = 4LL * N;
    s[k++] = Span{logits, (long long)N * V * dtype_bytes(dtype), dtype_bytes(dtype), false};
    s[k++] = Span{u, n, 4, false};
    s[k++] = Span{token, n, 4, true};
    s[k++] = Span{logp, n, 4, true};
    if (f)
        for (const void* p : {(const void*)f->temperatures, (const void*)f->top_ps, (const void*)f->min_ps,
                              (const void*)f->top_ks})
            if (p) s[k++] = Span{p, n, 4, false};
    return check_spans(s, k);
}

}  // namespace
}  // namespace ldyn

using namespace ldyn;

struct lstm_dyn_sample : OpsHandle {
    int N = 0, V = 0, dtype = 0, bits = 0;
};

extern "C" int lstm_dyn_check_sample_args(int N, int V, int dtype, const void* logits, const float* u,
                                          const lstm_dyn_sample_filter_t* filter, const int32_t* out_token,
                                          const float* out_logp) {
    const int rc = check_sizes(N, V, dtype);
    return rc != LSTM_DYN_OK ? rc : check_buffers(N, V, dtype, logits, u, filter, out_token, out_logp);
}

extern "C" int lstm_dyn_sample_create(lstm_dyn_sample_t** out, int N, int V, int dtype) {
    if (!out) return LSTM_DYN_ERR_INVALID;
    *out = nullptr;
    int rc = check_sizes(N, V, dtype);
    if (rc != LSTM_DYN_OK) return rc;
    auto* h = new (std::nothrow) lstm_dyn_sample();
    if (!h) return LSTM_DYN_ERR_NOMEM;
    h->N = N;
    h->V = V;
    h->dtype = dtype;
    h->bits = BITS;
    while ((long long)V > 1LL << (62 - h->bits)) --h->bits;
    if ((rc = ops_device(h)) == LSTM_DYN_OK) rc = ops_init(h, 256);
    if (rc != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    *out = h;
    return LSTM_DYN_OK;
}

extern "C" int lstm_dyn_sample_step(lstm_dyn_sample_t* h, const void* logits, const float* u,
                                    const lstm_dyn_sample_filter_t* filter, int32_t* out_token, float* out_logp,
                                    void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc = check_buffers(h->N, h->V, h->dtype, logits, u, filter, out_token, out_logp);
    if (rc != LSTM_DYN_OK || (rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const lstm_dyn_sample_filter_t none{1.0f, 1.0f, 0.0f, 0, nullptr, nullptr, nullptr, nullptr};
    const SampleParams p{logits, u, filter ? *filter : none, out_token, out_logp, h->V, h->bits};
    // A workgroup is a row.  Where a CU has one, 512 threads hold a short row's waits at joins down and 1024 take a long one's
    // work (us, k 200 and p 0.9, bf16: 64 rows of 4000 14.1 and 16.0 with 1024, 16 of 32768 26.4 and 30.2 with 512).  Where
    // a CU has two, 512 let both be there; where it has more, 256 let four be, which fill each other's waits
    // (1024 of 2000: 19.4, with 512 27.7, with 1024 52.3; 1500 of 8000: 51.8, 54.0, 87.2), but for rows so long that few such
    // workgroups end last (1100 of 32768 in fp32, p 0.9: 147 and 130 with 512).
    const int threads = h->N > 2 * h->num_cus && h->V <= 16384 ? 256 : h->N <= h->num_cus && h->V > 8192 ? 1024 : 512;
    auto launch = [&](auto of_bf16, auto of_f32) {
        hipLaunchKernelGGL(h->dtype == LSTM_DYN_BF16 ? of_bf16 : of_f32, dim3((unsigned)h->N), dim3(threads), 0, h->last_stream, p);
    };
    if (threads == 256) launch(sample_kernel<__bf16, 256>, sample_kernel<float, 256>);
    else if (threads == 512) launch(sample_kernel<__bf16, 512>, sample_kernel<float, 512>);
    else launch(sample_kernel<__bf16, 1024>, sample_kernel<float, 1024>);
    return ops_launched(h);
}

extern "C" int lstm_dyn_sample_query(lstm_dyn_sample_t* h, int what, long long* value) {
    return ops_query(h, what, value);
}

extern "C" int lstm_dyn_sample_destroy(lstm_dyn_sample_t* h) {
    if (!h) return LSTM_DYN_OK;
    const int rc = ops_free(h);
    delete h;
    return rc;
}
