// scan.hip -- the gated linear recurrence over whole sequences and its
// backward pass.
//
//   a_t = sigmoid(zf_t), k_t = 1 - a_t = sigmoid(-zf_t), s_t = sigmoid(zo_t)
//   h_t = a_t h_{t-1} + k_t v_t,   y_t = s_t h_t
// and back, with e_t the gradient of h_t from later steps (e_{L-1} = d_out_h):
//   g_t = s_t dy_t + e_t,   e_{t-1} = a_t g_t
//   dzf = g_t (h_{t-1} - v_t) a_t k_t,   dzv = g_t k_t,   dzo = dy_t h_t s_t (1 - s_t)
//
// a and k are both formed to their own relative error (the smaller from exp(-|zf|), the
// larger as one minus it), so a small k keeps its share over a long memory, and a
// small a leaves nothing of a large state in the candidate that replaces it.  The sum of
// the two products is finite where its operands are, and infinite where one of them
// is; a correction h + k (v - h) is neither.  All of it is fp32; y and dz are
// rounded once, to the data's type.
//
// Bound by memory: forward (3 + 1) and backward (4 + 3) elements of the data a step and
// channel, each read or written once.  A step is an affine map of the state, so the time
// axis is cut: a thread holds a run of R steps of two channels in registers (16 in bf16,
// 8 in fp32) and forms its map (A, S); the runs of a workgroup are joined by
// shuffles and through LDS (join_runs), the workgroups' shares of a row by one
// word a channel in memory (carry_on); then every thread goes through its run again
// from the state it starts from.  32 lanes along the channels (128 or 256 bytes of a row)
// and 16 runs along the time make the share long (256 steps), which keeps the chain
// of shares short.  For the backward the forward keeps the state every run
// starts from, 1/16 of the states (32 x 4096 x 2048 in bf16: 67 MB), and the runs'
// states are formed again.
//
// Measured: 32 x 4096 x 2048 in bf16, ragged, forward 0.34 ms (4.0 TB/s of what it has to
// move), backward 0.60 ms (4.5 TB/s); a 2 GiB copy reaches 4.9.  One row of
// 32768 x 2048: 0.126 ms (4.2 TB/s).  One thread a channel, step by step: 7.5 ms and 17.8.
#include "ops.h"

#include <type_traits>

namespace ldyn {
namespace {

// How a row's shares hang together: it has one; each waits for the one before;
// or for the one NW before and the maps between.
enum Way { ONE, CHAIN, WINDOW };

// Steps one thread holds, and between two kept states.
template <class E>
constexpr int run_of() { return sizeof(E) == 2 ? 16 : 8; }

// The largest workgroups.  The backward holds 140 registers a thread with bf16
// data, so three waves a SIMD: workgroups of 256 (a training step of 32 x 4096 x 2048
// 946 us, of 512 962).
constexpr int FWD_THREADS = 512, BWD_THREADS = 256;

constexpr long long FAR_BYTES = 32LL << 20;  // of y or dz; see the launch

struct ScanParams {
    const void* z;
    const int32_t* lengths;
    const float* h0;
    float* out_h;
    void* y;
    float* kept;  // [B][ceil(T / R)][H] the state each run starts from, or null
    const void* dy;
    const float* d_out_h;
    void* dz;
    float* dh0;
    int32_t* status;
    int B, T, H;
    int tiles, segs;      // column tiles of a row; shares of its steps
    unsigned long long* counters;  // [B tiles] shares taken, over all launches
    uint64_t* carry;      // [1 or 3][B][segs][H] {value, launch}: what a share passes on; its map
    unsigned long long timeout_ticks;
};

// 1 / (1 + e^x), which is 1 and 0 at the infinities.
__device__ inline float logistic_neg(float x) { return rcp_f(1.0f + __expf(x)); }

// The smaller of a = sigmoid(x) and k = sigmoid(-x), with x's sign: one register holds both, each to its
// own relative error.  gate_keep gives a, gate_take k; their product is gate_slope.
__device__ inline float gate_code(float x) {
    const float e = __expf(-fabsf(x));
    return copysignf(e * rcp_f(1.0f + e), x);
}
__device__ inline bool gate_low(float q) { return __float_as_int(q) < 0; }  // also where a is -0
__device__ inline float gate_keep(float q) { return gate_low(q) ? -q : 1.0f - q; }
__device__ inline float gate_take(float q) { return gate_low(q) ? 1.0f + q : q; }
__device__ inline float gate_slope(float q) { return fabsf(q) * (1.0f - fabsf(q)); }

// The compiler may not form anything of x before here, nor keep what it formed of it (a bf16 pair widened
// early, or both gates of a code kept, take twice the registers).
__device__ inline void hold(float& x) { asm volatile("" : "+v"(x)); }

// V elements as they lie in memory, in 32-bit words.
template <class E, int V>
struct Raw {
    static constexpr int N = sizeof(E) * V <= 4 ? 1 : 2;
    uint32_t w[N];

    __device__ float operator[](int i) const {
        if constexpr (sizeof(E) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i ? w[0] & 0xffff0000u : w[0] << 16);
    }
    __device__ void hold() {
#pragma unroll
        for (int i = 0; i < N; ++i) asm volatile("" : "+v"(w[i]));
    }
};

// Memory at a scalar base and a lane's own offset of 32 bits.
template <class E, int V>
__device__ inline Raw<E, V> load_raw(const E* base, unsigned off) {
    const char* q = reinterpret_cast<const char*>(base) + off;
    Raw<E, V> x;
    if constexpr (sizeof(E) * V == 2) {
        x.w[0] = *reinterpret_cast<const uint16_t*>(q);
    } else if constexpr (sizeof(E) * V == 4) {
        x.w[0] = *reinterpret_cast<const uint32_t*>(q);
    } else {
        const uint2 u = *reinterpret_cast<const uint2*>(q);
        x.w[0] = u.x;
        x.w[1] = u.y;
    }
    return x;
}
template <bool FAR, class E, int V>
__device__ inline void store_at(E* base, unsigned off, const float* in) {
    put<FAR, E, V>(reinterpret_cast<E*>(reinterpret_cast<char*>(base) + off), in);
}

// Which share of which row and columns this workgroup takes.  The shares of one
// row and tile are a chain, in the order of their dependence.  A workgroup's
// number names its chain; which share, the chain's counter: a workgroup then
// only ever waits for one that has started, whatever order they are started
// in.  Every launch takes each chain's shares once, so the counter also numbers
// the launches, and nothing is cleared between them.  (One counter for all
// chains: an atomic on one address takes 40 ns, 0.33 ms for 4096 shares.)
struct Item {
    int b, tile, seg;
    int length;  // as passed: loaded while the counter answers
    unsigned launch;
};
constexpr int COUNTER_WORDS = 8;  // a counter per 64 bytes
template <int WAY>
__device__ inline Item take_item(const ScanParams& p, bool last_first, unsigned (*lds)[2]) {
    const unsigned chains = (unsigned)p.B * p.tiles;
    Item it;
    const unsigned chain = WAY == ONE ? blockIdx.x : blockIdx.x % chains;
    unsigned seg = 0;
    it.launch = 0;
    it.b = (int)(chain / p.tiles);
    it.tile = (int)(chain - (unsigned)it.b * p.tiles);
    it.length = p.lengths[it.b];
    if constexpr (WAY != ONE) {
        if (threadIdx.x == 0) {
            const unsigned long long n = atomicAdd(p.counters + (long)chain * COUNTER_WORDS, 1ull);
            const unsigned long long l = n >> 32 ? n / (unsigned)p.segs : (unsigned)n / (unsigned)p.segs;
            (*lds)[0] = (unsigned)(n - l * (unsigned)p.segs);
            (*lds)[1] = (unsigned)l + 1;
        }
        __syncthreads();
        seg = (unsigned)__builtin_amdgcn_readfirstlane((int)(*lds)[0]);  // scalar addresses
        it.launch = (unsigned)__builtin_amdgcn_readfirstlane((int)(*lds)[1]);
    }
    it.seg = last_first ? p.segs - 1 - (int)seg : (int)seg;
    return it;
}

// A value and the launch it belongs to in one word: no flag beside it, and
// nothing to clear before a launch.
template <int V>
__device__ inline void publish(uint64_t* w, const float* x, unsigned launch) {
#pragma unroll
    for (int i = 0; i < V; ++i)
        __hip_atomic_store(w + i, (uint64_t)launch << 32 | __float_as_uint(x[i]), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
}
template <int V>
__device__ inline void await(const ScanParams& p, uint64_t* w, float* x, unsigned launch) {
    const unsigned long long t0 = wall_clock64();
    for (;;) {
        bool all = true;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint64_t q = __hip_atomic_load(w + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            all = all && (unsigned)(q >> 32) == launch;
            x[i] = __uint_as_float((unsigned)q);
        }
        if (all) return;
        if (wall_clock64() - t0 > p.timeout_ticks) {
            atomicOr(p.status, STATUS_TIMEOUT);
            return;
        }
        __builtin_amdgcn_s_sleep(1);
    }
}

// A thread holds R steps of V channels; CL lanes lie along the channels, so a
// workgroup holds NT / CL runs, S steps.  Each run is an affine map x -> A x + S
// of the state it starts from.  join_runs gives the map of all runs before
// this thread's (after, if REV), and in `total` that of the whole workgroup.
template <int V, int NT, int CL, bool REV>
__device__ inline void join_runs(float* A, float* S, float* total_A, float* total_S, float (*lds)[2][CL * V]) {
    constexpr int NW = NT / 64 < 1 ? 1 : NT / 64;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, cl = threadIdx.x % CL;
    float a[V], s[V];  // inclusive over the runs of this wave
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = A[i], s[i] = S[i];
#pragma unroll
    for (int o = CL; o < 64; o <<= 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float pa = REV ? __shfl_down(a[i], o) : __shfl_up(a[i], o);
            const float ps = REV ? __shfl_down(s[i], o) : __shfl_up(s[i], o);
            if (REV ? lane + o < 64 : lane >= o) {
                s[i] = fmaf(a[i], ps, s[i]);
                a[i] *= pa;
            }
        }
    }
    const bool last = REV ? lane < CL : lane >= 64 - CL;
    if (NW > 1 && last) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            lds[w][0][cl * V + i] = a[i];
            lds[w][1][cl * V + i] = s[i];
        }
    }
    // exclusive within the wave
    float xa[V], xs[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        xa[i] = 1.0f;
        xs[i] = 0.0f;
        if constexpr (CL < 64) {
            const float pa = REV ? __shfl_down(a[i], CL) : __shfl_up(a[i], CL);
            const float ps = REV ? __shfl_down(s[i], CL) : __shfl_up(s[i], CL);
            if (REV ? lane + CL < 64 : lane >= CL) xa[i] = pa, xs[i] = ps;
        }
    }
    if constexpr (NW > 1) {
        __syncthreads();
        float pa[V], ps[V];
#pragma unroll
        for (int i = 0; i < V; ++i) pa[i] = total_A[i] = 1.0f, ps[i] = total_S[i] = 0.0f;
        for (int j = 0; j < NW; ++j) {
            const int q = REV ? NW - 1 - j : j;
            if (q == w) {
#pragma unroll
                for (int i = 0; i < V; ++i) pa[i] = total_A[i], ps[i] = total_S[i];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float qa = lds[q][0][cl * V + i], qs = lds[q][1][cl * V + i];
                total_S[i] = fmaf(qa, total_S[i], qs);
                total_A[i] *= qa;
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            S[i] = fmaf(xa[i], ps[i], xs[i]);
            A[i] = xa[i] * pa[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int src = REV ? cl : 64 - CL + cl;
            total_A[i] = __shfl(a[i], src);
            total_S[i] = __shfl(s[i], src);
            A[i] = xa[i];
            S[i] = xs[i];
        }
    }
}

// What a workgroup's threads know of their place.
template <class E, int V, int NT, int CL>
struct Place {
    static constexpr int R = run_of<E>(), G = NT / CL;
    int b, seg, cl, g, c, t0, first, L;
    unsigned launch;
    bool on, full;
    unsigned zoff, yoff;  // bytes from the share's first step to this thread's

    __device__ Place(const ScanParams& p, const Item& it)
        : b(it.b), seg(it.seg), cl(threadIdx.x % CL), g(threadIdx.x / CL), launch(it.launch) {
        const int ch = (it.tile * CL + cl) * V;
        on = ch < p.H;
        c = on ? ch : 0;
        first = seg * G * R;
        t0 = first + g * R;
        L = clamp_length(it.length, p.T, p.status, it.tile == 0 && seg == 0 && threadIdx.x == 0);
        full = first + G * R <= L;
        zoff = ((unsigned)(g * R * 3) * p.H + c) * sizeof(E);
        yoff = ((unsigned)(g * R) * p.H + c) * sizeof(E);
    }
    __device__ long step0(const ScanParams& p) const { return (long)b * p.T + first; }
};

// The state (or gradient) a share starts from, into start[], and what it passes
// on.  `depth` shares of its row come before it, the nearest `dir` away; the
// row's first one starts from `base`.  Share j passes on P_j = A_j P_{j-1} + S_j.
// Where a row's chain is what takes the time (few chains), a share does not wait
// for P_{j-1}: every share first publishes its map, and each wave fetches one of
// the NW - 1 maps before this one, or P_{j-NW}, from which the same products and sums
// give P_{j-1}, to the bit: the chain is NW times shorter.
template <int WAY, class E, int V, int NT, int CL>
__device__ inline void carry_on(const ScanParams& p, const Place<E, V, NT, CL>& at, int depth, int dir, bool last,
                                const float* base, const float* A, const float* S, float* start,
                                float (*seen)[2][CL * V], float* out) {
    constexpr int NW = NT / 64;
    const int w = threadIdx.x >> 6;
    const long stride = (long)p.B * p.segs * p.H, cell = ((long)at.b * p.segs + at.seg) * p.H + at.c;
    const bool mine = threadIdx.x < CL && at.on;
    float x[V] = {};
    if constexpr (WAY == WINDOW) {
        // The base is read (into LDS) before the map goes out: whoever writes the row's result, which
        // may lie where h0 does, has awaited every share's map, its own or through another's.
        if (mine && depth < NW) {
#pragma unroll
            for (int i = 0; i < V; ++i) start[at.cl * V + i] = base ? base[i] : 0.0f;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (mine && !last) {
            publish<V>(p.carry + stride + cell, A, at.launch);
            publish<V>(p.carry + 2 * stride + cell, S, at.launch);
        }
        if (w < depth && (int)(threadIdx.x & 63) < CL && at.on) {
            uint64_t* q = p.carry + cell + (long)dir * (w + 1) * p.H;
            float a[V] = {}, s[V];
            if (w == NW - 1) {
                await<V>(p, q, s, at.launch);
            } else {
                await<V>(p, q + stride, a, at.launch);
                await<V>(p, q + 2 * stride, s, at.launch);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) seen[w][0][at.cl * V + i] = a[i], seen[w][1][at.cl * V + i] = s[i];
        }
        __syncthreads();
        if (mine) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[i] = depth >= NW ? seen[NW - 1][1][at.cl * V + i] : start[at.cl * V + i];
                for (int j = min(depth, NW - 1) - 1; j >= 0; --j)
                    x[i] = fmaf(seen[j][0][at.cl * V + i], x[i], seen[j][1][at.cl * V + i]);
            }
        }
    } else if (mine) {
        if (WAY == ONE || depth == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = base ? base[i] : 0.0f;
        } else {
            await<V>(p, p.carry + cell + (long)dir * p.H, x, at.launch);
        }
    }
    if (mine) {
        float e[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            start[at.cl * V + i] = x[i];
            e[i] = at.L == 0 ? x[i] : fmaf(A[i], x[i], S[i]);
        }
        if (WAY == ONE || last) {
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = e[i];
        } else {
            publish<V>(p.carry + cell, e, at.launch);
        }
    }
    __syncthreads();
}

// The steps of a share.  WHOLE: all of them are valid, so loads and selects
// depend on nothing; written out apart, because where the two ways would meet
// the compiler waits for every load.
template <bool WHOLE, bool FAR, int WAY, class E, int V, int NT, int CL>
__device__ inline void forward_share(const ScanParams& p, const Place<E, V, NT, CL>& at,
                                     float (*maps)[2][CL * V], float* start,
                                      float (*seen)[2][CL * V]) {
    constexpr int R = run_of<E>(), G = NT / CL;
    const int H = p.H, L = at.L, t0 = at.t0;
    const long row = (long)at.b * H + at.c;
    const E* z = static_cast<const E*>(p.z) + at.step0(p) * 3 * H;
    E* y = static_cast<E*>(p.y) + at.step0(p) * H;
    float q[R][V], A[V], S[V];
    Raw<E, V> f[R], v[R], o[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (!WHOLE) f[r] = v[r] = Raw<E, V>{};
        if (WHOLE || t0 + r < L) {
            f[r] = load_raw<E, V>(z + (long)r * 3 * H, at.zoff);
            v[r] = load_raw<E, V>(z + (long)r * 3 * H + H, at.zoff);
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) A[i] = 1.0f, S[i] = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            q[r][i] = gate_code(f[r][i]);
            const float a = gate_keep(q[r][i]);
            const float s = fmaf(a, S[i], gate_take(q[r][i]) * v[r][i]);
            if (WHOLE || t0 + r < L) S[i] = s, A[i] *= a;
        }
    }
    // The output gates are on their way while the runs are joined; earlier they would only
    // hold registers.
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (!WHOLE) o[r] = Raw<E, V>{};
        if (WHOLE || t0 + r < L) o[r] = load_raw<E, V>(z + (long)r * 3 * H + 2 * H, at.zoff);
    }
    float tA[V], tS[V], h[V] = {};
    join_runs<V, NT, CL, false>(A, S, tA, tS, maps);
    carry_on<WAY>(p, at, at.seg, -1, at.first + G * R >= L, p.h0 + row, tA, tS, start, seen, p.out_h + row);
    if (!at.on) return;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        v[r].hold(), o[r].hold();
#pragma unroll
        for (int i = 0; i < V; ++i) hold(q[r][i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = fmaf(A[i], start[at.cl * V + i], S[i]);
    if (p.kept && t0 < L) {
        float* kp = p.kept + ((long)at.b * ((p.T + R - 1) / R) + t0 / R) * H + at.c;
#pragma unroll
        for (int i = 0; i < V; ++i) kp[i] = h[i];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            h[i] = fmaf(gate_keep(q[r][i]), h[i], gate_take(q[r][i]) * v[r][i]);
            out[i] = logistic_neg(-o[r][i]) * h[i];
            if (!WHOLE && t0 + r >= L) out[i] = 0.0f;
        }
        if (WHOLE || t0 + r < p.T) store_at<FAR, E, V>(y + (long)r * H, at.yoff, out);
    }
}

template <bool FAR, int WAY, class E, int V, int NT, int CL>
__global__ void __launch_bounds__(NT, 4) scan_forward_kernel(ScanParams p) {
    constexpr int R = run_of<E>(), NW = NT / 64;
    __shared__ unsigned turn[1][2];
    __shared__ float maps[NW][2][CL * V];
    __shared__ float start[CL * V];
    __shared__ float seen[NW][2][CL * V];
    const Place<E, V, NT, CL> at(p, take_item<WAY>(p, false, turn));
    if (at.full) {
        forward_share<true, FAR, WAY, E, V, NT, CL>(p, at, maps, start, seen);
    } else if (at.first < at.L || at.first == 0) {
        forward_share<false, FAR, WAY, E, V, NT, CL>(p, at, maps, start, seen);
    } else if (at.on) {  // past the row's end
        E* y = static_cast<E*>(p.y) + at.step0(p) * p.H;
        float zero[V] = {};
        for (int r = 0; r < R && at.t0 + r < p.T; ++r) store_at<FAR, E, V>(y + (long)r * p.H, at.yoff, zero);
    }
}

template <bool WHOLE, bool FAR, int WAY, class E, int V, int NT, int CL>
__device__ inline void backward_share(const ScanParams& p, const Place<E, V, NT, CL>& at,
                                      float (*maps)[2][CL * V], float* start,
                                      float (*seen)[2][CL * V]) {
    constexpr int R = run_of<E>(), G = NT / CL;
    const int H = p.H, L = at.L, t0 = at.t0;
    const long row = (long)at.b * H + at.c;
    const E* z = static_cast<const E*>(p.z) + at.step0(p) * 3 * H;
    const E* dy = static_cast<const E*>(p.dy) + at.step0(p) * H;
    E* dz = static_cast<E*>(p.dz) + at.step0(p) * 3 * H;
    // per step: the gate's code, s dy, and dzf's factor of g
    float k[R][V], q[R][V], f[R][V], A[V], S[V], h[V] = {};
    Raw<E, V> zf[R], zv[R], zo[R], zd[R];
    if (WHOLE || t0 < L) {
        const float* kp = p.kept + ((long)at.b * ((p.T + R - 1) / R) + t0 / R) * H + at.c;
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = kp[i];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (!WHOLE) zf[r] = zv[r] = zo[r] = zd[r] = Raw<E, V>{};
        if (WHOLE || t0 + r < L) {
            zf[r] = load_raw<E, V>(z + (long)r * 3 * H, at.zoff);
            zv[r] = load_raw<E, V>(z + (long)r * 3 * H + H, at.zoff);
            zo[r] = load_raw<E, V>(z + (long)r * 3 * H + 2 * H, at.zoff);
            zd[r] = load_raw<E, V>(dy + (long)r * H, at.yoff);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float out[V];
        const bool valid = WHOLE || t0 + r < L;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float gf = gate_code(zf[r][i]), go = gate_code(zo[r][i]), d = zd[r][i];
            f[r][i] = (h[i] - zv[r][i]) * gate_slope(gf);
            h[i] = fmaf(gate_keep(gf), h[i], gate_take(gf) * zv[r][i]);
            out[i] = valid ? d * h[i] * gate_slope(go) : 0.0f;
            k[r][i] = valid ? gf : 0.0f;
            q[r][i] = valid ? gate_keep(go) * d : 0.0f;
            hold(f[r][i]), hold(q[r][i]);
        }
        if (at.on && (WHOLE || t0 + r < p.T)) store_at<FAR, E, V>(dz + ((long)r * 3 + 2) * H, at.zoff, out);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) A[i] = 1.0f, S[i] = 0.0f;
#pragma unroll
    for (int r = R - 1; r >= 0; --r) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            hold(k[r][i]);
            const float a = gate_keep(k[r][i]);
            S[i] = a * (q[r][i] + S[i]);
            A[i] *= a;
        }
    }
    float tA[V], tS[V], e[V] = {};
    join_runs<V, NT, CL, true>(A, S, tA, tS, maps);
    carry_on<WAY>(p, at, (L - 1) / (G * R) - at.seg, 1, at.seg == 0, p.d_out_h ? p.d_out_h + row : nullptr, tA, tS, start,
             seen, p.dh0 + row);
    if (!at.on) return;
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = fmaf(A[i], start[at.cl * V + i], S[i]);
#pragma unroll
    for (int r = R - 1; r >= 0; --r) {
        float df[V], dv[V];
        const bool valid = WHOLE || t0 + r < L;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            hold(k[r][i]);
            const float gr = q[r][i] + e[i];
            df[i] = valid ? gr * f[r][i] : 0.0f;
            dv[i] = valid ? gr * gate_take(k[r][i]) : 0.0f;
            e[i] = valid ? gate_keep(k[r][i]) * gr : e[i];
        }
        if (WHOLE || t0 + r < p.T) {
            store_at<FAR, E, V>(dz + (long)r * 3 * H, at.zoff, df);
            store_at<FAR, E, V>(dz + ((long)r * 3 + 1) * H, at.zoff, dv);
        }
    }
}

template <bool FAR, int WAY, class E, int V, int NT, int CL>
__global__ void __launch_bounds__(NT, sizeof(E) == 2 && V == 2 ? 3 : 4) scan_backward_kernel(ScanParams p) {
    constexpr int R = run_of<E>(), NW = NT / 64;
    __shared__ unsigned turn[1][2];
    __shared__ float maps[NW][2][CL * V];
    __shared__ float start[CL * V];
    __shared__ float seen[NW][2][CL * V];
    const Place<E, V, NT, CL> at(p, take_item<WAY>(p, true, turn));
    if (at.full) {
        backward_share<true, FAR, WAY, E, V, NT, CL>(p, at, maps, start, seen);
    } else if (at.first < at.L) {
        backward_share<false, FAR, WAY, E, V, NT, CL>(p, at, maps, start, seen);
    } else if (at.on) {  // past the row's end
        E* dz = static_cast<E*>(p.dz) + at.step0(p) * 3 * p.H;
        float zero[V] = {};
        for (int r = 0; r < R && at.t0 + r < p.T; ++r)
#pragma unroll
            for (int j = 0; j < 3; ++j) store_at<FAR, E, V>(dz + ((long)r * 3 + j) * p.H, at.zoff, zero);
        if (at.L == 0 && at.t0 == 0) {
            const long row = (long)at.b * p.H + at.c;
#pragma unroll
            for (int i = 0; i < V; ++i) p.dh0[row + i] = p.d_out_h ? p.d_out_h[row + i] : 0.0f;
        }
    }
}

// One step of each row: elementwise, V channels per thread.
template <class E, int V>
__global__ void __launch_bounds__(256)
scan_step_kernel(const E* z, const float* h, float* out_h, E* y, int rows, int H) {
    const int HV = H / V;
    const long i = blockIdx.x * 256L + threadIdx.x;
    if (i >= (long)rows * HV) return;
    const long r = i / HV;
    const int c = (int)(i - r * HV) * V;
    const E* zr = z + r * 3 * H + c;
    float f[V], v[V], o[V], s[V], out[V];
    load_vec<E, V>(zr, f);
    load_vec<E, V>(zr + H, v);
    load_vec<E, V>(zr + 2 * H, o);
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = h[r * H + c + j];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float q = gate_code(f[j]);
        s[j] = fmaf(gate_keep(q), s[j], gate_take(q) * v[j]);
        out[j] = logistic_neg(-o[j]) * s[j];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) out_h[r * H + c + j] = s[j];
    store_vec<E, V>(y + r * H + c, out);
}

struct Shape {
    int threads, lanes;  // of a workgroup; of those along the channels
    int steps;           // of a share
    int segs, tiles;
    int way;             // see carry_on
};

int scan_run_of(int dtype) { return dtype == LSTM_DYN_BF16 ? run_of<__bf16>() : run_of<float>(); }
int scan_vec_of(int H) { return H % 2 ? 1 : 2; }

// The smallest workgroup that holds all steps, up to `most` threads.
Shape scan_shape(int B, int H, int T, int dtype, int num_cus, int most) {
    const int run = scan_run_of(dtype), vec = scan_vec_of(H);
    Shape w{64, 64, 0, 0, 0, ONE};
    while (w.threads < most && w.threads / 64 * run < T) w.threads *= 2;
    if (w.threads == most && most / 64 * run < T) w.lanes = 32;  // the longer share: fewer in a row's chain
    w.steps = w.threads / w.lanes * run;
    w.segs = (int)(((long long)T + w.steps - 1) / w.steps);
    w.tiles = (H + w.lanes * vec - 1) / (w.lanes * vec);
    // Some 16 shares of a chain on the device at once hide its waits (two rows of 16384 x 2048,
    // 64 chains: 121 us in a plain chain, 127 with the maps); with fewer chains than that the chain's
    // own time counts (one row of 32768 x 2048, 32 chains: 141 and 127; x 512, 8
    // chains, with its backward: 256 and 128).
    if (w.segs > 1) w.way = w.segs > 2 && 8LL * B * w.tiles <= num_cus ? WINDOW : CHAIN;
    return w;
}

int check_scan_sizes(int B, int H, int T, int dtype) {
    if (B < 1 || H < 1 || T < 1 || !valid_dtype(dtype)) return LSTM_DYN_ERR_INVALID;
    if ((long long)B * T > 0x7fffffffLL || H >= 1 << 18) return LSTM_DYN_ERR_UNSUPPORTED;
    // the kernels count steps up to a share past T in 32 bits, a launch its threads
    for (int most : {FWD_THREADS, BWD_THREADS}) {
        const Shape w = scan_shape(B, H, T, dtype, 0, most);
        if ((long long)T + w.steps > 0x7fffffffLL) return LSTM_DYN_ERR_UNSUPPORTED;
        const long long per_row = (long long)w.tiles * w.segs * w.threads;  // under 2^49
        if (per_row > 0xffffffffLL || B * per_row > 0xffffffffLL) return LSTM_DYN_ERR_UNSUPPORTED;
    }
    return LSTM_DYN_OK;
}

int check_scan_forward(int B, int H, int T, int dtype, const void* z, const int32_t* lengths,
                       const float* h0, const float* out_h, const void* out_y) {
    const long long e = dtype_bytes(dtype), n = (long long)B * T * H, ns = 4LL * B * H;
    const Span s[] = {{z, 3 * n * e, 16, false}, {lengths, 4LL * B, 4, false}, {h0, ns, 4, false},
                      {out_h, ns, 4, true, h0}, {out_y, n * e, 16, true}};
    return check_spans(s, 5);
}

int check_scan_backward(int B, int H, int T, int dtype, const void* z, const int32_t* lengths,
                        const float* h0, const void* dy, const float* d_out_h, const void* dz,
                        const float* dh0) {
    const long long e = dtype_bytes(dtype), n = (long long)B * T * H, ns = 4LL * B * H;
    const Span s[] = {{z, 3 * n * e, 16, false}, {lengths, 4LL * B, 4, false}, {h0, ns, 4, false},
                      {dy, n * e, 16, false}, {dz, 3 * n * e, 16, true}, {dh0, ns, 4, true},
                      {d_out_h, ns, 4, false}};
    return check_spans(s, d_out_h ? 7 : 6);
}

}  // namespace
}  // namespace ldyn

using namespace ldyn;

struct lstm_dyn_scan : OpsHandle {
    int B, H, T, dtype;
    int run, vec;  // steps and channels of a thread
    Shape fwd, bwd;
    char* chains[2];  // forward's and backward's counters, then their carries
    float* kept = nullptr;  // made by the first forward for training
    bool has_kept = false;
};

template <bool FAR, class E, int V>
static void scan_launch(const lstm_dyn_scan* h, const ScanParams& p, bool back) {
    const Shape& w = back ? h->bwd : h->fwd;
    void (*k)(ScanParams);
    if (back)
        k = w.way == WINDOW    ? scan_backward_kernel<FAR, WINDOW, E, V, BWD_THREADS, 32>
            : w.way == CHAIN   ? scan_backward_kernel<FAR, CHAIN, E, V, BWD_THREADS, 32>
            : w.lanes == 32    ? scan_backward_kernel<FAR, ONE, E, V, BWD_THREADS, 32>
            : w.threads == 64  ? scan_backward_kernel<FAR, ONE, E, V, 64, 64>
            : w.threads == 128 ? scan_backward_kernel<FAR, ONE, E, V, 128, 64>
                               : scan_backward_kernel<FAR, ONE, E, V, 256, 64>;
    else
        k = w.way == WINDOW    ? scan_forward_kernel<FAR, WINDOW, E, V, FWD_THREADS, 32>
            : w.way == CHAIN   ? scan_forward_kernel<FAR, CHAIN, E, V, FWD_THREADS, 32>
            : w.lanes == 32    ? scan_forward_kernel<FAR, ONE, E, V, FWD_THREADS, 32>
            : w.threads == 64  ? scan_forward_kernel<FAR, ONE, E, V, 64, 64>
            : w.threads == 128 ? scan_forward_kernel<FAR, ONE, E, V, 128, 64>
            : w.threads == 256 ? scan_forward_kernel<FAR, ONE, E, V, 256, 64>
                               : scan_forward_kernel<FAR, ONE, E, V, 512, 64>;
    hipLaunchKernelGGL(k, dim3((unsigned)((long)h->B * w.tiles * w.segs)), dim3((unsigned)w.threads), 0,
                       h->last_stream, p);
}

static int scan_run(lstm_dyn_scan* h, const ScanParams& p, bool back) {
    const long long out = (long long)h->B * h->T * h->H * (back ? 3 : 1) * dtype_bytes(h->dtype);
    // Large outputs bypass the caches, which then keep what is read again (the kept states, and z in
    // the backward).  A training step with a product that reads dz behind it,
    // by the size of y: 24 MB 95 us either way, 32 MB 123 and 111 past them, 64 MB 233 and 227, 256
    // MB 856 and 845; the forward with a product behind it 64 MB 80 and 76, 128 MB 167 and 173, 256 MB
    // 320 and 315.
    const bool far = out > FAR_BYTES;
#define LDYN_RUN(E, V) (far ? scan_launch<true, E, V>(h, p, back) : scan_launch<false, E, V>(h, p, back))
    if (h->dtype == LSTM_DYN_BF16) {
        if (h->vec == 2) LDYN_RUN(__bf16, 2);
        else LDYN_RUN(__bf16, 1);
    } else {
        if (h->vec == 2) LDYN_RUN(float, 2);
        else LDYN_RUN(float, 1);
    }
#undef LDYN_RUN
    return ops_launched(h);
}

static ScanParams scan_params(const lstm_dyn_scan* h, const Shape& w, const void* z,
                              const int32_t* lengths, const float* h0) {
    ScanParams p{};
    p.z = z;
    p.lengths = lengths;
    p.h0 = h0;
    p.status = h->status();
    p.B = h->B;
    p.T = h->T;
    p.H = h->H;
    p.tiles = w.tiles;
    p.segs = w.segs;
    char* c = h->chains[&w == &h->bwd];
    p.counters = reinterpret_cast<unsigned long long*>(c);
    p.carry = reinterpret_cast<uint64_t*>(c + 8LL * COUNTER_WORDS * h->B * w.tiles);
    p.timeout_ticks = (unsigned long long)(5.0 * 1e3 * (double)h->wclk_khz);
    return p;
}

extern "C" int lstm_dyn_check_scan_args(int B, int H, int T, int dtype, const void* z,
                                        const int32_t* lengths, const float* h0,
                                        const float* out_h, const void* out_y, const void* dy,
                                        const float* d_out_h, const void* dz, const float* dh0) {
    const int rc = check_scan_sizes(B, H, T, dtype);
    if (rc != LSTM_DYN_OK) return rc;
    if (!dy && !dz && !dh0) return check_scan_forward(B, H, T, dtype, z, lengths, h0, out_h, out_y);
    return check_scan_backward(B, H, T, dtype, z, lengths, h0, dy, d_out_h, dz, dh0);
}

extern "C" int lstm_dyn_scan_create(lstm_dyn_scan_t** out, int B, int H, int T, int dtype) {
    if (!out) return LSTM_DYN_ERR_INVALID;
    *out = nullptr;
    int rc = check_scan_sizes(B, H, T, dtype);
    if (rc != LSTM_DYN_OK) return rc;
    lstm_dyn_scan* h = new (std::nothrow) lstm_dyn_scan();
    if (!h) return LSTM_DYN_ERR_NOMEM;
    h->B = B; h->H = H; h->T = T; h->dtype = dtype;
    if ((rc = ops_device(h)) != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    h->run = scan_run_of(dtype);
    h->vec = scan_vec_of(H);
    h->fwd = scan_shape(B, H, T, dtype, h->num_cus, FWD_THREADS);
    h->bwd = scan_shape(B, H, T, dtype, h->num_cus, BWD_THREADS);
    auto bytes = [&](const Shape& w) {
        return w.segs > 1 ? 8LL * COUNTER_WORDS * B * w.tiles + (w.way == WINDOW ? 24LL : 8LL) * B * w.segs * H : 0;
    };
    if ((rc = ops_init(h, 256 + bytes(h->fwd) + bytes(h->bwd))) != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    h->chains[0] = h->block + 256;
    h->chains[1] = h->chains[0] + bytes(h->fwd);
    *out = h;
    return LSTM_DYN_OK;
}

static int scan_forward_impl(lstm_dyn_scan* h, const void* z, const int32_t* lengths,
                             const float* h0, float* out_h, void* out_y, bool train, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc = check_scan_forward(h->B, h->H, h->T, h->dtype, z, lengths, h0, out_h, out_y);
    if (rc != LSTM_DYN_OK) return rc;
    if (train && out_h == h0) return LSTM_DYN_ERR_INVALID;  // the backward reads h0
    if (train && !h->kept) {  // memory is not allocated under a capture, which the attempt would end
        hipStreamCaptureStatus capture;
        if (hipStreamIsCapturing(static_cast<hipStream_t>(stream), &capture) != hipSuccess) {
            (void)hipGetLastError();
            return LSTM_DYN_ERR_HIP;
        }
        if (capture != hipStreamCaptureStatusNone) return LSTM_DYN_ERR_INVALID;
    }
    if ((rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    h->has_kept = false;
    if (train && !h->kept) {
        void* p = nullptr;
        const long long n = 4LL * h->B * ((h->T + h->run - 1) / h->run) * h->H;
        if (hipMalloc(&p, (size_t)n) != hipSuccess) {
            (void)hipGetLastError();
            return LSTM_DYN_ERR_NOMEM;
        }
        h->kept = static_cast<float*>(p);
        h->bytes += n;
    }
    ScanParams p = scan_params(h, h->fwd, z, lengths, h0);
    p.out_h = out_h;
    p.y = out_y;
    p.kept = train ? h->kept : nullptr;
    if ((rc = scan_run(h, p, false)) == LSTM_DYN_OK) h->has_kept = train;
    return rc;
}

extern "C" int lstm_dyn_scan_forward(lstm_dyn_scan_t* h, const void* z, const int32_t* lengths,
                                     const float* h0, float* out_h, void* out_y, void* stream) {
    return scan_forward_impl(h, z, lengths, h0, out_h, out_y, false, stream);
}

extern "C" int lstm_dyn_scan_forward_train(lstm_dyn_scan_t* h, const void* z,
                                           const int32_t* lengths, const float* h0, float* out_h,
                                           void* out_y, void* stream) {
    return scan_forward_impl(h, z, lengths, h0, out_h, out_y, true, stream);
}

extern "C" int lstm_dyn_scan_backward(lstm_dyn_scan_t* h, const void* z, const int32_t* lengths,
                                      const float* h0, const void* dy, const float* d_out_h,
                                      void* dz, float* dh0, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc = check_scan_backward(h->B, h->H, h->T, h->dtype, z, lengths, h0, dy, d_out_h, dz, dh0);
    if (rc != LSTM_DYN_OK) return rc;
    if (!h->has_kept) return LSTM_DYN_ERR_INVALID;  // no forward for training before it
    if ((rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    h->has_kept = false;
    ScanParams p = scan_params(h, h->bwd, z, lengths, h0);
    p.kept = h->kept;
    p.dy = dy;
    p.d_out_h = d_out_h;
    p.dz = dz;
    p.dh0 = dh0;
    return scan_run(h, p, true);
}

extern "C" int lstm_dyn_scan_step(int rows, int H, int dtype, const void* z, const float* h,
                                  float* out_h, void* out_y, void* stream) {
    if (rows < 1 || H < 1 || !valid_dtype(dtype)) return LSTM_DYN_ERR_INVALID;
    if (H >= 1 << 18) return LSTM_DYN_ERR_UNSUPPORTED;
    int rc;
    const long long e = dtype_bytes(dtype), n = (long long)rows * H;
    const Span s[] = {{z, 3 * n * e, (int)e, false}, {h, 4 * n, 4, false}, {out_h, 4 * n, 4, true, h},
                      {out_y, n * e, (int)e, true}};
    if ((rc = check_spans(s, 4)) != LSTM_DYN_OK) return rc;
    // four channels at once where z and y allow it: rows of a longer sequence need not
    const bool vec = H % 4 == 0 && ((reinterpret_cast<uintptr_t>(z) | reinterpret_cast<uintptr_t>(out_y)) &
                                    (uintptr_t)(4 * e - 1)) == 0;
    const int V = vec ? 4 : 1;
    if (n / V > 0xffffffffLL - 255) return LSTM_DYN_ERR_UNSUPPORTED;  // threads of a launch
    const unsigned grid = (unsigned)((n / V + 255) / 256);
    hipStream_t st = static_cast<hipStream_t>(stream);
#define LDYN_STEP(E, VV)                                                                              \
    hipLaunchKernelGGL((scan_step_kernel<E, VV>), dim3(grid), dim3(256), 0, st,                       \
                       static_cast<const E*>(z), h, out_h, static_cast<E*>(out_y), rows, H)
    if (dtype == LSTM_DYN_BF16) {
        if (V == 4) LDYN_STEP(__bf16, 4);
        else LDYN_STEP(__bf16, 1);
    } else {
        if (V == 4) LDYN_STEP(float, 4);
        else LDYN_STEP(float, 1);
    }
#undef LDYN_STEP
    return ops_launched(nullptr);
}

extern "C" int lstm_dyn_scan_query(lstm_dyn_scan_t* h, int what, long long* value) {
    return ops_query(h, what, value);
}

extern "C" int lstm_dyn_scan_destroy(lstm_dyn_scan_t* h) {
    if (!h) return LSTM_DYN_OK;
    int rc = ops_free(h);
    if (h->kept && hipFree(h->kept) != hipSuccess) rc = LSTM_DYN_ERR_HIP;
    delete h;
    return rc;
}
