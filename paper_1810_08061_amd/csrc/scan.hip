// scan.hip -- the gated linear recurrence over whole sequences and its
// backward pass.
//
//   a_t = sigmoid(zf_t), k_t = 1 - a_t = sigmoid(-zf_t), s_t = sigmoid(zo_t)
//   h_t = h_{t-1} + k_t (v_t - h_{t-1}),   y_t = s_t h_t
// and back, with e_t the gradient of h_t from later steps (e_{L-1} = d_out_h):
//   g_t = s_t dy_t + e_t,   e_{t-1} = a_t g_t
//   dzf = g_t (h_{t-1} - v_t) a_t k_t,   dzv = g_t k_t,   dzo = dy_t h_t s_t (1 - s_t)
//
// The time axis is split: see join_runs and take_item.
#include "ops.h"

#include <type_traits>

namespace ldyn {
namespace {

// Steps one thread holds, and between two kept states.
template <class E>
constexpr int run_of() { return sizeof(E) == 2 ? 16 : 8; }

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
    unsigned* counters;   // [0] the next item, [1] items done, [2] launches done
    uint64_t* carry;      // [B][segs][H] {value, launch} a share passes on
    unsigned long long timeout_ticks;
};

// 1 / (1 + e^x), which is 1 and 0 at the infinities.
__device__ inline float logistic_neg(float x) { return rcp_f(1.0f + __expf(x)); }

// V elements as they lie in memory.
template <class E, int V>
using raw_t = typename Vec<E, V>::type;
template <class E, int V>
__device__ inline float elem(const raw_t<E, V>& x, int i) {
    if constexpr (V == 1) return (float)x;
    else return (float)x[i];
}

// Which share of which row and columns this workgroup takes.  Shares come in
// the order of their dependence, by a counter, so that one whose turn it is only
// ever waits for workgroups that have started: no residency is assumed.
struct Item {
    int b, tile, seg;
};
__device__ inline Item take_item(const ScanParams& p, bool last_first, unsigned* lds) {
    unsigned n = blockIdx.x;
    if (p.segs > 1) {
        if (threadIdx.x == 0) *lds = atomicAdd(p.counters, 1u);
        __syncthreads();
        n = *lds;
    }
    const unsigned per = (unsigned)p.B * p.tiles, seg = n / per, rest = n - seg * per;
    Item it;
    it.b = (int)(rest / p.tiles);
    it.tile = (int)(rest - (unsigned)it.b * p.tiles);
    it.seg = last_first ? p.segs - 1 - (int)seg : (int)seg;
    return it;
}

// The last workgroup to end makes the counters ready for the next launch.
__device__ inline void end_item(const ScanParams& p) {
    if (p.segs > 1 && threadIdx.x == 0) {
        if (atomicAdd(p.counters + 1, 1u) == gridDim.x - 1) {
            __hip_atomic_store(p.counters, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(p.counters + 1, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_fetch_add(p.counters + 2, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
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

template <class E, int V, int NT, int CL>
__global__ void __launch_bounds__(NT) scan_forward_kernel(ScanParams p) {
    constexpr int R = run_of<E>(), G = NT / CL, NW = NT / 64;
    __shared__ unsigned turn;
    __shared__ float maps[NW][2][CL * V];
    __shared__ float start[CL * V];
    const Item it = take_item(p, false, &turn);
    const int H = p.H, T = p.T, cl = threadIdx.x % CL, g = threadIdx.x / CL;
    const int ch = (it.tile * CL + cl) * V;
    const bool on = ch < H;
    const int c = on ? ch : 0;
    const int L = row_length(p.lengths, it.b, T, p.status, it.tile == 0 && it.seg == 0 && threadIdx.x == 0);
    const int t0 = (it.seg * G + g) * R, first = it.seg * G * R;
    E* y = static_cast<E*>(p.y) + ((long)it.b * T + t0) * H + c;
    const unsigned launch = p.segs > 1 ? p.counters[2] + 1 : 0;
    const long row = (long)it.b * H + c;

    if (first >= L && !(first == 0)) {  // a share past the row's end
        float zero[V] = {};
        if (on)
            for (int r = 0; r < R && t0 + r < T; ++r) store_vec<E, V>(y + (long)r * H, zero);
        end_item(p);
        return;
    }
    float k[R][V], A[V], S[V];
    raw_t<E, V> v[R], o[R];
    const bool full = first + G * R <= L;
    if (L > 0) {
        // steps past the end read the last valid one, and are left out below
        const E* z = static_cast<const E*>(p.z) + (long)it.b * T * 3 * H + c;
        raw_t<E, V> f[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const E* q = z + (long)min(t0 + r, L - 1) * 3 * H;
            f[r] = *reinterpret_cast<const raw_t<E, V>*>(q);
            v[r] = *reinterpret_cast<const raw_t<E, V>*>(q + H);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            o[r] = *reinterpret_cast<const raw_t<E, V>*>(z + (long)min(t0 + r, L - 1) * 3 * H + 2 * H);
#pragma unroll
        for (int i = 0; i < V; ++i) A[i] = 1.0f, S[i] = 0.0f;
        auto maps_of = [&](auto whole) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    k[r][i] = logistic_neg(elem<E, V>(f[r], i));
                    const float s = fmaf(k[r][i], elem<E, V>(v[r], i) - S[i], S[i]);
                    const float a = fmaf(-k[r][i], A[i], A[i]);
                    if (whole.value || t0 + r < L) S[i] = s, A[i] = a;
                }
            }
        };
        if (full) maps_of(std::true_type{});
        else maps_of(std::false_type{});
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) A[i] = 1.0f, S[i] = 0.0f;
    }
    float tA[V], tS[V], h[V] = {};
    join_runs<V, NT, CL, false>(A, S, tA, tS, maps);
    if (threadIdx.x < CL) {
        uint64_t* w = p.carry + ((long)it.b * p.segs + it.seg) * H + c;
        if (it.seg == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = p.h0[row + i];
        } else if (on) {
            await<V>(p, w - H, h, launch);
        }
        float e[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            start[cl * V + i] = h[i];
            e[i] = fmaf(tA[i], h[i], tS[i]);
            if (L == 0) e[i] = h[i];
        }
        if (on) {
            if (first + G * R < L) {
                publish<V>(w, e, launch);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) p.out_h[row + i] = e[i];
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = fmaf(A[i], start[cl * V + i], S[i]);
    if (on) {
        if (p.kept && t0 < L) {
            float* kp = p.kept + ((long)it.b * ((T + R - 1) / R) + t0 / R) * H + c;
#pragma unroll
            for (int i = 0; i < V; ++i) kp[i] = h[i];
        }
        auto steps = [&](auto whole) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float out[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    h[i] = fmaf(k[r][i], elem<E, V>(v[r], i) - h[i], h[i]);
                    out[i] = logistic_neg(-elem<E, V>(o[r], i)) * h[i];
                    if (!whole.value && t0 + r >= L) out[i] = 0.0f;
                }
                if (whole.value || t0 + r < T) store_vec<E, V>(y + (long)r * H, out);
            }
        };
        if (full) {
            steps(std::true_type{});
        } else if (L > 0) {
            steps(std::false_type{});
        } else {
            float zero[V] = {};
            for (int r = 0; r < R && t0 + r < T; ++r) store_vec<E, V>(y + (long)r * H, zero);
        }
    }
    end_item(p);
}

template <class E, int V, int NT, int CL>
__global__ void __launch_bounds__(NT) scan_backward_kernel(ScanParams p) {
    constexpr int R = run_of<E>(), G = NT / CL, NW = NT / 64;
    __shared__ unsigned turn;
    __shared__ float maps[NW][2][CL * V];
    __shared__ float start[CL * V];
    const Item it = take_item(p, true, &turn);
    const int H = p.H, T = p.T, cl = threadIdx.x % CL, g = threadIdx.x / CL;
    const int ch = (it.tile * CL + cl) * V;
    const bool on = ch < H;
    const int c = on ? ch : 0;
    const int L = row_length(p.lengths, it.b, T, p.status, it.tile == 0 && it.seg == 0 && threadIdx.x == 0);
    const int t0 = (it.seg * G + g) * R, first = it.seg * G * R;
    E* dz = static_cast<E*>(p.dz) + ((long)it.b * T + t0) * 3 * H + c;
    const unsigned launch = p.segs > 1 ? p.counters[2] + 1 : 0;
    const long row = (long)it.b * H + c;

    if (first >= L) {  // a share past the row's end
        float zero[V] = {};
        if (on) {
            for (int r = 0; r < R && t0 + r < T; ++r)
#pragma unroll
                for (int j = 0; j < 3; ++j) store_vec<E, V>(dz + ((long)r * 3 + j) * H, zero);
            if (L == 0 && first == 0 && g == 0) {
#pragma unroll
                for (int i = 0; i < V; ++i) p.dh0[row + i] = p.d_out_h ? p.d_out_h[row + i] : 0.0f;
            }
        }
        end_item(p);
        return;
    }
    const bool full = first + G * R <= L;
    // per step: the gate's complement, s dy, and dzf's factor of g
    float k[R][V], q[R][V], f[R][V], A[V], S[V];
    {
        const E* z = static_cast<const E*>(p.z) + (long)it.b * T * 3 * H + c;
        const E* dy = static_cast<const E*>(p.dy) + (long)it.b * T * H + c;
        raw_t<E, V> zf[R], zv[R], zo[R], zd[R];
        float h[V];
        const float* kp = p.kept + ((long)it.b * ((T + R - 1) / R) + min(t0, L - 1) / R) * H + c;
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = kp[i];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long t = min(t0 + r, L - 1);
            zf[r] = *reinterpret_cast<const raw_t<E, V>*>(z + t * 3 * H);
            zv[r] = *reinterpret_cast<const raw_t<E, V>*>(z + t * 3 * H + H);
            zo[r] = *reinterpret_cast<const raw_t<E, V>*>(z + t * 3 * H + 2 * H);
            zd[r] = *reinterpret_cast<const raw_t<E, V>*>(dy + t * H);
        }
        auto again = [&](auto whole) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float out[V];
                const bool valid = whole.value || t0 + r < L;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float kk = logistic_neg(elem<E, V>(zf[r], i));
                    const float s = logistic_neg(-elem<E, V>(zo[r], i));
                    const float qq = s * elem<E, V>(zd[r], i);
                    const float diff = elem<E, V>(zv[r], i) - h[i];
                    h[i] = fmaf(kk, diff, h[i]);
                    out[i] = valid ? qq * h[i] * (1.0f - s) : 0.0f;
                    k[r][i] = valid ? kk : 0.0f;
                    q[r][i] = valid ? qq : 0.0f;
                    f[r][i] = -diff * kk * (1.0f - kk);
                }
                if (on && (whole.value || t0 + r < T)) store_vec<E, V>(dz + ((long)r * 3 + 2) * H, out);
            }
        };
        if (full) again(std::true_type{});
        else again(std::false_type{});
    }
#pragma unroll
    for (int i = 0; i < V; ++i) A[i] = 1.0f, S[i] = 0.0f;
#pragma unroll
    for (int r = R - 1; r >= 0; --r) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float t = q[r][i] + S[i];
            S[i] = fmaf(-k[r][i], t, t);
            A[i] = fmaf(-k[r][i], A[i], A[i]);
        }
    }
    float tA[V], tS[V], e[V] = {};
    join_runs<V, NT, CL, true>(A, S, tA, tS, maps);
    if (threadIdx.x < CL) {
        uint64_t* w = p.carry + ((long)it.b * p.segs + it.seg) * H + c;
        if (first + G * R >= L) {
#pragma unroll
            for (int i = 0; i < V; ++i) e[i] = p.d_out_h ? p.d_out_h[row + i] : 0.0f;
        } else if (on) {
            await<V>(p, w + H, e, launch);
        }
        float x[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            start[cl * V + i] = e[i];
            x[i] = fmaf(tA[i], e[i], tS[i]);
        }
        if (on) {
            if (it.seg > 0) {
                publish<V>(w, x, launch);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) p.dh0[row + i] = x[i];
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = fmaf(A[i], start[cl * V + i], S[i]);
    if (on) {
        auto steps = [&](auto whole) {
#pragma unroll
            for (int r = R - 1; r >= 0; --r) {
                float df[V], dv[V];
                const bool valid = whole.value || t0 + r < L;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float gr = q[r][i] + e[i];
                    df[i] = valid ? gr * f[r][i] : 0.0f;
                    dv[i] = valid ? gr * k[r][i] : 0.0f;
                    e[i] = valid ? fmaf(-k[r][i], gr, gr) : e[i];
                }
                if (whole.value || t0 + r < T) {
                    store_vec<E, V>(dz + (long)r * 3 * H, df);
                    store_vec<E, V>(dz + ((long)r * 3 + 1) * H, dv);
                }
            }
        };
        if (full) steps(std::true_type{});
        else steps(std::false_type{});
    }
    end_item(p);
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
        s[j] = fmaf(logistic_neg(f[j]), v[j] - s[j], s[j]);
        out[j] = logistic_neg(-o[j]) * s[j];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) out_h[r * H + c + j] = s[j];
    store_vec<E, V>(y + r * H + c, out);
}

int check_scan_sizes(int B, int H, int T, int dtype) {
    if (B < 1 || H < 1 || T < 1 || !valid_dtype(dtype)) return LSTM_DYN_ERR_INVALID;
    if ((long long)B * T > 0x7fffffffLL || H >= 1 << 24) return LSTM_DYN_ERR_UNSUPPORTED;
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
    int vec, threads, lanes;  // channels per thread, threads of a workgroup, lanes along the channels
    int run, segs, tiles;
    uint64_t* carry = nullptr;
    float* kept = nullptr;  // made by the first forward for training
    bool has_kept = false;
};

// The workgroup's shape.
static void scan_shape(lstm_dyn_scan* h) {
    h->run = h->dtype == LSTM_DYN_BF16 ? run_of<__bf16>() : run_of<float>();
    h->vec = h->H % 2 ? 1 : 2;
    h->lanes = 64;
    h->threads = 64;
    while (h->threads < 512 && h->threads / 64 * h->run < h->T) h->threads *= 2;
    if (h->threads == 512 && 8 * h->run < h->T) h->lanes = 32;  // the longer share: fewer shares in a row's chain
    const int steps = h->threads / h->lanes * h->run;
    h->segs = (h->T + steps - 1) / steps;
    h->tiles = (h->H + h->lanes * h->vec - 1) / (h->lanes * h->vec);
}

template <class E, int V>
static void scan_launch(const lstm_dyn_scan* h, const ScanParams& p, bool back) {
    const dim3 grid((unsigned)((long)h->B * h->tiles * h->segs)), block((unsigned)h->threads);
#define LDYN_SCAN(NT, CL) (back ? scan_backward_kernel<E, V, NT, CL> : scan_forward_kernel<E, V, NT, CL>)
    auto* k = h->lanes == 32       ? LDYN_SCAN(512, 32)
              : h->threads == 64  ? LDYN_SCAN(64, 64)
              : h->threads == 128 ? LDYN_SCAN(128, 64)
              : h->threads == 256 ? LDYN_SCAN(256, 64)
                                  : LDYN_SCAN(512, 64);
    hipLaunchKernelGGL(k, grid, block, 0, h->last_stream, p);
#undef LDYN_SCAN
}

static int scan_run(lstm_dyn_scan* h, const ScanParams& p, bool back) {
    if (h->dtype == LSTM_DYN_BF16) {
        if (h->vec == 2) scan_launch<__bf16, 2>(h, p, back);
        else scan_launch<__bf16, 1>(h, p, back);
    } else {
        if (h->vec == 2) scan_launch<float, 2>(h, p, back);
        else scan_launch<float, 1>(h, p, back);
    }
    return ops_launched(h);
}

static ScanParams scan_params(const lstm_dyn_scan* h, const void* z, const int32_t* lengths,
                              const float* h0) {
    ScanParams p{};
    p.z = z;
    p.lengths = lengths;
    p.h0 = h0;
    p.status = h->status();
    p.B = h->B;
    p.T = h->T;
    p.H = h->H;
    p.tiles = h->tiles;
    p.segs = h->segs;
    p.counters = reinterpret_cast<unsigned*>(h->block + 64);
    p.carry = h->carry;
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
    scan_shape(h);
    const long long carry = h->segs > 1 ? 8LL * B * h->segs * H : 0;
    if ((rc = ops_init(h, 256 + carry)) != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    h->carry = reinterpret_cast<uint64_t*>(h->block + 256);
    *out = h;
    return LSTM_DYN_OK;
}

static int scan_forward_impl(lstm_dyn_scan* h, const void* z, const int32_t* lengths,
                             const float* h0, float* out_h, void* out_y, bool train, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc = check_scan_forward(h->B, h->H, h->T, h->dtype, z, lengths, h0, out_h, out_y);
    if (rc != LSTM_DYN_OK) return rc;
    if (train && out_h == h0) return LSTM_DYN_ERR_INVALID;  // the backward reads h0
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
    ScanParams p = scan_params(h, z, lengths, h0);
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
    ScanParams p = scan_params(h, z, lengths, h0);
    p.kept = h->kept;
    p.dy = dy;
    p.d_out_h = d_out_h;
    p.dz = dz;
    p.dh0 = dh0;
    return scan_run(h, p, true);
}

extern "C" int lstm_dyn_scan_step(int rows, int H, int dtype, const void* z, const float* h,
                                  float* out_h, void* out_y, void* stream) {
    int rc = check_scan_sizes(rows, H, 1, dtype);
    if (rc != LSTM_DYN_OK) return rc;
    const long long e = dtype_bytes(dtype), n = (long long)rows * H;
    const Span s[] = {{z, 3 * n * e, (int)e, false}, {h, 4 * n, 4, false}, {out_h, 4 * n, 4, true, h},
                      {out_y, n * e, (int)e, true}};
    if ((rc = check_spans(s, 4)) != LSTM_DYN_OK) return rc;
    // four channels at once where z and y allow it: rows of a longer sequence need not
    const bool vec = H % 4 == 0 && ((reinterpret_cast<uintptr_t>(z) | reinterpret_cast<uintptr_t>(out_y)) &
                                    (uintptr_t)(4 * e - 1)) == 0;
    const int V = vec ? 4 : 1;
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
