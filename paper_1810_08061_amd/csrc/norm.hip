// norm.hip -- layer norm over the last axis of [B][T][D] and its backward pass.
//
//   n = (x - mean) r, r = 1 / sqrt(var + eps), y = n w + b
//   g = dy w,  dx = r (g - mean g - n mean (g n)),  dw = sum dy n,  db = sum dy
//
// Bound by memory: x read and y written; back x and dy read and dx written.  A row lives in
// the registers of W waves, so its mean and then its squared deviations come from one
// reading (squares of x itself would cancel where the mean is large), and the backward
// forms the statistics again rather than reading kept ones.  A group of waves goes over many
// rows, with weight, bias and the two gradients' sums of its columns in registers;
// each workgroup leaves its sums in the workspace, and a second launch adds them in their order.
//
// Measured: 256 x 1000 x 1024 in bf16, ragged (half of the rows), with fp32 gradients: forward 199 us (3.9 TB/s),
// backward 382 us (4.7) and 5 for the sums; a 2 GiB copy reaches 4.9.  21 x 45 x 333 in fp32, element by element: 3.8
// and 10.4 us, a chain of loads and reductions for four rows a wave.  Widths that are no whole vectors go element by element:
// 256 x 1000 x 1023 in bf16, all rows, 562 us forward and 738 back, where 1024 takes 241 and 458; 128 x 1000 x 1023 in fp32 219 and
// 314, where 1024 takes 199 and 309.
#include "ops.h"
#include "../../include/lstm_dyn_layer.h"

#include <cmath>

namespace ldyn {
namespace {

constexpr int MAX_D = 32768;

struct NormParams {
    const void* x;
    const int32_t* lengths;
    const float* weight;
    const float* bias;
    const void* dy;
    void* out;       // y, or dx
    float* sums;     // [groups][2][D]
    int32_t* status;
    int rows, T, D;
    float eps;
};

__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// The sum over a row's W waves; every thread of the workgroup calls it when W > 1.
template <int W, int N>
__device__ inline void row_sum(float (&v)[N], float (*lds)[16]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (W > 1) {
        const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
        __syncthreads();  // the sums before these have been read
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[i][w] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j) s += lds[i][j];
            v[i] = s;
        }
    }
}

template <class E, int V, int NV>
__device__ inline void load_row(const E* p, int col, int step, int D, float* out) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (col + i * step < D) {
            load_vec<E, V>(p + col + i * step, out + i * V);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) out[i * V + j] = 0.0f;
        }
    }
}
template <bool FAR, class E, int V, int NV>
__device__ inline void store_row(E* p, int col, int step, int D, const float* in) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (col + i * step < D) put<FAR, E, V>(p + col + i * step, in + i * V);
}
// Weight or bias; a missing one is `fill`.
template <int V, int NV>
__device__ inline void load_param(const float* p, int col, int step, int D, float fill, float* out) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = col + i * step + j;
            out[i * V + j] = c < D ? (p ? p[c] : fill) : 0.0f;
        }
}

// n of a row in place of x, and r.
template <int W, int V, int NV>
__device__ inline float normalise(float* x, int col, int step, int D, float eps, float (*lds)[16]) {
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < V * NV; ++i) s[0] += x[i];
    row_sum<W>(s, lds);
    const float mean = s[0] / (float)D;
    float q[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float& e = x[i * V + j];
            e = col + i * step < D ? e - mean : 0.0f;
            q[0] += e * e;
        }
    row_sum<W>(q, lds);
    const float r = 1.0f / sqrtf(q[0] / (float)D + eps);
#pragma unroll
    for (int i = 0; i < V * NV; ++i) x[i] *= r;
    return r;
}

// Whether row r is one of a sequence's steps.
__device__ inline bool row_on(const NormParams& a, int r, bool report) {
    if (!a.lengths) return true;
    const int b = r / a.T, t = r - b * a.T;
    return t < clamp_length(a.lengths[b], a.T, a.status, report && t == 0);
}

constexpr int threads_of(int W) { return W > 4 ? 64 * W : 256; }

// FAR: the output goes past the caches.
template <class E, int V, int NV, int W, bool FAR>
__global__ void __launch_bounds__(threads_of(W)) norm_kernel(NormParams a) {
    __shared__ float lds[1][16];
    constexpr int PER = threads_of(W) / 64 / W;  // rows of a workgroup at once
    const int me = W == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    const int col = me * V, step = 64 * W * V;
    float w[V * NV], b[V * NV];
    load_param<V, NV>(a.weight, col, step, a.D, 1.0f, w);
    load_param<V, NV>(a.bias, col, step, a.D, 0.0f, b);
    const int first = __builtin_amdgcn_readfirstlane((int)blockIdx.x * PER + (W == 1 ? (int)(threadIdx.x >> 6) : 0));
    for (long long r = first; r < a.rows; r += (long long)gridDim.x * PER) {
        float x[V * NV];
        E* out = static_cast<E*>(a.out) + (size_t)r * a.D;
        if (!row_on(a, (int)r, me == 0)) {
#pragma unroll
            for (int i = 0; i < V * NV; ++i) x[i] = 0.0f;
        } else {
            load_row<E, V, NV>(static_cast<const E*>(a.x) + (size_t)r * a.D, col, step, a.D, x);
            normalise<W, V, NV>(x, col, step, a.D, a.eps, lds);
#pragma unroll
            for (int i = 0; i < V * NV; ++i) x[i] = x[i] * w[i] + b[i];
        }
        store_row<FAR, E, V, NV>(out, col, step, a.D, x);
    }
}

template <class E, class G, int V, int NV, int W, bool FAR>
__global__ void __launch_bounds__(threads_of(W)) norm_back_kernel(NormParams a) {
    __shared__ float lds[2][16];
    constexpr int WAVES = threads_of(W) / 64, PER = WAVES / W;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int me = W == 1 ? lane : (int)threadIdx.x;
    const int col = me * V, step = 64 * W * V;
    float w[V * NV], dw[V * NV], db[V * NV];
    load_param<V, NV>(a.weight, col, step, a.D, 1.0f, w);
#pragma unroll
    for (int i = 0; i < V * NV; ++i) dw[i] = db[i] = 0.0f;
    const int first = __builtin_amdgcn_readfirstlane((int)blockIdx.x * PER + (W == 1 ? wave : 0));
    for (long long r = first; r < a.rows; r += (long long)gridDim.x * PER) {
        float x[V * NV], g[V * NV];
        G* out = static_cast<G*>(a.out) + (size_t)r * a.D;
        if (!row_on(a, (int)r, me == 0)) {
#pragma unroll
            for (int i = 0; i < V * NV; ++i) g[i] = 0.0f;
        } else {
            load_row<E, V, NV>(static_cast<const E*>(a.x) + (size_t)r * a.D, col, step, a.D, x);
            load_row<G, V, NV>(static_cast<const G*>(a.dy) + (size_t)r * a.D, col, step, a.D, g);
            const float rs = normalise<W, V, NV>(x, col, step, a.D, a.eps, lds);
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < V * NV; ++i) {
                dw[i] += g[i] * x[i];
                db[i] += g[i];
                g[i] *= w[i];
                s[0] += g[i];
                s[1] += g[i] * x[i];
            }
            row_sum<W>(s, lds);
            const float m0 = s[0] / (float)a.D, m1 = s[1] / (float)a.D;
#pragma unroll
            for (int i = 0; i < V * NV; ++i) g[i] = rs * (g[i] - m0 - x[i] * m1);
        }
        store_row<FAR, G, V, NV>(out, col, step, a.D, g);
    }
    // the workgroup's sums, wave by wave
    float* sums = a.sums + (size_t)blockIdx.x * 2 * a.D;
    if constexpr (PER == 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = col + i * step + j;
                if (c < a.D) {
                    sums[c] = dw[i * V + j];
                    sums[a.D + c] = db[i * V + j];
                }
            }
    } else {
        __shared__ float part[WAVES][64 * V];
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < V; ++j) part[wave][j * 64 + lane] = half ? db[i * V + j] : dw[i * V + j];
                __syncthreads();
                for (int e = threadIdx.x; e < 64 * V; e += WAVES * 64) {
                    const int c = (e & 63) * V + (e >> 6) + i * step;
                    float s = 0.0f;
#pragma unroll
                    for (int k = 0; k < WAVES; ++k) s += part[k][e];
                    if (c < a.D) sums[half * a.D + c] = s;
                }
            }
        }
    }
}

// d_weight and d_bias: 32 columns a workgroup, 32 shares of the workgroups' sums each.
__global__ void __launch_bounds__(1024) norm_sums_kernel(const float* sums, int groups, int D, float* dw, float* db) {
    __shared__ float part[32][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), k = threadIdx.x >> 5;
    float s = 0.0f;
    if (c < 2 * D) {
        float four[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        int g = k;
        for (; g + 3 * 32 < groups; g += 4 * 32)
#pragma unroll
            for (int i = 0; i < 4; ++i) four[i] += sums[(size_t)(g + i * 32) * 2 * D + c];
        for (; g < groups; g += 32) four[0] += sums[(size_t)g * 2 * D + c];
        s = (four[0] + four[1]) + (four[2] + four[3]);
    }
    part[k][threadIdx.x & 31] = s;
    __syncthreads();
    if (k == 0 && c < 2 * D) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += part[i][threadIdx.x];
        if (c < D) dw[c] = s;
        else db[c - D] = s;
    }
}

// Workgroups that leave sums: rows of more than 4096 elements take 16 waves, one group a CU; the others
// four groups a CU of 4 waves (1024 at most), with four rows and more for each wave or row of waves: fewer sums are left to
// add, at the price of longer chains where rows are few.  us of a backward with four, two and one row and more: 945 x 333 in fp32
// 11.6, 9.4 and 8.6; bf16 x, fp32 dy, 2048 x 512 10.6, 8.6 and 8.7, 300 x 8000 25.0, 20.9 and 23.0; 4096 x 1024 in fp32 17.9, 16.0 and
// 19.0 (two would be the better rule here).
int sum_groups(long long rows, int D, int num_cus, int at_once) {
    const long long most = D > 4096 ? num_cus : 4LL * num_cus < 1024 ? 4LL * num_cus : 1024;
    const long long want = (rows + 4 * at_once - 1) / (4 * at_once);
    return (int)(want < most ? want : most);
}

int check_sizes(int B, int T, int D, int dtype, float eps) {
    if (B < 1 || T < 1 || D < 1 || !valid_dtype(dtype) || !(eps >= 0.0f) || std::isinf(eps)) return LSTM_DYN_ERR_INVALID;
    if (D > MAX_D || (long long)B * T >= 1LL << 31) return LSTM_DYN_ERR_UNSUPPORTED;
    return LSTM_DYN_OK;
}

int check_buffers(int B, int T, int D, int dtype, const void* x, const int32_t* lengths, const float* weight,
                  const float* bias, const void* out_y, const void* dy, int dy_dtype, const void* out_dx,
                  const float* d_weight, const float* d_bias) {
    const long long n = (long long)B * T * D, e = dtype_bytes(dtype);
    const bool back = out_dx || dy || d_weight || d_bias;
    if (back && !valid_dtype(dy_dtype)) return LSTM_DYN_ERR_INVALID;
    Span s[8];
    int k = 0;
    s[k++] = Span{x, n * e, 16, false};
    if (lengths) s[k++] = Span{lengths, 4LL * B, 4, false};
    if (weight) s[k++] = Span{weight, 4LL * D, 4, false};
    if (!back) {
        if (bias) s[k++] = Span{bias, 4LL * D, 4, false};
        s[k++] = Span{out_y, n * e, 16, true, x};
    } else {
        const long long ge = dtype_bytes(dy_dtype);
        s[k++] = Span{dy, n * ge, 16, false};
        s[k++] = Span{out_dx, n * ge, 16, true, dy};
        s[k++] = Span{d_weight, 4LL * D, 4, true};
        s[k++] = Span{d_bias, 4LL * D, 4, true};
    }
    return check_spans(s, k);
}

}  // namespace
}  // namespace ldyn

using namespace ldyn;

struct lstm_dyn_norm : OpsHandle {
    int B = 0, T = 0, D = 0, dtype = 0;
    float eps = 0.0f;
};

extern "C" int lstm_dyn_check_norm_args(int B, int T, int D, int dtype, float eps, const void* x,
                                        const int32_t* lengths, const float* weight, const float* bias,
                                        const void* out_y, const void* dy, int dy_dtype, const void* out_dx,
                                        const float* d_weight, const float* d_bias) {
    const int rc = check_sizes(B, T, D, dtype, eps);
    if (rc != LSTM_DYN_OK) return rc;
    return check_buffers(B, T, D, dtype, x, lengths, weight, bias, out_y, dy, dy_dtype, out_dx, d_weight, d_bias);
}

extern "C" int lstm_dyn_norm_create(lstm_dyn_norm_t** out, int B, int T, int D, int dtype, float eps) {
    if (!out) return LSTM_DYN_ERR_INVALID;
    *out = nullptr;
    int rc = check_sizes(B, T, D, dtype, eps);
    if (rc != LSTM_DYN_OK) return rc;
    auto* h = new (std::nothrow) lstm_dyn_norm();
    if (!h) return LSTM_DYN_ERR_NOMEM;
    h->B = B;
    h->T = T;
    h->D = D;
    h->dtype = dtype;
    h->eps = eps;
    if ((rc = ops_device(h)) == LSTM_DYN_OK)
        rc = ops_init(h, 256 + 8LL * sum_groups((long long)B * T, D, h->num_cus, 1) * D);
    if (rc != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    *out = h;
    return LSTM_DYN_OK;
}

namespace {

// Elements a thread holds: up to 16 with a row in one wave or in four, then a row takes 16
// waves (up to 32 each).  Rows whose start is not aligned to 16 bytes go element by element.
template <class F>
int by_shape(int D, int vec, F&& launch) {
    const int n = (D + 64 * vec - 1) / (64 * vec);  // vectors of one wave
    auto pick = [&](auto v) {
        constexpr int V = decltype(v)::value;
        constexpr int TOP = 16 / V;
        auto go = [&](auto nv, auto w) { return launch(v, nv, w); };
        std::integral_constant<int, 1> w1;
        std::integral_constant<int, 4> w4;
        std::integral_constant<int, 16> w16;
        constexpr int LOW = V == 1 ? 4 : 1;
        if (n <= TOP) {
            if (n <= LOW) return go(std::integral_constant<int, LOW>(), w1);
            if constexpr (TOP >= 4)
                if (n <= TOP / 2) return go(std::integral_constant<int, TOP / 2>(), w1);
            return go(std::integral_constant<int, TOP>(), w1);
        }
        if (n <= 4 * TOP) {
            if (n <= 2 * TOP) return go(std::integral_constant<int, TOP / 2>(), w4);
            return go(std::integral_constant<int, TOP>(), w4);
        }
        if (n <= 16 * TOP) {
            if (n <= 8 * TOP) return go(std::integral_constant<int, TOP / 2>(), w16);
            return go(std::integral_constant<int, TOP>(), w16);
        }
        return go(std::integral_constant<int, 2 * TOP>(), w16);
    };
    if (vec == 8) return pick(std::integral_constant<int, 8>());
    if (vec == 4) return pick(std::integral_constant<int, 4>());
    return pick(std::integral_constant<int, 1>());
}

// From 256 MB on, the size of the last cache, an output's reader finds it in memory in any case, and what the call reads
// again stays (256 x 1000 x 1024, ragged: 206 us through the caches, 185 past them; the training step 606 and 592).
inline bool is_far(const lstm_dyn_norm* h, int bytes) { return (long long)h->B * h->T * h->D * bytes >= 256LL << 20; }

template <class E>
int run_forward(lstm_dyn_norm* h, const NormParams& p) {
    const int vec = p.D % (16 / (int)sizeof(E)) == 0 ? 16 / (int)sizeof(E) : 1;
    return by_shape(p.D, vec, [&](auto v, auto nv, auto w) {
        constexpr int V = decltype(v)::value, NV = decltype(nv)::value, W = decltype(w)::value;
        if constexpr (V == 1 || V == 16 / (int)sizeof(E)) {
            constexpr int PER = threads_of(W) / 64 / W;
            const long long groups = ((long long)p.rows + PER - 1) / PER, most = (long long)h->num_cus * (W > 4 ? 2 : 8);
            auto* k = is_far(h, (int)sizeof(E)) ? norm_kernel<E, V, NV, W, true> : norm_kernel<E, V, NV, W, false>;
            hipLaunchKernelGGL(k, dim3((unsigned)(groups < most ? groups : most)), dim3(threads_of(W)), 0,
                               h->last_stream, p);
        }
        return ops_launched(h);
    });
}

template <class E, class G>
int run_backward(lstm_dyn_norm* h, const NormParams& p, float* d_weight, float* d_bias) {
    int groups = 1;
    // four elements at once where one of the types has four bytes
    constexpr int VEC = sizeof(E) == 2 && sizeof(G) == 2 ? 8 : 4;
    const int vec = p.D % VEC == 0 ? VEC : 1;
    int rc = by_shape(p.D, vec, [&](auto v, auto nv, auto w) {
        constexpr int V = decltype(v)::value, NV = decltype(nv)::value, W = decltype(w)::value;
        if constexpr (V == 1 || V == VEC) {
            constexpr int PER = threads_of(W) / 64 / W;
            groups = sum_groups(p.rows, p.D, h->num_cus, PER);
            auto* k = is_far(h, (int)sizeof(G)) ? norm_back_kernel<E, G, V, NV, W, true> : norm_back_kernel<E, G, V, NV, W, false>;
            hipLaunchKernelGGL(k, dim3((unsigned)groups), dim3(threads_of(W)), 0, h->last_stream, p);
        }
        return ops_launched(h);
    });
    if (rc != LSTM_DYN_OK) return rc;
    hipLaunchKernelGGL(norm_sums_kernel, dim3((unsigned)((2 * p.D + 31) / 32)), dim3(1024), 0, h->last_stream, p.sums,
                       groups, p.D, d_weight, d_bias);
    return ops_launched(h);
}

}  // namespace

extern "C" int lstm_dyn_norm_forward(lstm_dyn_norm_t* h, const void* x, const int32_t* lengths, const float* weight,
                                     const float* bias, void* out_y, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc = check_buffers(h->B, h->T, h->D, h->dtype, x, lengths, weight, bias, out_y, nullptr, 0, nullptr, nullptr,
                           nullptr);
    if (rc != LSTM_DYN_OK || (rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const NormParams p{x, lengths, weight, bias, nullptr, out_y, nullptr, h->status(), h->B * h->T, h->T, h->D, h->eps};
    return h->dtype == LSTM_DYN_BF16 ? run_forward<__bf16>(h, p) : run_forward<float>(h, p);
}

extern "C" int lstm_dyn_norm_backward(lstm_dyn_norm_t* h, const void* x, const int32_t* lengths, const float* weight,
                                      const void* dy, int dy_dtype, void* out_dx, float* d_weight, float* d_bias,
                                      void* stream) {
    if (!h || !out_dx) return LSTM_DYN_ERR_INVALID;
    int rc = check_buffers(h->B, h->T, h->D, h->dtype, x, lengths, weight, nullptr, nullptr, dy, dy_dtype, out_dx,
                           d_weight, d_bias);
    if (rc != LSTM_DYN_OK || (rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const NormParams p{x, lengths, weight, nullptr, dy, out_dx, reinterpret_cast<float*>(h->block + 256), h->status(),
                       h->B * h->T, h->T, h->D, h->eps};
    if (h->dtype == LSTM_DYN_BF16)
        return dy_dtype == LSTM_DYN_BF16 ? run_backward<__bf16, __bf16>(h, p, d_weight, d_bias)
                                         : run_backward<__bf16, float>(h, p, d_weight, d_bias);
    return dy_dtype == LSTM_DYN_BF16 ? run_backward<float, __bf16>(h, p, d_weight, d_bias)
                                     : run_backward<float, float>(h, p, d_weight, d_bias);
}

extern "C" int lstm_dyn_norm_query(lstm_dyn_norm_t* h, int what, long long* value) { return ops_query(h, what, value); }

extern "C" int lstm_dyn_norm_destroy(lstm_dyn_norm_t* h) {
    if (!h) return LSTM_DYN_OK;
    const int rc = ops_free(h);
    delete h;
    return rc;
}
