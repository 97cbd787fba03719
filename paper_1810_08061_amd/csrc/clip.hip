// clip.hip -- the norm of all gradients of a model, and the gradients clipped to it.
//
//   norm = |gs| sqrt(sum g^2),  factor = gs min(1, max_norm / norm)
//
// Bound by memory: every gradient read once for the norm; once more, and written, for
// clipping.  Squares are formed and added in 64 bits (a square of two fp32 numbers is exact there, and one
// product-sum an element is far below what memory lets through), so nothing
// overflows or vanishes on the way and no scaling pass is needed.  A workgroup takes CHUNK
// elements of one tensor and leaves its sum; the sums are added in an order that the sizes
// decide, so the same call gives the same bits.  Up to FEW workgroups, as many as it has threads, the last one to end adds
// them; beyond, a launch of its own does: a counter that all count on takes 20 to 40 ns each
// (159 M elements, 9731 workgroups: 631 us so; 139 us and 5 with the launch, 4.6 TB/s).  us with the counter and with the launch: 8
// workgroups 4.4 and 4.9, 64 4.9 and 5.0, 128 6.3 and 5.0, 256 9.3 and 5.7.  2.9 M elements: 10.6 us, and 7.8 for clipping them.
//
// One launch for up to 256 tensors (128 for clipping), whose addresses come with it.
#include "ops.h"
#include "../../include/lstm_dyn_layer.h"

#include <algorithm>
#include <cmath>
#include <vector>

namespace ldyn {
namespace {

constexpr int CHUNK = 16384;  // elements per workgroup
constexpr int GROUP = 256;    // tensors per launch
constexpr int THREADS = 256;
constexpr uint32_t FEW = THREADS;  // workgroups

struct Piece {        // what a workgroup takes
    uint32_t tensor;
    uint32_t part;    // its CHUNK of the tensor
};

struct Reads {
    const void* g[GROUP];
};
struct Pairs {
    const void* g[GROUP / 2];
    void* out[GROUP / 2];
};

struct ClipParams {
    const Piece* pieces;
    const long long* n;     // elements of the tensors
    double* sums;           // one a workgroup
    uint32_t* arrived;
    float* result;
    uint32_t piece0, all;   // first workgroup of the launch; of the whole call
    uint32_t tensor0;
    double gs, max_norm;
};

__device__ inline double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
template <int WAVES>
__device__ inline double group_sum(double v, double* lds) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) v += lds[i];
    return v;
}

__device__ inline void write_result(const ClipParams& a, double sum) {
    const double norm = fabs(a.gs) * sqrt(sum);
    a.result[0] = (float)norm;
    // not (norm <= max): what is not a number goes on into the factor
    a.result[1] = (float)(norm <= a.max_norm ? a.gs : a.gs * (a.max_norm / norm));
}

template <class E>
__global__ void __launch_bounds__(THREADS) clip_norm_kernel(ClipParams a, Reads in) {
    constexpr int V = 16 / (int)sizeof(E);
    __shared__ double lds[4];
    __shared__ bool last;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    if (a.all) {
        const Piece piece = a.pieces[a.piece0 + blockIdx.x];
        const long long base = (long long)piece.part * CHUNK;
        const long long left = a.n[piece.tensor] - base;
        const int n = left < CHUNK ? (int)left : CHUNK;
        const E* g = static_cast<const E*>(in.g[piece.tensor - a.tensor0]) + base;
        if (n == CHUNK && (reinterpret_cast<uintptr_t>(g) & 15) == 0) {
#pragma unroll 8
            for (int i = 0; i < CHUNK / (V * THREADS); ++i) {
                float x[V];
                load_vec<E, V>(g + (i * THREADS + (int)threadIdx.x) * V, x);
#pragma unroll
                for (int j = 0; j < V; ++j) s[j & 3] += (double)x[j] * (double)x[j];
            }
        } else {
            for (int i = threadIdx.x; i < n; i += THREADS) {
                const double x = (double)(float)g[i];
                s[0] += x * x;
            }
        }
    }
    const double mine = group_sum<THREADS / 64>((s[0] + s[1]) + (s[2] + s[3]), lds);
    if (a.all > FEW) {
        if (threadIdx.x == 0) a.sums[a.piece0 + blockIdx.x] = mine;
        return;
    }
    if (threadIdx.x == 0) {
        last = true;
        if (a.all) {
            __hip_atomic_store(a.sums + a.piece0 + blockIdx.x, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last = __hip_atomic_fetch_add(a.arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == a.all - 1;
        }
    }
    __syncthreads();
    if (!last) return;
    double t = threadIdx.x < a.all
                   ? __hip_atomic_load(a.sums + threadIdx.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
    t = group_sum<THREADS / 64>(t, lds);
    if (threadIdx.x == 0) {
        write_result(a, t);
        __hip_atomic_store(a.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

__global__ void __launch_bounds__(1024) clip_sums_kernel(ClipParams a) {
    __shared__ double lds[16];
    double t[4] = {0.0, 0.0, 0.0, 0.0};
    uint32_t i = threadIdx.x;
    for (; i + 3 * 1024 < a.all; i += 4 * 1024)
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] += a.sums[i + k * 1024];
    for (; i < a.all; i += 1024) t[0] += a.sums[i];
    const double sum = group_sum<16>((t[0] + t[1]) + (t[2] + t[3]), lds);
    if (threadIdx.x == 0) write_result(a, sum);
}

template <class E>
__global__ void __launch_bounds__(THREADS) clip_apply_kernel(ClipParams a, Pairs io) {
    constexpr int V = 16 / (int)sizeof(E);
    const float f = a.result[1];
    const Piece piece = a.pieces[a.piece0 + blockIdx.x];
    const long long base = (long long)piece.part * CHUNK;
    const long long left = a.n[piece.tensor] - base;
    const int n = left < CHUNK ? (int)left : CHUNK;
    const E* g = static_cast<const E*>(io.g[piece.tensor - a.tensor0]) + base;
    E* out = static_cast<E*>(io.out[piece.tensor - a.tensor0]) + base;
    if (n == CHUNK && ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(out)) & 15) == 0) {
        constexpr int N = CHUNK / (V * THREADS), AT_ONCE = 4;
        for (int i = 0; i < N; i += AT_ONCE) {
            float x[AT_ONCE][V];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) load_vec<E, V>(g + ((i + k) * THREADS + (int)threadIdx.x) * V, x[k]);
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
#pragma unroll
                for (int j = 0; j < V; ++j) x[k][j] *= f;
                store_vec<E, V>(out + ((i + k) * THREADS + (int)threadIdx.x) * V, x[k]);
            }
        }
    } else {
        for (int i = threadIdx.x; i < n; i += THREADS) out[i] = (E)((float)g[i] * f);
    }
}

bool is_aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int check_counts(const long long* n, int count) {
    if (!n || count < 1) return LSTM_DYN_ERR_INVALID;
    long long pieces = 0;
    for (int i = 0; i < count; ++i) {
        if (n[i] < 0) return LSTM_DYN_ERR_INVALID;
        if (n[i] >= 1LL << 40) return LSTM_DYN_ERR_UNSUPPORTED;
        pieces += (n[i] + CHUNK - 1) / CHUNK;
        if (pieces >= 1LL << 22) return LSTM_DYN_ERR_UNSUPPORTED;  // 2^36 elements
    }
    return LSTM_DYN_OK;
}

int check_grads(const long long* n, int count, const void* const* grads, int dtype, const float* result) {
    if (!grads || !valid_dtype(dtype) || !result || !is_aligned(result, 4)) return LSTM_DYN_ERR_INVALID;
    const int e = dtype_bytes(dtype);
    const Span r{result, 8, 4, true};
    for (int i = 0; i < count; ++i)
        if (n[i] && (!grads[i] || !is_aligned(grads[i], (uintptr_t)e) ||
                     span_overlap(r, Span{grads[i], n[i] * e, e, false})))
            return LSTM_DYN_ERR_INVALID;
    return LSTM_DYN_OK;
}

// Outputs: each apart from every other buffer of the call, but for its own gradient.
int check_out(const long long* n, int count, const void* const* grads, int dtype, const float* result,
              void* const* out) {
    if (!out) return LSTM_DYN_ERR_INVALID;
    struct Range {
        uintptr_t lo, hi;
        int tensor;
        bool written;
    };
    std::vector<Range> all;
    const int e = dtype_bytes(dtype);
    const Span r{result, 8, 4, false};
    for (int i = 0; i < count; ++i) {
        if (!n[i]) continue;
        if (!out[i] || !is_aligned(out[i], (uintptr_t)e) || span_overlap(r, Span{out[i], n[i] * e, e, true}))
            return LSTM_DYN_ERR_INVALID;
        const uintptr_t g = reinterpret_cast<uintptr_t>(grads[i]), o = reinterpret_cast<uintptr_t>(out[i]);
        const uintptr_t bytes = (uintptr_t)(n[i] * e);
        all.push_back(Range{o, o + bytes, i, true});
        if (g != o) all.push_back(Range{g, g + bytes, i, false});
    }
    std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
    // a written range may not meet any other: against the furthest end so far of each kind
    uintptr_t written = 0, read = 0;
    for (const Range& x : all) {
        if (x.lo < written || (x.written && x.lo < read)) return LSTM_DYN_ERR_INVALID;
        (x.written ? written : read) = std::max(x.written ? written : read, x.hi);
    }
    return LSTM_DYN_OK;
}

}  // namespace
}  // namespace ldyn

using namespace ldyn;

struct lstm_dyn_clip : OpsHandle {
    int count = 0;
    std::vector<long long> n;
    std::vector<uint32_t> first;  // [count + 1] first workgroup of each tensor
    const Piece* pieces = nullptr;
    const long long* dev_n = nullptr;
    double* sums = nullptr;
};

extern "C" int lstm_dyn_check_clip_args(const long long* n, int count, const void* const* grads, int grad_dtype,
                                        const float* result, void* const* out) {
    try {
        int rc = check_counts(n, count);
        if (rc != LSTM_DYN_OK || (!grads && !out)) return rc;
        rc = check_grads(n, count, grads, grad_dtype, result);
        return rc != LSTM_DYN_OK || !out ? rc : check_out(n, count, grads, grad_dtype, result, out);
    } catch (...) {
        return LSTM_DYN_ERR_NOMEM;
    }
}

static int clip_make(lstm_dyn_clip* h, const long long* n, int count) {
    h->count = count;
    h->n.assign(n, n + count);
    std::vector<Piece> pieces;
    for (int i = 0; i < count; ++i) {
        h->first.push_back((uint32_t)pieces.size());
        for (long long k = 0; k < (n[i] + CHUNK - 1) / CHUNK; ++k) pieces.push_back(Piece{(uint32_t)i, (uint32_t)k});
    }
    h->first.push_back((uint32_t)pieces.size());
    int rc = ops_device(h);
    if (rc != LSTM_DYN_OK) return rc;
    const long long np = (long long)(sizeof(Piece) * pieces.size() + 255) / 256 * 256, nn = (8LL * count + 255) / 256 * 256;
    if ((rc = ops_init(h, 256 + np + nn + 8LL * (long long)(pieces.size() + 1))) != LSTM_DYN_OK) return rc;
    h->pieces = reinterpret_cast<const Piece*>(h->block + 256);
    h->dev_n = reinterpret_cast<const long long*>(h->block + 256 + np);
    h->sums = reinterpret_cast<double*>(h->block + 256 + np + nn);
    if ((!pieces.empty() && hipMemcpy(h->block + 256, pieces.data(), sizeof(Piece) * pieces.size(), hipMemcpyHostToDevice) != hipSuccess) ||
        hipMemcpy(h->block + 256 + np, n, 8 * (size_t)count, hipMemcpyHostToDevice) != hipSuccess) {
        (void)hipGetLastError();
        (void)ops_free(h);
        return LSTM_DYN_ERR_HIP;
    }
    return LSTM_DYN_OK;
}

extern "C" int lstm_dyn_clip_create(lstm_dyn_clip_t** out, const long long* n, int count) {
    if (!out) return LSTM_DYN_ERR_INVALID;
    *out = nullptr;
    const int ok = check_counts(n, count);
    if (ok != LSTM_DYN_OK) return ok;
    lstm_dyn_clip* h = nullptr;
    try {
        h = new lstm_dyn_clip();
        const int rc = clip_make(h, n, count);
        if (rc != LSTM_DYN_OK) {
            delete h;
            return rc;
        }
    } catch (...) {
        if (h) (void)ops_free(h);
        delete h;
        return LSTM_DYN_ERR_NOMEM;
    }
    *out = h;
    return LSTM_DYN_OK;
}

static ClipParams clip_params(const lstm_dyn_clip* h, float* result) {
    return ClipParams{h->pieces, h->dev_n, h->sums, reinterpret_cast<uint32_t*>(h->block + 64), result, 0,
                      h->first[(size_t)h->count], 0, 1.0, 0.0};
}

extern "C" int lstm_dyn_clip_norm(lstm_dyn_clip_t* h, const void* const* grads, int grad_dtype, double grad_scale,
                                  double max_norm, float* result, void* stream) {
    if (!h || !(max_norm >= 0.0) || !std::isfinite(grad_scale)) return LSTM_DYN_ERR_INVALID;
    int rc = check_grads(h->n.data(), h->count, grads, grad_dtype, result);
    if (rc != LSTM_DYN_OK || (rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    ClipParams a = clip_params(h, result);
    a.gs = grad_scale;
    a.max_norm = max_norm;
    auto* k = grad_dtype == LSTM_DYN_BF16 ? clip_norm_kernel<__bf16> : clip_norm_kernel<float>;
    if (!a.all) {  // nothing to add: one workgroup writes the result
        hipLaunchKernelGGL(k, dim3(1), dim3(THREADS), 0, h->last_stream, a, Reads{});
        return ops_launched(h);
    }
    for (int i0 = 0; i0 < h->count; i0 += GROUP) {
        const int n = std::min(GROUP, h->count - i0);
        const uint32_t p0 = h->first[(size_t)i0], pn = h->first[(size_t)(i0 + n)] - p0;
        if (!pn) continue;
        Reads in;
        for (int i = 0; i < GROUP; ++i) in.g[i] = i < n ? grads[i0 + i] : nullptr;
        a.piece0 = p0;
        a.tensor0 = (uint32_t)i0;
        hipLaunchKernelGGL(k, dim3(pn), dim3(THREADS), 0, h->last_stream, a, in);
        if ((rc = ops_launched(h)) != LSTM_DYN_OK) return rc;
    }
    if (a.all <= FEW) return LSTM_DYN_OK;
    hipLaunchKernelGGL(clip_sums_kernel, dim3(1), dim3(1024), 0, h->last_stream, a);
    return ops_launched(h);
}

extern "C" int lstm_dyn_clip_apply(lstm_dyn_clip_t* h, const void* const* grads, int grad_dtype, const float* result,
                                   void* const* out, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc;
    try {
        rc = check_grads(h->n.data(), h->count, grads, grad_dtype, result);
        if (rc == LSTM_DYN_OK) rc = check_out(h->n.data(), h->count, grads, grad_dtype, result, out);
    } catch (...) {
        return LSTM_DYN_ERR_NOMEM;
    }
    if (rc != LSTM_DYN_OK || (rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    ClipParams a = clip_params(h, const_cast<float*>(result));
    auto* k = grad_dtype == LSTM_DYN_BF16 ? clip_apply_kernel<__bf16> : clip_apply_kernel<float>;
    for (int i0 = 0; i0 < h->count; i0 += GROUP / 2) {
        const int n = std::min(GROUP / 2, h->count - i0);
        const uint32_t p0 = h->first[(size_t)i0], pn = h->first[(size_t)(i0 + n)] - p0;
        if (!pn) continue;
        Pairs io{};
        for (int i = 0; i < n; ++i) {
            io.g[i] = grads[i0 + i];
            io.out[i] = out[i0 + i];
        }
        a.piece0 = p0;
        a.tensor0 = (uint32_t)i0;
        hipLaunchKernelGGL(k, dim3(pn), dim3(THREADS), 0, h->last_stream, a, io);
        if ((rc = ops_launched(h)) != LSTM_DYN_OK) return rc;
    }
    return LSTM_DYN_OK;
}

extern "C" int lstm_dyn_clip_query(lstm_dyn_clip_t* h, int what, long long* value) { return ops_query(h, what, value); }

extern "C" int lstm_dyn_clip_destroy(lstm_dyn_clip_t* h) {
    if (!h) return LSTM_DYN_OK;
    const int rc = ops_free(h);
    delete h;
    return rc;
}
