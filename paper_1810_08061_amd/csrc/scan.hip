// scan.hip -- the gated linear recurrence over whole sequences and its
// backward pass.
//
//   a_t = sigmoid(zf_t), k_t = 1 - a_t = sigmoid(-zf_t), s_t = sigmoid(zo_t)
//   h_t = h_{t-1} + k_t (v_t - h_{t-1}),   y_t = s_t h_t
// and back, with e_t the gradient of h_t from later steps (e_{L-1} = d_out_h):
//   g_t = s_t dy_t + e_t,   e_{t-1} = a_t g_t
//   dzf = g_t (h_{t-1} - v_t) a_t k_t,   dzv = g_t k_t,   dzo = dy_t h_t s_t (1 - s_t)
//
// The simple form: one thread per row and channel, step by step.
#include "ops.h"

namespace ldyn {
namespace {

constexpr int RUN = 16;  // steps between two kept states

// sigmoid(z) and sigmoid(-z), each to its own relative accuracy.
__device__ inline void sigmoid_both(float z, float& pos, float& neg) {
    const float e = __expf(-fabsf(z));
    const float r = rcp_f(1.0f + e), q = e * r;
    pos = z >= 0.0f ? r : q;
    neg = z >= 0.0f ? q : r;
    if (z != z) pos = neg = z;
}

struct ScanParams {
    const void* z;
    const int32_t* lengths;
    const float* h0;
    float* out_h;
    void* y;
    float* kept;  // [B][ceil(T / RUN)][H] the state each run of steps starts from, or null
    const void* dy;
    const float* d_out_h;
    void* dz;
    float* dh0;
    int32_t* status;
    int B, T, H;
};

template <class E>
__global__ void __launch_bounds__(64) scan_forward_simple(ScanParams p) {
    const long i = blockIdx.x * 64L + threadIdx.x;
    if (i >= (long)p.B * p.H) return;
    const int b = (int)(i / p.H), c = (int)(i - (long)b * p.H), H = p.H, T = p.T;
    const int L = row_length(p.lengths, b, T, p.status, c == 0);
    const E* z = static_cast<const E*>(p.z) + (long)b * T * 3 * H + c;
    E* y = static_cast<E*>(p.y) + (long)b * T * H + c;
    float h = p.h0[i];
    for (int t = 0; t < T; ++t) {
        if (t >= L) {
            y[(long)t * H] = (E)0.0f;
            continue;
        }
        if (p.kept && t % RUN == 0) p.kept[((long)b * ((T + RUN - 1) / RUN) + t / RUN) * H + c] = h;
        const E* zt = z + (long)t * 3 * H;
        float a, k, s, ns;
        sigmoid_both((float)zt[0], a, k);
        sigmoid_both((float)zt[2 * H], s, ns);
        h = fmaf(k, (float)zt[H] - h, h);
        y[(long)t * H] = (E)(s * h);
    }
    p.out_h[i] = h;
}

template <class E>
__global__ void __launch_bounds__(64) scan_backward_simple(ScanParams p) {
    const long i = blockIdx.x * 64L + threadIdx.x;
    if (i >= (long)p.B * p.H) return;
    const int b = (int)(i / p.H), c = (int)(i - (long)b * p.H), H = p.H, T = p.T;
    const int L = row_length(p.lengths, b, T, p.status, c == 0);
    const E* z = static_cast<const E*>(p.z) + (long)b * T * 3 * H + c;
    const E* dy = static_cast<const E*>(p.dy) + (long)b * T * H + c;
    E* dz = static_cast<E*>(p.dz) + (long)b * T * 3 * H + c;
    for (int t = L; t < T; ++t)
        for (int j = 0; j < 3; ++j) dz[((long)t * 3 + j) * H] = (E)0.0f;
    float e = p.d_out_h ? p.d_out_h[i] : 0.0f;
    for (int r = (L + RUN - 1) / RUN - 1; r >= 0; --r) {
        float hs[RUN + 1];
        hs[0] = p.kept[((long)b * ((T + RUN - 1) / RUN) + r) * H + c];
        const int n = min(RUN, L - r * RUN);
        for (int j = 0; j < n; ++j) {
            const E* zt = z + (long)(r * RUN + j) * 3 * H;
            float a, k;
            sigmoid_both((float)zt[0], a, k);
            hs[j + 1] = fmaf(k, (float)zt[H] - hs[j], hs[j]);
        }
        for (int j = n - 1; j >= 0; --j) {
            const long t = r * RUN + j;
            const E* zt = z + t * 3 * H;
            float a, k, s, ns;
            sigmoid_both((float)zt[0], a, k);
            sigmoid_both((float)zt[2 * H], s, ns);
            const float d = (float)dy[t * H], g = fmaf(s, d, e);
            E* dzt = dz + t * 3 * H;
            dzt[0] = (E)(g * (hs[j] - (float)zt[H]) * a * k);
            dzt[H] = (E)(g * k);
            dzt[2 * H] = (E)(d * hs[j + 1] * s * ns);
            e = a * g;
        }
    }
    p.dh0[i] = e;
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
        float a, k, so, ns;
        sigmoid_both(f[j], a, k);
        sigmoid_both(o[j], so, ns);
        s[j] = fmaf(k, v[j] - s[j], s[j]);
        out[j] = so * s[j];
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
    float* kept = nullptr;  // made by the first forward for training
    bool has_kept = false;
};

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
    if ((rc = ops_init(h, 256)) != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
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
        const long long n = 4LL * h->B * ((h->T + RUN - 1) / RUN) * h->H;
        if (hipMalloc(&p, (size_t)n) != hipSuccess) {
            (void)hipGetLastError();
            return LSTM_DYN_ERR_NOMEM;
        }
        h->kept = static_cast<float*>(p);
        h->bytes += n;
    }
    ScanParams p{z, lengths, h0, out_h, out_y, train ? h->kept : nullptr, nullptr, nullptr, nullptr,
                 nullptr, h->status(), h->B, h->T, h->H};
    const unsigned grid = (unsigned)(((long)h->B * h->H + 63) / 64);
    auto* k = h->dtype == LSTM_DYN_BF16 ? scan_forward_simple<__bf16> : scan_forward_simple<float>;
    hipLaunchKernelGGL(k, dim3(grid), dim3(64), 0, h->last_stream, p);
    if ((rc = ops_launched(h)) == LSTM_DYN_OK) h->has_kept = train;
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
    ScanParams p{z, lengths, h0, nullptr, nullptr, h->kept, dy, d_out_h, dz, dh0, h->status(), h->B,
                 h->T, h->H};
    const unsigned grid = (unsigned)(((long)h->B * h->H + 63) / 64);
    auto* k = h->dtype == LSTM_DYN_BF16 ? scan_backward_simple<__bf16> : scan_backward_simple<float>;
    hipLaunchKernelGGL(k, dim3(grid), dim3(64), 0, h->last_stream, p);
    return ops_launched(h);
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
