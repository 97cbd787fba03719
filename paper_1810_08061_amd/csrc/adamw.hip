// adamw.hip -- one AdamW step over all tensors of a model, states in 32 bits
// or in 8.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p - lr (m c1 / (sqrt(v) sqrt(c2) + eps) + wd p),  c1 = 1/(1 - b1^t), c2 = 1/(1 - b2^t)
//
// 8 bits: m and r = sqrt(v) in e4m3 with one power of two per 256 elements.
// One wave holds such a block, four elements a lane, so the block's largest
// magnitudes are two reductions over the wave and the old and the new codes
// are read and written once.  r instead of v: e4m3 with a power of two per
// block spans 2^18, which v would need twice over.
//
// Bound by memory: 28 bytes an element with states in 32 bits, 16 with 8, 2 more with
// a bf16 copy.  159 M elements, 8 bits and copies: 570 us (5.0 TB/s), their states'
// values 175 us (5.4 TB/s); 2.9 M elements, 32 bits: 15 us (5.3 TB/s).
//
// One launch for up to 256 tensors: a workgroup takes CHUNK elements of one
// tensor, found in a table made at create.  The gradients' addresses come with
// the launch, since a program may have its gradients elsewhere in every step.
#include "ops.h"

#include <algorithm>
#include <cmath>
#include <vector>

namespace ldyn {
namespace {

constexpr int BLOCK = 256;    // elements that share an exponent
constexpr int CHUNK = 4096;   // elements per workgroup
constexpr int GROUP = 256;    // tensors per launch

struct Tensor {
    float* p;
    __bf16* p16;
    void* m;
    void* v;
    uint8_t* me;
    uint8_t* ve;
    long long n;
    float wd;
    uint32_t first;    // its first chunk
    int32_t aligned;   // p, m, v and p16 take four elements at once
};

struct Grads {
    const void* g[GROUP];
};
struct Values {
    __bf16* m[GROUP / 2];
    __bf16* v[GROUP / 2];
};

struct AdamwParams {
    const Tensor* tensors;
    const uint32_t* owner;   // [chunks] the chunk's tensor
    uint32_t chunk0;
    int tensor0;
    float lr, b1, nb1, b2, nb2, eps, gs, c1, rc2;  // nb = 1 - b, rounded once
};

template <class E>
__device__ inline void load4(const E* p, int n, bool vec, float* out) {
    if (vec && n >= 4) {
        load_vec<E, 4>(p, out);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = i < n ? (float)p[i] : 0.0f;
    }
}
template <class E>
__device__ inline void store4(E* p, int n, bool vec, const float* in) {
    if (vec && n >= 4) {
        store_vec<E, 4>(p, in);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (E)in[i];
    }
}
__device__ inline uint32_t load_codes(const uint8_t* p, int n, bool vec) {
    if (vec && n >= 4) return *reinterpret_cast<const uint32_t*>(p);
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) c |= (uint32_t)p[i] << (8 * i);
    return c;
}
__device__ inline void store_codes(uint8_t* p, int n, bool vec, uint32_t c) {
    if (vec && n >= 4) {
        *reinterpret_cast<uint32_t*>(p) = c;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (uint8_t)(c >> (8 * i));
    }
}

__device__ inline float pow2_of(int biased) { return __int_as_float(biased << 23); }

typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ inline void from_codes(uint32_t c, float scale, float* out) {
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
    const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    out[0] = lo[0] * scale;
    out[1] = lo[1] * scale;
    out[2] = hi[0] * scale;
    out[3] = hi[1] * scale;
}

// The codes of a wave's 256 values and their exponent (biased by 127).  UP:
// a positive value is not rounded to zero.
template <bool UP>
__device__ inline uint32_t to_codes(const float* x, int* biased) {
    float mx = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = fabsf(x[i]);
        mx = a < __builtin_inff() ? fmaxf(mx, a) : mx;  // neither an infinity nor a NaN
    }
    for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    const uint32_t u = __float_as_uint(mx);
    // 448 = 1.75 2^8: mx = f 2^(E - 127) needs 2^(E - 135), or twice that for f > 1.75
    int e = (int)(u >> 23) - 135 + ((u & 0x7fffff) > 0x600000);
    e = e < -100 ? -100 : e;
    *biased = e + 127;
    const float inv = pow2_of(127 - e);
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        q[i] = x[i] * inv;
        if (UP && q[i] > 0.0f) q[i] = fmaxf(q[i], 0x1p-9f);
        if (!(fabsf(q[i]) <= 448.0f)) q[i] = __builtin_nanf("");
    }
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], c, true);
}

template <bool EIGHT, class G>
__global__ void __launch_bounds__(256) adamw_kernel(AdamwParams a, Grads grads) {
    const uint32_t chunk = a.chunk0 + blockIdx.x;
    const int ti = (int)a.owner[chunk];
    const Tensor t = a.tensors[ti];
    const G* g = static_cast<const G*>(grads.g[ti - a.tensor0]);
    const bool gvec = (reinterpret_cast<uintptr_t>(g) & (4 * sizeof(G) - 1)) == 0;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const long long base = (long long)(chunk - t.first) * CHUNK;
    for (int j = w; j < CHUNK / BLOCK; j += 4) {
        const long long b0 = base + j * BLOCK;
        if (b0 >= t.n) return;  // the whole wave
        const long long at = b0 + 4 * lane;
        const int n = (int)min(4LL, max(0LL, t.n - at));
        float p[4], gr[4], m[4], v[4];
        load4<float>(t.p + at, n, t.aligned, p);
        load4<G>(g + at, n, gvec, gr);
        if constexpr (EIGHT) {
            const uint32_t cm = load_codes(static_cast<const uint8_t*>(t.m) + at, n, t.aligned);
            const uint32_t cv = load_codes(static_cast<const uint8_t*>(t.v) + at, n, t.aligned);
            from_codes(cm, pow2_of(t.me[b0 / BLOCK]), m);
            from_codes(cv, pow2_of(t.ve[b0 / BLOCK]), v);
        } else {
            load4<float>(static_cast<const float*>(t.m) + at, n, t.aligned, m);
            load4<float>(static_cast<const float*>(t.v) + at, n, t.aligned, v);
        }
        float r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // Every product and sum is rounded by itself (no fused multiply-add),
            // so the same formula in plain fp32 gives the same codes.
#pragma clang fp contract(off)
            const float gi = gr[i] * a.gs;
            m[i] = a.b1 * m[i] + a.nb1 * gi;
            if constexpr (EIGHT) {
                // v[i] holds r.  Where both squares would leave fp32's range below, they are
                // formed 2^128 times larger, so that an r that is not zero stays so.
                const float up = fmaxf(v[i], fabsf(gi)) < 0x1p-60f ? 0x1p64f : 1.0f;
                const float rs = v[i] * up, gs = gi * up;
                const float sq = a.b2 * (rs * rs) + a.nb2 * gs * gs;
                r[i] = sqrtf(sq) * (up == 1.0f ? 1.0f : 0x1p-64f);
            } else {
                v[i] = a.b2 * v[i] + a.nb2 * gi * gi;
                r[i] = sqrtf(v[i]);
            }
            p[i] -= a.lr * (m[i] * a.c1 / (r[i] * a.rc2 + a.eps) + t.wd * p[i]);
        }
        store4<float>(t.p + at, n, t.aligned, p);
        if (t.p16) store4<__bf16>(t.p16 + at, n, t.aligned, p);
        if constexpr (EIGHT) {
            int em, ev;
            const uint32_t cm = to_codes<false>(m, &em), cv = to_codes<true>(r, &ev);
            store_codes(static_cast<uint8_t*>(t.m) + at, n, t.aligned, cm);
            store_codes(static_cast<uint8_t*>(t.v) + at, n, t.aligned, cv);
            if (lane == 0) {
                t.me[b0 / BLOCK] = (uint8_t)em;
                t.ve[b0 / BLOCK] = (uint8_t)ev;
            }
        } else {
            store4<float>(static_cast<float*>(t.m) + at, n, t.aligned, m);
            store4<float>(static_cast<float*>(t.v) + at, n, t.aligned, v);
        }
    }
}

// The values of the codes, as bf16: three mantissa bits times a power of two.
__global__ void __launch_bounds__(256) adamw_states_kernel(AdamwParams a, Values out) {
    const uint32_t chunk = a.chunk0 + blockIdx.x;
    const int ti = (int)a.owner[chunk];
    const Tensor t = a.tensors[ti];
    __bf16 *dm = out.m[ti - a.tensor0], *dv = out.v[ti - a.tensor0];
    const bool vec = ((reinterpret_cast<uintptr_t>(dm) | reinterpret_cast<uintptr_t>(dv)) & 7) == 0;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const long long base = (long long)(chunk - t.first) * CHUNK;
    for (int j = w; j < CHUNK / BLOCK; j += 4) {
        const long long b0 = base + j * BLOCK;
        if (b0 >= t.n) return;
        const long long at = b0 + 4 * lane;
        const int n = (int)min(4LL, max(0LL, t.n - at));
        float m[4], r[4];
        from_codes(load_codes(static_cast<const uint8_t*>(t.m) + at, n, t.aligned), pow2_of(t.me[b0 / BLOCK]), m);
        from_codes(load_codes(static_cast<const uint8_t*>(t.v) + at, n, t.aligned), pow2_of(t.ve[b0 / BLOCK]), r);
        store4<__bf16>(dm + at, n, vec, m);
        store4<__bf16>(dv + at, n, vec, r);
    }
}

bool is_aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

struct Range {
    uintptr_t lo, hi;
};

// The written buffers of all tensors in order of address; false if two overlap.
bool written_ranges(const lstm_dyn_adamw_tensor_t* t, int count, int bits, std::vector<Range>* out) {
    const long long e = bits == 8 ? 1 : 4;
    for (int i = 0; i < count; ++i) {
        const long long n = t[i].n, nb = (n + BLOCK - 1) / BLOCK;
        auto add = [&](const void* p, long long bytes) {
            const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
            if (p && bytes) out->push_back(Range{lo, lo + (uintptr_t)bytes});
        };
        add(t[i].p, 4 * n);
        add(t[i].p_bf16, 2 * n);
        add(t[i].m, e * n);
        add(t[i].v, e * n);
        if (bits == 8) {
            add(t[i].m_exp, nb);
            add(t[i].v_exp, nb);
        }
    }
    std::sort(out->begin(), out->end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
    for (size_t i = 1; i < out->size(); ++i)
        if ((*out)[i].lo < (*out)[i - 1].hi) return false;
    return true;
}

bool on_written(const std::vector<Range>& w, const void* p, long long bytes) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p), hi = lo + (uintptr_t)bytes;
    auto it = std::upper_bound(w.begin(), w.end(), lo, [](uintptr_t x, const Range& r) { return x < r.hi; });
    return it != w.end() && it->lo < hi;
}

int check_tensors(const lstm_dyn_adamw_tensor_t* t, int count, int bits, std::vector<Range>* w) {
    if (!t || count < 1 || (bits != 32 && bits != 8)) return LSTM_DYN_ERR_INVALID;
    long long chunks = 0;
    for (int i = 0; i < count; ++i) {
        const lstm_dyn_adamw_tensor_t& x = t[i];
        if (x.n < 0 || x.weight_decay != x.weight_decay) return LSTM_DYN_ERR_INVALID;
        if (x.n == 0) continue;
        if (x.n >= 1LL << 40) return LSTM_DYN_ERR_UNSUPPORTED;
        chunks += (x.n + CHUNK - 1) / CHUNK;
        if (!x.p || !x.m || !x.v || !is_aligned(x.p, 4) || !is_aligned(x.p_bf16, 2)) return LSTM_DYN_ERR_INVALID;
        if (bits == 32 && (!is_aligned(x.m, 4) || !is_aligned(x.v, 4))) return LSTM_DYN_ERR_INVALID;
        if (bits == 8 && (!x.m_exp || !x.v_exp)) return LSTM_DYN_ERR_INVALID;
    }
    if (chunks >= 1LL << 24) return LSTM_DYN_ERR_UNSUPPORTED;  // 2^36 elements
    return written_ranges(t, count, bits, w) ? LSTM_DYN_OK : LSTM_DYN_ERR_INVALID;
}

int check_grads(const std::vector<Range>& w, const long long* n, int count, const void* const* grads,
                int dtype) {
    if (!grads || !valid_dtype(dtype)) return LSTM_DYN_ERR_INVALID;
    const int e = dtype_bytes(dtype);
    for (int i = 0; i < count; ++i)
        if (n[i] && (!grads[i] || !is_aligned(grads[i], (uintptr_t)e) || on_written(w, grads[i], n[i] * e)))
            return LSTM_DYN_ERR_INVALID;
    return LSTM_DYN_OK;
}

}  // namespace
}  // namespace ldyn

using namespace ldyn;

struct lstm_dyn_adamw : OpsHandle {
    int bits = 0, count = 0;
    std::vector<Range> written;
    std::vector<long long> n;
    std::vector<uint32_t> first;  // [count + 1] first chunk of each tensor
    const Tensor* tensors = nullptr;
    const uint32_t* owner = nullptr;
};

extern "C" int lstm_dyn_check_adamw_args(const lstm_dyn_adamw_tensor_t* tensors, int count, int bits,
                                         const void* const* grads, int grad_dtype) {
    try {
        std::vector<Range> w;
        const int rc = check_tensors(tensors, count, bits, &w);
        if (rc != LSTM_DYN_OK || !grads) return rc;
        std::vector<long long> n((size_t)count);
        for (int i = 0; i < count; ++i) n[(size_t)i] = tensors[i].n;
        return check_grads(w, n.data(), count, grads, grad_dtype);
    } catch (...) {
        return LSTM_DYN_ERR_NOMEM;
    }
}

static int adamw_make(lstm_dyn_adamw* h, const lstm_dyn_adamw_tensor_t* t, int count, int bits) {
    int rc = check_tensors(t, count, bits, &h->written);
    if (rc != LSTM_DYN_OK) return rc;
    h->bits = bits;
    h->count = count;
    std::vector<Tensor> dev((size_t)count);
    std::vector<uint32_t> owner;
    for (int i = 0; i < count; ++i) {
        h->n.push_back(t[i].n);
        h->first.push_back((uint32_t)owner.size());
        const uintptr_t sa = bits == 8 ? 4 : 16;
        dev[(size_t)i] = Tensor{t[i].p, static_cast<__bf16*>(t[i].p_bf16), t[i].m, t[i].v, t[i].m_exp,
                                t[i].v_exp, t[i].n, t[i].weight_decay, (uint32_t)owner.size(),
                                is_aligned(t[i].p, 16) && is_aligned(t[i].m, sa) &&
                                    is_aligned(t[i].v, sa) && is_aligned(t[i].p_bf16, 8)};
        owner.insert(owner.end(), (size_t)((t[i].n + CHUNK - 1) / CHUNK), (uint32_t)i);
    }
    h->first.push_back((uint32_t)owner.size());
    const long long nt = ((long long)sizeof(Tensor) * count + 255) / 256 * 256;
    if ((rc = ops_device(h)) != LSTM_DYN_OK) return rc;
    if ((rc = ops_init(h, 256 + nt + 4LL * (long long)owner.size())) != LSTM_DYN_OK) return rc;
    h->tensors = reinterpret_cast<const Tensor*>(h->block + 256);
    h->owner = reinterpret_cast<const uint32_t*>(h->block + 256 + nt);
    if (hipMemcpy(h->block + 256, dev.data(), sizeof(Tensor) * (size_t)count, hipMemcpyHostToDevice) != hipSuccess ||
        (!owner.empty() && hipMemcpy(h->block + 256 + nt, owner.data(), 4 * owner.size(), hipMemcpyHostToDevice) != hipSuccess)) {
        (void)hipGetLastError();
        (void)ops_free(h);
        return LSTM_DYN_ERR_HIP;
    }
    return LSTM_DYN_OK;
}

extern "C" int lstm_dyn_adamw_create(lstm_dyn_adamw_t** out, const lstm_dyn_adamw_tensor_t* tensors,
                                     int count, int state_bits) {
    if (!out) return LSTM_DYN_ERR_INVALID;
    *out = nullptr;
    lstm_dyn_adamw* h = nullptr;
    try {
        h = new lstm_dyn_adamw();
        const int rc = adamw_make(h, tensors, count, state_bits);
        if (rc != LSTM_DYN_OK) {
            delete h;
            return rc;
        }
    } catch (...) {
        delete h;
        return LSTM_DYN_ERR_NOMEM;
    }
    *out = h;
    return LSTM_DYN_OK;
}

extern "C" int lstm_dyn_adamw_step(lstm_dyn_adamw_t* h, const void* const* grads, int grad_dtype,
                                   double lr, double beta1, double beta2, double eps,
                                   double grad_scale, long long step, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0 && eps >= 0.0) || lr != lr ||
        grad_scale != grad_scale || step < 1)
        return LSTM_DYN_ERR_INVALID;
    int rc = check_grads(h->written, h->n.data(), h->count, grads, grad_dtype);
    if (rc != LSTM_DYN_OK) return rc;
    if ((rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const double c1 = 1.0 / (1.0 - std::pow(beta1, (double)step));
    const double c2 = 1.0 / (1.0 - std::pow(beta2, (double)step));
    for (int i0 = 0; i0 < h->count; i0 += GROUP) {
        const int n = h->count - i0 < GROUP ? h->count - i0 : GROUP;
        const uint32_t c0 = h->first[(size_t)i0], cn = h->first[(size_t)(i0 + n)] - c0;
        if (!cn) continue;
        Grads g;
        for (int i = 0; i < GROUP; ++i) g.g[i] = i < n ? grads[i0 + i] : nullptr;
        const AdamwParams a{h->tensors, h->owner, c0, i0, (float)lr, (float)beta1, (float)(1.0 - beta1),
                            (float)beta2, (float)(1.0 - beta2), (float)eps, (float)grad_scale,
                            (float)c1, (float)std::sqrt(c2)};
        auto* k = h->bits == 8 ? (grad_dtype == LSTM_DYN_BF16 ? adamw_kernel<true, __bf16> : adamw_kernel<true, float>)
                               : (grad_dtype == LSTM_DYN_BF16 ? adamw_kernel<false, __bf16> : adamw_kernel<false, float>);
        hipLaunchKernelGGL(k, dim3(cn), dim3(256), 0, h->last_stream, a, g);
        if ((rc = ops_launched(h)) != LSTM_DYN_OK) return rc;
    }
    return LSTM_DYN_OK;
}

extern "C" int lstm_dyn_adamw_states(lstm_dyn_adamw_t* h, void* const* out_m, void* const* out_v,
                                     void* stream) {
    if (!h || !out_m || !out_v) return LSTM_DYN_ERR_INVALID;
    if (h->bits != 8) return LSTM_DYN_ERR_UNSUPPORTED;
    int rc;
    for (int i = 0; i < h->count; ++i) {
        const long long n = h->n[(size_t)i];
        if (!n) continue;
        for (const void* p : {(const void*)out_m[i], (const void*)out_v[i]})
            if (!p || !is_aligned(p, 2) || on_written(h->written, p, 2 * n)) return LSTM_DYN_ERR_INVALID;
    }
    if ((rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    for (int i0 = 0; i0 < h->count; i0 += GROUP / 2) {
        const int n = h->count - i0 < GROUP / 2 ? h->count - i0 : GROUP / 2;
        const uint32_t c0 = h->first[(size_t)i0], cn = h->first[(size_t)(i0 + n)] - c0;
        if (!cn) continue;
        Values o{};
        for (int i = 0; i < n; ++i) {
            o.m[i] = static_cast<__bf16*>(out_m[i0 + i]);
            o.v[i] = static_cast<__bf16*>(out_v[i0 + i]);
        }
        const AdamwParams a{h->tensors, h->owner, c0, i0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        hipLaunchKernelGGL(adamw_states_kernel, dim3(cn), dim3(256), 0, h->last_stream, a, o);
        if ((rc = ops_launched(h)) != LSTM_DYN_OK) return rc;
    }
    return LSTM_DYN_OK;
}

extern "C" int lstm_dyn_adamw_query(lstm_dyn_adamw_t* h, int what, long long* value) {
    return ops_query(h, what, value);
}

extern "C" int lstm_dyn_adamw_destroy(lstm_dyn_adamw_t* h) {
    if (!h) return LSTM_DYN_OK;
    const int rc = ops_free(h);
    delete h;
    return rc;
}
