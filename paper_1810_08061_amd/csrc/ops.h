// ops.h -- what the operators around the loop share: argument checks, the
// part of a handle that all of them have, vector loads and stores.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <new>

#include "../../include/lstm_dyn_ops.h"
#include "common.h"

namespace ldyn {

constexpr int32_t STATUS_BAD_TOKENS = 4;

// --- host: argument checks ---------------------------------------------------

// One buffer of a call: its bytes, its alignment, whether it is written.
struct Span {
    const void* p;
    long long bytes;
    int align;
    bool written;
    const void* may_be = nullptr;  // a written buffer may be exactly this input
};

inline bool span_overlap(const Span& a, const Span& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

// No NULL, every buffer aligned, no written buffer on another one.
inline int check_spans(const Span* s, int n) {
    for (int i = 0; i < n; ++i)
        if (!s[i].p || (reinterpret_cast<uintptr_t>(s[i].p) & (uintptr_t)(s[i].align - 1)))
            return LSTM_DYN_ERR_INVALID;
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n; ++j)
            if (s[i].written && i != j && span_overlap(s[i], s[j]) &&
                !(s[i].may_be == s[j].p && s[i].p == s[j].p && !s[j].written))
                return LSTM_DYN_ERR_INVALID;
    return LSTM_DYN_OK;
}

inline bool valid_dtype(int dtype) { return dtype == LSTM_DYN_F32 || dtype == LSTM_DYN_BF16; }
inline int dtype_bytes(int dtype) { return dtype == LSTM_DYN_BF16 ? 2 : 4; }

// --- host: handles -------------------------------------------------------------

// The part every operator's handle has.  The workspace is zeroed at create;
// its first word is the device status.
struct OpsHandle {
    int device = 0, num_cus = 0, wclk_khz = 0;
    char* block = nullptr;
    long long bytes = 0;
    hipStream_t last_stream = nullptr;
    bool has_work = false;
    int launches = 0;

    int32_t* status() const { return reinterpret_cast<int32_t*>(block); }
};

// The current device, for a handle that is being made.
inline int ops_device(OpsHandle* h) {
    if (hipGetDevice(&h->device) != hipSuccess ||
        hipDeviceGetAttribute(&h->num_cus, hipDeviceAttributeMultiprocessorCount, h->device) != hipSuccess ||
        hipDeviceGetAttribute(&h->wclk_khz, hipDeviceAttributeWallClockRate, h->device) != hipSuccess) {
        (void)hipGetLastError();
        return LSTM_DYN_ERR_HIP;
    }
    return LSTM_DYN_OK;
}

// Its workspace (after ops_device).
inline int ops_init(OpsHandle* h, long long bytes) {
    void* p = nullptr;
    if (hipMalloc(&p, (size_t)bytes) != hipSuccess) {
        (void)hipGetLastError();
        return LSTM_DYN_ERR_NOMEM;
    }
    // the caller's streams need not wait for the default stream: the zeros are there on return
    if (hipMemset(p, 0, (size_t)bytes) != hipSuccess || hipDeviceSynchronize() != hipSuccess) {
        (void)hipGetLastError();
        (void)hipFree(p);
        return LSTM_DYN_ERR_HIP;
    }
    h->block = static_cast<char*>(p);
    h->bytes = bytes;
    return LSTM_DYN_OK;
}

// Before a call's launches: the handle's device has to be current.
inline int ops_begin(OpsHandle* h, void* stream) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) {
        (void)hipGetLastError();
        return LSTM_DYN_ERR_HIP;
    }
    if (dev != h->device) return LSTM_DYN_ERR_INVALID;
    h->last_stream = static_cast<hipStream_t>(stream);
    h->has_work = true;
    h->launches = 0;
    return LSTM_DYN_OK;
}

inline int ops_launched(OpsHandle* h) {
    if (hipGetLastError() != hipSuccess) return LSTM_DYN_ERR_HIP;
    if (h) ++h->launches;
    return LSTM_DYN_OK;
}

inline int ops_query(OpsHandle* h, int what, long long* value) {
    if (!h || !value) return LSTM_DYN_ERR_INVALID;
    if (what == LSTM_DYN_OPS_Q_WORKSPACE_BYTES) {
        *value = h->bytes;
        return LSTM_DYN_OK;
    }
    if (what == LSTM_DYN_OPS_Q_LAUNCHES) {
        *value = h->launches;
        return LSTM_DYN_OK;
    }
    if (what != LSTM_DYN_OPS_Q_STATUS) return LSTM_DYN_ERR_INVALID;
    int32_t s = 0;
    const int32_t zero = 0;
    if ((h->has_work && hipStreamSynchronize(h->last_stream) != hipSuccess) ||
        hipMemcpy(&s, h->status(), 4, hipMemcpyDeviceToHost) != hipSuccess ||
        (s && hipMemcpy(h->status(), &zero, 4, hipMemcpyHostToDevice) != hipSuccess)) {
        (void)hipGetLastError();
        return LSTM_DYN_ERR_HIP;
    }
    *value = (s & STATUS_TIMEOUT)       ? LSTM_DYN_ERR_TIMEOUT
             : (s & STATUS_BAD_LENGTHS) ? LSTM_DYN_ERR_BAD_LENGTHS
             : (s & STATUS_BAD_TOKENS)  ? LSTM_DYN_ERR_BAD_TOKENS
                                        : LSTM_DYN_OK;
    return LSTM_DYN_OK;
}

// Waits for the stream of the handle's last call, then frees its memory.
inline int ops_free(OpsHandle* h) {
    int rc = LSTM_DYN_OK;
    if (h->has_work && hipStreamSynchronize(h->last_stream) != hipSuccess) rc = LSTM_DYN_ERR_HIP;
    if (h->block && hipFree(h->block) != hipSuccess) rc = LSTM_DYN_ERR_HIP;
    if (rc != LSTM_DYN_OK) (void)hipGetLastError();
    return rc;
}

// --- device ----------------------------------------------------------------------

// V elements of E at once (p aligned to the vector).
template <class E, int V>
struct Vec {
    typedef E type __attribute__((ext_vector_type(V)));
};
template <class E>
struct Vec<E, 1> {
    typedef E type;
};
template <class E, int V>
__device__ inline void load_vec(const E* p, float* out) {
    const typename Vec<E, V>::type x = *reinterpret_cast<const typename Vec<E, V>::type*>(p);
    if constexpr (V == 1) {
        out[0] = (float)x;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = (float)x[i];
    }
}
// The same store; FAR: past the caches, for an output that its reader finds in memory anyway.
template <bool FAR, class E, int V>
__device__ inline void put(E* p, const float* in) {
    typename Vec<E, V>::type x;
    if constexpr (V == 1) {
        x = (E)in[0];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (E)in[i];
    }
    auto* q = reinterpret_cast<typename Vec<E, V>::type*>(p);
    if constexpr (FAR) __builtin_nontemporal_store(x, q);
    else *q = x;
}
template <class E, int V>
__device__ inline void store_vec(E* p, const float* in) { put<false, E, V>(p, in); }

// A row's length, clamped to [0, T]; a bad one is reported once.
__device__ inline int clamp_length(int L, int T, int32_t* status, bool report) {
    if ((unsigned)L <= (unsigned)T) return L;
    if (report) atomicOr(status, STATUS_BAD_LENGTHS);
    return L < 0 ? 0 : T;
}
__device__ inline int row_length(const int32_t* lengths, int b, int T, int32_t* status, bool report) {
    return lengths ? clamp_length(lengths[b], T, status, report) : T;
}

}  // namespace ldyn
