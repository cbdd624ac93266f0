// sk_routed.h -- launchers and device helpers of the routed-layer operators: the router, the experts' products,
// dropout and the combination of expert rows.
#pragma once

#include "sk_device.h"
#include "sk_internal.h"

namespace sk {

struct RouteArgs {
    const void *logits;
    const float *bias;    // may be null
    const uint8_t *mask;  // may be null
    float *weights;
    int32_t *experts, *counts, *offsets, *tokens, *slots;
    float *balance, *z_loss;
    float *state;  // [2 T + 1]: per token the largest logit and the sum of exponentials; then the live tokens
    void *ws;
    int T, E, k, dtype, renormalize;
};
size_t route_workspace_bytes(int T, int E, int k);
hipError_t launch_route_forward(const RouteArgs &a, hipStream_t st);

struct RouteBwdArgs {
    const void *logits;
    const float *weights;
    const int32_t *experts, *counts;
    const float *state;
    const float *g_weights, *g_balance, *g_z;  // each may be null: no gradient from there
    void *g_logits;
    int T, E, k, dtype, renormalize;
};
hipError_t launch_route_backward(const RouteBwdArgs &a, hipStream_t st);

// Threshold and scale of dropout: 16 random bits per element, dropped where they are below `threshold`.
struct DropArgs {
    uint64_t seed, offset;
    uint32_t threshold;  // 0: nothing is dropped
    float scale;
};
hipError_t launch_dropout(const void *x, const void *residual, void *y, int64_t n, int dtype, const DropArgs &d,
                          hipStream_t st);

struct CombineArgs {
    const void *z, *residual, *gy;  // residual may be null
    const float *weights;
    const int32_t *slots, *used;  // used: device pointer to the number of experts' rows
    void *y, *gz;
    float *g_weights;
    int T, D, k, dtype;
    DropArgs drop;
};
hipError_t launch_combine_forward(const CombineArgs &a, hipStream_t st);
hipError_t launch_combine_backward(const CombineArgs &a, hipStream_t st);

// ---- element types ----

struct alignas(16) Words4 {
    uint32_t w[4];
};

// Eight consecutive elements as 32-bit floats, at any alignment (the memory takes 16 bytes from anywhere).
template <class T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
    typedef T T8 __attribute__((ext_vector_type(8)));
    T8 a;
    __builtin_memcpy(&a, p, sizeof(a));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
}

// The one rounding of a result held in 32 bits to its type, to nearest even.
template <class T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    typedef T T8 __attribute__((ext_vector_type(8)));
    T8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (T)v[i];
    __builtin_memcpy(p, &a, sizeof(a));
}

// The same for the elements [lo, hi) of the eight; the others are 0 and stay.
template <class T>
__device__ __forceinline__ void load_some(const T *p, int lo, int hi, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i >= lo && i < hi ? (float)p[i] : 0.f;
}
template <class T>
__device__ __forceinline__ void store_some(T *p, int lo, int hi, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i >= lo && i < hi) p[i] = (T)v[i];
}

// Calls f with a value of the element type of dtype (an sk_dtype).
template <class F>
hipError_t with_type(int dtype, F f) {
    if (dtype == SK_BF16) return f(__bf16{});
    if (dtype == SK_F16) return f(_Float16{});
    return f(float{});
}

inline bool aligned16(const void *p) { return ((uintptr_t)p % 16) == 0; }

}  // namespace sk
