// sk_dropout.hip -- dropout from a counter-based generator, and the combination of a token's expert rows with it.
//
//   dropout   y = r + s keep x                      gx = s keep gy
//   combine   y[t] = r[t] + s keep sum_j w[t,j] z[slot(t,j)]
//             gz[slot(t,j)] = w[t,j] s keep gy[t]   gw[t,j] = sum_d s keep gy[t,d] z[slot(t,j),d]
//
// keep of element i (row-major) depends on (seed, offset, i) alone, so no mask is stored: the backward pass draws it
// again.  The generator is Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy
// as 1, 2, 3", 2011).  One block of four words serves eight elements, 16 bits each: the drop rate is then a multiple
// of 2^-16 (scale is of that rate, so the mean is kept exactly), and the generator costs half of what a word per
// element would.
#include "sk_routed.h"

namespace sk {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ Words4 philox(uint64_t block, const DropArgs &d) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)d.offset,
             c3 = (uint32_t)(d.offset >> 32);
    uint32_t k0 = (uint32_t)d.seed, k1 = (uint32_t)(d.seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// v = s keep v for the eight elements of a block.
__device__ __forceinline__ void drop8(float (&v)[8], uint64_t block, const DropArgs &d) {
    const Words4 r = philox(block, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = i & 1 ? r.w[i / 2] >> 16 : r.w[i / 2] & 0xFFFFu;
        v[i] = u >= d.threshold ? v[i] * d.scale : 0.f;
    }
}

// One thread per block of eight elements.  VEC: every pointer is aligned to 16 bytes; the last block may be short.
template <class T, bool VEC, bool RES>
__global__ __launch_bounds__(kThreads) void sk_dropout_kernel(const T *x, const T *res, T *y, int64_t n, DropArgs d) {
    const int64_t block = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t i0 = block * 8;
    if (i0 >= n) return;
    float v[8], r[8];
    if (VEC && i0 + 8 <= n) {
        load8(x + i0, v);
        if (RES) load8(res + i0, r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = i0 + i < n ? (float)x[i0 + i] : 0.f;
            if (RES) r[i] = i0 + i < n ? (float)res[i0 + i] : 0.f;
        }
    }
    drop8(v, block, d);
    if (RES) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    if (VEC && i0 + 8 <= n) {
        store8(y + i0, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i0 + i < n) y[i0 + i] = (T)v[i];
    }
}

// A slot outside [0, rows) names no row.
__device__ __forceinline__ bool names_row(int32_t slot, int64_t rows) { return slot >= 0 && slot < rows; }

// One thread per block of eight elements of y.  VEC: D is a multiple of 8 and every pointer is aligned to 16 bytes,
// so that a block lies in one row; otherwise each element is on its own.
template <class T, bool VEC>
__global__ __launch_bounds__(kThreads) void sk_combine_fwd(CombineArgs A) {
    const int64_t n = (int64_t)A.T * A.D, rows = (int64_t)A.T * A.k;
    const int64_t block = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t i0 = block * 8;
    if (i0 >= n) return;
    const T *z = static_cast<const T *>(A.z), *res = static_cast<const T *>(A.residual);
    T *y = static_cast<T *>(A.y);
    float v[8] = {};
    if (VEC) {
        const int64_t t = i0 / A.D;
        const int64_t col = i0 - t * A.D;
        for (int j = 0; j < A.k; ++j) {
            const int32_t s = A.slots[t * A.k + j];
            if (!names_row(s, rows)) continue;
            const float w = A.weights[t * A.k + j];
            float a[8];
            load8(z + (int64_t)s * A.D + col, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(w, a[i], v[i]);
        }
    } else {
        for (int i = 0; i < 8 && i0 + i < n; ++i) {
            const int64_t t = (i0 + i) / A.D;
            const int64_t col = i0 + i - t * A.D;
            float sum = 0.f;
            for (int j = 0; j < A.k; ++j) {
                const int32_t s = A.slots[t * A.k + j];
                if (names_row(s, rows))
                    sum = __builtin_fmaf(A.weights[t * A.k + j], (float)z[(int64_t)s * A.D + col], sum);
            }
            v[i] = sum;
        }
    }
    if (A.drop.threshold) drop8(v, block, A.drop);
    if (VEC) {
        if (res) {
            float r[8];
            load8(res + i0, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += r[i];
        }
        store8(y + i0, v);
    } else {
        for (int i = 0; i < 8 && i0 + i < n; ++i) y[i0 + i] = (T)(v[i] + (res ? (float)res[i0 + i] : 0.f));
    }
}

// One wavefront per token: gy's row is read and dropped out once, then goes to every slot's row and product.  The
// rows that no slot names (from *used on) are zeroed by the same wavefronts.  KS: slots per pass (registers).
template <class T, bool VEC, int KS>
__global__ __launch_bounds__(kThreads) void sk_combine_bwd(CombineArgs A) {
    const int64_t rows = (int64_t)A.T * A.k;
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (t >= A.T) return;
    const T *z = static_cast<const T *>(A.z), *gy = static_cast<const T *>(A.gy);
    T *gz = static_cast<T *>(A.gz);
    const int D = A.D;
    for (int j0 = 0; j0 < A.k; j0 += KS) {
        int32_t slot[KS];
        float w[KS], dot[KS];
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const bool in = j0 + j < A.k;
            slot[j] = in ? A.slots[t * A.k + j0 + j] : -1;
            w[j] = in ? A.weights[t * A.k + j0 + j] : 0.f;
            if (!names_row(slot[j], rows)) slot[j] = -1;
            dot[j] = 0.f;
        }
        if (VEC) {
            for (int c = lane * 8; c < D; c += 64 * 8) {
                float g[8];
                load8(gy + t * D + c, g);
                if (A.drop.threshold) drop8(g, (uint64_t)(t * D + c) / 8, A.drop);
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    if (slot[j] < 0) continue;
                    const int64_t at = (int64_t)slot[j] * D + c;
                    float a[8], o[8];
                    load8(z + at, a);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        dot[j] = __builtin_fmaf(g[i], a[i], dot[j]);
                        o[i] = w[j] * g[i];
                    }
                    store8(gz + at, o);
                }
            }
        } else {
            // Blocks of the generator do not begin with rows here: each lane draws the block of its element.
            for (int c = lane; c < D; c += 64) {
                const int64_t i = t * D + c;
                float g = (float)gy[i];
                if (A.drop.threshold) {
                    float v[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
                    drop8(v, (uint64_t)i / 8, A.drop);
                    float keep = 0.f;
#pragma unroll
                    for (int q = 0; q < 8; ++q) keep = (i & 7) == q ? v[q] : keep;
                    g = keep > 0.f ? g * keep : 0.f;
                }
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    if (slot[j] < 0) continue;
                    const int64_t at = (int64_t)slot[j] * D + c;
                    dot[j] = __builtin_fmaf(g, (float)z[at], dot[j]);
                    gz[at] = (T)(w[j] * g);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const float sum = wave_sum(dot[j]);
            if (lane == 0 && j0 + j < A.k) A.g_weights[t * A.k + j0 + j] = sum;
        }
    }
    int64_t used = *A.used;
    used = used < 0 ? 0 : used;
    for (int64_t r = used + t; r < rows; r += A.T)
        for (int c = lane; c < D; c += 64) gz[r * D + c] = (T)0.f;
}

}  // namespace

hipError_t launch_dropout(const void *x, const void *residual, void *y, int64_t n, int dtype, const DropArgs &d,
                          hipStream_t st) {
    if (n == 0) return hipSuccess;
    const dim3 grid((unsigned)((n + 8 * kThreads - 1) / (8 * kThreads)));
    const bool vec = aligned16(x) && aligned16(y) && (!residual || aligned16(residual));
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, static_cast<const T *>(x),
                               static_cast<const T *>(residual), static_cast<T *>(y), n, d);
            return hipGetLastError();
        };
        if (vec) return residual ? go(sk_dropout_kernel<T, true, true>) : go(sk_dropout_kernel<T, true, false>);
        return residual ? go(sk_dropout_kernel<T, false, true>) : go(sk_dropout_kernel<T, false, false>);
    });
}

hipError_t launch_combine_forward(const CombineArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    const int64_t n = (int64_t)a.T * a.D;
    const dim3 grid((unsigned)((n + 8 * kThreads - 1) / (8 * kThreads)));
    const bool vec = a.D % 8 == 0 && aligned16(a.z) && aligned16(a.y) && (!a.residual || aligned16(a.residual));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        if (vec)
            hipLaunchKernelGGL((sk_combine_fwd<T, true>), grid, dim3(kThreads), 0, st, a);
        else
            hipLaunchKernelGGL((sk_combine_fwd<T, false>), grid, dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

hipError_t launch_combine_backward(const CombineArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    const dim3 grid((unsigned)(((int64_t)a.T + 3) / 4));
    const bool vec = a.D % 8 == 0 && aligned16(a.z) && aligned16(a.gy) && aligned16(a.gz);
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, a);
            return hipGetLastError();
        };
        if (vec) return go(sk_combine_bwd<T, true, 4>);
        return go(sk_combine_bwd<T, false, 4>);
    });
}

}  // namespace sk
