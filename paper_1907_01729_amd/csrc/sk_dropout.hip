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
// element would: its 20 multiplications then fit beside the memory's time.  All of these are bound by memory.  67M bf16
// elements with a residual 72 us (5.6 TB/s), without 44 us (6.1 TB/s); 16384 tokens of 2048 from four rows each,
// forward 96 us (4.2 TB/s), backward 128 us (4.7 TB/s) after 5 for the pairs.
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

// One thread per block of eight elements; the last block may be short.
template <class T, bool RES>
__global__ __launch_bounds__(kThreads) void sk_dropout_kernel(const T *x, const T *res, T *y, int64_t n, DropArgs d) {
    const int64_t block = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t i0 = block * 8;
    if (i0 >= n) return;
    const bool whole = i0 + 8 <= n;
    const int left = whole ? 8 : (int)(n - i0);
    float v[8], r[8];
    if (whole) {
        load8(x + i0, v);
        if (RES) load8(res + i0, r);
    } else {
        load_some(x + i0, 0, left, v);
        if (RES) load_some(res + i0, 0, left, r);
    }
    drop8(v, block, d);
    if (RES) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    if (whole)
        store8(y + i0, v);
    else
        store_some(y + i0, 0, left, v);
}

// A slot outside [0, rows) names no row.
__device__ __forceinline__ bool names_row(int32_t slot, int64_t rows) { return slot >= 0 && slot < rows; }

// One thread per block of eight elements of y.  A block that lies in one row goes as a whole; one that does not (D no
// multiple of eight, or the last block) element by element.
template <class T>
__global__ __launch_bounds__(kThreads) void sk_combine_fwd(CombineArgs A) {
    const int64_t n = (int64_t)A.T * A.D, rows = (int64_t)A.T * A.k;
    const int64_t block = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t i0 = block * 8;
    if (i0 >= n) return;
    const T *z = static_cast<const T *>(A.z), *res = static_cast<const T *>(A.residual);
    T *y = static_cast<T *>(A.y);
    const int64_t t = i0 / A.D, col = i0 - t * A.D;
    const bool whole = col + 8 <= A.D;
    float v[8] = {};
    if (whole) {
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
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i0 + i >= n) continue;
            const int64_t ti = (i0 + i) / A.D, ci = i0 + i - ti * A.D;
            for (int j = 0; j < A.k; ++j) {
                const int32_t s = A.slots[ti * A.k + j];
                if (names_row(s, rows))
                    v[i] = __builtin_fmaf(A.weights[ti * A.k + j], (float)z[(int64_t)s * A.D + ci], v[i]);
            }
        }
    }
    if (A.drop.threshold) drop8(v, block, A.drop);
    const int left = i0 + 8 <= n ? 8 : (int)(n - i0);
    if (res) {
        float r[8];
        if (left == 8)
            load8(res + i0, r);
        else
            load_some(res + i0, 0, left, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    if (left == 8)
        store8(y + i0, v);
    else
        store_some(y + i0, 0, left, v);
}

// The pair that names a row, for every row that one does: pair_of[slots[i]] = i.  The other places keep what they had,
// so a reader looks whether the pair that it finds there names the row.
__global__ __launch_bounds__(kThreads) void sk_combine_pairs(const int32_t *slots, int64_t rows, float *pair_of) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= rows) return;
    const int32_t s = slots[i];
    if (names_row(s, rows)) pair_of[s] = __int_as_float((int32_t)i);
}

// One wavefront per token, its lanes over the generator's blocks that the token's row meets: gy's row is read and
// dropped out once, then goes to the rows and products of up to KS slots at a time (their sums are in registers).
//
// The rows that no slot names are zeroed: those from *used on and those whose pair was left out (slot -1).  The pairs
// that name rows (above) stand in g_weights until the results do: token t's wavefront sees to the rows t k .. t k + k,
// whose places there are the ones that it alone writes.
template <class T, int KS>
__global__ __launch_bounds__(kThreads) void sk_combine_bwd(CombineArgs A) {
    const int64_t rows = (int64_t)A.T * A.k;
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (t >= A.T) return;
    const T *z = static_cast<const T *>(A.z), *gy = static_cast<const T *>(A.gy);
    T *gz = static_cast<T *>(A.gz);
    const int64_t D = A.D, first = t * D, last = first + D;  // elements of the row
    bool clear = false;  // lane j: row t k + j
    if (lane < A.k) {
        const int64_t r = t * A.k + lane;
        clear = r >= *A.used;
        if (!clear) {
            const int32_t pair = __float_as_int(A.g_weights[r]);
            clear = !names_row(pair, rows) || A.slots[pair] != r;
        }
    }
    uint64_t cleared = __builtin_amdgcn_ballot_w64(clear);
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
        for (int64_t block = first / 8 + lane; block * 8 < last; block += 64) {
            const int64_t i0 = block * 8, col = i0 - first;  // col < 0: the block begins in the row before
            const bool whole = col >= 0 && col + 8 <= D;
            const int lo = col < 0 ? (int)-col : 0, hi = col + 8 <= D ? 8 : (int)(D - col);
            float g[8];
            if (whole)
                load8(gy + i0, g);
            else
                load_some(gy + i0, lo, hi, g);
            if (A.drop.threshold) drop8(g, (uint64_t)block, A.drop);
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                if (slot[j] < 0) continue;
                const int64_t at = slot[j] * D + col;
                float a[8], o[8];
                if (whole)
                    load8(z + at, a);
                else
                    load_some(z + at, lo, hi, a);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dot[j] = __builtin_fmaf(g[i], a[i], dot[j]);
                    o[i] = w[j] * g[i];
                }
                if (whole)
                    store8(gz + at, o);
                else
                    store_some(gz + at, lo, hi, o);
            }
        }
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const float sum = wave_sum(dot[j]);
            if (lane == 0 && j0 + j < A.k) A.g_weights[t * A.k + j0 + j] = sum;
        }
    }
    for (; cleared; cleared &= cleared - 1) {
        T *row = gz + (t * A.k + __builtin_ctzll(cleared)) * D;
        const float none[8] = {};
        for (int64_t c = lane * 8; c < D; c += 64 * 8) {
            if (c + 8 <= D)
                store8(row + c, none);
            else
                store_some(row + c, 0, (int)(D - c), none);
        }
    }
}

}  // namespace

hipError_t launch_dropout(const void *x, const void *residual, void *y, int64_t n, int dtype, const DropArgs &d,
                          hipStream_t st) {
    if (n == 0) return hipSuccess;
    const dim3 grid((unsigned)((n + 8 * kThreads - 1) / (8 * kThreads)));
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, static_cast<const T *>(x),
                               static_cast<const T *>(residual), static_cast<T *>(y), n, d);
            return hipGetLastError();
        };
        return residual ? go(sk_dropout_kernel<T, true>) : go(sk_dropout_kernel<T, false>);
    });
}

hipError_t launch_combine_forward(const CombineArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    const int64_t n = (int64_t)a.T * a.D;
    const dim3 grid((unsigned)((n + 8 * kThreads - 1) / (8 * kThreads)));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        hipLaunchKernelGGL(sk_combine_fwd<T>, grid, dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

hipError_t launch_combine_backward(const CombineArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    const int64_t rows = (int64_t)a.T * a.k;
    hipLaunchKernelGGL(sk_combine_pairs, dim3((unsigned)((rows + kThreads - 1) / kThreads)), dim3(kThreads), 0, st,
                       a.slots, rows, a.g_weights);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)(((int64_t)a.T + 3) / 4));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        hipLaunchKernelGGL((sk_combine_bwd<T, 4>), grid, dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

}  // namespace sk
