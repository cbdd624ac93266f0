// sk_experts.hip -- the experts' products: each expert's rows times that expert's matrix, and both gradients.
//
//   forward   y[r, n]     = sum_k x[src(r), k] w[e, n, k]                 offsets[e] <= r < offsets[e + 1]
//   input     gr[r, k]    = sum_n gy[r, n] w[e, n, k]                     gx[t] = sum_s gr[slots[t, s]]
//   weight    gw[e, n, k] = sum_r gy[r, n] x[src(r), k]
//
// src(r) = tokens[r] where the rows are gathered from the tokens, else r.  Products of 16-bit factors on the matrix
// cores, sums in 32 bits, one rounding at the end.
#include "sk_experts.h"

namespace sk {
namespace {

constexpr int kThreads = 256;

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <class T>
__device__ __forceinline__ f32x4 mfma16(const Frag8<T> &a, const Frag8<T> &b, f32x4 c) {
    if constexpr (std::is_same_v<T, __bf16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// ---- any sizes and alignment: 64 x 64 tiles, elements loaded one by one ----

constexpr int kAnyTile = 64, kAnyDeep = 32, kAnyPitch = kAnyDeep + 8;

template <class T, int MODE>
__global__ __launch_bounds__(kThreads) void sk_experts_any(ExpertArgs A) {
    __shared__ T la[kAnyTile * kAnyPitch], lb[kAnyTile * kAnyPitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T *x = static_cast<const T *>(A.x), *w = static_cast<const T *>(A.w), *gy = static_cast<const T *>(A.gy);
    const int K = A.K, N = A.N;

    int e, r0, r1, c0, m0 = 0;  // the expert, its rows here, the first column; weight: the first row of gw's tile
    if constexpr (MODE == kWeight) {
        const int tk = (K + kAnyTile - 1) / kAnyTile, tn = (N + kAnyTile - 1) / kAnyTile;
        e = blockIdx.x / (tk * tn);
        const int rest = blockIdx.x - e * (tk * tn);
        m0 = rest / tk * kAnyTile;
        c0 = rest % tk * kAnyTile;
        const RowRange rr = expert_rows(A, e);
        r0 = rr.begin, r1 = rr.end;
    } else {
        const int cols = MODE == kForward ? N : K;
        const int tc = (cols + kAnyTile - 1) / kAnyTile;
        const RowTile t = find_row_tile(A, kAnyTile, blockIdx.x / tc);
        if (t.expert < 0) return;
        e = t.expert, r0 = t.begin, r1 = t.end;
        c0 = blockIdx.x % tc * kAnyTile;
    }
    const T *we = w + (size_t)(e < A.E ? e : 0) * N * K;
    const int deep = MODE == kForward ? K : MODE == kInput ? N : r1 - r0;
    const bool none = MODE != kWeight && e >= A.E;  // rows of no expert: zeros

    auto source = [&](int r) -> int64_t {  // x's row of a row, -1: none
        if (!A.tokens) return r;
        const int t = A.tokens[r];
        return t >= 0 && t < A.T ? t : -1;
    };
    auto load_a = [&](int i, int d) -> T {  // row i of the tile, d of the contraction
        if (d >= deep) return (T)0.f;
        if constexpr (MODE == kWeight) {
            return m0 + i < N ? gy[(int64_t)(r0 + d) * N + m0 + i] : (T)0.f;
        } else {
            if (r0 + i >= r1) return (T)0.f;
            if constexpr (MODE == kInput) return gy[(int64_t)(r0 + i) * N + d];
            const int64_t s = source(r0 + i);
            return s >= 0 ? x[s * K + d] : (T)0.f;
        }
    };
    auto load_b = [&](int j, int d) -> T {  // column j of the tile
        if (d >= deep) return (T)0.f;
        if constexpr (MODE == kForward) return c0 + j < N ? we[(int64_t)(c0 + j) * K + d] : (T)0.f;
        if constexpr (MODE == kInput) return c0 + j < K ? we[(int64_t)d * K + c0 + j] : (T)0.f;
        const int64_t s = source(r0 + d);
        return c0 + j < K && s >= 0 ? x[s * K + c0 + j] : (T)0.f;
    };

    f32x4 acc[2][2] = {};
    const int wi = (wave >> 1) * 32, wj = (wave & 1) * 32;
    for (int d0 = 0; !none && d0 < deep; d0 += kAnyDeep) {
        __syncthreads();
        for (int q = tid; q < kAnyTile * kAnyDeep; q += kThreads) {
            // neighbours in memory to neighbouring lanes
            const int i = MODE == kWeight ? q % kAnyTile : q / kAnyDeep, d = MODE == kWeight ? q / kAnyTile : q % kAnyDeep;
            la[i * kAnyPitch + d] = load_a(i, d0 + d);
            const int j = MODE == kForward ? q / kAnyDeep : q % kAnyTile, f = MODE == kForward ? q % kAnyDeep : q / kAnyTile;
            lb[j * kAnyPitch + f] = load_b(j, d0 + f);
        }
        __syncthreads();
        Frag8<T> fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            fa[i] = *reinterpret_cast<const Frag8<T> *>(la + (wi + i * 16 + (lane & 15)) * kAnyPitch + (lane >> 4) * 8);
            fb[i] = *reinterpret_cast<const Frag8<T> *>(lb + (wj + i * 16 + (lane & 15)) * kAnyPitch + (lane >> 4) * 8);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = mfma16<T>(fa[i], fb[j], acc[i][j]);
    }
    // lane: column lane % 16, rows (lane / 16) * 4 + v of a 16 x 16 block
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int row = wi + i * 16 + (lane >> 4) * 4 + v, col = c0 + wj + j * 16 + (lane & 15);
                if constexpr (MODE == kWeight) {
                    if (m0 + row < N && col < K)
                        static_cast<T *>(A.out)[((size_t)e * N + m0 + row) * K + col] = (T)acc[i][j][v];
                } else {
                    const int cols = MODE == kForward ? N : K;
                    if (r0 + row >= r1 || col >= cols) continue;
                    const int64_t at = (int64_t)(r0 + row) * cols + col;
                    if (A.out32)
                        A.out32[at] = acc[i][j][v];
                    else
                        static_cast<T *>(A.out)[at] = (T)acc[i][j][v];
                }
            }
}

// gx[t] = sum over the token's slots of the rows' gradients, kept in 32 bits until here.  Eight elements of gx to a
// thread; VEC: K is a multiple of eight and gx aligned to 16 bytes, so that they lie in one row.
template <class T, bool VEC>
__global__ __launch_bounds__(kThreads) void sk_experts_sum_slots(ExpertArgs A, const float *rows, T *gx) {
    const int64_t n = (int64_t)A.T * A.K, all = (int64_t)A.T * A.k;
    const int64_t i0 = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 8;
    if (i0 >= n) return;
    if (VEC) {
        const int64_t t = i0 / A.K, c = i0 - t * A.K;
        float sum[8] = {};
        for (int s = 0; s < A.k; ++s) {
            const int32_t r = A.slots[t * A.k + s];
            if (r < 0 || r >= all) continue;
            float v[8];
            load8(rows + (int64_t)r * A.K + c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        }
        store8(gx + i0, sum);
    } else {
        for (int64_t i = i0; i < i0 + 8 && i < n; ++i) {
            const int64_t t = i / A.K, c = i - t * A.K;
            float sum = 0.f;
            for (int s = 0; s < A.k; ++s) {
                const int32_t r = A.slots[t * A.k + s];
                if (r >= 0 && r < all) sum += rows[(int64_t)r * A.K + c];
            }
            gx[i] = (T)sum;
        }
    }
}

template <class F>
hipError_t with_half(int dtype, F f) {
    return dtype == SK_BF16 ? f(__bf16{}) : f(_Float16{});
}

// Row tiles that E experts' rows and the rows of none can take at most.
int64_t most_row_tiles(const ExpertArgs &a, int tile) {
    const int64_t rows = (int64_t)a.T * a.k;
    return rows / tile + (rows < a.E + 1 ? rows : a.E + 1);
}

template <int MODE>
hipError_t launch_rows(const ExpertArgs &a, hipStream_t st) {
    const int cols = MODE == kForward ? a.N : a.K;
    const int64_t grid = most_row_tiles(a, kAnyTile) * ((cols + kAnyTile - 1) / kAnyTile);
    return with_half(a.dtype, [&](auto type) {
        using T = decltype(type);
        hipLaunchKernelGGL((sk_experts_any<T, MODE>), dim3((unsigned)grid), dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

}  // namespace

size_t experts_workspace_bytes(int T, int k, int K) { return (size_t)T * k * K * 4; }

hipError_t launch_experts_forward(const ExpertArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    return launch_rows<kForward>(a, st);
}

hipError_t launch_experts_input(const ExpertArgs &a, void *ws, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    if (!a.slots) return launch_rows<kInput>(a, st);
    ExpertArgs r = a;
    r.out32 = static_cast<float *>(ws);
    const hipError_t e = launch_rows<kInput>(r, st);
    if (e != hipSuccess) return e;
    return with_half(a.dtype, [&](auto type) {
        using T = decltype(type);
        const dim3 grid((unsigned)(((int64_t)a.T * a.K + 8 * kThreads - 1) / (8 * kThreads)));
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, a, static_cast<const float *>(ws),
                               static_cast<T *>(a.out));
            return hipGetLastError();
        };
        return a.K % 8 == 0 && aligned16(ws) && aligned16(a.out) ? go(sk_experts_sum_slots<T, true>)
                                                                 : go(sk_experts_sum_slots<T, false>);
    });
}

hipError_t launch_experts_weight(const ExpertArgs &a, hipStream_t st) {
    const int64_t grid = (int64_t)a.E * ((a.N + kAnyTile - 1) / kAnyTile) * ((a.K + kAnyTile - 1) / kAnyTile);
    return with_half(a.dtype, [&](auto type) {
        using T = decltype(type);
        hipLaunchKernelGGL((sk_experts_any<T, kWeight>), dim3((unsigned)grid), dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

}  // namespace sk
