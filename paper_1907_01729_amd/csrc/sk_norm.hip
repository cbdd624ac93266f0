// sk_norm.hip -- the norms around a block, fused with its gate and its residual, and their gradients.
//
//   norm(x) = xh w + b,  xh = (x - m) r,  r = (mean((x - m)^2) + eps)^-1/2,  m = mean(x) or 0
//   forward   n = norm_after(h) or h,  out = scale residual + gate n,  next = norm_before(out)
//   backward  of a norm, with d = gy w:  gx = r (d - [m] mean(d) - xh mean(d xh)),  gw = sum_t gy xh,  gb = sum_t gy
//             g = g_out + (norm_before's),  g_residual = scale g,  g_gate = g n,  dn = gate g,  g_h = (norm_after's of dn)
#include "sk_norm.h"

#include <type_traits>

#include "sk_rows.h"

namespace sk {
namespace {

constexpr int kMostLanes = 1024;

// Eight of a parameter's values, of type T or float.
template <class T>
__device__ __forceinline__ void load_param(const void *p, int f32, int64_t at, int left, float (&v)[8]) {
    if (f32)
        load_left(static_cast<const float *>(p) + at, left, v);
    else
        load_left(static_cast<const T *>(p) + at, left, v);
}
template <class T>
__device__ __forceinline__ void load_weight(const void *p, int f32, int64_t at, int left, float (&v)[8]) {
    if (p) {
        load_param<T>(p, f32, at, left, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.f;
    }
}
template <class T>
__device__ __forceinline__ void load_bias(const void *p, int f32, int64_t at, int left, float (&v)[8]) {
    if (p) {
        load_param<T>(p, f32, at, left, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
}
template <class T>
__device__ __forceinline__ void store_param(void *p, int f32, int64_t at, float v) {
    if (f32)
        static_cast<float *>(p)[at] = v;
    else
        static_cast<T *>(p)[at] = (T)v;
}

// The gate's values for eight columns of a row.
template <class T>
__device__ __forceinline__ void load_gate(const NormArgs &A, int64_t row, int c, int left, float (&v)[8]) {
    if (A.gate_kind == SK_GATE_COLUMNS) {
        load_param<T>(A.gate, A.gf32, c, left, v);
    } else if (A.gate_kind == SK_GATE_FULL) {
        load_param<T>(A.gate, A.gf32, row * A.N + c, left, v);
    } else {
        const float one = A.gate_kind == SK_GATE_NONE ? 1.f
                          : A.gf32                    ? static_cast<const float *>(A.gate)[row]
                                                      : (float)static_cast<const T *>(A.gate)[row];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = one;
    }
}

__device__ __forceinline__ float sum8(const float (&v)[8]) { return tree_sum<8>(v); }

// Each step is rounded by itself, as a program's own steps in 32 bits are: a sum that lies next to a border between two
// 16-bit numbers then falls to the same side for both.
__device__ __forceinline__ void norm8_of(const float (&x)[8], float mean, float r, const float (&w)[8],
                                         const float (&b)[8], float (&y)[8]) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float xh = (x[i] - mean) * r;
        y[i] = xh * w[i] + b[i];
    }
}
__device__ __forceinline__ void sum8_of(float (&y)[8], const float (&gate)[8], const float (&n)[8], float scale) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = scale * y[i] + gate[i] * n[i];
}

// A row to a group of lanes.  V: the chunks that a lane holds in registers; 0: rows wider than that, read again from
// the caches for each pass over them.  END: the block's end; else the norm alone, of `residual`.
template <class T, int V, bool END>
__global__ __launch_bounds__(kMostLanes) void sk_norm_forward(NormArgs A) {
    constexpr int H = V ? V : 1;
    __shared__ float lds[2][1][kRowWaves];
    const RowGroup g(A.lanes);
    const int64_t all = (int64_t)blockIdx.x * g.groups + g.group, row = min(all, (int64_t)A.T - 1);
    const bool mine = all < A.T;
    const int N = A.N;
    const float each_n = 1.f / (float)N;
    int turn = 0;
    // f(chunk held, column, columns left)
    auto each = [&](auto f) {
        if constexpr (V > 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (v * g.lanes + g.lane) * 8;
                f(v, c, N - c);
            }
        } else {
            for (int c = g.lane * 8; c < N; c += g.lanes * 8) f(0, c, N - c);
        }
    };
    // Mean and r of a row that `load` puts in x, eight columns at a time.
    auto statistics = [&](int kind, float eps, float (&x)[H][8], auto load, float &mean, float &r) {
        mean = 0.f;
        if (kind == SK_NORM_CENTRED) {
            float s[1] = {};
            each([&](int v, int c, int left) {
                if (V == 0) load(v, c, left);
                s[0] += sum8(x[v]);
            });
            group_reduce<Sum>(g, s, lds, turn);
            mean = s[0] * each_n;
        }
        float s[1] = {};
        each([&](int v, int c, int left) {
            if (V == 0) load(v, c, left);
            float q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = i < left ? (x[v][i] - mean) * (x[v][i] - mean) : 0.f;
            s[0] += sum8(q);
        });
        group_reduce<Sum>(g, s, lds, turn);
        r = rsqrtf(s[0] * each_n + eps);
    };
    auto normed = [&](const float (&x)[8], float mean, float r, const void *w, const void *b, int c, int left,
                      float (&y)[8]) {
        float wv[8], bv[8];
        load_weight<T>(w, A.wf32, c, left, wv);
        load_bias<T>(b, A.wf32, c, left, bv);
        norm8_of(x, mean, r, wv, bv, y);
    };

    const T *residual = static_cast<const T *>(A.residual) + row * N;
    float y[H][8];  // the sum, or the norm's input
    float4 stats = {0.f, 1.f, 0.f, 1.f};
    T *out = static_cast<T *>(A.out) + row * N;
    if constexpr (END) {
        const T *h = static_cast<const T *>(A.h) + row * N;
        float x[H][8];
        auto load_h = [&](int v, int c, int left) { load_left(h + c, left, x[v]); };
        if constexpr (V > 0) {
            each([&](int v, int c, int left) {
                load_h(v, c, left);
                load_left(residual + c, left, y[v]);
            });
        }
        if (A.after) statistics(A.after, A.eps_after, x, load_h, stats.x, stats.y);
        each([&](int v, int c, int left) {
            if (V == 0) {
                load_h(v, c, left);
                load_left(residual + c, left, y[v]);
            }
            float n[8], gate[8];
            if (A.after) {
                normed(x[v], stats.x, stats.y, A.after_w, A.after_b, c, left, n);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) n[i] = x[v][i];
            }
            load_gate<T>(A, row, c, left, gate);
            sum8_of(y[v], gate, n, A.scale);
            // Rounded here: the next norm, and the backward pass of it, take the sum as it is stored.
#pragma unroll
            for (int i = 0; i < 8; ++i) y[v][i] = i < left ? (float)(T)y[v][i] : 0.f;
            if (mine) store_left(out + c, left, y[v]);
        });
    } else if constexpr (V > 0) {
        each([&](int v, int c, int left) { load_left(residual + c, left, y[v]); });
    }
    if (A.before) {
        auto load_y = [&](int v, int c, int left) { load_left((END ? out : residual) + c, left, y[v]); };
        statistics(A.before, A.eps_before, y, load_y, stats.z, stats.w);
        each([&](int v, int c, int left) {
            if (V == 0) load_y(v, c, left);
            float z[8];
            normed(y[v], stats.z, stats.w, A.before_w, A.before_b, c, left, z);
            if (mine) store_left(static_cast<T *>(A.next) + row * N + c, left, z);
        });
    }
    if (A.stats && mine && g.lane == 0) reinterpret_cast<float4 *>(A.stats)[row] = stats;
}

// The sums over the rows.
enum { kAfterW, kBeforeW, kAfterB, kBeforeB, kGate, kArrays };
template <int A>
using Array = std::integral_constant<int, A>;

// A work-group's groups go through rows; the sums over the rows stay in registers (WIDE: in the work-group's own part
// of memory, and the row is read again from the caches for each pass over it) and are added up over the groups at the
// end, into one part a work-group.  MORE: there are biases, or a gate that is more than a number a row; without them
// fewer registers are taken.
template <class T, bool WIDE, bool END, bool MORE, int THREADS>
__global__ __launch_bounds__(THREADS) void sk_norm_backward(NormArgs A) {
    constexpr int kSums = MORE ? kArrays : kAfterB;
    __shared__ float lds[2][3][kRowWaves];
    __shared__ __attribute__((aligned(16))) float total[WIDE ? 8 : THREADS * 8];
    const RowGroup g(A.lanes);
    const int N = A.N;
    const float each_n = 1.f / (float)N;
    const bool before = A.before && A.g_next, after = END && A.after;
    const bool wants_h = after || (END && A.g_gate), sums_gate = END && A.gate_kind == SK_GATE_ROWS && A.g_gate;
    int turn = 0;
    float sums[WIDE ? 1 : kSums][8] = {};
    auto part_of = [&](int array) {
        return A.place[array] < 0 ? nullptr
                                  : A.parts + ((int64_t)blockIdx.x * A.arrays + A.place[array]) * N;
    };
    bool first = true;  // WIDE: the work-group's first row
    auto add = [&](auto which, int c, int left, const float (&v)[8]) {
        constexpr int array = decltype(which)::value;
        if constexpr (array >= kSums) {
        } else if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[array][i] += v[i];
        } else if (float *to = part_of(array)) {
            float s[8] = {};
            if (!first) load_left(to + c, left, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += v[i];
            store_left(to + c, left, s);
        }
    };
    float x[8], dy[8], go[8], h[8], gate[8];
    float wb[8], wa[8], ba[8] = {};
    auto load_weights = [&](int c, int left) {
        load_weight<T>(A.before_w, A.wf32, c, left, wb);
        if (END) {
            load_weight<T>(A.after_w, A.wf32, c, left, wa);
            if (MORE) load_bias<T>(A.after_b, A.wf32, c, left, ba);
        }
    };
    if (!WIDE) load_weights(g.lane * 8, N - g.lane * 8);
    const int64_t step = (int64_t)gridDim.x * g.groups;
    for (int64_t r0 = (int64_t)blockIdx.x * g.groups; r0 < A.T; r0 += step) {
        const bool mine = r0 + g.group < A.T;
        const int64_t row = mine ? r0 + g.group : A.T - 1, at = row * N;
        const float4 stats = reinterpret_cast<const float4 *>(A.stats)[row];
        auto load = [&](int c, int left) {
            if (before) {
                load_left(static_cast<const T *>(A.out) + at + c, left, x);
                load_left(static_cast<const T *>(A.g_next) + at + c, left, dy);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = dy[i] = 0.f;
            }
            if (END && A.g_out) {
                load_left(static_cast<const T *>(A.g_out) + at + c, left, go);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) go[i] = 0.f;
            }
            if (wants_h) load_left(static_cast<const T *>(A.h) + at + c, left, h);
            if (MORE && END) {
                load_gate<T>(A, row, c, left, gate);
            } else {
                const float one = !END || A.gate_kind == SK_GATE_NONE ? 1.f
                                  : A.gf32 ? static_cast<const float *>(A.gate)[row]
                                           : (float)static_cast<const T *>(A.gate)[row];
#pragma unroll
                for (int i = 0; i < 8; ++i) gate[i] = one;
            }
        };
        auto each = [&](auto f) {
            if constexpr (!WIDE) {
                f(g.lane * 8, N - g.lane * 8);
            } else {
                for (int c = g.lane * 8; c < N; c += g.lanes * 8) {
                    load(c, N - c);
                    load_weights(c, N - c);
                    f(c, N - c);
                }
            }
        };
        if (!WIDE) load(g.lane * 8, N - g.lane * 8);
        float s[2] = {0.f, 0.f};
        if (before) {
            each([&](int c, int left) {
                float a[8], b[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    a[i] = i < left ? dy[i] * wb[i] : 0.f;
                    b[i] = a[i] * ((x[i] - stats.z) * stats.w);
                }
                s[0] += sum8(a), s[1] += sum8(b);
            });
            group_reduce<Sum>(g, s, lds, turn);
            s[0] = A.before == SK_NORM_CENTRED ? s[0] * each_n : 0.f;
            s[1] *= each_n;
        }
        // The sum's gradient.
        auto gradient = [&](int left, float (&d)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] = go[i];
                if (before) d[i] += stats.w * (dy[i] * wb[i] - s[0] - (x[i] - stats.z) * stats.w * s[1]);
                if (i >= left) d[i] = 0.f;
            }
        };
        float d[8], q[3] = {0.f, 0.f, 0.f};
        each([&](int c, int left) {
            gradient(left, d);
            if ((before || WIDE) && mine) {  // WIDE: zeros are written, too
                float xd[8], yd[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    yd[i] = i < left ? dy[i] : 0.f;
                    xd[i] = yd[i] * ((x[i] - stats.z) * stats.w);
                }
                add(Array<kBeforeW>{}, c, left, xd);
                add(Array<kBeforeB>{}, c, left, yd);
            }
            if constexpr (!END) {
                if (mine && A.g_residual) store_left(static_cast<T *>(A.g_residual) + at + c, left, d);
            } else {
                float n[8], e[8];
                if (mine && A.g_residual) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = A.scale * d[i];
                    store_left(static_cast<T *>(A.g_residual) + at + c, left, e);
                }
                if (wants_h) {
                    float hh[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        hh[i] = after ? (h[i] - stats.x) * stats.y : h[i];
                        n[i] = after ? hh[i] * wa[i] + ba[i] : h[i];
                    }
                    if (A.g_gate) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) e[i] = i < left ? d[i] * n[i] : 0.f;
                        if (sums_gate) q[2] += sum8(e);
                        if (MORE && A.gate_kind == SK_GATE_COLUMNS && mine) add(Array<kGate>{}, c, left, e);
                        if (MORE && A.gate_kind == SK_GATE_FULL && mine) {
                            if (A.gf32)
                                store_left(static_cast<float *>(A.g_gate) + at + c, left, e);
                            else
                                store_left(static_cast<T *>(A.g_gate) + at + c, left, e);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] = i < left ? d[i] * gate[i] : 0.f;
                    if (after) {
                        float a[8], b[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            a[i] = d[i] * wa[i];
                            b[i] = a[i] * hh[i];
                            e[i] = d[i] * hh[i];
                        }
                        q[0] += sum8(a), q[1] += sum8(b);
                        if (mine) {
                            add(Array<kAfterW>{}, c, left, e);
                            add(Array<kAfterB>{}, c, left, d);
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] = i < left ? d[i] * gate[i] : 0.f;
                }
                if (!after && mine && A.g_h) store_left(static_cast<T *>(A.g_h) + at + c, left, d);
            }
        });
        if (END && (after || sums_gate)) {
            group_reduce<Sum>(g, q, lds, turn);
            q[0] = A.after == SK_NORM_CENTRED ? q[0] * each_n : 0.f;
            q[1] *= each_n;
            if (sums_gate && mine && g.lane == 0) store_param<T>(A.g_gate, A.gf32, row, q[2]);
            if (after && A.g_h && mine)
                each([&](int c, int left) {
                    if (WIDE) {
                        gradient(left, d);
#pragma unroll
                        for (int i = 0; i < 8; ++i) d[i] *= gate[i];
                    }
                    float e[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        e[i] = stats.y * (d[i] * wa[i] - q[0] - (h[i] - stats.x) * stats.y * q[1]);
                    store_left(static_cast<T *>(A.g_h) + at + c, left, e);
                });
        }
        first = false;
    }
    if constexpr (!WIDE) {
#pragma unroll
        for (int a = 0; a < kSums; ++a) {
            float *to = part_of(a);
            if (!to) continue;
            // Eight columns a lane, the groups one after the other.
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) total[threadIdx.x * 8 + i] = sums[a][i];
            __syncthreads();
            for (int c = threadIdx.x; c < N; c += blockDim.x) {
                float s = 0.f;
                for (int q = 0; q < g.groups; ++q) s += total[q * g.lanes * 8 + c];
                to[c] = s;
            }
        }
    }
}

// The work-groups' parts of the sums over the rows, added up in order: 16 columns of one array to a work-group, four a
// thread, over 64 runs of parts whose sums meet in LDS.
constexpr int kSumThreads = 256, kSumColumns = 16;

struct SumArgs {
    const float *parts;
    void *to[kArrays];
    int f32[kArrays];
    int blocks, arrays, N;
};

template <class T>
__global__ __launch_bounds__(kSumThreads) void sk_norm_sums(SumArgs A) {
    constexpr int kLanes = kSumColumns / 4, kRuns = kSumThreads / kLanes;
    __shared__ float4 part[kRuns][kLanes];
    const int lane = threadIdx.x % kLanes, run = threadIdx.x / kLanes, array = blockIdx.y;
    const int c = blockIdx.x * kSumColumns + lane * 4, left = A.N - c;
    const int each = (A.blocks + kRuns - 1) / kRuns, end = min(A.blocks, (run + 1) * each);
    float4 s = {0.f, 0.f, 0.f, 0.f};
    for (int b = run * each; b < end; ++b) {
        const float *from = A.parts + ((int64_t)b * A.arrays + array) * A.N + c;
        if (left >= 4) {
            float4 v;
            __builtin_memcpy(&v, from, 16);
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        } else {
            if (left > 0) s.x += from[0];
            if (left > 1) s.y += from[1];
            if (left > 2) s.z += from[2];
        }
    }
    part[run][lane] = s;
    __syncthreads();
    if (threadIdx.x < kSumColumns) {
        const int column = blockIdx.x * kSumColumns + threadIdx.x;
        float total = 0.f;
        for (int q = 0; q < kRuns; ++q) total += reinterpret_cast<const float *>(&part[q][0])[threadIdx.x];
        if (column < A.N) store_param<T>(A.to[array], A.f32[array], column, total);
    }
}

// Rows wider than a work-group's chunks of eight.
bool wide(int N) { return N > kMostLanes * 8; }

// Threads and work-groups of the backward pass.
int backward_threads(int lanes) { return lanes <= 512 ? 512 : 1024; }
int backward_blocks(int T, int N) {
    const int lanes = row_lanes(N, kMostLanes), groups = backward_threads(lanes) / lanes;
    const int64_t most = (1 << 22) / N < 128 ? 128 : (1 << 22) / N > 512 ? 512 : (1 << 22) / N;
    const int64_t all = ((int64_t)T + groups - 1) / groups;
    return (int)(all < most ? all : most);
}

}  // namespace

size_t norm_workspace_bytes(int T, int N) { return (size_t)backward_blocks(T, N) * kArrays * N * 4; }

hipError_t launch_norm_forward(NormArgs a, hipStream_t st) {
    a.lanes = row_lanes(a.N, kMostLanes);
    const int threads = a.lanes < 256 ? 256 : a.lanes, groups = threads / a.lanes;
    const dim3 grid((unsigned)(((int64_t)a.T + groups - 1) / groups));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, a);
            return hipGetLastError();
        };
        if (a.end) return wide(a.N) ? go(sk_norm_forward<T, 0, true>) : go(sk_norm_forward<T, 1, true>);
        return wide(a.N) ? go(sk_norm_forward<T, 0, false>) : go(sk_norm_forward<T, 1, false>);
    });
}

hipError_t launch_norm_backward(NormArgs a, void *ws, hipStream_t st) {
    a.lanes = row_lanes(a.N, kMostLanes);
    a.parts = static_cast<float *>(ws);
    SumArgs s = {};
    void *const wanted[kArrays] = {a.g_after_w, a.g_before_w, a.g_after_b, a.g_before_b,
                                   a.gate_kind == SK_GATE_COLUMNS ? a.g_gate : nullptr};
    for (int i = 0; i < kArrays; ++i) {
        a.place[i] = -1;
        if (!wanted[i]) continue;
        s.to[a.arrays] = wanted[i];
        s.f32[a.arrays] = i == kGate ? a.gf32 : a.wf32;
        a.place[i] = a.arrays++;
    }
    const bool more = a.gate_kind > SK_GATE_ROWS || a.after_b || a.g_after_b || a.g_before_b;
    s.parts = a.parts;
    s.blocks = backward_blocks(a.T, a.N);
    s.arrays = a.arrays;
    s.N = a.N;
    const int threads = backward_threads(a.lanes);
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)s.blocks), dim3(threads), 0, st, a);
            return hipGetLastError();
        };
        auto by_more = [&](auto is_wide, auto end, auto most) {
            constexpr bool W = decltype(is_wide)::value, B = decltype(end)::value;
            constexpr int M = decltype(most)::value;
            return more ? go(sk_norm_backward<T, W, B, true, M>) : go(sk_norm_backward<T, W, B, false, M>);
        };
        auto by_size = [&](auto end) {
            constexpr std::integral_constant<int, 512> half{};
            constexpr std::integral_constant<int, 1024> full{};
            if (wide(a.N)) return by_more(std::true_type{}, end, full);
            return threads == 512 ? by_more(std::false_type{}, end, half) : by_more(std::false_type{}, end, full);
        };
        const hipError_t e = a.T == 0 ? hipSuccess : a.end ? by_size(std::true_type{}) : by_size(std::false_type{});
        if (e != hipSuccess || !a.arrays) return e;
        hipLaunchKernelGGL((sk_norm_sums<T>), dim3((unsigned)((a.N + kSumColumns - 1) / kSumColumns), a.arrays),
                           dim3(kSumThreads), 0, st, s);
        return hipGetLastError();
    });
}

}  // namespace sk
