// sk_norm.hip -- the norms around a block, fused with its gate and its residual, and their gradients.
//
//   norm(x) = xh w + b,  xh = (x - m) r,  r = (mean((x - m)^2) + eps)^-1/2,  m = mean(x) or 0
//   forward   n = norm_after(h) or h,  out = scale residual + gate n,  next = norm_before(out)
//   backward  of a norm, with d = gy w:  gx = r (d - [m] mean(d) - xh mean(d xh)),  gw = sum_t gy xh,  gb = sum_t gy
//             g = g_out + (norm_before's),  g_residual = scale g,  g_gate = g n,  dn = gate g,  g_h = (norm_after's of dn)
//
// Bound by memory: each array is read or written once, a row stays in registers between its passes, statistics and sums
// are in 32 bits.  65536 x 2048, bf16: the norm 96 us (5.6 TB/s), its gradients 158 (5.1); a block's end with two norms
// 186 (5.8), its gradients 328 (4.9); a 2 GiB copy reaches 4.9 TB/s here.  Rows of odd width cost little more (16384 x
// 1001: 25 us, 53 for the gradients).
#include "sk_norm.h"

#include <type_traits>

#include "sk_rows.h"

namespace sk {
namespace {

constexpr int kMostLanes = 1024;

// ---- eight columns ----

template <class T>
using Raw8 = T __attribute__((ext_vector_type(8)));

// A lane's columns [c, c + 8).  Where a row is no whole number of eights its last window lies back over the one before:
// the lane's own columns are those from c + lo on, the others are computed and stored twice, with the same bits, and
// masked in sums.  lo = 8: none.  Rows of less than eight columns have hi of them.
struct Window {
    int c, lo, hi;
    __device__ __forceinline__ Window(int at, int N) {
        c = max(min(at, N - 8), 0);
        lo = min(at - c, 8);
        hi = min(N, 8);
    }
    __device__ __forceinline__ bool any() const { return lo < hi; }
    __device__ __forceinline__ bool own(int i) const { return i >= lo && i < hi; }
};

template <class T>
__device__ __forceinline__ Raw8<T> load_raw(const T *p, const Window &w) {
    Raw8<T> v = {};
    if (w.hi == 8) {
        __builtin_memcpy(&v, p + w.c, sizeof(v));
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < w.hi) v[i] = p[i];
    }
    return v;
}
template <class T>
__device__ __forceinline__ void store_window(T *p, const Window &w, const float (&v)[8]) {
    if (!w.any()) return;
    if (w.hi == 8)
        store8(p + w.c, v);
    else
        store_some(p, 0, w.hi, v);
}
// Eight of a parameter's values, of type T or float.
template <class T>
__device__ __forceinline__ void load_param(const void *p, int f32, const Window &w, float (&v)[8]) {
    if (f32) {
        const Raw8<float> r = load_raw(static_cast<const float *>(p), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = r[i];
    } else {
        const Raw8<T> r = load_raw(static_cast<const T *>(p), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)r[i];
    }
}
// Of a parameter that may not be there.
template <class T>
__device__ __forceinline__ void load_param(const void *p, int f32, const Window &w, float none, float (&v)[8]) {
    if (p) {
        load_param<T>(p, f32, w, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = none;
    }
}
template <class T>
__device__ __forceinline__ float param_at(const void *p, int f32, int64_t at) {
    return f32 ? static_cast<const float *>(p)[at] : (float)static_cast<const T *>(p)[at];
}
template <class T>
__device__ __forceinline__ void store_param(void *p, int f32, int64_t at, float v) {
    if (f32)
        static_cast<float *>(p)[at] = v;
    else
        static_cast<T *>(p)[at] = (T)v;
}
// The gate of a window of a row.
template <class T>
__device__ __forceinline__ void load_gate(const NormArgs &A, int64_t row, const Window &w, float (&v)[8]) {
    if (A.gate_kind > SK_GATE_ROWS) {
        const int64_t at = A.gate_kind == SK_GATE_FULL ? row * A.N : 0;
        const char *p = static_cast<const char *>(A.gate) + at * (A.gf32 ? 4 : (int)sizeof(T));
        load_param<T>(p, A.gf32, w, v);
    } else {
        const float one = A.gate_kind == SK_GATE_NONE ? 1.f : param_at<T>(A.gate, A.gf32, row);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = one;
    }
}

// A lane's own of eight numbers, added up.
__device__ __forceinline__ float sum_own(const Window &w, const float (&v)[8]) {
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = w.own(i) ? v[i] : 0.f;
    return tree_sum<8>(s);
}

// Each step is rounded by itself, as a program's own steps in 32 bits are: a sum that lies next to a border between two
// 16-bit numbers then falls to the same side for both.
template <class T>
__device__ __forceinline__ void norm8(const Raw8<T> &x, float mean, float r, const float (&w)[8], const float (&b)[8],
                                      float (&y)[8]) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float xh = ((float)x[i] - mean) * r;
        y[i] = xh * w[i] + b[i];
    }
}
template <class T>
__device__ __forceinline__ void residual8(const Raw8<T> &residual, float scale, const float (&gate)[8],
                                          const float (&n)[8], float (&y)[8]) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = scale * (float)residual[i] + gate[i] * n[i];
}

// ---- forward ----

// A row to a group of lanes.  V: the windows that a lane holds in registers; 0: rows wider than that, read again from
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
    // f(window held, window)
    auto each = [&](auto f) {
        if constexpr (V > 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) f(v, Window((v * g.lanes + g.lane) * 8, N));
        } else {
            for (int c = g.lane * 8; c < N; c += g.lanes * 8) f(0, Window(c, N));
        }
    };
    // Mean and r of a row that `load` gives a window of.
    auto statistics = [&](int kind, float eps, auto load, float &mean, float &r) {
        mean = 0.f;
        float s[1] = {0.f};
        if (kind == SK_NORM_CENTRED) {
            each([&](int v, const Window &w) {
                const Raw8<T> x = load(v, w);
                float q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) q[i] = (float)x[i];
                s[0] += sum_own(w, q);
            });
            group_reduce<Sum>(g, s, lds, turn);
            mean = s[0] * each_n;
            s[0] = 0.f;
        }
        each([&](int v, const Window &w) {
            const Raw8<T> x = load(v, w);
            float q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = ((float)x[i] - mean) * ((float)x[i] - mean);
            s[0] += sum_own(w, q);
        });
        group_reduce<Sum>(g, s, lds, turn);
        r = rsqrtf(s[0] * each_n + eps);
    };

    const T *residual = static_cast<const T *>(A.residual) + row * N;
    T *out = static_cast<T *>(A.out) + row * N;
    Raw8<T> y[H];  // the residual, then the sum; or the norm's input
    float4 stats = {0.f, 1.f, 0.f, 1.f};
    if constexpr (V > 0) each([&](int v, const Window &w) { y[v] = load_raw(residual, w); });
    if constexpr (END) {
        const T *h = static_cast<const T *>(A.h) + row * N;
        Raw8<T> x[H];
        if constexpr (V > 0) each([&](int v, const Window &w) { x[v] = load_raw(h, w); });
        auto load_h = [&](int v, const Window &w) { return V > 0 ? x[v] : load_raw(h, w); };
        if (A.after) statistics(A.after, A.eps_after, load_h, stats.x, stats.y);
        each([&](int v, const Window &w) {
            const Raw8<T> hv = load_h(v, w);
            float n[8], gate[8], wv[8], bv[8], sum[8];
            if (A.after) {
                load_param<T>(A.after_w, A.wf32, w, 1.f, wv);
                load_param<T>(A.after_b, A.wf32, w, 0.f, bv);
                norm8<T>(hv, stats.x, stats.y, wv, bv, n);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) n[i] = (float)hv[i];
            }
            load_gate<T>(A, row, w, gate);
            residual8<T>(V > 0 ? y[v] : load_raw(residual, w), A.scale, gate, n, sum);
            // Rounded here: the next norm, and the backward pass of it, take the sum as it is stored.
#pragma unroll
            for (int i = 0; i < 8; ++i) y[v][i] = (T)sum[i];
            if (mine) store_window(out, w, sum);
        });
    }
    if (A.before) {
        auto load_y = [&](int v, const Window &w) { return V > 0 ? y[v] : load_raw(END ? out : residual, w); };
        statistics(A.before, A.eps_before, load_y, stats.z, stats.w);
        each([&](int v, const Window &w) {
            float z[8], wv[8], bv[8];
            load_param<T>(A.before_w, A.wf32, w, 1.f, wv);
            load_param<T>(A.before_b, A.wf32, w, 0.f, bv);
            norm8<T>(load_y(v, w), stats.z, stats.w, wv, bv, z);
            if (mine) store_window(static_cast<T *>(A.next) + row * N, w, z);
        });
    }
    if (A.stats && mine && g.lane == 0) reinterpret_cast<float4 *>(A.stats)[row] = stats;
}

// ---- backward ----

// The sums over the rows.
enum { kAfterW, kBeforeW, kAfterB, kBeforeB, kGate, kArrays };
template <int A>
using Array = std::integral_constant<int, A>;

// A work-group's groups go through rows, the next row's loads under way while a row is worked on (65536 x 2048, bf16,
// without / with that, in us: the norm's gradients 197 / 161, a block's end with two norms 359 / 332, with the next norm
// alone and one gradient for both 224 / 223).  The sums over the rows stay in registers and are added up over the groups
// at the end, into one part a work-group; WIDE: rows of more windows than lanes, whose sums lie in the work-group's own
// part of memory and which are read again from the caches for each pass over them.  BIAS: there are sums for biases; GATE: the gate is more than a number a row.  Without them fewer
// registers are taken: two work-groups of 512 threads fit on a CU with up to 128 (16-bit rows, no such gate).  Of 1024
// threads one does; where its registers do not hold the next row, too, that is loaded when it is its turn.
template <class T, bool WIDE, bool END, bool BIAS, bool GATE, int THREADS>
__global__ __launch_bounds__(THREADS, GATE || (END && sizeof(T) == 4) ? 2 : 4) void sk_norm_backward(NormArgs A) {
    constexpr bool kAhead = !WIDE && (THREADS < 1024 || !END || (sizeof(T) == 2 && !BIAS && !GATE));
    constexpr auto has = [](int array) { return array < kAfterB || (array == kGate ? GATE : BIAS); };
    __shared__ float lds[2][3][kRowWaves];
    __shared__ float total[WIDE ? 8 : THREADS * 8];
    const RowGroup g(A.lanes);
    const int N = A.N;
    const float each_n = 1.f / (float)N;
    const bool before = A.before && A.g_next, after = END && A.after;
    const bool wants_h = after || (END && A.g_gate), sums_gate = END && A.gate_kind == SK_GATE_ROWS && A.g_gate;
    int turn = 0;
    float sums[WIDE ? 1 : kArrays][8] = {};
    auto part_of = [&](int array) {
        return A.place[array] < 0 ? nullptr
                                  : A.parts + ((int64_t)blockIdx.x * A.arrays + A.place[array]) * N;
    };
    bool first = true;  // WIDE: the work-group's first row
    auto add = [&](auto which, const Window &w, const float (&v)[8]) {
        constexpr int array = decltype(which)::value;
        if constexpr (!has(array)) {
        } else if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[array][i] += v[i];
        } else if (float *to = part_of(array)) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (w.own(i)) to[w.c + i] = first ? v[i] : to[w.c + i] + v[i];
        }
    };
    // A window of a row.
    struct Row {
        Raw8<T> x, dy, go, h, gate;
        float one;  // the gate, where it is a number
    };
    auto load = [&](int64_t row, const Window &w) {
        Row v = {};
        const int64_t at = row * N;
        if (before) {
            v.x = load_raw(static_cast<const T *>(A.out) + at, w);
            v.dy = load_raw(static_cast<const T *>(A.g_next) + at, w);
        }
        if (END && A.g_out) v.go = load_raw(static_cast<const T *>(A.g_out) + at, w);
        if (wants_h) v.h = load_raw(static_cast<const T *>(A.h) + at, w);
        if constexpr (GATE) {
            if (A.gate_kind == SK_GATE_FULL && !A.gf32) v.gate = load_raw(static_cast<const T *>(A.gate) + at, w);
        }
        v.one = !END || A.gate_kind != SK_GATE_ROWS ? 1.f : param_at<T>(A.gate, A.gf32, row);
        return v;
    };
    float wb[8], wa[8];
    auto load_weights = [&](const Window &w) {
        load_param<T>(A.before_w, A.wf32, w, 1.f, wb);
        if (END) load_param<T>(A.after_w, A.wf32, w, 1.f, wa);
    };
    const Window fixed(g.lane * 8, N);
    if (!WIDE) load_weights(fixed);
    const int64_t step = (int64_t)gridDim.x * g.groups, last = A.T - 1;
    int64_t r0 = (int64_t)blockIdx.x * g.groups;
    Row v, ahead;
    float4 stats, stats_ahead;
    if (kAhead) ahead = load(min(r0 + g.group, last), fixed);
    stats_ahead = reinterpret_cast<const float4 *>(A.stats)[min(r0 + g.group, last)];
    for (; r0 < A.T; r0 += step) {
        const bool mine = r0 + g.group < A.T;
        const int64_t row = min(r0 + g.group, last), at = row * N;
        stats = stats_ahead;
        if (kAhead)
            v = ahead;
        else if (!WIDE)
            v = load(row, fixed);
        if (r0 + step < A.T) {
            const int64_t next = min(r0 + step + g.group, last);
            if (kAhead) ahead = load(next, fixed);
            stats_ahead = reinterpret_cast<const float4 *>(A.stats)[next];
        }
        auto each = [&](auto f) {
            if constexpr (!WIDE) {
                f(fixed);
            } else {
                for (int c = g.lane * 8; c < N; c += g.lanes * 8) {
                    const Window w(c, N);
                    v = load(row, w);
                    load_weights(w);
                    f(w);
                }
            }
        };
        // d times the gate.
        auto gated = [&](const Window &w, float (&d)[8]) {
            if (GATE && (A.gate_kind == SK_GATE_COLUMNS || (A.gate_kind == SK_GATE_FULL && A.gf32))) {
                float gate[8];
                load_gate<T>(A, row, w, gate);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] *= gate[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] *= GATE && A.gate_kind == SK_GATE_FULL ? (float)v.gate[i] : v.one;
            }
        };
        auto xh = [&](int i) { return ((float)v.x[i] - stats.z) * stats.w; };
        auto hh = [&](int i) { return after ? ((float)v.h[i] - stats.x) * stats.y : (float)v.h[i]; };
        float s[2] = {0.f, 0.f};
        if (before) {
            each([&](const Window &w) {
                float a[8], b[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    a[i] = (float)v.dy[i] * wb[i];
                    b[i] = a[i] * xh(i);
                }
                s[0] += sum_own(w, a), s[1] += sum_own(w, b);
            });
            group_reduce<Sum>(g, s, lds, turn);
            s[0] = A.before == SK_NORM_CENTRED ? s[0] * each_n : 0.f;
            s[1] *= each_n;
        }
        // The sum's gradient.
        auto gradient = [&](float (&d)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] = (float)v.go[i];
                if (before) d[i] += stats.w * ((float)v.dy[i] * wb[i] - s[0] - xh(i) * s[1]);
            }
        };
        float d[8], q[3] = {0.f, 0.f, 0.f};
        each([&](const Window &w) {
            gradient(d);
            if (before && mine) {
                float xd[8], yd[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) yd[i] = (float)v.dy[i], xd[i] = yd[i] * xh(i);
                add(Array<kBeforeW>{}, w, xd);
                add(Array<kBeforeB>{}, w, yd);
            }
            if constexpr (!END) {
                if (mine && A.g_residual) store_window(static_cast<T *>(A.g_residual) + at, w, d);
            } else {
                float e[8];
                if (mine && A.g_residual) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = A.scale * d[i];
                    store_window(static_cast<T *>(A.g_residual) + at, w, e);
                }
                if (A.g_gate) {
                    float ba[8];
                    load_param<T>(A.after_b, A.wf32, w, 0.f, ba);
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = d[i] * (after ? hh(i) * wa[i] + ba[i] : hh(i));
                    if (sums_gate) q[2] += sum_own(w, e);
                    if (GATE && A.gate_kind == SK_GATE_COLUMNS && mine) add(Array<kGate>{}, w, e);
                    if (GATE && A.gate_kind == SK_GATE_FULL && mine) {
                        if (A.gf32)
                            store_window(static_cast<float *>(A.g_gate) + at, w, e);
                        else
                            store_window(static_cast<T *>(A.g_gate) + at, w, e);
                    }
                }
                gated(w, d);
                if (after) {
                    float a[8], b[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        a[i] = d[i] * wa[i];
                        b[i] = a[i] * hh(i);
                        e[i] = d[i] * hh(i);
                    }
                    q[0] += sum_own(w, a), q[1] += sum_own(w, b);
                    if (mine) {
                        add(Array<kAfterW>{}, w, e);
                        add(Array<kAfterB>{}, w, d);
                    }
                } else if (mine && A.g_h) {
                    store_window(static_cast<T *>(A.g_h) + at, w, d);
                }
            }
        });
        if (END && (after || sums_gate)) {
            group_reduce<Sum>(g, q, lds, turn);
            q[0] = A.after == SK_NORM_CENTRED ? q[0] * each_n : 0.f;
            q[1] *= each_n;
            if (sums_gate && mine && g.lane == 0) store_param<T>(A.g_gate, A.gf32, row, q[2]);
            if (after && A.g_h && mine)
                each([&](const Window &w) {
                    if (WIDE) {
                        gradient(d);
                        gated(w, d);
                    }
                    float e[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = stats.y * (d[i] * wa[i] - q[0] - hh(i) * q[1]);
                    store_window(static_cast<T *>(A.g_h) + at, w, e);
                });
        }
        first = false;
    }
    if constexpr (!WIDE) {
#pragma unroll
        for (int a = 0; a < kArrays; ++a) {
            float *to = has(a) ? part_of(a) : nullptr;
            if (!to) continue;
            // The groups one after the other, by columns.
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (fixed.own(i)) total[g.group * g.lanes * 8 + fixed.c + i] = sums[a][i];
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
    int f32[kArrays], from[kArrays];  // from: its place among the parts' arrays; -1: none, its sum is zero
    int blocks, arrays, N;
};

template <class T>
__global__ __launch_bounds__(kSumThreads) void sk_norm_sums(SumArgs A) {
    constexpr int kLanes = kSumColumns / 4, kRuns = kSumThreads / kLanes;
    __shared__ float4 part[kRuns][kLanes];
    const int lane = threadIdx.x % kLanes, run = threadIdx.x / kLanes, array = blockIdx.y, place = A.from[array];
    const int c = blockIdx.x * kSumColumns + lane * 4, left = A.N - c;
    const int blocks = place < 0 ? 0 : A.blocks, each = (blocks + kRuns - 1) / kRuns, end = min(blocks, (run + 1) * each);
    float4 s = {0.f, 0.f, 0.f, 0.f};
    for (int b = run * each; b < end; ++b) {
        const float *from = A.parts + ((int64_t)b * A.arrays + place) * A.N + c;
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

// Threads and work-groups of the backward pass.
bool wide(int N) { return N > kMostLanes * 8; }
int backward_threads(int lanes) { return lanes <= 512 ? 512 : 1024; }
// few: as many as fit on the CUs one by one.
int backward_blocks(int T, int N, bool few) {
    const int lanes = row_lanes(N, kMostLanes), groups = backward_threads(lanes) / lanes;
    const int64_t most = lanes <= 512 && !few ? 512 : 256;
    const int64_t all = ((int64_t)T + groups - 1) / groups;
    return (int)(all < most ? all : most);
}

}  // namespace

size_t norm_workspace_bytes(int T, int N) { return (size_t)backward_blocks(T, N, false) * kArrays * N * 4; }

hipError_t launch_norm_forward(NormArgs a, hipStream_t st) {
    // Two windows a lane, which wait for memory together: the norm of 65536 x 2048 in 95 us, with one 110; a block's end
    // with two norms, 16384 x 2048, in 47, with one 54.  A block's end loads two arrays at once already: with one norm
    // or none 181 us with a window, 191 with two.
    const bool two = !a.end || (a.after && a.before);
    a.lanes = row_lanes(two ? (a.N + 1) / 2 : a.N, kMostLanes);
    const int windows = (a.N + a.lanes * 8 - 1) / (a.lanes * 8), V = windows <= 2 ? windows : windows <= 4 ? 4 : 0;
    const int threads = a.lanes < 256 ? 256 : a.lanes, groups = threads / a.lanes;
    const dim3 grid((unsigned)(((int64_t)a.T + groups - 1) / groups));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, a);
            return hipGetLastError();
        };
        auto by_end = [&](auto windows) {
            constexpr int W = decltype(windows)::value;
            return a.end ? go(sk_norm_forward<T, W, true>) : go(sk_norm_forward<T, W, false>);
        };
        if (V == 1) return by_end(std::integral_constant<int, 1>{});
        if (V == 2) return by_end(std::integral_constant<int, 2>{});
        if (V == 4) return by_end(std::integral_constant<int, 4>{});
        return by_end(std::integral_constant<int, 0>{});
    });
}

hipError_t launch_norm_backward(NormArgs a, void *ws, hipStream_t st) {
    a.lanes = row_lanes(a.N, kMostLanes);
    a.parts = static_cast<float *>(ws);
    SumArgs s = {};
    int outputs = 0;
    void *const wanted[kArrays] = {a.g_after_w, a.g_before_w, a.g_after_b, a.g_before_b,
                                   a.gate_kind == SK_GATE_COLUMNS ? a.g_gate : nullptr};
    for (int i = 0; i < kArrays; ++i) {
        a.place[i] = -1;
        if (!wanted[i]) continue;
        s.to[outputs] = wanted[i];
        s.f32[outputs] = i == kGate ? a.gf32 : a.wf32;
        if (a.g_next || (i != kBeforeW && i != kBeforeB)) a.place[i] = a.arrays++;
        s.from[outputs++] = a.place[i];
    }
    const bool bias = a.g_after_b || a.g_before_b, gate = a.gate_kind > SK_GATE_ROWS;
    s.parts = a.parts;
    s.blocks = backward_blocks(a.T, a.N, gate || (a.end && a.dtype == SK_F32));
    s.arrays = a.arrays;
    s.N = a.N;
    const int threads = backward_threads(a.lanes);
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)s.blocks), dim3(threads), 0, st, a);
            return hipGetLastError();
        };
        auto by_sums = [&](auto is_wide, auto end, auto most) {
            constexpr bool W = decltype(is_wide)::value, B = decltype(end)::value;
            constexpr int M = decltype(most)::value;
            if constexpr (B) {
                if (gate)
                    return bias ? go(sk_norm_backward<T, W, B, true, true, M>)
                                : go(sk_norm_backward<T, W, B, false, true, M>);
            }
            return bias ? go(sk_norm_backward<T, W, B, true, false, M>)
                        : go(sk_norm_backward<T, W, B, false, false, M>);
        };
        auto by_size = [&](auto end) {
            constexpr std::integral_constant<int, 512> half{};
            constexpr std::integral_constant<int, 1024> full{};
            if (wide(a.N)) return by_sums(std::true_type{}, end, full);
            return threads == 512 ? by_sums(std::false_type{}, end, half) : by_sums(std::false_type{}, end, full);
        };
        const hipError_t e = a.T == 0 ? hipSuccess : a.end ? by_size(std::true_type{}) : by_size(std::false_type{});
        if (e != hipSuccess || !outputs) return e;
        hipLaunchKernelGGL((sk_norm_sums<T>), dim3((unsigned)((a.N + kSumColumns - 1) / kSumColumns), outputs),
                           dim3(kSumThreads), 0, st, s);
        return hipGetLastError();
    });
}

}  // namespace sk
