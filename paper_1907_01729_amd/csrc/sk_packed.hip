// sk_packed.hip -- rows in 8 bits, and the activations whose input is kept so for the backward pass.
//
//   s = max |x| / 127 over a row or 128 columns of it,  q = x / s to nearest even,  x~ = s q
//   y = act(x), or act(v) u of the two halves (v, u) of a row
//   backward  y = act(x~),  gx = gy act'(x~);  gated: gv = gy u~ act'(v~), gu = gy act(v~)
//
// Bound by memory.  bf16: packing 16384 x 2048 by rows 20 us (4.9 TB/s), by blocks 13 (7.8, partly from the last-level
// cache), unpacking it 12; the gated activation of 32768 x 2048 with its rows kept 47 us (5.7 TB/s; vector issue, too, is 83 % of it), from the
// kept rows again with the gradient 57 (5.9).
#include "sk_packed.h"

#include <type_traits>

#include "sk_rows.h"

namespace sk {
namespace {

constexpr int kThreads = 256;
constexpr int kMostLanes = 1024;
constexpr int kBlockLanes = kPackBlock / 8;  // lanes of a block of columns

// ---- rounding to 8 bits ----

// The scale of numbers up to `most`.  Where it is so small that its reciprocal would overflow, numbers and scale are
// multiplied by a power of two first (exactly).
struct Scale {
    float s, scaled, inverse;
    bool tiny;
};
constexpr float kUp = 0x1p64f;
__device__ __forceinline__ Scale scale_of(float most) {
    Scale c;
    c.s = most / 127.f;
    if (!(most < __builtin_inff())) c.s = __builtin_nanf("");
    c.tiny = most < 0x1p-96f;
    c.scaled = c.tiny ? c.s * kUp : c.s;
    c.inverse = c.scaled > 0.f ? __builtin_amdgcn_rcpf(c.scaled) : 0.f;  // NaN and 0: 0
    return c;
}

// Eight whole numbers x / s, to nearest even of the exact quotient, as bytes.  Added to 1.5 2^23, a number has its whole
// part in its lowest bits.  The quotient by the reciprocal is off by less than 2^-15, so it rounds as the exact one does
// unless it lies that near to a half.  There the remainder x - q s decides, which a fused multiplication and addition
// gives exactly (it is a multiple of the last place of s or of x, and no larger than s).
struct Bytes8 {
    uint32_t w[2];
};
__device__ __forceinline__ Bytes8 round8(const float (&x)[8], const Scale &c) {
    constexpr float kMagic = 12582912.f;
    float v[8], f[8], far = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i];
    if (c.tiny) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= kUp;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f[i] = fmaf(v[i], c.inverse, kMagic);
        far = fmaxf(far, fabsf(fmaf(v[i], c.inverse, kMagic - f[i])));
    }
    if (c.tiny || far > 0.5f - 0x1p-14f) {
        const uint32_t half = __float_as_uint(0.5f * c.scaled);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float q = f[i] - kMagic;
            const float left = fmaf(-q, c.scaled, v[i]);
            // above a half, or a half away from an odd number
            if (__float_as_uint(fabsf(left)) + ((uint32_t)(int)q & 1) > half) q += left < 0.f ? -1.f : 1.f;
            f[i] = __builtin_amdgcn_fmed3f(q, -127.f, 127.f) + kMagic;  // a scale of few bits: past 127
        }
    }
    Bytes8 b;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(f[h * 4 + i]);
        const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400), hi = __builtin_amdgcn_perm(u[3], u[2], 0x04000c0c);
        b.w[h] = c.inverse > 0.f ? lo | hi : 0;  // infinities and NaN under a scale of NaN: 0, too
    }
    return b;
}

__device__ __forceinline__ float largest8(const float (&v)[8]) {
    const Largest op;
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = op(m, fabsf(v[i]));
    return m;
}

// Eight of the values as floats; the first `left` of them.
__device__ __forceinline__ void load_bytes(const int8_t *p, int left, float (&v)[8]) {
    if (left >= 8) {
        Bytes8 b;
        __builtin_memcpy(&b, p, 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(b.w[i / 4] >> (8 * (i % 4)));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? (float)p[i] : 0.f;
    }
}
// x~ = s q of eight columns of a row.
__device__ __forceinline__ void load_kept(const PackArgs &A, int64_t row, int c, int left, float (&v)[8]) {
    load_bytes(A.values + row * A.pitch + c, left, v);
    const float *s = A.scales + row * A.blocks;
    if (A.blocks == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= s[0];
    } else if (c % 8 == 0) {
        const float one = left > 0 ? s[c / kPackBlock] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= one;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? v[i] * s[(c + i) / kPackBlock] : 0.f;
    }
}

// ---- activations ----
//
// The activated rows are rounded to 16 bits, since the products' matrix instructions take such factors, and so is in bf16
// their gradient between the product and the activation's derivative: each adds an error of the size of the result's own
// rounding (0.0023 of the norm in all, against 0.0017).  That gradient in 32 bits costs 134 MB more, 22 of 659 us, for 32768
// rows of 1024.  In fp16, whose range would lose numbers there, it is kept so (the gradient's type is a parameter of its
// own).

// exp(x) and 1 / x for rows of type T.  In 16-bit rows by the hardware's power of two, off by one of its units and by |x|
// for its argument's rounding, and its reciprocal, off by one: far below their own rounding.
template <class T>
__device__ __forceinline__ float exp_of(float x) {
    return sizeof(T) == 4 ? expf(x) : ex2(x * kLog2e);
}
template <class T>
__device__ __forceinline__ float inverse_of(float x) {
    return sizeof(T) == 4 ? 1.f / x : __builtin_amdgcn_rcpf(x);
}

// act(x), and its derivative in d.
template <class T, int KIND>
__device__ __forceinline__ float activate(float x, float &d) {
    if constexpr (KIND == SK_ACT_RELU) {
        d = x > 0.f ? 1.f : 0.f;
        return x > 0.f ? x : x != x ? x : 0.f;
    } else if constexpr (KIND == SK_ACT_SILU) {
        const float p = inverse_of<T>(1.f + exp_of<T>(-x));
        d = p * (1.f + x * (1.f - p));
        return x * p;
    } else if constexpr (KIND == SK_ACT_GELU) {
        const float p = 0.5f * erfcf(x * -0.70710678118654752f);  // (1 + erf) / 2 without its cancellation
        d = p + x * exp_of<T>(-0.5f * x * x) * 0.39894228040143268f;
        return x * p;
    } else {
        d = 1.f;
        return x;
    }
}
// Of eight numbers; one choice for all of them.
template <class T>
__device__ __forceinline__ void activate8(int kind, const float (&x)[8], float (&y)[8], float (&d)[8]) {
    auto all = [&](auto k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = activate<T, decltype(k)::value>(x[i], d[i]);
    };
    if (kind == SK_ACT_RELU)
        all(std::integral_constant<int, SK_ACT_RELU>{});
    else if (kind == SK_ACT_SILU)
        all(std::integral_constant<int, SK_ACT_SILU>{});
    else if (kind == SK_ACT_GELU)
        all(std::integral_constant<int, SK_ACT_GELU>{});
    else
        all(std::integral_constant<int, SK_ACT_NONE>{});
}

// ---- a scale a row ----

// V: the chunks that a lane holds in registers; 0: wider rows, read twice.
template <class T, int V>
__global__ __launch_bounds__(kMostLanes) void sk_pack_rows(PackArgs A) {
    __shared__ float lds[2][1][kRowWaves];
    const RowGroup g(A.lanes);
    const int64_t all = (int64_t)blockIdx.x * g.groups + g.group, row = min(all, A.rows - 1);
    const bool mine = all < A.rows;
    const T *x = static_cast<const T *>(A.x) + row * A.columns;
    int turn = 0;
    float v[V ? V : 1][8], most[1] = {0.f};
    const Largest op;
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (i * g.lanes + g.lane) * 8;
            load_left(x + c, A.columns - c, v[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) most[0] = op(most[0], largest8(v[i]));
    } else {
        for (int c = g.lane * 8; c < A.columns; c += g.lanes * 8) {
            load_left(x + c, A.columns - c, v[0]);
            most[0] = op(most[0], largest8(v[0]));
        }
    }
    group_reduce<Largest>(g, most, lds, turn);
    const Scale s = scale_of(most[0]);
    if (!mine) return;
    int8_t *to = A.values + row * A.pitch;
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (i * g.lanes + g.lane) * 8;
            if (c < A.pitch) *reinterpret_cast<Bytes8 *>(to + c) = round8(v[i], s);
        }
    } else {
        for (int c = g.lane * 8; c < A.pitch; c += g.lanes * 8) {
            load_left(x + c, A.columns - c, v[0]);
            *reinterpret_cast<Bytes8 *>(to + c) = round8(v[0], s);
        }
    }
    if (g.lane == 0) A.scales[row] = s.s;
}

// ---- a scale for 128 columns of a row ----

// Sixteen lanes take a block of columns.  ACT: the activation of the rows, too; GATED: of a block of each half.
template <class T, bool ACT, bool GATED>
__global__ __launch_bounds__(kThreads) void sk_pack_blocks(PackArgs A) {
    const int cols = GATED ? A.columns / 2 : A.columns, blocks = (cols + kPackBlock - 1) / kPackBlock;
    const int64_t all = A.rows * blocks, i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kBlockLanes;
    const uint32_t at = (uint32_t)min(i, all - 1), row = at / (uint32_t)blocks;
    const int b = (int)(at - row * (uint32_t)blocks), lane = threadIdx.x % kBlockLanes, c = b * kPackBlock + lane * 8;
    const int left = cols - c;
    float x[GATED ? 2 : 1][8];
#pragma unroll
    for (int h = 0; h < (GATED ? 2 : 1); ++h)
        load_left(static_cast<const T *>(A.x) + (int64_t)row * A.columns + h * cols + c, left, x[h]);
#pragma unroll
    for (int h = 0; h < (GATED ? 2 : 1); ++h) {
        const Scale s = scale_of(lanes_reduce<Largest>(largest8(x[h]), kBlockLanes));
        if (i < all) {
            // GATED: halves of whole blocks
            if (GATED || c < A.pitch)
                *reinterpret_cast<Bytes8 *>(A.values + (int64_t)row * A.pitch + h * cols + c) = round8(x[h], s);
            if (lane == 0) A.scales[(int64_t)row * A.blocks + h * blocks + b] = s.s;
        }
    }
    if constexpr (ACT) {
        float y[8], d[8];
        activate8<T>(A.kind, x[0], y, d);
        if constexpr (GATED) {
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] *= x[1][j];
        }
        if (i < all) store_left(static_cast<T *>(A.y) + (int64_t)row * cols + c, left, y);
    }
}

// ---- eight columns to a thread ----

struct Place {
    int64_t row;
    int c, left;
};
// Thread's row and columns; left <= 0: none.
__device__ __forceinline__ Place place_of(int64_t rows, int cols) {
    const int chunks = (cols + 7) / 8;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t row = i / chunks;
    const int c = (int)(i - row * chunks) * 8;
    return {row, c, row < rows ? cols - c : 0};
}

template <class T, bool GATED>
__global__ __launch_bounds__(kThreads) void sk_activation(PackArgs A) {
    const int cols = GATED ? A.columns / 2 : A.columns;
    const Place p = place_of(A.rows, cols);
    if (p.left <= 0) return;
    const T *x = static_cast<const T *>(A.x) + p.row * A.columns + p.c;
    float v[8], u[8], y[8], d[8];
    load_left(x, p.left, v);
    activate8<T>(A.kind, v, y, d);
    if (GATED) {
        load_left(x + cols, p.left, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] *= u[j];
    }
    store_left(static_cast<T *>(A.y) + p.row * cols + p.c, p.left, y);
}

template <class T>
__global__ __launch_bounds__(kThreads) void sk_unpack(PackArgs A) {
    const Place p = place_of(A.rows, A.columns);
    if (p.left <= 0) return;
    float v[8];
    load_kept(A, p.row, p.c, p.left, v);
    store_left(static_cast<T *>(A.y) + p.row * A.columns + p.c, p.left, v);
}

template <class T, class G, bool GATED>  // G: the type of gy
__global__ __launch_bounds__(kThreads) void sk_activation_backward(PackArgs A) {
    const int cols = GATED ? A.columns / 2 : A.columns;
    const Place p = place_of(A.rows, cols);
    if (p.left <= 0) return;
    float v[8], u[8], g[8], y[8], d[8];
    load_kept(A, p.row, p.c, p.left, v);
    if (GATED) load_kept(A, p.row, cols + p.c, p.left, u);
    if (A.gx) load_left(static_cast<const G *>(A.gy) + p.row * cols + p.c, p.left, g);
    activate8<T>(A.kind, v, y, d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (A.gx) v[j] = g[j] * d[j] * (GATED ? u[j] : 1.f);
        if (GATED) {
            const float a = y[j];
            y[j] = a * u[j];
            if (A.gx) u[j] = g[j] * a;
        }
    }
    if (A.y) store_left(static_cast<T *>(A.y) + p.row * cols + p.c, p.left, y);
    if (A.gx) {
        T *gx = static_cast<T *>(A.gx) + p.row * A.columns + p.c;
        store_left(gx, p.left, v);
        if (GATED) store_left(gx + cols, p.left, u);
    }
}

dim3 grid_of(int64_t threads) { return dim3((unsigned)((threads + kThreads - 1) / kThreads)); }

template <bool ACT>
hipError_t launch_blocks(const PackArgs &a, hipStream_t st) {
    const bool gated = ACT && a.gated;
    const int cols = gated ? a.columns / 2 : a.columns;
    const dim3 grid = grid_of(a.rows * ((cols + kPackBlock - 1) / kPackBlock) * kBlockLanes);
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        if constexpr (ACT) {
            if (gated) {
                hipLaunchKernelGGL((sk_pack_blocks<T, true, true>), grid, dim3(kThreads), 0, st, a);
                return hipGetLastError();
            }
        }
        hipLaunchKernelGGL((sk_pack_blocks<T, ACT, false>), grid, dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_pack(const PackArgs &p, hipStream_t st) {
    if (p.blocks != 1 || p.columns <= kPackBlock) return launch_blocks<false>(p, st);
    PackArgs a = p;
    constexpr int kHeld = 2;  // 16384 x 2048 in 20.6 us, with one chunk 26.6, with four 23.2
    a.lanes = row_lanes((a.columns + kHeld - 1) / kHeld, kMostLanes);
    const int threads = a.lanes < kThreads ? kThreads : a.lanes, groups = threads / a.lanes;
    const dim3 grid((unsigned)((a.rows + groups - 1) / groups));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, a);
            return hipGetLastError();
        };
        return a.pitch > a.lanes * 8 * kHeld ? go(sk_pack_rows<T, 0>) : go(sk_pack_rows<T, kHeld>);
    });
}

hipError_t launch_unpack(const PackArgs &a, hipStream_t st) {
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        hipLaunchKernelGGL((sk_unpack<T>), grid_of(a.rows * ((a.columns + 7) / 8)), dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

hipError_t launch_activation_forward(const PackArgs &a, hipStream_t st) {
    if (a.values) {
        // In one pass where the halves are whole blocks.
        if (!a.gated || a.columns % (2 * kPackBlock) == 0) return launch_blocks<true>(a, st);
        const hipError_t e = launch_blocks<false>(a, st);
        if (e != hipSuccess) return e;
    }
    const int cols = a.gated ? a.columns / 2 : a.columns;
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        const dim3 grid = grid_of(a.rows * ((cols + 7) / 8));
        if (a.gated)
            hipLaunchKernelGGL((sk_activation<T, true>), grid, dim3(kThreads), 0, st, a);
        else
            hipLaunchKernelGGL((sk_activation<T, false>), grid, dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

hipError_t launch_activation_backward(const PackArgs &a, hipStream_t st) {
    const int cols = a.gated ? a.columns / 2 : a.columns;
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        const dim3 grid = grid_of(a.rows * ((cols + 7) / 8));
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, a);
            return hipGetLastError();
        };
        if (a.gy32) return a.gated ? go(sk_activation_backward<T, float, true>) : go(sk_activation_backward<T, float, false>);
        return a.gated ? go(sk_activation_backward<T, T, true>) : go(sk_activation_backward<T, T, false>);
    });
}

}  // namespace sk
