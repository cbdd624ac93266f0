// sk_rows.h -- rows shared out over groups of lanes, for the norms and the rows in 8 bits.
#pragma once

#include "sk_routed.h"

namespace sk {

// A work-group takes rows by groups of `lanes` threads, a power of two of 8 or more; a lane takes chunks of eight
// columns, `lanes` chunks apart.
struct RowGroup {
    int lanes, lane, group, groups;
    __device__ __forceinline__ explicit RowGroup(int lanes_)
        : lanes(lanes_), lane((int)threadIdx.x & (lanes_ - 1)), group((int)threadIdx.x / lanes_),
          groups((int)blockDim.x / lanes_) {}
};

// Lanes for rows of `columns`: as many as there are chunks, up to `most`.
inline int row_lanes(int64_t columns, int most) {
    int lanes = 8;
    while (lanes < most && (int64_t)lanes * 8 < columns) lanes *= 2;
    return lanes;
}

struct Sum {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
// Of numbers that are not negative, by their bits: NaN counts as the largest, so it is not lost.
struct Largest {
    __device__ __forceinline__ float operator()(float a, float b) const {
        const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
        return __uint_as_float(x > y ? x : y);
    }
};

// Over `lanes` <= 64 neighbouring lanes of a wavefront; every lane gets the same bits.
template <class Op>
__device__ __forceinline__ float lanes_reduce(float v, int lanes) {
    const Op op;
    v = op(v, dpp<kQuadXor1>(v));
    v = op(v, dpp<kQuadXor2>(v));
    v = op(v, dpp<kHalfMirror>(v));
    if (lanes > 8) v = op(v, dpp<kRowRor8>(v));
    if (lanes > 16) {
        const LanePair p = swap16(v);
        v = op(p.lo, p.hi);
    }
    if (lanes > 32) {
        const LanePair p = swap32(v);
        v = op(p.lo, p.hi);
    }
    return v;
}

constexpr int kRowWaves = 16;  // of a work-group at most

// Over each group's lanes.  `turn` counts the reductions of a kernel: two places in LDS take turns, so that one barrier
// a reduction is enough.  Every thread of the work-group calls it.
template <class Op, int NV, int MOST>
__device__ __forceinline__ void group_reduce(const RowGroup &g, float (&v)[NV], float (&lds)[2][MOST][kRowWaves],
                                             int &turn) {
    static_assert(NV <= MOST);
    const Op op;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = lanes_reduce<Op>(v[i], g.lanes);
    if (g.lanes <= 64) return;
    const int here = turn & 1, waves = g.lanes / 64;
    ++turn;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) lds[here][i][threadIdx.x >> 6] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const float *from = &lds[here][i][g.group * waves];
        float s = from[0];
        for (int w = 1; w < waves; ++w) s = op(s, from[w]);
        v[i] = s;
    }
}

// The first `left` of eight elements; zeros for the others.  left may be anything.
template <class T>
__device__ __forceinline__ void load_left(const T *p, int left, float (&v)[8]) {
    if (left >= 8)
        load8(p, v);
    else
        load_some(p, 0, left, v);
}
template <class T>
__device__ __forceinline__ void store_left(T *p, int left, const float (&v)[8]) {
    if (left >= 8)
        store8(p, v);
    else
        store_some(p, 0, left, v);
}

}  // namespace sk
