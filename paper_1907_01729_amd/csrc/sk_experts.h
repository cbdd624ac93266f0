// sk_experts.h -- arguments of the experts' products, and the tiles of their rows.
#pragma once

#include <type_traits>

#include "sk_routed.h"

namespace sk {

enum { kForward = 0, kInput = 1, kWeight = 2 };

struct ExpertArgs {
    const void *x, *w, *gy;
    const int32_t *offsets, *tokens, *slots;  // tokens (slots): null where x (gx) has one row for each row
    void *out;
    float *out32;  // where set, the rows' result in 32 bits goes here instead
    int T, k, E, K, N, dtype;
};
size_t experts_workspace_bytes(int T, int k, int K);
hipError_t launch_experts_forward(const ExpertArgs &a, hipStream_t st);
hipError_t launch_experts_input(const ExpertArgs &a, void *ws, hipStream_t st);
hipError_t launch_experts_weight(const ExpertArgs &a, hipStream_t st);

template <class T>
using Frag8 = T __attribute__((ext_vector_type(8)));

// Rows [begin, end) of an expert; e = E: the rows of none.  Whatever the offsets hold, within the rows there are.
struct RowRange {
    int begin, end;
};
__device__ __forceinline__ RowRange expert_rows(const ExpertArgs &A, int e) {
    const int rows = A.T * A.k;
    RowRange r;
    r.begin = min(max(A.offsets[e], 0), rows);
    r.end = e < A.E ? min(max(A.offsets[e + 1], 0), rows) : rows;
    if (r.end < r.begin) r.end = r.begin;
    return r;
}

// The expert and the rows of the id-th tile of up to `tile` rows, tiles counted over the experts in order (E: the
// rows of none); expert = -1 past the last.  Every lane of the wavefront calls it and gets the answer.
struct RowTile {
    int expert, begin, end;
};
__device__ __forceinline__ RowTile find_row_tile(const ExpertArgs &A, int tile, int id) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int e0 = 0; e0 <= A.E; e0 += 64) {
        const int e = e0 + lane;
        RowRange r = {0, 0};
        if (e <= A.E) r = expert_rows(A, e);
        const int n = (r.end - r.begin + tile - 1) / tile;
        int upto = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(upto, d, 64);
            if (lane >= d) upto += up;
        }
        upto += before;
        const bool mine = id < upto && id >= upto - n;
        const uint64_t who = __builtin_amdgcn_ballot_w64(mine);
        if (who) {
            const int q = __builtin_ctzll(who);
            const int begin = __builtin_amdgcn_readlane(r.begin + (id - (upto - n)) * tile, q);
            const int end = __builtin_amdgcn_readlane(r.end, q);
            return {e0 + q, begin, min(begin + tile, end)};
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return {-1, 0, 0};
}

}  // namespace sk
