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
    int parts;  // weight: parts of the rows
    // Rows in 8 bits: x and w hold pairs of whole numbers, K counts pairs, dtype is the result's.
    const float *x_scale, *w_scale;
    bool whole_out;  // their results are stored in whole 16 bytes
};
// packed: of rows in 8 bits, whose results have any type.
sk_status check_experts(const sk_experts *p, bool packed);
size_t experts_workspace_bytes(int T, int k, int K);
size_t experts_weight_workspace_bytes(const ExpertArgs &a);
hipError_t launch_experts_forward(const ExpertArgs &a, hipStream_t st);
hipError_t launch_experts_packed(const ExpertArgs &a, hipStream_t st);
hipError_t launch_experts_input(const ExpertArgs &a, void *ws, hipStream_t st);
hipError_t launch_experts_weight(const ExpertArgs &a, void *ws, hipStream_t st);

template <class T>
using Frag8 = T __attribute__((ext_vector_type(8)));

// Rows [begin, end) of an expert; e = E: the rows of none.  Whatever the offsets hold, within the rows there are.
// Without offsets all are the first expert's.
struct RowRange {
    int begin, end;
};
__device__ __forceinline__ RowRange expert_rows(const ExpertArgs &A, int e) {
    const int rows = A.T * A.k;
    RowRange r;
    if (!A.offsets) return {e ? rows : 0, rows};
    r.begin = min(max(A.offsets[e], 0), rows);
    r.end = e < A.E ? min(max(A.offsets[e + 1], 0), rows) : rows;
    if (r.end < r.begin) r.end = r.begin;
    return r;
}

// Work-groups go round the eight XCDs in turn; each XCD has its own L2.  This gives XCD b % 8 a run of consecutive
// tiles, so that neighbours share what they read; -1: no tile for this work-group (a grid of a multiple of eight that
// has at least `tiles`).
__device__ __forceinline__ int xcd_order(int b, int tiles) {
    const int run = (tiles + 7) / 8, t = (b & 7) * run + (b >> 3);
    return (b >> 3) < run && t < tiles ? t : -1;
}

// The tile of work-group b: up to `tile` rows of an expert (E: the rows of none), and one of `columns` column tiles.
// Tiles are counted over the experts in order, within an expert by groups of four row tiles that go over the columns
// together.  How many there are is known here alone, from the offsets.  expert = -1: none.  Every lane of the
// wavefront calls it and gets the answer.
struct Tile {
    int expert, begin, end, column;
};
// The inclusive sum over the wavefront's lanes.
__device__ __forceinline__ int lane_sums(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);   // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);   // row_shr:2
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);   // row_shr:4
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);   // row_shr:8
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31 to rows 2 and 3
    return v;
}
__device__ __forceinline__ Tile find_tile(const ExpertArgs &A, int tile, int columns, int b) {
    const int lane = threadIdx.x & 63;
    const auto row_tiles = [&](RowRange r) { return (r.end - r.begin + tile - 1) / tile; };
    const RowRange none = expert_rows(A, A.E);
    // The first 64 experts' ranges and sums stay at hand.
    RowRange mine = {0, 0};
    if (lane < A.E) mine = expert_rows(A, lane);
    int n = row_tiles(mine), upto = lane_sums(n);
    int in_experts = __builtin_amdgcn_readlane(upto, 63);
    for (int e0 = 64; e0 < A.E; e0 += 64)
        in_experts += __builtin_amdgcn_readlane(lane_sums(e0 + lane < A.E ? row_tiles(expert_rows(A, e0 + lane)) : 0), 63);
    const int t = xcd_order(b, (in_experts + row_tiles(none)) * columns);
    if (t < 0) return {-1, 0, 0, 0};
    const int row = t / columns;
    RowRange r = none;
    int expert = A.E, before = in_experts;
    if (row < in_experts) {
        before = 0;
        for (int e0 = 0;;) {
            const uint64_t who = __builtin_amdgcn_ballot_w64(row < upto && row >= upto - n);
            if (who) {
                const int q = __builtin_ctzll(who);
                expert = e0 + q;
                before = __builtin_amdgcn_readlane(upto - n, q);
                r.begin = __builtin_amdgcn_readlane(mine.begin, q);
                r.end = __builtin_amdgcn_readlane(mine.end, q);
                break;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
            e0 += 64;
            if (e0 >= A.E) return {-1, 0, 0, 0};
            mine = {0, 0};
            if (e0 + lane < A.E) mine = expert_rows(A, e0 + lane);
            n = row_tiles(mine);
            upto = lane_sums(n) + before;
        }
    }
    const int i = t - before * columns, m = row_tiles(r);
    const int group = i / (4 * columns), j = i - group * 4 * columns;
    const int high = min(4, m - group * 4);
    const int begin = r.begin + (group * 4 + j % high) * tile;
    return {expert, begin, min(begin + tile, r.end), j / high};
}

}  // namespace sk
