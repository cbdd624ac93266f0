// sk_norm.h -- launchers of the norms around a block.
#pragma once

#include "sk_routed.h"

namespace sk {

struct NormArgs {
    int end;  // 1: a block's end; 0: the norm alone, of `residual` (in the backward pass of `out`)
    const void *h, *residual, *gate;
    const void *after_w, *after_b, *before_w, *before_b;
    void *out, *next;
    float *stats;  // [T, 4]: mean and r of h, of out; may be null in the forward pass
    const void *g_out, *g_next;
    void *g_h, *g_residual, *g_gate, *g_after_w, *g_after_b, *g_before_w, *g_before_b;
    float *parts;  // [blocks, arrays, N]
    int T, N, dtype, wf32, gate_kind, gf32, after, before;
    float scale, eps_after, eps_before;
    int lanes, arrays;
    int place[5];  // of each of the sums over the rows among the arrays; -1: not wanted
};
size_t norm_workspace_bytes(int T, int N);
hipError_t launch_norm_forward(NormArgs a, hipStream_t st);
hipError_t launch_norm_backward(NormArgs a, void *ws, hipStream_t st);

}  // namespace sk
