// sk_route.hip -- the router: experts of each token, their weights, counts per expert, the balance and z losses, and
// the order of the (token, slot) pairs by expert; and the gradient of the logits.
//
// A token's logits are held by a group of L lanes, V consecutive ones to a lane (E <= L V), so one read serves the
// softmax, the k largest and the sums over tokens.  A group takes a run of consecutive tokens, one after the other, and
// counts each expert's pairs in LDS as it goes: the count is a pair's rank among the run's pairs of that expert, so the
// order by (expert, token, slot) needs no sort, and no two lanes count the same expert at a time:
//   sk_route_tokens   one work-group per block of tokens; ranks within the block; counts, probability sums per block
//   sk_route_scan     per expert, the blocks' counts summed into starts; totals
//   sk_route_place    start of the expert + start of the block + rank; the losses
// Few tokens are one block, which finishes in the first launch.  All sums are taken in a fixed order in 32 bits.
//
// 65536 tokens, 256 experts, k = 8, fp32: tokens 54 us, bound by vector issue (450 instructions a token, three fifths
// of them the k maxima; reading the logits would take 14 us), scan 9, place 8, gradient 31 us (131 MB, 4.2 TB/s).
#include <type_traits>

#include "sk_routed.h"

namespace sk {
namespace {

constexpr int kThreads = 256;
constexpr int kRowBcast15 = 0x142;  // DPP: lane 15 of a row of 16 to the next row
constexpr int kRowBcast31 = 0x143;  // DPP: lane 31 to the upper 32
constexpr int kMaxK = 16;
constexpr int kMaxRun = 32;         // tokens of a group: ranks within a run stay below 2^16 and the pairs in LDS
constexpr int kBlocksWanted = 512;
constexpr int kManyThreads = 1024;
constexpr uint32_t kNoPair = 0xFFFFFFFFu;

// 1 / x and a / x for x from 1 on: v_rcp_f32, which may be off by a unit in the last place, and one step of Newton's,
// after which the result is off by little more than half of one (1 / x for x = 1 .. 1024 is the nearest float from
// any start within a unit, enumerated).  A division that also takes infinities and the smallest numbers is ten
// instructions.
__device__ __forceinline__ float reciprocal(float x) {
    const float r = __builtin_amdgcn_rcpf(x);
    return __builtin_fmaf(__builtin_fmaf(-x, r, 1.f), r, r);
}
__device__ __forceinline__ float quotient(float a, float x) {
    const float r = __builtin_amdgcn_rcpf(x), q = a * r;
    return __builtin_fmaf(__builtin_fmaf(-q, x, a), r, q);
}

// Reductions over aligned groups of L lanes; every lane of the group ends with the same bits.
template <int L>
__device__ __forceinline__ float group_sum(float v) {
    v = sum_q(v);
    if constexpr (L >= 16) v += dpp<kRowRor8>(v);
    if constexpr (L >= 32) {
        const LanePair a = swap16(v);
        v = a.lo + a.hi;
    }
    if constexpr (L >= 64) {
        const LanePair b = swap32(v);
        v = b.lo + b.hi;
    }
    return v;
}
template <int L>
__device__ __forceinline__ float group_max(float v) {
    v = max_q(v);
    if constexpr (L >= 16) v = fmaxf(v, dpp<kRowRor8>(v));
    if constexpr (L >= 32) {
        const LanePair a = swap16(v);
        v = fmaxf(a.lo, a.hi);
    }
    if constexpr (L >= 64) {
        const LanePair b = swap32(v);
        v = fmaxf(b.lo, b.hi);
    }
    return v;
}
// The largest key of a group.  Keys are whole numbers (the larger of two floats costs two instructions more, which make
// NaN quiet); over a whole wavefront by broadcasts to its last lane and a scalar.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint32_t key_dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
template <int L>
__device__ __forceinline__ uint32_t group_best(uint32_t v) {
    v = max(v, key_dpp<kQuadXor1>(v));
    v = max(v, key_dpp<kQuadXor2>(v));
    v = max(v, key_dpp<kHalfMirror>(v));
    if constexpr (L >= 16) v = max(v, key_dpp<kRowRor8>(v));
    if constexpr (L == 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max((uint32_t)r[0], (uint32_t)r[1]);
    }
    if constexpr (L == 64) {
        v = max(v, key_dpp<kRowBcast15, 0xA>(v));
        v = max(v, key_dpp<kRowBcast31, 0xC>(v));
        v = (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
    }
    return v;
}
// Keys in the order of the scores, above 0; 0: not to be taken (-inf, NaN).  -0 and 0 are the same.
__device__ __forceinline__ uint32_t score_key(float s) {
    const uint32_t u = __float_as_uint(s + 0.f);
    return s > neg_inf() ? u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u) : 0u;
}
// The group's bits of a wavefront's ballot.
template <int L>
__device__ __forceinline__ uint64_t group_ballot(bool b) {
    const uint64_t all = __builtin_amdgcn_ballot_w64(b);
    if constexpr (L == 64) return all;
    return (all >> (threadIdx.x & 63 & ~(L - 1))) & ((1ull << (L & 63)) - 1);
}

// This lane's V logits of token t; -inf past the last expert.
template <class T, int L, int V, bool VEC>
__device__ __forceinline__ void load_logits(const T *row, int E, int first, float (&x)[V]) {
    if constexpr (VEC) {
        static_assert(V == 4, "vector loads are of four logits");
        if (first < E) {  // E is a multiple of four
            if constexpr (sizeof(T) == 4) {
                const float4 a = *reinterpret_cast<const float4 *>(row + first);
                x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
            } else {
                typedef T T4 __attribute__((ext_vector_type(4)));
                const T4 a = *reinterpret_cast<const T4 *>(row + first);
#pragma unroll
                for (int v = 0; v < 4; ++v) x[v] = (float)a[v];
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = neg_inf();
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = first + v < E ? (float)row[first + v] : neg_inf();
    }
}

struct RoutePlan {
    int run;     // tokens of a group
    int groups;  // groups of a work-group
    int blocks;  // work-groups
};

// Workspace: counts [blocks][E], probability sums [blocks][E], z sums [blocks], live tokens [blocks]; totals of the
// probability sums [E], of z and of the live tokens.
struct RouteSpace {
    int32_t *cnt;
    float *prob, *z, *live, *prob_all, *z_all, *live_all;
};
__host__ __device__ inline RouteSpace route_space(void *ws, int blocks, int E) {
    RouteSpace s;
    s.cnt = static_cast<int32_t *>(ws);
    s.prob = reinterpret_cast<float *>(s.cnt + (size_t)blocks * E);
    s.z = s.prob + (size_t)blocks * E;
    s.live = s.z + blocks;
    s.prob_all = s.live + blocks;
    s.z_all = s.prob_all + E;
    s.live_all = s.z_all + 1;
    return s;
}

// Exclusive sums over E experts of counts read through `count`, by the whole work-group, into off[0..E] (LDS).
template <class Count>
__device__ __forceinline__ void expert_offsets(int E, int32_t *off, int32_t *wave_total, Count count) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int32_t base = 0;
    for (int e0 = 0; e0 < E; e0 += kThreads) {
        const int e = e0 + threadIdx.x;
        const int32_t c = e < E ? count(e) : 0;
        int32_t sum = c;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int32_t up = __shfl_up(sum, d, 64);
            if (lane >= d) sum += up;
        }
        if (lane == 63) wave_total[w] = sum;
        __syncthreads();
        int32_t before = base;
        for (int q = 0; q < w; ++q) before += wave_total[q];
        if (e < E) off[e] = before + sum - c;
        for (int q = 0; q < kThreads / 64; ++q) base += wave_total[q];
        __syncthreads();
    }
    if (threadIdx.x == 0) off[E] = base;
    __syncthreads();
}

// The losses from the totals, by one work-group: balance = E sum_e f_e P_e, z.
template <class Count, class Prob>
__device__ __forceinline__ void route_losses(const RouteArgs &A, float live, float z, float *red, Count count,
                                             Prob prob) {
    const float n = fmaxf(live, 1.f);
    float s = 0.f;
    for (int e = threadIdx.x; e < A.E; e += kThreads) s += ((float)count(e) / ((float)A.k * n)) * (prob(e) / n);
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        float all = 0.f;
        for (int q = 0; q < kThreads / 64; ++q) all += red[q];
        *A.balance = (float)A.E * all;
        *A.z_loss = z / n;
        if (A.state) A.state[2 * (size_t)A.T] = live;
    }
}

// NT threads.  ONE: the only work-group; writes the order and the losses too.
template <class T, int L, int V, bool VEC, bool ONE, int NT>
__global__ __launch_bounds__(NT) void sk_route_tokens(RouteArgs A, RoutePlan P) {
    constexpr int G = NT / L;
    extern __shared__ int32_t lds[];
    int32_t *cnt_lds = lds;                                      // [G][L V]
    float *prob_lds = reinterpret_cast<float *>(lds + G * L * V);  // [G][L V]
    uint32_t *pair = reinterpret_cast<uint32_t *>(prob_lds + G * L * V);  // [G][run][k]: expert << 16 | rank
    __shared__ float z_lds[G], live_lds[G], red[NT / 64];
    __shared__ int32_t off[ONE ? L * V + 1 : 1], wave_total[NT / 64];

    const int E = A.E, k = A.k;
    const int lane = threadIdx.x & (L - 1), g = threadIdx.x / L;
    const int first = lane * V;
    const int64_t t0 = ((int64_t)blockIdx.x * G + g) * P.run;
    uint32_t *mine = pair + (size_t)g * P.run * k;
    int32_t *cnt = cnt_lds + g * L * V;  // pairs so far

    float bias[V], psum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bias[v] = A.bias && first + v < E ? A.bias[first + v] : 0.f;
        psum[v] = 0.f;
        cnt[first + v] = 0;
    }
    __builtin_amdgcn_wave_barrier();
    float zsum = 0.f, nlive = 0.f;

    for (int q = 0; q < P.run; ++q) {
        const int64_t t = t0 + q;
        const bool here = t < A.T;  // one answer for the group; the wavefront's groups stay together
        float x[V];
        load_logits<T, L, V, VEC>(static_cast<const T *>(A.logits) + (here ? t : 0) * (int64_t)E, E,
                                  here ? first : E, x);
        bool live = here && (!A.mask || A.mask[t]);

        // softmax: the largest logit, the sum of exponentials
        float mx = x[0];
#pragma unroll
        for (int v = 1; v < V; ++v) mx = fmaxf(mx, x[v]);
        mx = group_max<L>(mx);
        if (__builtin_amdgcn_ballot_w64(live && mx == neg_inf())) {
            // Nothing above -inf: no row, unless a NaN is in it (fmaxf passes over NaN), which then shows in the row.
            bool nan = false;
#pragma unroll
            for (int v = 0; v < V; ++v) nan |= x[v] != x[v];
            nan = group_ballot<L>(nan) != 0;
            if (mx == neg_inf()) {
                if (nan) mx = __builtin_nanf("");
                else live = false;
            }
        }
        float ex[V], sum = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ex[v] = first + v < E ? ex2((x[v] - mx) * kLog2e) : 0.f;
            sum += ex[v];
        }
        sum = group_sum<L>(sum);
        if (live) {
            const float inv = reciprocal(sum);
#pragma unroll
            for (int v = 0; v < V; ++v) psum[v] += ex[v] * inv;
            const float lse = mx + lg2(sum) * kLn2;
            zsum += lse * lse;
            nlive += 1.f;
        }
        if (here && lane == 0 && A.state) {
            A.state[2 * t] = live ? mx : neg_inf();
            A.state[2 * t + 1] = sum;
        }

        // the k largest scores, ties to the lowest expert; scores of -inf and NaN are not taken
        uint32_t key[V];
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = live && first + v < E ? score_key(x[v] + bias[v]) : 0u;
        // Each lane keeps the first of its best scores at hand; the lane whose it is notes the expert in LDS and looks for
        // its next.  Nothing goes between lanes but the maximum.
        uint32_t m = 0;
        int at = 0;
        auto look = [&] {
            m = key[0], at = 0;
#pragma unroll
            for (int v = 1; v < V; ++v)
                if (key[v] > m) m = key[v], at = v;
        };
        look();
        for (int s = 0; s < k; ++s) {
            const uint32_t best = group_best<L>(m);
            const uint64_t holders = group_ballot<L>(m == best);
            if (lane == __builtin_ctzll(holders)) {
                mine[q * k + s] = best ? (uint32_t)(first + at) << 16 : kNoPair;
#pragma unroll
                for (int v = 0; v < V; ++v) key[v] = v == at ? 0u : key[v];
                look();
            }
        }
        __builtin_amdgcn_wave_barrier();  // a wavefront's LDS operations complete in order
        // lane s has slot s: its rank, its logit
        int my_expert = -1;
        float my_logit = neg_inf();
        if (lane < k) {
            uint32_t word = mine[q * k + lane];
            if (word != kNoPair) {
                my_expert = (int)(word >> 16);
                my_logit = (float)static_cast<const T *>(A.logits)[t * (int64_t)E + my_expert];
                word |= (uint32_t)atomicAdd(&cnt[my_expert], 1);
                mine[q * k + lane] = word;
            }
        }
        __builtin_amdgcn_wave_barrier();

        // weights of the chosen: lane s has slot s
        float w = 0.f;
        if (A.renormalize) {
            const float top = group_max<L>(my_logit);
            // A chosen logit that is not finite shows in the weights, as in any softmax.
            const float u = my_expert >= 0 ? ex2((my_logit - top) * kLog2e) : 0.f;
            const float all = group_sum<L>(u);
            // The row's own sum is used for NaN alone: a NaN logit is never chosen, and its row must not look sound.
            w = my_expert >= 0 ? (sum != sum ? sum : quotient(u, all)) : 0.f;
        } else {
            w = my_expert >= 0 ? quotient(ex2((my_logit - mx) * kLog2e), sum) : 0.f;
        }
        if (here && lane < k) {
            A.weights[t * k + lane] = w;
            A.experts[t * k + lane] = my_expert;
        }
    }

    // The block's totals, and each group's start among them.
#pragma unroll
    for (int v = 0; v < V; ++v) prob_lds[g * L * V + first + v] = psum[v];
    if (lane == 0) z_lds[g] = zsum, live_lds[g] = nlive;
    __syncthreads();
    const RouteSpace S = route_space(A.ws, P.blocks, E);
    for (int e = threadIdx.x; e < E; e += NT) {
        int32_t c = 0;
        float p = 0.f;
        for (int q = 0; q < G; ++q) {
            const int32_t n = cnt_lds[q * L * V + e];
            cnt_lds[q * L * V + e] = c;
            c += n;
            p += prob_lds[q * L * V + e];
        }
        if constexpr (ONE) {
            A.counts[e] = c;
            prob_lds[e] = p;  // the totals take the places of groups 0 and 1, which this thread alone has read
            reinterpret_cast<int32_t *>(prob_lds)[L * V + e] = c;
        } else {
            S.cnt[(size_t)blockIdx.x * E + e] = c;
            S.prob[(size_t)blockIdx.x * E + e] = p;
        }
    }
    float z = 0.f, live = 0.f;
    for (int q = 0; q < G; ++q) z += z_lds[q], live += live_lds[q];
    __syncthreads();
    if constexpr (ONE) {
        const int32_t *total = reinterpret_cast<const int32_t *>(prob_lds) + L * V;
        expert_offsets(E, off, wave_total, [&](int e) { return total[e]; });
        for (int e = threadIdx.x; e <= E; e += NT) A.offsets[e] = off[e];
        route_losses(A, live, z, red, [&](int e) { return total[e]; }, [&](int e) { return prob_lds[e]; });
    } else if (threadIdx.x == 0) {
        S.z[blockIdx.x] = z;
        S.live[blockIdx.x] = live;
    }

    for (int q = lane; q < P.run * k; q += L) {
        const int64_t at = t0 * k + q;
        if (at >= (int64_t)A.T * k) break;
        const uint32_t word = mine[q];
        int32_t slot = -1;
        if (word != kNoPair) {
            const int e = (int)(word >> 16);
            slot = cnt_lds[g * L * V + e] + (int32_t)(word & 0xFFFFu);
            if constexpr (ONE) {
                slot += off[e];
                A.tokens[slot] = (int32_t)(t0 + q / k);
            }
        }
        A.slots[at] = slot;  // !ONE: the rank within the block until sk_route_place
    }
    if constexpr (ONE)
        for (int64_t r = off[E] + threadIdx.x; r < (int64_t)A.T * k; r += NT) A.tokens[r] = -1;
}

// One wavefront an expert, its lanes a run of blocks each: the blocks' counts become starts, in place; totals of counts
// and probabilities.  The last work-group sums z and the live tokens.
__global__ __launch_bounds__(kThreads) void sk_route_scan(RouteArgs A, RoutePlan P) {
    __shared__ float red[2][kThreads / 64];
    const RouteSpace S = route_space(A.ws, P.blocks, A.E);
    if (blockIdx.x + 1 == gridDim.x) {
        float z = 0.f, n = 0.f;
        for (int b = threadIdx.x; b < P.blocks; b += kThreads) z += S.z[b], n += S.live[b];
        z = wave_sum(z), n = wave_sum(n);
        if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6] = z, red[1][threadIdx.x >> 6] = n;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int q = 1; q < kThreads / 64; ++q) z += red[0][q], n += red[1][q];
            *S.z_all = z;
            *S.live_all = n;
        }
        return;
    }
    constexpr int kAtOnce = 8;  // loads under way together
    const int lane = threadIdx.x & 63, e = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (e >= A.E) return;
    const int per = (P.blocks + 63) / 64;
    const int b0 = min(lane * per, P.blocks), b1 = min(b0 + per, P.blocks);
    int32_t c = 0;
    float p = 0.f;
    for (int b = b0; b < b1; b += kAtOnce) {
        int32_t n[kAtOnce];
        float f[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            n[i] = b + i < b1 ? S.cnt[(size_t)(b + i) * A.E + e] : 0;
            f[i] = b + i < b1 ? S.prob[(size_t)(b + i) * A.E + e] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) c += n[i], p += f[i];
    }
    int32_t upto = c;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t up = __shfl_up(upto, d, 64);
        if (lane >= d) upto += up;
    }
    p = wave_sum(p);
    if (lane == 63) {
        A.counts[e] = upto;
        S.prob_all[e] = p;
    }
    int32_t start = upto - c;
    for (int b = b0; b < b1; b += kAtOnce) {
        int32_t n[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) n[i] = b + i < b1 ? S.cnt[(size_t)(b + i) * A.E + e] : 0;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (b + i < b1) S.cnt[(size_t)(b + i) * A.E + e] = start;
            start += n[i];
        }
    }
}

__global__ __launch_bounds__(kThreads) void sk_route_place(RouteArgs A, RoutePlan P) {
    extern __shared__ int32_t off[];  // [E + 1]
    __shared__ int32_t wave_total[kThreads / 64];
    __shared__ float red[kThreads / 64];
    const RouteSpace S = route_space(A.ws, P.blocks, A.E);
    expert_offsets(A.E, off, wave_total, [&](int e) { return A.counts[e]; });
    if (blockIdx.x == 0) {
        for (int e = threadIdx.x; e <= A.E; e += kThreads) A.offsets[e] = off[e];
        route_losses(A, *S.live_all, *S.z_all, red, [&](int e) { return A.counts[e]; },
                     [&](int e) { return S.prob_all[e]; });
    }
    const int64_t pairs = (int64_t)A.T * A.k, stride = (int64_t)gridDim.x * kThreads;
    const int tokens_of_block = P.groups * P.run;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < pairs; i += stride) {
        const int32_t e = A.experts[i];
        if (e >= 0) {
            const int32_t t = (int32_t)(i / A.k);
            const int32_t slot = off[e] + S.cnt[(size_t)(t / tokens_of_block) * A.E + e] + A.slots[i];
            A.slots[i] = slot;
            A.tokens[slot] = t;
        }
        if (i >= off[A.E]) A.tokens[i] = -1;
    }
}

// dl_e = p_e (c_e - sum p c + 2 g_z lse / n) + the weights' part at the chosen, c_e = g_balance E f_e / n.
template <class T, int L, int V, bool VEC>
__global__ __launch_bounds__(kThreads) void sk_route_bwd(RouteBwdArgs A) {
    constexpr int G = kThreads / L;
    const int E = A.E, k = A.k;
    const int lane = threadIdx.x & (L - 1), g = threadIdx.x / L;
    const int first = lane * V;
    const float n = fmaxf(A.state[2 * (size_t)A.T], 1.f);
    const float gb = A.g_balance ? *A.g_balance : 0.f, gz = A.g_z ? *A.g_z : 0.f;
    float coef[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        coef[v] = first + v < E ? gb * (float)E * ((float)A.counts[first + v] / ((float)k * n)) / n : 0.f;

    for (int64_t t0 = (int64_t)blockIdx.x * G; t0 < A.T; t0 += (int64_t)gridDim.x * G) {
        const int64_t t = t0 + g;
        const bool here = t < A.T;
        const int64_t tt = here ? t : t0;
        float x[V];
        load_logits<T, L, V, VEC>(static_cast<const T *>(A.logits) + tt * E, E, first, x);
        const float mx = A.state[2 * tt], sum = A.state[2 * tt + 1];
        const bool live = mx != neg_inf();
        const float inv = reciprocal(sum), lse = mx + lg2(sum) * kLn2;
        float p[V], pc = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            p[v] = first + v < E ? ex2((x[v] - mx) * kLog2e) * inv : 0.f;
            pc = __builtin_fmaf(p[v], coef[v], pc);
        }
        pc = group_sum<L>(pc);
        // lane s has slot s
        float w = 0.f, gw = 0.f;
        int expert = -1;
        if (A.g_weights && lane < k) {
            expert = A.experts[tt * k + lane];
            w = A.weights[tt * k + lane];
            gw = A.g_weights[tt * k + lane];
            if (expert < 0) w = gw = 0.f;
        }
        const float wg = group_sum<L>(w * gw);
        const float all = 2.f * gz * lse / n - pc - (A.renormalize ? 0.f : wg);
        const float own = A.renormalize ? w * (gw - wg) : w * gw;
        float d[V];
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = p[v] * (coef[v] + all);
        if (A.g_weights) {
            for (int s = 0; s < k; ++s) {
                const int e = __shfl(expert, s, L);
                const float add = __shfl(own, s, L);
#pragma unroll
                for (int v = 0; v < V; ++v) d[v] += e == first + v ? add : 0.f;
            }
        }
        if (!here) continue;
        T *out = static_cast<T *>(A.g_logits) + t * E;
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = live ? d[v] : 0.f;
        if constexpr (VEC) {
            if (first < E) {
                if constexpr (sizeof(T) == 4) {
                    *reinterpret_cast<float4 *>(out + first) = make_float4(d[0], d[1], d[2], d[3]);
                } else {
                    typedef T T4 __attribute__((ext_vector_type(4)));
                    T4 o;
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[v] = (T)d[v];
                    *reinterpret_cast<T4 *>(out + first) = o;
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (first + v < E) out[first + v] = (T)d[v];
        }
    }
}

// Lanes of a group: as few as hold the experts at four (beyond 256 experts: up to 16) to a lane, so that small rows
// share a wavefront, but not fewer than 16, which carry the k <= 16 slots (eight for up to eight experts).
int group_lanes(int E) { return E <= 8 ? 8 : E <= 64 ? 16 : E <= 128 ? 32 : 64; }

template <int N>
using Int = std::integral_constant<int, N>;

// Calls f(L, V, vector loads) for the shape that holds E experts.
template <class F>
hipError_t with_shape(int E, bool vec, F f) {
    if (E <= 8) return f(Int<8>{}, Int<1>{}, std::false_type{});
    if (E <= 16) return f(Int<16>{}, Int<1>{}, std::false_type{});
    if (E <= 64) return vec ? f(Int<16>{}, Int<4>{}, std::true_type{}) : f(Int<16>{}, Int<4>{}, std::false_type{});
    if (E <= 128) return vec ? f(Int<32>{}, Int<4>{}, std::true_type{}) : f(Int<32>{}, Int<4>{}, std::false_type{});
    if (E <= 256) return vec ? f(Int<64>{}, Int<4>{}, std::true_type{}) : f(Int<64>{}, Int<4>{}, std::false_type{});
    if (E <= 512) return f(Int<64>{}, Int<8>{}, std::false_type{});
    return f(Int<64>{}, Int<16>{}, std::false_type{});
}

// One block while each group has at most four tokens: two more launches take longer than those in turn.  One launch /
// three, in us: 64 tokens of 64 experts, k = 2, 8.2 / 9.7, 128 of them 12.9 / 9.9; 8 of 256, k = 8, 7.8 / 10.7, 16 of
// them 12.1 / 11.1.  Beyond, up to 512 blocks: fewer leave wavefronts out, more are as many more partial sums for the
// scan.  512 / 256 / 1024 of them: 65536 tokens of 64, k = 2, 25.8 / 37.8 / 30.4; of 256, k = 8, 70.5 / 74.4 / 75.6;
// 20000 of 128, k = 4, 27.3 / 21.1 / 32.2.
//
// The blocks are of 256 threads, two wavefronts a SIMD, or, from 65 experts on, of 1024: the k rounds of maxima are
// one chain of latencies, which four wavefronts a SIMD (up to 128 experts, for want of registers) or eight hide.
// With up to 64 experts a group is 16 lanes or fewer, and a work-group of 1024 threads has 64 of them or more: its
// sums over the groups then take longer than the wavefronts save, and want more registers than there are.  1024
// threads / 256: 65536 tokens of 256, k = 8, 71 / 104; of 128, k = 8, 51 / 61; of 100, k = 4, 41 / 48; 20000 of 128,
// k = 4, 27 / 25; 65536 of 64, k = 8, 37 / 38; of 64, k = 2, 29 / 26; of 16, k = 2, 25 / 21; a million of 64, k = 2,
// 274 / 173.
RoutePlan route_plan(int T, int E) {
    RoutePlan P;
    const int L = group_lanes(E);
    P.groups = kThreads / L;
    if (T <= 4 * P.groups) {
        P.run = T > 0 ? (T + P.groups - 1) / P.groups : 1;
        P.blocks = 1;
        return P;
    }
    if (E > 64 && E <= 256 && T > kBlocksWanted * P.groups) P.groups = kManyThreads / L;
    const int64_t wanted = (int64_t)kBlocksWanted * P.groups;
    // the pairs of a work-group of 1024 threads: at most 16 KB of LDS
    const int most = P.groups * L == kManyThreads ? kMaxRun * L / 128 : kMaxRun;
    int64_t run = (T + wanted - 1) / wanted;
    P.run = (int)(run > most ? most : run);
    const int per = P.groups * P.run;
    P.blocks = (int)(((int64_t)T + per - 1) / per);
    return P;
}

bool vector_rows(const void *p, int E, int dtype) {
    return E % 4 == 0 && ((uintptr_t)p % (dtype == SK_F32 ? 16 : 8)) == 0;
}

}  // namespace

size_t route_workspace_bytes(int T, int E, int k) {
    (void)k;
    const RoutePlan P = route_plan(T, E);
    if (P.blocks == 1) return 0;
    return ((size_t)P.blocks * E * 2 + (size_t)P.blocks * 2 + E + 2) * 4;
}

hipError_t launch_route_forward(const RouteArgs &a, hipStream_t st) {
    const RoutePlan P = route_plan(a.T, a.E);
    hipError_t err = with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        return with_shape(a.E, vector_rows(a.logits, a.E, a.dtype), [&](auto l, auto v, auto vec) {
            constexpr int L = decltype(l)::value, V = decltype(v)::value;
            constexpr bool VEC = decltype(vec)::value;
            const size_t lds = (size_t)P.groups * (2 * L * V + (size_t)P.run * a.k) * 4;
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3(P.blocks), dim3(P.groups * L), lds, st, a, P);
                return hipGetLastError();
            };
            if (P.blocks == 1) return go(sk_route_tokens<T, L, V, VEC, true, kThreads>);
            if constexpr (L >= 32 && V <= 4) {
                if (P.groups * L == kManyThreads) return go(sk_route_tokens<T, L, V, VEC, false, kManyThreads>);
            }
            return go(sk_route_tokens<T, L, V, VEC, false, kThreads>);
        });
    });
    if (err != hipSuccess || P.blocks == 1) return err;
    hipLaunchKernelGGL(sk_route_scan, dim3((a.E + kThreads / 64 - 1) / (kThreads / 64) + 1), dim3(kThreads), 0, st, a, P);
    const int64_t pairs = (int64_t)a.T * a.k;
    int64_t grid = (pairs + 4 * kThreads - 1) / (4 * kThreads);
    if (grid > 1024) grid = 1024;
    hipLaunchKernelGGL(sk_route_place, dim3((unsigned)grid), dim3(kThreads), ((size_t)a.E + 1) * 4, st, a, P);
    return hipGetLastError();
}

hipError_t launch_route_backward(const RouteBwdArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    const int G = kThreads / group_lanes(a.E);
    int64_t grid = ((int64_t)a.T + G - 1) / G;
    if (grid > 2048) grid = 2048;
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        const bool vec = vector_rows(a.logits, a.E, a.dtype) && vector_rows(a.g_logits, a.E, a.dtype);
        return with_shape(a.E, vec, [&](auto l, auto v, auto ve) {
            hipLaunchKernelGGL((sk_route_bwd<T, decltype(l)::value, decltype(v)::value, decltype(ve)::value>),
                               dim3((unsigned)grid), dim3(kThreads), 0, st, a);
            return hipGetLastError();
        });
    });
}

}  // namespace sk
