// sk_api_routed.hip -- the C ABI of the routed-layer operators: argument checks and launches.
#include <math.h>
#include <stdint.h>

#include "sk_experts.h"

namespace {

constexpr int32_t kMaxTokens = 1 << 24;
constexpr int64_t kMaxElements = int64_t(1) << 34;  // eight to a thread: a grid of fewer than 2^32 threads
constexpr int32_t kMaxExperts = 1024;
constexpr int32_t kMaxSlots = 16;
constexpr int32_t kMaxColumns = 1 << 16;

sk_status status_of(hipError_t e) { return e == hipSuccess ? SK_OK : SK_ERR_HIP; }

bool is_dtype(int32_t d) { return d == SK_F32 || d == SK_BF16 || d == SK_F16; }

sk_status check_router(const sk_router *r) {
    if (!r) return SK_ERR_NULLPTR;
    if (r->T < 0 || r->T > kMaxTokens || r->E < 1 || r->E > kMaxExperts) return SK_ERR_SHAPE;
    if (r->k < 1 || r->k > kMaxSlots || r->k > r->E) return SK_ERR_SHAPE;
    if (!is_dtype(r->dtype) || (r->renormalize != 0 && r->renormalize != 1)) return SK_ERR_ARG;
    return SK_OK;
}

sk_status check_combine(const sk_combine *c) {
    if (!c) return SK_ERR_NULLPTR;
    if (c->T < 0 || c->T > kMaxTokens || c->D < 1 || c->D > kMaxTokens || c->k < 1 || c->k > kMaxSlots)
        return SK_ERR_SHAPE;
    if ((int64_t)c->T * c->k > kMaxElements / c->D) return SK_ERR_SHAPE;
    if (!is_dtype(c->dtype)) return SK_ERR_ARG;
    return SK_OK;
}

// The rate to 16 bits; p in [0, 1).
bool drop_args(double p, uint64_t seed, uint64_t offset, sk::DropArgs *d) {
    if (!(p >= 0.0 && p < 1.0)) return false;
    const int64_t t = (int64_t)(p * 65536.0 + 0.5);
    d->threshold = (uint32_t)(t > 65535 ? 65535 : t);
    d->scale = (float)(65536.0 / (65536.0 - (double)d->threshold));
    d->seed = seed;
    d->offset = offset;
    return true;
}

sk_status check_experts(const sk_experts *p) {
    if (!p) return SK_ERR_NULLPTR;
    if (p->T < 0 || p->T > kMaxTokens || p->k < 1 || p->k > kMaxSlots || p->E < 1 || p->E > kMaxExperts)
        return SK_ERR_SHAPE;
    if (p->K < 1 || p->N < 1 || p->K > kMaxColumns || p->N > kMaxColumns) return SK_ERR_SHAPE;
    const int64_t rows = (int64_t)p->T * p->k, wide = p->K > p->N ? p->K : p->N;
    if (rows * wide > kMaxElements || (int64_t)p->E * p->N * p->K > kMaxElements) return SK_ERR_SHAPE;
    if (p->dtype != SK_BF16 && p->dtype != SK_F16) return SK_ERR_ARG;
    return SK_OK;
}

sk::ExpertArgs expert_args(const sk_experts *p) {
    sk::ExpertArgs a = {};
    a.T = p->T;
    a.k = p->k;
    a.E = p->E;
    a.K = p->K;
    a.N = p->N;
    a.dtype = p->dtype;
    return a;
}

}  // namespace

extern "C" {

size_t sinkhorn_route_workspace_bytes(const sk_router *r) {
    if (check_router(r) != SK_OK) return 0;
    return sk::route_workspace_bytes(r->T, r->E, r->k);
}

sk_status sinkhorn_route_forward(const sk_router *r, const void *logits, const float *bias, const uint8_t *mask,
                                 float *weights, int32_t *experts, int32_t *counts, int32_t *offsets,
                                 int32_t *tokens, int32_t *slots, float *balance, float *z_loss, float *state,
                                 void *workspace, size_t ws_bytes, void *stream) {
    const sk_status st = check_router(r);
    if (st != SK_OK) return st;
    if (!counts || !offsets || !balance || !z_loss) return SK_ERR_NULLPTR;
    if (r->T > 0 && (!logits || !weights || !experts || !tokens || !slots)) return SK_ERR_NULLPTR;
    const size_t need = sk::route_workspace_bytes(r->T, r->E, r->k);
    if (ws_bytes < need) return SK_ERR_WORKSPACE;
    if (need && !workspace) return SK_ERR_NULLPTR;
    sk::RouteArgs a;
    a.logits = logits;
    a.bias = bias;
    a.mask = mask;
    a.weights = weights;
    a.experts = experts;
    a.counts = counts;
    a.offsets = offsets;
    a.tokens = tokens;
    a.slots = slots;
    a.balance = balance;
    a.z_loss = z_loss;
    a.state = state;
    a.ws = workspace;
    a.T = r->T;
    a.E = r->E;
    a.k = r->k;
    a.dtype = r->dtype;
    a.renormalize = r->renormalize;
    return status_of(sk::launch_route_forward(a, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_route_backward(const sk_router *r, const void *logits, const float *weights,
                                  const int32_t *experts, const int32_t *counts, const float *state,
                                  const float *grad_weights, const float *grad_balance, const float *grad_z,
                                  void *grad_logits, void *stream) {
    const sk_status st = check_router(r);
    if (st != SK_OK) return st;
    if (r->T == 0) return SK_OK;
    if (!logits || !weights || !experts || !counts || !state || !grad_logits) return SK_ERR_NULLPTR;
    sk::RouteBwdArgs a;
    a.logits = logits;
    a.weights = weights;
    a.experts = experts;
    a.counts = counts;
    a.state = state;
    a.g_weights = grad_weights;
    a.g_balance = grad_balance;
    a.g_z = grad_z;
    a.g_logits = grad_logits;
    a.T = r->T;
    a.E = r->E;
    a.k = r->k;
    a.dtype = r->dtype;
    a.renormalize = r->renormalize;
    return status_of(sk::launch_route_backward(a, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_dropout(int64_t n, int32_t dtype, const void *x, const void *residual, void *y, double p,
                           uint64_t seed, uint64_t offset, void *stream) {
    if (n < 0 || n > kMaxElements) return SK_ERR_SHAPE;
    sk::DropArgs d;
    if (!is_dtype(dtype) || !drop_args(p, seed, offset, &d)) return SK_ERR_ARG;
    if (n == 0) return SK_OK;
    if (!x || !y) return SK_ERR_NULLPTR;
    return status_of(sk::launch_dropout(x, residual, y, n, dtype, d, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_combine_forward(const sk_combine *c, const void *z, const float *weights, const int32_t *slots,
                                   const void *residual, void *y, double p, uint64_t seed, uint64_t offset,
                                   void *stream) {
    const sk_status st = check_combine(c);
    if (st != SK_OK) return st;
    sk::CombineArgs a = {};
    if (!drop_args(p, seed, offset, &a.drop)) return SK_ERR_ARG;
    if (c->T == 0) return SK_OK;
    if (!z || !weights || !slots || !y) return SK_ERR_NULLPTR;
    a.z = z;
    a.residual = residual;
    a.weights = weights;
    a.slots = slots;
    a.y = y;
    a.T = c->T;
    a.D = c->D;
    a.k = c->k;
    a.dtype = c->dtype;
    return status_of(sk::launch_combine_forward(a, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_combine_backward(const sk_combine *c, const void *z, const float *weights, const int32_t *slots,
                                    const int32_t *used_rows, const void *grad_y, void *grad_z,
                                    float *grad_weights, double p, uint64_t seed, uint64_t offset, void *stream) {
    const sk_status st = check_combine(c);
    if (st != SK_OK) return st;
    sk::CombineArgs a = {};
    if (!drop_args(p, seed, offset, &a.drop)) return SK_ERR_ARG;
    if (c->T == 0) return SK_OK;
    if (!z || !weights || !slots || !used_rows || !grad_y || !grad_z || !grad_weights) return SK_ERR_NULLPTR;
    a.z = z;
    a.weights = weights;
    a.slots = slots;
    a.used = used_rows;
    a.gy = grad_y;
    a.gz = grad_z;
    a.g_weights = grad_weights;
    a.T = c->T;
    a.D = c->D;
    a.k = c->k;
    a.dtype = c->dtype;
    return status_of(sk::launch_combine_backward(a, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_experts_forward(const sk_experts *p, const void *x, const void *w, const int32_t *offsets,
                                   const int32_t *tokens, void *y, void *stream) {
    const sk_status st = check_experts(p);
    if (st != SK_OK) return st;
    if (p->T == 0) return SK_OK;
    if (!x || !w || !offsets || !y) return SK_ERR_NULLPTR;
    sk::ExpertArgs a = expert_args(p);
    a.x = x;
    a.w = w;
    a.offsets = offsets;
    a.tokens = tokens;
    a.out = y;
    return status_of(sk::launch_experts_forward(a, static_cast<hipStream_t>(stream)));
}

size_t sinkhorn_experts_workspace_bytes(const sk_experts *p) {
    if (check_experts(p) != SK_OK) return 0;
    return sk::experts_workspace_bytes(p->T, p->k, p->K);
}

sk_status sinkhorn_experts_backward_input(const sk_experts *p, const void *grad_y, const void *w,
                                          const int32_t *offsets, const int32_t *slots, void *grad_x,
                                          void *workspace, size_t ws_bytes, void *stream) {
    const sk_status st = check_experts(p);
    if (st != SK_OK) return st;
    if (p->T == 0) return SK_OK;
    if (!grad_y || !w || !offsets || !grad_x) return SK_ERR_NULLPTR;
    if (slots) {
        if (ws_bytes < sk::experts_workspace_bytes(p->T, p->k, p->K)) return SK_ERR_WORKSPACE;
        if (!workspace) return SK_ERR_NULLPTR;
    }
    sk::ExpertArgs a = expert_args(p);
    a.gy = grad_y;
    a.w = w;
    a.offsets = offsets;
    a.slots = slots;
    a.out = grad_x;
    return status_of(sk::launch_experts_input(a, workspace, static_cast<hipStream_t>(stream)));
}

size_t sinkhorn_experts_weight_workspace_bytes(const sk_experts *p) {
    if (check_experts(p) != SK_OK) return 0;
    return sk::experts_weight_workspace_bytes(expert_args(p));
}

sk_status sinkhorn_experts_backward_weight(const sk_experts *p, const void *grad_y, const void *x,
                                           const int32_t *offsets, const int32_t *tokens, void *grad_w,
                                           void *workspace, size_t ws_bytes, void *stream) {
    const sk_status st = check_experts(p);
    if (st != SK_OK) return st;
    if (!offsets || !grad_w) return SK_ERR_NULLPTR;
    if (p->T > 0 && (!grad_y || !x)) return SK_ERR_NULLPTR;
    sk::ExpertArgs a = expert_args(p);
    const size_t need = sk::experts_weight_workspace_bytes(a);
    if (ws_bytes < need) return SK_ERR_WORKSPACE;
    if (need && !workspace) return SK_ERR_NULLPTR;
    a.gy = grad_y;
    a.x = x;
    a.offsets = offsets;
    a.tokens = tokens;
    a.out = grad_w;
    return status_of(sk::launch_experts_weight(a, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
