// sk_api_block.hip -- the C ABI of the operators around a routed layer: the norms of its block, rows in 8 bits, their
// activations and products.
#include <math.h>
#include <stdint.h>

#include "sk_experts.h"
#include "sk_norm.h"
#include "sk_packed.h"

namespace {

constexpr int32_t kMaxRows = 1 << 24;
constexpr int64_t kMaxPackedRows = 1 << 26;
constexpr int64_t kMaxElements = int64_t(1) << 34;  // eight to a thread: a grid of fewer than 2^32 threads
constexpr int32_t kMaxColumns = 1 << 16;
constexpr int32_t kMaxPackedColumns = 1 << 17;

sk_status status_of(hipError_t e) { return e == hipSuccess ? SK_OK : SK_ERR_HIP; }

bool is_dtype(int32_t d) { return d == SK_F32 || d == SK_BF16 || d == SK_F16; }
bool is_norm(int32_t k) { return k == SK_NORM_NONE || k == SK_NORM_RMS || k == SK_NORM_CENTRED; }
bool is_eps(float e) { return e >= 0.f && e < INFINITY; }

// end: a block's end; else the norm alone.
sk_status check_norms(const sk_norms *p, bool end) {
    if (!p) return SK_ERR_NULLPTR;
    if (p->T < 0 || p->T > kMaxRows || p->N < 1 || p->N > kMaxColumns) return SK_ERR_SHAPE;
    if ((int64_t)p->T * p->N > kMaxElements) return SK_ERR_SHAPE;
    if (!is_dtype(p->dtype) || (p->wdtype != p->dtype && p->wdtype != SK_F32)) return SK_ERR_ARG;
    if (!is_norm(p->before) || !is_eps(p->eps_before)) return SK_ERR_ARG;
    if (!end) return p->before == SK_NORM_NONE ? SK_ERR_ARG : SK_OK;
    if (p->gate < SK_GATE_NONE || p->gate > SK_GATE_FULL) return SK_ERR_ARG;
    if (p->gate != SK_GATE_NONE && p->gdtype != p->dtype && p->gdtype != SK_F32) return SK_ERR_ARG;
    if (!is_norm(p->after) || !is_eps(p->eps_after) || !isfinite(p->scale)) return SK_ERR_ARG;
    return SK_OK;
}

sk::NormArgs norm_args(const sk_norms *p, bool end) {
    sk::NormArgs a = {};
    a.end = end;
    a.T = p->T;
    a.N = p->N;
    a.dtype = p->dtype;
    a.wf32 = p->wdtype == SK_F32;
    a.before = p->before;
    a.eps_before = p->eps_before;
    if (end) {
        a.gate_kind = p->gate;
        a.gf32 = p->gdtype == SK_F32;
        a.after = p->after;
        a.eps_after = p->eps_after;
        a.scale = p->scale;
    }
    return a;
}

sk_status check_packing(const sk_packing *p) {
    if (!p) return SK_ERR_NULLPTR;
    if (p->rows < 0 || p->rows > kMaxPackedRows || p->columns < 1 || p->columns > kMaxPackedColumns)
        return SK_ERR_SHAPE;
    if (p->rows * p->columns > kMaxElements) return SK_ERR_SHAPE;
    if (!is_dtype(p->dtype) || (p->block != 0 && p->block != sk::kPackBlock)) return SK_ERR_ARG;
    return SK_OK;
}

sk_status check_activation(const sk_packing *p, int32_t activation, int32_t gated, bool kept) {
    const sk_status st = check_packing(p);
    if (st != SK_OK) return st;
    if (activation < SK_ACT_NONE || activation > SK_ACT_GELU || (gated != 0 && gated != 1)) return SK_ERR_ARG;
    if (kept && p->block != sk::kPackBlock) return SK_ERR_ARG;
    return gated && p->columns % 2 ? SK_ERR_SHAPE : SK_OK;
}

sk::PackArgs pack_args(const sk_packing *p) {
    sk::PackArgs a = {};
    a.rows = p->rows;
    a.columns = p->columns;
    a.pitch = sk::pack_pitch(p->columns);
    a.blocks = p->block ? (p->columns + p->block - 1) / p->block : 1;
    a.dtype = p->dtype;
    return a;
}

}  // namespace

extern "C" {

sk_status sinkhorn_norm_forward(const sk_norms *p, const void *x, const void *w, const void *b, void *y, float *stats,
                                void *stream) {
    const sk_status st = check_norms(p, false);
    if (st != SK_OK) return st;
    if (p->T == 0) return SK_OK;
    if (!x || !y) return SK_ERR_NULLPTR;
    sk::NormArgs a = norm_args(p, false);
    a.residual = x;
    a.before_w = w;
    a.before_b = b;
    a.next = y;
    a.stats = stats;
    return status_of(sk::launch_norm_forward(a, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_residual_norm_forward(const sk_norms *p, const void *h, const void *residual, const void *gate,
                                         const void *after_w, const void *after_b, const void *before_w,
                                         const void *before_b, void *out, void *next, float *stats, void *stream) {
    const sk_status st = check_norms(p, true);
    if (st != SK_OK) return st;
    if (p->T == 0) return SK_OK;
    if (!h || !residual || !out || (p->gate && !gate) || (p->before && !next)) return SK_ERR_NULLPTR;
    sk::NormArgs a = norm_args(p, true);
    a.h = h;
    a.residual = residual;
    a.gate = gate;
    a.after_w = after_w;
    a.after_b = after_b;
    a.before_w = before_w;
    a.before_b = before_b;
    a.out = out;
    a.next = next;
    a.stats = stats;
    return status_of(sk::launch_norm_forward(a, static_cast<hipStream_t>(stream)));
}

size_t sinkhorn_norm_workspace_bytes(const sk_norms *p) {
    if (check_norms(p, true) != SK_OK) return 0;
    return sk::norm_workspace_bytes(p->T, p->N);
}

sk_status sinkhorn_norm_backward(const sk_norms *p, const void *x, const void *w, const float *stats,
                                 const void *grad_y, void *grad_x, void *grad_w, void *grad_b, void *workspace,
                                 size_t ws_bytes, void *stream) {
    const sk_status st = check_norms(p, false);
    if (st != SK_OK) return st;
    if (p->T > 0 && (!x || !stats || !grad_y)) return SK_ERR_NULLPTR;
    const size_t need = grad_w || grad_b ? sk::norm_workspace_bytes(p->T, p->N) : 0;
    if (ws_bytes < need) return SK_ERR_WORKSPACE;
    if (need && !workspace) return SK_ERR_NULLPTR;
    sk::NormArgs a = norm_args(p, false);
    a.out = const_cast<void *>(x);
    a.before_w = w;
    a.stats = const_cast<float *>(stats);
    a.g_next = grad_y;
    a.g_residual = grad_x;
    a.g_before_w = grad_w;
    a.g_before_b = grad_b;
    return status_of(sk::launch_norm_backward(a, workspace, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_residual_norm_backward(const sk_norms *p, const void *h, const void *out, const void *gate,
                                          const void *after_w, const void *after_b, const void *before_w,
                                          const float *stats, const void *grad_out, const void *grad_next,
                                          void *grad_h, void *grad_residual, void *grad_gate, void *grad_after_w,
                                          void *grad_after_b, void *grad_before_w, void *grad_before_b,
                                          void *workspace, size_t ws_bytes, void *stream) {
    const sk_status st = check_norms(p, true);
    if (st != SK_OK) return st;
    if (!p->after && (grad_after_w || grad_after_b)) return SK_ERR_ARG;
    if (!p->before && (grad_before_w || grad_before_b || grad_next)) return SK_ERR_ARG;
    if (!p->gate && grad_gate) return SK_ERR_ARG;
    if (p->T > 0 && (!stats || (p->gate && !gate))) return SK_ERR_NULLPTR;
    if (p->T > 0 && ((!h && (p->after || grad_gate)) || (!out && grad_next))) return SK_ERR_NULLPTR;
    const bool sums = grad_after_w || grad_after_b || grad_before_w || grad_before_b ||
                      (grad_gate && p->gate == SK_GATE_COLUMNS);
    const size_t need = sums ? sk::norm_workspace_bytes(p->T, p->N) : 0;
    if (ws_bytes < need) return SK_ERR_WORKSPACE;
    if (need && !workspace) return SK_ERR_NULLPTR;
    sk::NormArgs a = norm_args(p, true);
    a.h = h;
    a.out = const_cast<void *>(out);
    a.gate = gate;
    a.after_w = after_w;
    a.after_b = after_b;
    a.before_w = before_w;
    a.stats = const_cast<float *>(stats);
    a.g_out = grad_out;
    a.g_next = grad_next;
    a.g_h = grad_h;
    a.g_residual = grad_residual;
    a.g_gate = grad_gate;
    a.g_after_w = grad_after_w;
    a.g_after_b = grad_after_b;
    a.g_before_w = grad_before_w;
    a.g_before_b = grad_before_b;
    return status_of(sk::launch_norm_backward(a, workspace, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_pack(const sk_packing *p, const void *x, void *values, float *scales, void *stream) {
    const sk_status st = check_packing(p);
    if (st != SK_OK) return st;
    if (p->rows == 0) return SK_OK;
    if (!x || !values || !scales) return SK_ERR_NULLPTR;
    if (!sk::aligned16(values)) return SK_ERR_ARG;
    sk::PackArgs a = pack_args(p);
    a.x = x;
    a.values = static_cast<int8_t *>(values);
    a.scales = scales;
    return status_of(sk::launch_pack(a, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_unpack(const sk_packing *p, const void *values, const float *scales, void *x, void *stream) {
    const sk_status st = check_packing(p);
    if (st != SK_OK) return st;
    if (p->rows == 0) return SK_OK;
    if (!x || !values || !scales) return SK_ERR_NULLPTR;
    if (!sk::aligned16(values)) return SK_ERR_ARG;
    sk::PackArgs a = pack_args(p);
    a.values = static_cast<int8_t *>(const_cast<void *>(values));
    a.scales = const_cast<float *>(scales);
    a.y = x;
    return status_of(sk::launch_unpack(a, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_activation_forward(const sk_packing *p, int32_t activation, int32_t gated, const void *x, void *y,
                                      void *values, float *scales, void *stream) {
    const sk_status st = check_activation(p, activation, gated, values != nullptr);
    if (st != SK_OK) return st;
    if (p->rows == 0) return SK_OK;
    if (!x || !y || !values != !scales) return SK_ERR_NULLPTR;
    if (!sk::aligned16(values)) return SK_ERR_ARG;
    sk::PackArgs a = pack_args(p);
    a.kind = activation;
    a.gated = gated;
    a.x = x;
    a.y = y;
    a.values = static_cast<int8_t *>(values);
    a.scales = scales;
    return status_of(sk::launch_activation_forward(a, static_cast<hipStream_t>(stream)));
}

static sk_status activation_backward(const sk_packing *p, int32_t activation, int32_t gated, const void *values,
                                     const float *scales, const void *grad_y, bool gy32, void *y, void *grad_x,
                                     void *stream) {
    const sk_status st = check_activation(p, activation, gated, true);
    if (st != SK_OK) return st;
    if (p->rows == 0 || (!y && !grad_x)) return SK_OK;
    if (!values || !scales || !grad_y != !grad_x) return SK_ERR_NULLPTR;
    if (!sk::aligned16(values)) return SK_ERR_ARG;
    sk::PackArgs a = pack_args(p);
    a.kind = activation;
    a.gated = gated;
    a.values = static_cast<int8_t *>(const_cast<void *>(values));
    a.scales = const_cast<float *>(scales);
    a.gy = grad_y;
    a.gy32 = gy32;
    a.y = y;
    a.gx = grad_x;
    return status_of(sk::launch_activation_backward(a, static_cast<hipStream_t>(stream)));
}

sk_status sinkhorn_activation_backward(const sk_packing *p, int32_t activation, int32_t gated, const void *values,
                                       const float *scales, const void *grad_y, void *y, void *grad_x, void *stream) {
    return activation_backward(p, activation, gated, values, scales, grad_y, false, y, grad_x, stream);
}

sk_status sinkhorn_activation_backward32(const sk_packing *p, int32_t activation, int32_t gated, const void *values,
                                         const float *scales, const float *grad_y, void *y, void *grad_x, void *stream) {
    return activation_backward(p, activation, gated, values, scales, grad_y, true, y, grad_x, stream);
}

sk_status sinkhorn_experts_forward_packed(const sk_experts *p, const void *xv, const float *xs, const void *wv,
                                          const float *ws, const int32_t *offsets, const int32_t *tokens, void *y,
                                          void *stream) {
    const sk_status st = sk::check_experts(p, true);
    if (st != SK_OK) return st;
    if (p->T == 0) return SK_OK;
    if (!xv || !xs || !wv || !ws || !y || (!offsets && p->E != 1)) return SK_ERR_NULLPTR;
    if (!sk::aligned16(xv) || !sk::aligned16(wv)) return SK_ERR_ARG;
    sk::ExpertArgs a = {};
    a.T = p->T;
    a.k = p->k;
    a.E = p->E;
    a.K = sk::pack_pitch(p->K) / 2;
    a.N = p->N;
    a.dtype = p->dtype;
    a.x = xv;
    a.x_scale = xs;
    a.w = wv;
    a.w_scale = ws;
    a.offsets = offsets;
    a.tokens = tokens;
    a.out = y;
    return status_of(sk::launch_experts_packed(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
