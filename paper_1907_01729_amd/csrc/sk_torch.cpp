// sk_torch.cpp -- the operators around a routed layer as calls on torch tensors, with their nodes of the autograd graph:
// argument checks, allocation and calls of the C ABI.  In C++ and not through ctypes, because these calls are short: a
// norm with its gradients takes the host 62 us a step, with a node written in Python 115.
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/VariableTypeUtils.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>

#include <mutex>
#include <optional>
#include <string>
#include <tuple>
#include <vector>

#include "../../include/sinkhorn.h"

namespace {

namespace py = pybind11;
using at::Tensor;
using torch::autograd::SavedVariable;
using torch::autograd::variable_list;
using Maybe = std::optional<Tensor>;

// A call that the library refused; becomes the package's SinkhornError.
struct Refused : std::runtime_error {
    sk_status status;
    const char *where;
    Refused(sk_status st, const char *w)
        : std::runtime_error(std::string(w) + ": " + sinkhorn_status_string(st)), status(st), where(w) {}
};
void check(sk_status st, const char *where) {
    if (st != SK_OK) throw Refused(st, where);
}

// ---- tensors ----

int32_t type_of(at::ScalarType t) {
    return t == at::kFloat ? SK_F32 : t == at::kBFloat16 ? SK_BF16 : t == at::kHalf ? SK_F16 : -1;
}

Tensor or_none(const Maybe &t) { return t ? *t : Tensor(); }
void *data(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
template <class T>
T *data_of(const Tensor &t) {
    return t.defined() ? static_cast<T *>(t.data_ptr()) : nullptr;
}
Tensor contiguous(const Tensor &t) { return t.defined() ? t.contiguous() : t; }

// A GPU tensor of one of the element types the operators take.
void typed(const Tensor &t, const char *name, bool half = false) {
    TORCH_CHECK_TYPE(t.defined() && t.is_cuda(), name, " must be a GPU tensor");
    const int32_t type = type_of(t.scalar_type());
    TORCH_CHECK_TYPE(type >= 0 && !(half && type == SK_F32), name, " must be ",
                     half ? "bfloat16 or float16" : "float32, bfloat16 or float16", ", got ", t.scalar_type());
}
// On ref's device, of its type or the one given.
void like(const Tensor &t, const char *name, const Tensor &ref, at::ScalarType type) {
    TORCH_CHECK_TYPE(t.is_cuda(), name, " must be a GPU tensor");
    TORCH_CHECK_TYPE(t.scalar_type() == type, name, " must be ", type, ", got ", t.scalar_type());
    TORCH_CHECK_VALUE(t.device() == ref.device(), name, " must be on ", ref.device(), ", got ", t.device());
}
void shaped(const Tensor &t, const char *name, at::IntArrayRef shape) {
    TORCH_CHECK_VALUE(t.sizes() == shape, name, " must be ", shape, ", got ", t.sizes());
}
// Whole numbers that the router gives: contiguous, since their address goes to the kernels.
void indices(const Tensor &t, const char *name, const Tensor &ref) {
    like(t, name, ref, at::kInt);
    TORCH_CHECK_VALUE(t.is_contiguous(), name, " must be contiguous");
}
// Sizes for fields of 32 bits: refused, not cut off.
int32_t size32(int64_t n, const char *where) {
    if (n < INT32_MIN || n > INT32_MAX) throw Refused(SK_ERR_SHAPE, where);
    return static_cast<int32_t>(n);
}

Tensor empty(at::IntArrayRef shape, const Tensor &ref, at::ScalarType type) {
    return at::empty(shape, ref.options().dtype(type));
}
Tensor empty_bytes(size_t n, const Tensor &ref) {
    return n ? empty({static_cast<int64_t>(n)}, ref, at::kByte) : Tensor();
}

// The device of a call, and its current stream there.
struct On {
    c10::DeviceGuard guard;
    void *stream;
    explicit On(const Tensor &t)
        : guard(t.device()), stream(c10::hip::getCurrentHIPStream(t.device().index()).stream()) {}
};

// ---- autograd ----

// torch.jit.trace and make_fx record torch's own operations alone: of a call of these its allocations, whose memory a
// replay would give out as nobody wrote it.
void not_traced(const char *what) {
    using Mode = c10::impl::TorchDispatchModeKey;
    TORCH_CHECK_NOT_IMPLEMENTED(!torch::jit::tracer::isTracing() && !c10::impl::TorchDispatchModeTLS::get_mode(Mode::PROXY),
                                what, " cannot be traced");
}
// These have no derivative in forward mode, and a result without one would pass for zero.
void no_tangent(const char *what, std::initializer_list<Tensor> inputs) {
    for (const Tensor &t : inputs)
        TORCH_CHECK_NOT_IMPLEMENTED(!torch::autograd::isFwGradDefined(t), what,
                                    " has no derivative in forward mode AD");
}
bool recorded(std::initializer_list<Tensor> inputs) {
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor &t : inputs)
        if (t.defined() && t.requires_grad()) return true;
    return false;
}

// A backward pass that has no derivative itself: who differentiates its results gets an error.
struct Node : torch::autograd::Node {
    const char *what;
    explicit Node(const char *w) : what(w) {}
    std::string name() const override { return what; }
    virtual variable_list gradients(const variable_list &grads) = 0;
    bool wants(size_t i) const { return task_should_compute_output(i); }

    // The engine has the stream of whoever takes a gradient wait for the stream of this node.  While this one is captured
    // and that one is the default stream, as of a leaf that an eager graph still holds, the wait cannot be recorded, and
    // the error ends the process.
    void check_capture() const {
        if (c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None) return;
        for (size_t i = 0; i < num_outputs(); ++i) {
            if (!next_edge(i).is_valid() || !wants(i)) continue;
            const auto taker = next_edge(i).function->stream();
            TORCH_CHECK(!taker || taker->id() != 0, what, ": a backward pass cannot be captured while a graph made on the "
                        "default stream holds one of its leaves; delete that graph's results first");
        }
    }

    variable_list apply(variable_list &&grads) override {
        const std::lock_guard<std::mutex> lock(mutex_);  // two backward passes through one graph
        not_traced(what);
        check_capture();
        const bool again = at::GradMode::is_enabled();
        for (const Tensor &g : grads) no_tangent(what, {g});
        variable_list out;
        {
            at::AutoGradMode off(false);
            for (Tensor &g : grads) g = contiguous(g);
            out = gradients(grads);
        }
        if (!again) return out;
        auto refuses = std::make_shared<torch::autograd::DelayedError>(
            std::string(what) + ": the gradients have no derivative", out.size());
        for (Tensor &t : out)
            if (t.defined()) t = t.detach().requires_grad_();
        return (*refuses)(std::move(out));
    }
};
template <class N>
void attach(std::shared_ptr<N> node, const variable_list &outputs, torch::autograd::edge_list &&edges) {
    node->set_next_edges(std::move(edges));
    for (const Tensor &t : outputs) torch::autograd::set_history(t, node);
}
template <class N, class... A>
std::shared_ptr<N> new_node(A &&...a) {
    return std::shared_ptr<N>(new N(std::forward<A>(a)...), torch::autograd::deleteNode);
}
SavedVariable keep(const Tensor &t) { return SavedVariable(t, false); }
// What a node kept, in the layout that the kernels take: hooks on saved tensors may give the same values back with other
// strides, and at another address.
Tensor restored(const SavedVariable &v) { return contiguous(v.unpack()); }
// Of what the node allocated itself, which begins at whole 16 bytes.
Tensor restored_own(const SavedVariable &v) {
    const Tensor t = restored(v);
    return t.defined() && reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 ? t.clone() : t;
}

// ---- norms ----

struct Norm {
    Tensor w, b;
    double eps;
    bool center;
};
using NormOf = std::tuple<Maybe, Maybe, double, bool>;  // as the package's Norm
Norm norm_of(const NormOf &n) {
    return {contiguous(or_none(std::get<0>(n))), contiguous(or_none(std::get<1>(n))), std::get<2>(n), std::get<3>(n)};
}

void parameter(const Tensor &t, const std::string &name, const Tensor &x, int32_t &type) {
    if (!t.defined()) return;
    typed(t, name.c_str());
    TORCH_CHECK_VALUE(t.device() == x.device(), name, " must be on ", x.device(), ", got ", t.device());
    TORCH_CHECK_VALUE(t.dim() == 1 && t.size(0) == x.size(1), name, " must be [", x.size(1), "], got ", t.sizes());
    TORCH_CHECK_TYPE(t.scalar_type() == x.scalar_type() || t.scalar_type() == at::kFloat, name, " must be ",
                     x.scalar_type(), " or float32, got ", t.scalar_type());
    const int32_t mine = type_of(t.scalar_type());
    TORCH_CHECK_TYPE(type < 0 || type == mine, "all weights and biases must have one type");
    type = mine;
}
void parameters(const Norm &n, const char *name, const Tensor &x, int32_t &type) {
    parameter(n.w, std::string(name) + ".weight", x, type);
    parameter(n.b, std::string(name) + ".bias", x, type);
}
void rows(const Tensor &t, const char *name) {
    typed(t, name);
    TORCH_CHECK_VALUE(t.dim() == 2, name, " must be [T, N], got ", t.sizes());
}

struct NormNode : Node {
    SavedVariable x, w, b, stats;
    sk_norms p;
    NormNode() : Node("sinkhorn_norm") {}

    variable_list gradients(const variable_list &grads) override {
        if (!grads[0].defined()) return variable_list(3);
        const Tensor xv = restored(x), wv = restored(w), bv = restored(b), sv = restored_own(stats);
        const On on(xv);
        const Tensor gx = wants(0) ? at::empty_like(xv) : Tensor(),
                     gw = wv.defined() && wants(1) ? at::empty_like(wv) : Tensor(),
                     gb = bv.defined() && wants(2) ? at::empty_like(bv) : Tensor();
        const size_t need = gw.defined() || gb.defined() ? sinkhorn_norm_workspace_bytes(&p) : 0;
        const Tensor ws = empty_bytes(need, xv);
        check(sinkhorn_norm_backward(&p, data(xv), data(wv), data_of<float>(sv), data(grads[0]), data(gx), data(gw),
                                     data(gb), data(ws), need, on.stream),
              "sinkhorn_norm_backward");
        return {gx, gw, gb};
    }
    void release_variables() override {
        const std::lock_guard<std::mutex> lock(mutex_);
        for (SavedVariable *v : {&x, &w, &b, &stats}) v->reset_data();
    }
};

Tensor norm(const Tensor &x_, const NormOf &norm_) {
    not_traced("sinkhorn_norm");
    const Tensor x = contiguous(x_);
    const Norm n = norm_of(norm_);
    rows(x, "x");
    int32_t type = -1;
    parameters(n, "norm", x, type);
    no_tangent("sinkhorn_norm", {x, n.w, n.b});
    sk_norms p = {};
    p.T = size32(x.size(0), "sinkhorn_norm"), p.N = size32(x.size(1), "sinkhorn_norm");
    p.dtype = type_of(x.scalar_type());
    p.wdtype = type < 0 ? p.dtype : type;
    p.before = n.center ? SK_NORM_CENTRED : SK_NORM_RMS;
    p.scale = 1.f, p.eps_before = static_cast<float>(n.eps);
    const bool rec = recorded({x, n.w, n.b});
    Tensor y, stats;
    {
        at::AutoGradMode off(false);
        const On on(x);
        y = at::empty_like(x);
        if (rec) stats = empty({p.T, 4}, x, at::kFloat);
        check(sinkhorn_norm_forward(&p, data(x), data(n.w), data(n.b), data(y), data_of<float>(stats), on.stream),
              "sinkhorn_norm_forward");
    }
    if (rec) {
        auto node = new_node<NormNode>();
        node->x = keep(x), node->w = keep(n.w), node->b = keep(n.b);
        node->stats = keep(stats), node->p = p;
        attach(node, {y}, torch::autograd::collect_next_edges(x, n.w, n.b));
    }
    return y;
}

struct ResidualNode : Node {
    SavedVariable h, out, gate, aw, ab, bw, bb, stats;
    sk_norms p;
    bool has_out = false;
    at::TensorOptions options;
    ResidualNode() : Node("sinkhorn_residual_norm") {}

    variable_list gradients(const variable_list &grads) override {
        const Tensor g_out = grads[0], g_next = grads.size() > 1 ? grads[1] : Tensor();
        if (!g_out.defined() && !g_next.defined()) return variable_list(7);
        const Tensor hv = restored(h), gv = restored(gate), awv = restored(aw), abv = restored(ab), bwv = restored(bw),
                     bbv = restored(bb), sv = restored_own(stats);
        const Tensor ov = has_out ? contiguous(out.unpack(shared_from_this())) : Tensor();
        const On on(sv);
        auto made = [&](size_t i, const Tensor &as) {
            return as.defined() && wants(i) ? at::empty_like(as) : Tensor();
        };
        // Where out = residual + h both have one gradient: it is written once, and is one tensor for both, as of a sum.
        const bool same = !p.after && !p.gate && p.scale == 1.f && wants(0) && wants(1);
        const Tensor gr = wants(1) ? at::empty({p.T, p.N}, options) : Tensor(),
                     gh = wants(0) && !same ? at::empty({p.T, p.N}, options) : Tensor();
        const Tensor gg = made(2, gv), gaw = made(3, awv), gab = made(4, abv), gbw = made(5, bwv), gbb = made(6, bbv);
        const bool sums = gaw.defined() || gab.defined() || gbw.defined() || gbb.defined() ||
                          (gg.defined() && p.gate == SK_GATE_COLUMNS);
        const size_t need = sums ? sinkhorn_norm_workspace_bytes(&p) : 0;
        const Tensor ws = empty_bytes(need, sv);
        check(sinkhorn_residual_norm_backward(&p, data(hv), data(ov), data(gv), data(awv), data(abv), data(bwv),
                                              data_of<float>(sv), data(g_out), data(g_next), data(gh), data(gr),
                                              data(gg), data(gaw), data(gab), data(gbw), data(gbb), data(ws), need,
                                              on.stream),
              "sinkhorn_residual_norm_backward");
        return {same ? gr : gh, gr, gg, gaw, gab, gbw, gbb};
    }
    void release_variables() override {
        const std::lock_guard<std::mutex> lock(mutex_);
        for (SavedVariable *v : {&h, &out, &gate, &aw, &ab, &bw, &bb, &stats}) v->reset_data();
    }
};

variable_list residual_norm(const Tensor &h_, const Tensor &residual_, const Maybe &gate_, double scale,
                            const std::optional<NormOf> &after_, const std::optional<NormOf> &before_) {
    const char *what = "sinkhorn_residual_norm";
    not_traced(what);
    const Tensor h = contiguous(h_), residual = contiguous(residual_), gate = contiguous(or_none(gate_));
    const Norm after = after_ ? norm_of(*after_) : Norm{}, before = before_ ? norm_of(*before_) : Norm{};
    rows(h, "h");
    like(residual, "residual", h, h.scalar_type());
    shaped(residual, "residual", h.sizes());
    sk_norms p = {};
    p.T = size32(h.size(0), what), p.N = size32(h.size(1), what);
    p.dtype = type_of(h.scalar_type());
    if (gate.defined()) {
        typed(gate, "gate");
        TORCH_CHECK_VALUE(gate.device() == h.device(), "gate must be on ", h.device(), ", got ", gate.device());
        TORCH_CHECK_TYPE(gate.scalar_type() == h.scalar_type() || gate.scalar_type() == at::kFloat, "gate must be ",
                         h.scalar_type(), " or float32, got ", gate.scalar_type());
        const int64_t T = p.T, N = p.N;
        p.gdtype = type_of(gate.scalar_type());
        p.gate = gate.dim() != 2                              ? -1
                 : gate.size(0) == T && gate.size(1) == N     ? SK_GATE_FULL
                 : gate.size(0) == T && gate.size(1) == 1     ? SK_GATE_ROWS
                 : gate.size(0) == 1 && gate.size(1) == N     ? SK_GATE_COLUMNS
                                                              : -1;
        TORCH_CHECK_VALUE(p.gate >= 0, "gate must be [", T, ", ", N, "], [", T, ", 1] or [1, ", N, "], got ",
                          gate.sizes());
    }
    int32_t type = -1;
    parameters(after, "after", h, type);
    parameters(before, "before", h, type);
    no_tangent(what, {h, residual, gate, after.w, after.b, before.w, before.b});
    p.wdtype = type < 0 ? p.dtype : type;
    p.after = !after_ ? SK_NORM_NONE : after.center ? SK_NORM_CENTRED : SK_NORM_RMS;
    p.before = !before_ ? SK_NORM_NONE : before.center ? SK_NORM_CENTRED : SK_NORM_RMS;
    p.scale = static_cast<float>(scale);
    p.eps_after = static_cast<float>(after.eps), p.eps_before = static_cast<float>(before.eps);
    const bool rec = recorded({h, residual, gate, after.w, after.b, before.w, before.b});
    Tensor out, next, stats;
    {
        at::AutoGradMode off(false);
        const On on(h);
        out = at::empty_like(h);
        if (before_) next = at::empty_like(h);
        if (rec) stats = empty({p.T, 4}, h, at::kFloat);
        check(sinkhorn_residual_norm_forward(&p, data(h), data(residual), data(gate), data(after.w), data(after.b),
                                             data(before.w), data(before.b), data(out), data(next),
                                             data_of<float>(stats), on.stream),
              "sinkhorn_residual_norm_forward");
    }
    variable_list results = {out};
    if (before_) results.push_back(next);
    if (rec) {
        auto node = new_node<ResidualNode>();
        // Without a norm after the block its output is needed for the gate's gradient alone; without one before the
        // next, the sum is not needed.
        if (after_ || (gate.defined() && gate.requires_grad())) node->h = keep(h);
        node->gate = keep(gate), node->aw = keep(after.w), node->ab = keep(after.b);
        node->bw = keep(before.w), node->bb = keep(before.b);
        node->stats = keep(stats), node->p = p, node->options = h.options();
        attach(node, results,
               torch::autograd::collect_next_edges(h, residual, gate, after.w, after.b, before.w, before.b));
        if (before_) node->out = SavedVariable(out, true), node->has_out = true;
    }
    return results;
}

// ---- rows in 8 bits ----

constexpr int64_t kKeptBlock = 128;  // columns under one scale of a kept row

int64_t pitch(int64_t columns) { return (columns + 15) / 16 * 16; }
int64_t row_count(at::IntArrayRef lead) {
    int64_t n = 1;
    for (int64_t s : lead) n *= s;
    return n;
}
void check_block(int64_t block) {
    TORCH_CHECK_VALUE(block == 0 || block == kKeptBlock, "block must be 0 (a scale a row) or ", kKeptBlock, ", got ",
                      block);
}
std::vector<int64_t> scales_shape(at::IntArrayRef lead, int64_t columns, int64_t block) {
    std::vector<int64_t> s = lead.vec();
    if (block) s.push_back((columns + block - 1) / block);
    return s;
}
sk_packing packing(int64_t rows, int64_t columns, int64_t block, at::ScalarType type) {
    sk_packing p = {};
    p.rows = rows, p.columns = size32(columns, "rows in 8 bits"), p.block = static_cast<int32_t>(block);
    p.dtype = type_of(type);
    return p;
}
void columns_of(const Tensor &x, const char *name) {
    typed(x, name);
    TORCH_CHECK_VALUE(x.dim() >= 1 && x.size(-1) >= 1, name, " must be [..., columns], got ", x.sizes());
}
std::pair<Tensor, Tensor> new_packed(const Tensor &x, int64_t block) {
    const int64_t columns = x.size(-1);
    std::vector<int64_t> shape = x.sizes().vec();
    shape.back() = pitch(columns);
    return {empty(shape, x, at::kChar), empty(scales_shape(x.sizes().slice(0, x.dim() - 1), columns, block), x, at::kFloat)};
}

struct Packed {
    Tensor values, scales;
    int64_t columns, block;
};
using PackedOf = std::tuple<Tensor, Tensor, int64_t, int64_t>;  // as the package's Packed
// Of the shapes that its columns and block say.
Packed packed_of(const PackedOf &given, const std::string &name, bool by_rows) {
    const Packed p = {std::get<0>(given), std::get<1>(given), std::get<2>(given), std::get<3>(given)};
    check_block(p.block);
    TORCH_CHECK_VALUE(!by_rows || p.block == 0, name, " must have a scale for each row, got block = ", p.block);
    like(p.values, (name + ".values").c_str(), p.values, at::kChar);
    TORCH_CHECK_VALUE(p.values.is_contiguous(), name, ".values must be contiguous");
    TORCH_CHECK_VALUE(p.values.dim() >= 1 && p.columns >= 1 && p.values.size(-1) == pitch(p.columns), name,
                      ".values must be [..., ", pitch(p.columns), "] for ", p.columns, " columns, got ",
                      p.values.sizes());
    TORCH_CHECK_VALUE(reinterpret_cast<uintptr_t>(p.values.data_ptr()) % 16 == 0, name,
                      ".values must be aligned to 16 bytes");
    like(p.scales, (name + ".scales").c_str(), p.values, at::kFloat);
    TORCH_CHECK_VALUE(p.scales.is_contiguous(), name, ".scales must be contiguous");
    shaped(p.scales, (name + ".scales").c_str(),
           scales_shape(p.values.sizes().slice(0, p.values.dim() - 1), p.columns, p.block));
    return p;
}

std::pair<Tensor, Tensor> pack(const Tensor &x_, int64_t block) {
    not_traced("sinkhorn_pack");
    at::AutoGradMode off(false);
    const Tensor x = contiguous(x_);
    columns_of(x, "x");
    check_block(block);
    const On on(x);
    const sk_packing p = packing(row_count(x.sizes().slice(0, x.dim() - 1)), x.size(-1), block, x.scalar_type());
    const auto made = new_packed(x, block);
    check(sinkhorn_pack(&p, data(x), data(made.first), data_of<float>(made.second), on.stream), "sinkhorn_pack");
    return made;
}

Tensor unpack_values(const Packed &p, at::ScalarType type) {
    const On on(p.values);
    std::vector<int64_t> shape = p.values.sizes().vec();
    shape.back() = p.columns;
    const Tensor y = empty(shape, p.values, type);
    const sk_packing s = packing(row_count(p.values.sizes().slice(0, p.values.dim() - 1)), p.columns, p.block, type);
    check(sinkhorn_unpack(&s, data(p.values), data_of<float>(p.scales), data(y), on.stream), "sinkhorn_unpack");
    return y;
}
void result_type(at::ScalarType type) {
    TORCH_CHECK_TYPE(type_of(type) >= 0, "dtype must be float32, bfloat16 or float16, got ", type);
}
Tensor unpack(const PackedOf &packed, at::ScalarType type) {
    not_traced("sinkhorn_unpack");
    at::AutoGradMode off(false);
    const Packed p = packed_of(packed, "packed", false);
    result_type(type);
    return unpack_values(p, type);
}

// ---- experts ----

sk_experts experts(int64_t T, int64_t k, int64_t E, int64_t K, int64_t N, at::ScalarType type) {
    const char *where = "experts' product";
    return {size32(T, where), size32(k, where), size32(E, where), size32(K, where), size32(N, where), type_of(type)};
}
// Pairs of a token, where `rows` rows belong to T tokens.
int64_t rows_of(int64_t rows, int64_t T, const char *name) {
    if (T == 0) {
        TORCH_CHECK_VALUE(rows == 0, name, ": ", rows, " rows of no token");
        return 1;
    }
    TORCH_CHECK_VALUE(rows > 0 && rows % T == 0, name, ": ", rows, " rows are not a whole number for each of ", T,
                      " tokens");
    return rows / T;
}
// (T, k) for rows that are not gathered, where only T k counts: a token has up to 16 rows, so there are more of them
// than the library takes tokens.
std::pair<int64_t, int64_t> rows_in_order(int64_t rows) {
    for (int64_t k = 1; k <= 16; ++k)
        if (rows <= k << 24 && rows % k == 0) return {rows / k, k};
    return {rows, 1};  // the library refuses it
}

// A call without a gradient: its result counts as computed from the inputs, and who differentiates it gets an error, not
// a gradient without this path's part.
struct Constant : torch::autograd::Node {
    variable_list apply(variable_list &&) override {
        TORCH_CHECK_NOT_IMPLEMENTED(false, "sinkhorn_expert_product_packed has no gradient");
    }
};

Tensor product_packed(const Maybe &x_, const std::optional<PackedOf> &packed_, const PackedOf &weight_,
                      const Maybe &offsets_, const Maybe &tokens_, const std::optional<at::ScalarType> &type_) {
    not_traced("sinkhorn_expert_product_packed");
    TORCH_CHECK_TYPE(x_ || packed_, "x must be a GPU tensor or a Packed");
    const Packed weight = packed_of(weight_, "weight", true);
    const Tensor offsets = or_none(offsets_), tokens = or_none(tokens_);
    const int64_t dims = weight.values.dim();
    TORCH_CHECK_VALUE((dims == 3 && (offsets.defined() || weight.values.size(0) == 1)) || (dims == 2 && !offsets.defined()),
                      "weight must be packed from [E, N, K] (without offsets from [N, K]), got values ",
                      weight.values.sizes());
    const int64_t E = dims == 3 ? weight.values.size(0) : 1, N = weight.values.size(dims - 2), K = weight.columns;
    Packed x = {};
    Tensor given;
    at::ScalarType type = at::kBFloat16;
    int64_t columns, lead, rank;
    if (packed_) {
        x = packed_of(*packed_, "x", true);
        rank = x.values.dim(), lead = x.values.size(0), columns = x.columns;
    } else {
        given = contiguous(*x_);
        typed(given, "x");
        type = given.scalar_type();
        rank = given.dim(), lead = rank ? given.size(0) : 0, columns = rank ? given.size(-1) : 0;
    }
    const Tensor &rows = packed_ ? x.values : given;
    TORCH_CHECK_VALUE(rank == 2 && columns == K, "x must have rows of ", K, " columns, got ", rows.sizes());
    TORCH_CHECK_VALUE(weight.values.device() == rows.device(), "weight must be on ", rows.device(), ", got ",
                      weight.values.device());
    if (type_) result_type(type = *type_);
    if (offsets.defined()) {
        indices(offsets, "offsets", rows);
        shaped(offsets, "offsets", {E + 1});
    }
    std::pair<int64_t, int64_t> pairs;
    if (tokens.defined()) {
        TORCH_CHECK_VALUE(offsets.defined(), "tokens go with offsets");
        indices(tokens, "tokens", rows);
        pairs = {lead, rows_of(tokens.numel(), lead, "tokens")};
    } else {
        pairs = rows_in_order(lead);
    }
    no_tangent("sinkhorn_expert_product_packed", {given, x.scales, weight.scales});
    Tensor y;
    {
        at::AutoGradMode off(false);
        const On on(rows);
        void *values = data(x.values);
        float *scales = data_of<float>(x.scales);
        Tensor space;
        if (!packed_) {  // the scales behind the values
            const int64_t wide = pitch(K);
            space = empty({lead * (wide + 4)}, rows, at::kChar);
            values = data(space);
            scales = reinterpret_cast<float *>(static_cast<char *>(values) + lead * wide);
            const sk_packing s = packing(lead, K, 0, given.scalar_type());
            check(sinkhorn_pack(&s, data(given), values, scales, on.stream), "sinkhorn_pack");
        }
        y = empty({pairs.first * pairs.second, N}, rows, type);
        const sk_experts p = experts(pairs.first, pairs.second, E, K, N, type);
        check(sinkhorn_experts_forward_packed(&p, values, scales, data(weight.values), data_of<float>(weight.scales),
                                              data_of<int32_t>(offsets), data_of<int32_t>(tokens), data(y), on.stream),
              "sinkhorn_experts_forward_packed");
    }
    if (recorded({given, x.scales, weight.scales}))
        attach(new_node<Constant>(), {y}, torch::autograd::collect_next_edges(given, x.scales, weight.scales));
    return y;
}

// ---- activations, and products that keep their rows in 8 bits ----

void activation_of(int64_t kind, bool gated, int64_t columns) {
    TORCH_CHECK_VALUE(kind >= 0, "activation must be one of none, relu, silu, gelu");
    TORCH_CHECK_VALUE(!gated || columns % 2 == 0, "a gated activation takes an even number of columns, got ", columns);
}
std::vector<int64_t> activated_shape(at::IntArrayRef x, int64_t columns, bool gated) {
    std::vector<int64_t> s = x.vec();
    s.back() = gated ? columns / 2 : columns;
    return s;
}
// The activated rows; x in 8 bits goes to `kept`, where that is given.
Tensor activate(const Tensor &x, int64_t kind, bool gated, Packed *kept, const On &on) {
    const int64_t columns = x.size(-1);
    const Tensor y = empty(activated_shape(x.sizes(), columns, gated), x, x.scalar_type());
    if (kept) {
        std::tie(kept->values, kept->scales) = new_packed(x, kKeptBlock);
        kept->columns = columns, kept->block = kKeptBlock;
    }
    const sk_packing p = packing(row_count(x.sizes().slice(0, x.dim() - 1)), columns, kKeptBlock, x.scalar_type());
    check(sinkhorn_activation_forward(&p, static_cast<int32_t>(kind), gated, data(x), data(y),
                                      kept ? data(kept->values) : nullptr, kept ? data_of<float>(kept->scales) : nullptr,
                                      on.stream),
          "sinkhorn_activation_forward");
    return y;
}
// (activated rows again, gradient of x): each where wanted.
std::pair<Tensor, Tensor> activate_backward(const Packed &kept, int64_t kind, bool gated, at::ScalarType type,
                                            const Tensor &gy, bool wants_y, const On &on) {
    std::vector<int64_t> shape = kept.values.sizes().vec();
    shape.back() = kept.columns;
    const Tensor y = wants_y ? empty(activated_shape(kept.values.sizes(), kept.columns, gated), kept.values, type) : Tensor();
    const Tensor gx = gy.defined() ? empty(shape, kept.values, type) : Tensor();
    const bool wide = gy.defined() && gy.scalar_type() != type;  // gy in 32 bits
    const sk_packing p =
        packing(row_count(kept.values.sizes().slice(0, kept.values.dim() - 1)), kept.columns, kKeptBlock, type);
    check(wide ? sinkhorn_activation_backward32(&p, static_cast<int32_t>(kind), gated, data(kept.values),
                                                data_of<float>(kept.scales), data_of<float>(gy), data(y), data(gx),
                                                on.stream)
               : sinkhorn_activation_backward(&p, static_cast<int32_t>(kind), gated, data(kept.values),
                                              data_of<float>(kept.scales), data(gy), data(y), data(gx), on.stream),
          "sinkhorn_activation_backward");
    return {y, gx};
}

// Rows that a node keeps: as saved tensors, so that hooks on those (checkpoints, copies to the host) have them too.
struct KeptRows {
    SavedVariable values, scales;
    int64_t columns = 0;
    KeptRows() = default;
    explicit KeptRows(const Packed &p) : values(keep(p.values)), scales(keep(p.scales)), columns(p.columns) {}
    Packed unpack() const { return {restored_own(values), restored_own(scales), columns, kKeptBlock}; }
    void release() { values.reset_data(), scales.reset_data(); }
};

struct ActivationNode : Node {
    KeptRows rows;
    int64_t kind;
    bool gated;
    at::ScalarType type;
    ActivationNode() : Node("sinkhorn_activation") {}
    variable_list gradients(const variable_list &grads) override {
        if (!grads[0].defined()) return variable_list(1);
        const Packed kept = rows.unpack();
        const On on(kept.values);
        return {activate_backward(kept, kind, gated, type, grads[0], false, on).second};
    }
    void release_variables() override {
        const std::lock_guard<std::mutex> lock(mutex_);
        rows.release();
    }
};

Tensor activation(const Tensor &x_, int64_t kind, bool gated) {
    not_traced("sinkhorn_activation");
    const Tensor x = contiguous(x_);
    columns_of(x, "x");
    activation_of(kind, gated, x.size(-1));
    no_tangent("sinkhorn_activation", {x});
    const bool rec = recorded({x});
    Packed kept = {};
    Tensor y;
    {
        at::AutoGradMode off(false);
        const On on(x);
        y = activate(x, kind, gated, rec ? &kept : nullptr, on);
    }
    if (rec) {
        auto node = new_node<ActivationNode>();
        node->rows = KeptRows(kept), node->kind = kind, node->gated = gated, node->type = x.scalar_type();
        attach(node, {y}, torch::autograd::collect_next_edges(x));
    }
    return y;
}

struct KeptNode : Node {
    SavedVariable weight, offsets, tokens, slots;
    KeptRows rows;
    int64_t kind;
    bool gated;
    sk_experts p;
    at::ScalarType type;
    KeptNode() : Node("sinkhorn_expert_product_kept") {}

    variable_list gradients(const variable_list &grads) override {
        if (!grads[0].defined()) return variable_list(2);
        const Tensor w = restored(weight), off = restored(offsets), tok = restored(tokens), sl = restored(slots);
        const Packed kept = rows.unpack();
        const Tensor &gy = grads[0];
        const On on(w);
        Tensor gx, a, gw;
        if (wants(0)) {
            // What an activation's derivative and the other half still multiply stays in 32 bits in float16, whose range
            // would lose a gradient (past 65504, or below 3e-8) that these bring back into it.  bfloat16 has the range.
            const bool wide = (kind || gated) && type == at::kHalf;
            gx = empty({sl.defined() ? p.T : static_cast<int64_t>(p.T) * p.k, p.K}, w, wide ? at::kFloat : type);
            const size_t need = sl.defined() ? sinkhorn_experts_workspace_bytes(&p) : 0;
            const Tensor ws = empty_bytes(need, w);
            const auto run = [&](auto entry, auto *to) {
                check(entry(&p, data(gy), data(w), data_of<int32_t>(off), data_of<int32_t>(sl), to, data(ws), need, on.stream),
                      "sinkhorn_experts_backward_input");
            };
            if (wide)
                run(sinkhorn_experts_backward_input32, data_of<float>(gx));
            else
                run(sinkhorn_experts_backward_input, data(gx));
        }
        if (kind || gated)
            std::tie(a, gx) = activate_backward(kept, kind, gated, type, gx, wants(1), on);
        else if (wants(1))
            a = unpack_values(kept, type);
        if (wants(1)) {
            gw = at::empty_like(w);
            const size_t need = sinkhorn_experts_weight_workspace_bytes(&p);
            const Tensor ws = empty_bytes(need, w);
            check(sinkhorn_experts_backward_weight(&p, data(gy), data(a), data_of<int32_t>(off), data_of<int32_t>(tok),
                                                   data(gw), data(ws), need, on.stream),
                  "sinkhorn_experts_backward_weight");
        }
        return {gx, gw};
    }
    void release_variables() override {
        const std::lock_guard<std::mutex> lock(mutex_);
        for (SavedVariable *v : {&weight, &offsets, &tokens, &slots}) v->reset_data();
        rows.release();
    }
};

Tensor product_kept(const Tensor &x_, const Tensor &weight_, const Tensor &offsets, const Maybe &tokens_,
                    const Maybe &slots_, int64_t kind, bool gated) {
    const char *what = "sinkhorn_expert_product_kept";
    not_traced(what);
    const Tensor tokens = or_none(tokens_), slots = or_none(slots_);
    TORCH_CHECK_VALUE(tokens.defined() == slots.defined(), "tokens and slots go together");
    const Tensor x = contiguous(x_), weight = contiguous(weight_);
    typed(weight, "weight", true);
    TORCH_CHECK_VALUE(weight.dim() == 3, "weight must be [E, N, K], got ", weight.sizes());
    const int64_t E = weight.size(0), N = weight.size(1), K = weight.size(2), wide = gated ? 2 * K : K;
    typed(x, "x", true);
    TORCH_CHECK_VALUE(x.dim() == 2 && x.size(1) == wide, "x must have ", wide, " columns, got ", x.sizes());
    like(x, "x", weight, weight.scalar_type());
    activation_of(kind, gated, x.size(1));
    indices(offsets, "offsets", x);
    shaped(offsets, "offsets", {E + 1});
    std::pair<int64_t, int64_t> pairs;
    if (tokens.defined()) {
        indices(tokens, "tokens", x);
        indices(slots, "slots", x);
        pairs = {x.size(0), rows_of(tokens.numel(), x.size(0), "tokens")};
        TORCH_CHECK_VALUE(slots.dim() == 2 && slots.size(0) == x.size(0) &&
                              (x.size(0) == 0 || slots.size(1) == pairs.second),
                          "slots must be [", x.size(0), ", ", pairs.second, "], got ", slots.sizes());
    } else {
        pairs = rows_in_order(x.size(0));
    }
    no_tangent(what, {x, weight});
    const sk_experts p = experts(pairs.first, pairs.second, E, K, N, x.scalar_type());
    const bool rec = recorded({x, weight}), plain = !kind && !gated;
    Packed kept = {};
    Tensor y;
    {
        at::AutoGradMode off(false);
        const On on(x);
        Tensor a = x;
        if (!plain) {
            a = activate(x, kind, gated, rec ? &kept : nullptr, on);
        } else if (rec && weight.requires_grad()) {  // the gradient of x needs the weight alone
            kept.columns = K, kept.block = kKeptBlock;
            std::tie(kept.values, kept.scales) = pack(x, kKeptBlock);
        }
        y = empty({pairs.first * pairs.second, N}, x, x.scalar_type());
        check(sinkhorn_experts_forward(&p, data(a), data(weight), data_of<int32_t>(offsets), data_of<int32_t>(tokens),
                                       data(y), on.stream),
              "sinkhorn_experts_forward");
    }
    if (rec) {
        auto node = new_node<KeptNode>();
        node->weight = keep(weight), node->offsets = keep(offsets), node->tokens = keep(tokens);
        node->slots = keep(slots), node->rows = KeptRows(kept), node->kind = kind, node->gated = gated, node->p = p;
        node->type = x.scalar_type();
        attach(node, {y}, torch::autograd::collect_next_edges(x, weight));
    }
    return y;
}

}  // namespace

PYBIND11_MODULE(_sinkhorn_torch, m) {
    py::register_exception_translator([](std::exception_ptr e) {
        try {
            if (e) std::rethrow_exception(e);
        } catch (const Refused &r) {
            const py::object type = py::module_::import("paper_1907_01729_amd._binding").attr("SinkhornError");
            const py::object made = type(static_cast<int>(r.status), r.where);
            PyErr_SetObject(type.ptr(), made.ptr());
        }
    });
    m.def("norm", &norm);
    m.def("residual_norm", &residual_norm);
    m.def("pack", &pack);
    m.def("unpack", &unpack);
    m.def("product_packed", &product_packed);
    m.def("activation", &activation);
    m.def("product_kept", &product_kept);
}
