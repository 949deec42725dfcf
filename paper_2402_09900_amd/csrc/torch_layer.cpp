// torch_layer.cpp -- the gated recurrence, layer norm and dropout on torch tensors: checks
// of the arguments, outputs and workspaces, calls of the library (include/memoroid.h) on the
// current stream, and nodes of torch's autograd engine.  binding.py has the Python side
// with the documentation.
//
// In C++ because the call is what small ones cost: a gated step of 16 x 256 floats, 2.4 us
// on the GPU, takes 3.9 us a call and took 7.6 through ctypes, scan_gated 4.8 and 11; a
// backward pass in Python, on a thread of the engine's, costs about twice what the same calls
// do on the caller's own (5997 x 250 fp32, norm and gradient: 115 us, 67 here).
#include <torch/extension.h>

#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include "memoroid.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::Function;
using torch::autograd::variable_list;
using OptTensor = std::optional<Tensor>;
using Shape = std::initializer_list<int64_t>;

// ------------------------------------------------------------- checks, calls

// (thrown to Python, with the interpreter's lock: never from a node's backward pass)
void type_if(bool bad, const char* what) {
    if (bad) throw py::type_error(what);
}
void value_if(bool bad, const char* what) {
    if (bad) throw py::value_error(what);
}
bool is(const Tensor& t, at::ScalarType type, Shape shape) {
    return t.scalar_type() == type && t.sizes() == at::IntArrayRef(shape);
}
Tensor given(const OptTensor& t) { return t.has_value() ? *t : Tensor(); }

// The library is no torch operator: what records operators (a trace, a graph of them, shapes
// without memory) would see the results' new memory and not the call that fills it.  Modes
// that only look on are no reason to refuse.
void refuse_recording() {
    using c10::impl::TorchDispatchModeKey;
    using Modes = c10::impl::TorchDispatchModeTLS;
    bool records = torch::jit::tracer::isTracing();
    if (Modes::any_modes_set())
        for (const auto key : {TorchDispatchModeKey::FAKE, TorchDispatchModeKey::PROXY, TorchDispatchModeKey::FUNCTIONAL})
            records = records || Modes::get_mode(key).has_value();
    if (records)
        throw std::runtime_error("calls of the gated recurrence, layer norm and dropout cannot be traced or run without memory");
}
struct Unrecorded {
    Unrecorded() { refuse_recording(); }
};
// Device memory that kernels may index: of one device, without gaps, there
void check_places(std::initializer_list<const Tensor*> tensors) {
    const Tensor* first = nullptr;
    for (const Tensor* t : tensors) {
        if (!t->defined()) continue;
        value_if(!t->is_cuda(), "tensors must live on a CUDA (HIP) device");
        value_if(!t->is_contiguous(), "tensors must be contiguous");
        // (a tensor of no memory of its own, as in functionalize: an optional one would count as not given)
        value_if(t->numel() != 0 && !t->data_ptr(), "tensors must have memory");
        if (!first) first = t;
        value_if(t->device() != first->device(), "tensors must live on one device");
    }
}
int dtype_of(const Tensor& t) { return t.scalar_type() == at::kBFloat16 ? MEMOROID_BF16 : MEMOROID_F32; }
void check_dtype(const Tensor& x, const char* what) {
    type_if(x.scalar_type() != at::kFloat && x.scalar_type() != at::kBFloat16, what);
}

// A call that the library refused, MemoroidError in Python
struct StatusError : std::runtime_error {
    StatusError(const char* where_, int status_)
        : std::runtime_error(std::string(where_) + " failed: " + memoroid_status_string(status_) + " (status " +
                             std::to_string(status_) + ")"),
          where(where_), status(status_) {}
    std::string where;
    int status;
};

void* ptr(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
float* floats(const Tensor& t) { return (float*)ptr(t); }
const int64_t* numbers(const Tensor& t) { return (const int64_t*)ptr(t); }
Tensor dense(const Tensor& t) { return t.defined() ? t.contiguous() : t; }
Tensor new_floats(const Tensor& like, at::IntArrayRef size) { return at::empty(size, like.options().dtype(at::kFloat)); }

// fn(args..., stream) on `like`'s device and that device's current stream
template <class F, class... A>
void launch(const char* name, F fn, const Tensor& like, A... args) {
    const c10::OptionalDeviceGuard guard(like.device());
    const int st = fn(args..., (void*)c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(like.device().index()).stream());
    if (st != MEMOROID_OK) throw StatusError(name, st);
}
// A call's workspace: the caller's if it is large enough, else one of its own
Tensor workspace(const Tensor& like, size_t bytes, const Tensor& callers = Tensor()) {
    if (callers.defined()) {
        value_if(callers.device() != like.device(), "the workspace must live on the tensors' device");
        value_if(!callers.is_contiguous(), "the workspace must be contiguous");
        if ((size_t)callers.numel() >= bytes) return callers;
    }
    return at::empty({(int64_t)std::max<size_t>(bytes, 256)}, like.options().dtype(at::kByte));
}

// ------------------------------------------------------- gated recurrence

int64_t kept_states(int64_t T) { return (T + MEMOROID_GATED_STATE_STEPS - 1) / MEMOROID_GATED_STATE_STEPS; }

void check_gates(const Tensor& x, const Tensor& gates, const Tensor& alpha) {
    const int64_t d = x.size(-1);
    if (x.dim() == 3) value_if(gates.sizes() != at::IntArrayRef({x.size(0), x.size(1), 2, d}), "gates must be [B,T,2,d]");
    else value_if(gates.sizes() != at::IntArrayRef({x.size(0), 2, d}), "gates must be [B,2,d]");
    type_if(gates.scalar_type() != x.scalar_type(), "x and gates must share a dtype");
    check_dtype(x, "the gated recurrence takes float32 or bfloat16");
    type_if(!is(alpha, at::kFloat, {d}), "alpha must be float32 [d]");
}
void check_tapes(const Tensor& x, const Tensor& gates, const Tensor& alpha, const Tensor& start) {
    value_if(x.dim() != 3, "x must be [B,T,d]");
    check_gates(x, gates, alpha);
    type_if(!is(start, at::kByte, {x.size(0), x.size(1)}), "start must be uint8 [B,T]");
}
void check_state(const Tensor& x, const Tensor& state, const char* what) {
    type_if(state.defined() && !is(state, at::kFloat, {x.size(0), x.size(-1)}), what);
}

struct Scanned {
    Tensor h, last, kept;
};
Scanned gated_forward(const Tensor& x, const Tensor& gates, const Tensor& alpha, const Tensor& start, const Tensor& state,
                      bool final_state, bool keep_states, const Tensor& callers) {
    const at::NoGradGuard off;
    const int64_t B = x.size(0), T = x.size(1), d = x.size(2);
    Scanned got;
    got.h = at::empty_like(x);
    if (final_state) got.last = new_floats(x, {B, d});
    if (keep_states) got.kept = new_floats(x, {B, kept_states(T), d});
    if (T == 0 && final_state) {                             // no step: the state stays
        if (state.defined()) got.last.copy_(state);
        else got.last.zero_();
    }
    const int dt = dtype_of(x);
    const Tensor ws = workspace(x, memoroid_scan_gated_workspace_bytes(B, T, d, dt), callers);
    launch("memoroid_scan_gated", memoroid_scan_gated, x, ptr(x), ptr(gates), floats(alpha), (const uint8_t*)ptr(start),
           floats(state), ptr(got.h), floats(got.last), floats(got.kept), B, T, d, dt, ptr(ws), (size_t)ws.numel());
    return got;
}
// (dx, dgates, dalpha, dstate), the last two where they are wanted
variable_list gated_backward(const Tensor& x, const Tensor& gates, const Tensor& alpha, const Tensor& start, const Tensor& kept,
                             const Tensor& grad_h, const Tensor& grad_state, bool want_alpha, bool want_state,
                             const Tensor& callers) {
    const at::NoGradGuard off;
    const int64_t B = x.size(0), T = x.size(1), d = x.size(2);
    Tensor gx = at::empty_like(x), gg = at::empty_like(gates), ga, gs;
    if (want_alpha) ga = at::empty_like(alpha);
    if (want_state) gs = new_floats(x, {B, d});
    if (B == 0 || T == 0) {                                  // no step: the state stays, nothing decays
        if (want_alpha) ga.zero_();
        if (want_state && grad_state.defined()) gs.copy_(grad_state);
        else if (want_state) gs.zero_();
    } else {
        const int dt = dtype_of(x);
        const Tensor ws = workspace(x, memoroid_scan_gated_bwd_workspace_bytes(B, T, d, dt), callers);
        launch("memoroid_scan_gated_bwd", memoroid_scan_gated_bwd, x, ptr(x), ptr(gates), floats(alpha),
               (const uint8_t*)ptr(start), floats(kept), ptr(grad_h), floats(grad_state), ptr(gx), ptr(gg), floats(ga),
               floats(gs), B, T, d, dt, ptr(ws), (size_t)ws.numel());
    }
    return {gx, gg, ga, gs};
}

// ---------------------------------------------------- layer norm and dropout

struct Rows {
    int64_t n, d;
    explicit Rows(const Tensor& x) : d(x.size(-1)) { n = d ? x.numel() / d : 0; }
};
void check_rows(const Tensor& x, const Tensor& residual, double p, const Tensor& rng, int64_t site) {
    value_if(x.dim() < 1, "x must be [...,d]");
    check_dtype(x, "x must be float32 or bfloat16");
    type_if(residual.defined() && (residual.scalar_type() != x.scalar_type() || residual.sizes() != x.sizes()),
            "the residual must be like x");
    value_if(!(p >= 0.0 && p <= 1.0), "p must be in [0, 1]");
    value_if(p > 0 && !rng.defined(), "dropout needs rng, int64 [2] on x's device: seed and step");
    type_if(rng.defined() && !is(rng, at::kLong, {2}), "rng must be int64 [2]");
    value_if(site < 0 || site >= (int64_t)1 << 32, "site must be in [0, 2^32)");
}
void check_weights(const Tensor& x, const Tensor& weight, const Tensor& bias) {
    for (const Tensor* w : {&weight, &bias})
        type_if(w->defined() && !is(*w, at::kFloat, {x.size(-1)}), "weight and bias must be float32 [d]");
}
std::vector<int64_t> stats_size(const Tensor& x) {
    std::vector<int64_t> size = x.sizes().vec();
    size.back() = 2;
    return size;
}

struct Normed {
    Tensor y, s, stats;
};
Normed norm_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, double eps, const Tensor& residual, double p,
                    const Tensor& rng, int64_t site, bool keep_stats) {
    const Rows r(x);
    Normed got;
    got.y = at::empty_like(x);
    if (residual.defined() || p > 0) got.s = at::empty_like(x);
    if (keep_stats) got.stats = new_floats(x, stats_size(x));
    launch("memoroid_layer_norm", memoroid_layer_norm, x, ptr(x), ptr(residual), floats(weight), floats(bias), numbers(rng),
           ptr(got.y), ptr(got.s), floats(got.stats), (float)eps, p, site, r.n, r.d, dtype_of(x));
    return got;
}
// (dx, dresidual, dweight, dbias): the second undefined without a residual, the last two
// where they are not wanted
variable_list norm_backward(const Tensor& x, const Tensor& stats, const Tensor& grad_y, const Tensor& weight,
                            const Tensor& residual, const Tensor& grad_s, double p, const Tensor& rng, int64_t site,
                            bool want_weight, bool want_bias, const Tensor& callers) {
    const at::NoGradGuard off;
    const Rows r(x);
    Tensor gx = at::empty_like(x), gr, gw, gb, ws;
    if (residual.defined()) gr = p > 0 ? at::empty_like(x) : gx;
    if (want_weight) gw = new_floats(x, {r.d});
    if (want_bias) gb = new_floats(x, {r.d});
    if (r.n == 0) {                                          // no rows: sums of nothing
        if (want_weight) gw.zero_();
        if (want_bias) gb.zero_();
    }
    if (want_weight || want_bias) ws = workspace(x, memoroid_layer_norm_bwd_workspace_bytes(r.n, r.d), callers);
    launch("memoroid_layer_norm_bwd", memoroid_layer_norm_bwd, x, ptr(x), ptr(residual), floats(weight), numbers(rng),
           floats(stats), ptr(grad_y), ptr(grad_s), ptr(gx), p > 0 ? ptr(gr) : nullptr, floats(gw), floats(gb), p, site, r.n,
           r.d, dtype_of(x), ptr(ws), (size_t)(ws.defined() ? ws.numel() : 0));
    return {gx, gr, gw, gb};
}

Tensor drop(const Tensor& x, double p, const Tensor& rng, int64_t site, const Tensor& residual) {
    const Rows r(x);
    Tensor out = at::empty_like(x);
    launch("memoroid_dropout", memoroid_dropout, x, ptr(x), ptr(residual), numbers(rng), ptr(out), p, site, r.n, r.d,
           dtype_of(x));
    return out;
}

// ------------------------------------------------------------- autograd nodes
// (gradients that arrive are like their outputs: the engine has seen to it)

// Gradients here have none of their own.  Where the engine builds a graph of them, a node
// that raises stands behind them, in front of all that they hang on: the inputs of the node
// that has formed them, and the gradients that it was given.
variable_list once(variable_list got, const variable_list& upstream) {
    if (!at::GradMode::is_enabled()) return got;
    const auto by = torch::autograd::get_current_node();
    if (!by) throw std::runtime_error("a graph of gradients needs torch's engine to call the backward pass");
    torch::autograd::edge_list to;
    for (const auto& e : by->next_edges())
        if (e.is_valid()) to.push_back(e);
    for (const Tensor& g : upstream)
        if (g.defined() && g.requires_grad()) to.push_back(torch::autograd::impl::gradient_edge(g));
    const auto node = std::make_shared<torch::autograd::Error>(
        "trying to differentiate twice a function that has one derivative", std::move(to));
    for (Tensor& t : got)
        if (t.defined()) {
            // (two gradients may be one tensor, which could stand behind one of them only)
            t = t.detach();
            torch::autograd::create_gradient_edge(t, node);
        }
    return got;
}

struct GatedScan : Function<GatedScan> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& gates, const Tensor& alpha,
                                 const Tensor& start, const OptTensor& state, bool final_state) {
        const Scanned got = gated_forward(x, gates, alpha, start, given(state), final_state, true, Tensor());
        ctx->save_for_backward({x, gates, alpha, start, got.kept});
        ctx->saved_data["state"] = state.has_value();
        ctx->set_materialize_grads(false);
        return final_state ? variable_list{got.h, got.last} : variable_list{got.h};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        refuse_recording();
        const variable_list s = ctx->get_saved_variables();
        const Tensor gh = grads[0].defined() ? grads[0].contiguous() : at::zeros_like(s[0]);
        // (inputs that are tensors are counted: x, gates, alpha, start, state)
        const bool want_state = ctx->saved_data["state"].toBool() && ctx->needs_input_grad(4);
        const variable_list g = once(gated_backward(s[0], s[1], s[2], s[3], s[4], gh, grads.size() > 1 ? dense(grads[1]) : Tensor(),
                                                    ctx->needs_input_grad(2), want_state, Tensor()), grads);
        return {g[0], g[1], g[2], Tensor(), g[3], Tensor()};
    }
};

struct LayerNorm : Function<LayerNorm> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const OptTensor& weight, const OptTensor& bias,
                                 double eps, const OptTensor& residual, double p, const OptTensor& rng, int64_t site) {
        const Normed got = norm_forward(x, given(weight), given(bias), eps, given(residual), p, given(rng), site, true);
        ctx->save_for_backward({x, given(weight), given(residual), p > 0 ? given(rng) : Tensor(), got.stats});
        ctx->saved_data["p"] = p;
        ctx->saved_data["site"] = site;
        ctx->saved_data["bias"] = bias.has_value();
        ctx->set_materialize_grads(false);
        return got.s.defined() ? variable_list{got.y, got.s} : variable_list{got.y};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        refuse_recording();
        const variable_list s = ctx->get_saved_variables();
        const Tensor gy = grads[0].defined() ? grads[0].contiguous() : at::zeros_like(s[0]);
        // (inputs that are tensors are counted: x, weight and bias where they are given)
        const bool weight = s[1].defined(), bias = ctx->saved_data["bias"].toBool();
        const variable_list g =
            once(norm_backward(s[0], s[4], gy, s[1], s[2], grads.size() > 1 ? dense(grads[1]) : Tensor(),
                               ctx->saved_data["p"].toDouble(), s[3], ctx->saved_data["site"].toInt(),
                               weight && ctx->needs_input_grad(1), bias && ctx->needs_input_grad(weight ? 2 : 1), Tensor()), grads);
        return {g[0], g[2], g[3], Tensor(), g[1], Tensor(), Tensor(), Tensor()};
    }
};

struct Dropout : Function<Dropout> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, double p, const OptTensor& rng, int64_t site,
                          const OptTensor& residual) {
        ctx->save_for_backward({p > 0 ? given(rng) : Tensor()});
        ctx->saved_data["p"] = p;
        ctx->saved_data["site"] = site;
        ctx->saved_data["residual"] = residual.has_value();
        return drop(x, p, given(rng), site, given(residual));
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        refuse_recording();
        const double p = ctx->saved_data["p"].toDouble();
        const Tensor& g = grads[0];
        Tensor gx;
        if (p == 0) gx = g;
        else if (ctx->needs_input_grad(0))
            gx = once({drop(g.contiguous(), p, ctx->get_saved_variables()[0], ctx->saved_data["site"].toInt(), Tensor())}, grads)[0];
        return {gx, Tensor(), Tensor(), Tensor(), ctx->saved_data["residual"].toBool() ? g : Tensor()};
    }
};

// ------------------------------------------------------------------ for Python

// f() without the interpreter's lock, which other threads may want while it waits for a queue
template <class F>
auto unlocked(F&& f) {
    const py::gil_scoped_release free;
    return f();
}
// The tensors that are there: one by itself, else a tuple
py::object result(std::initializer_list<Tensor> tensors) {
    py::list there;
    for (const Tensor& t : tensors)
        if (t.defined()) there.append(t);
    if (there.size() == 1) return there[0];
    return py::tuple(there);
}
py::object result(const variable_list& got) {
    return got.size() == 1 ? py::cast(got[0]) : py::object(py::make_tuple(got[0], got[1]));
}

// Forward mode has no derivative here, and a result without a tangent would count as one
// whose tangent is zero: refused wherever forward mode is on, under no_grad too
void refuse_tangents(std::initializer_list<const Tensor*> inputs) {
    for (const Tensor* t : inputs)
        if (t->defined() && t->_fw_grad(0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode())
            throw std::runtime_error("the gated recurrence, layer norm and dropout have no derivative in forward mode");
}
// Whether a call belongs in the engine's graph; outside it nothing is kept for a gradient
bool in_graph(std::initializer_list<const Tensor*> inputs) {
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor* t : inputs)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}

py::object scan_gated(const Tensor& x, const Tensor& gates, const Tensor& alpha, const Tensor& start, const OptTensor& state_,
                      bool final_state, bool keep_states, const OptTensor& callers) {
    const Tensor state = given(state_);
    check_tapes(x, gates, alpha, start);
    check_state(x, state, "state must be float32 [B,d]");
    check_places({&x, &gates, &alpha, &start, &state});
    const Scanned got =
        unlocked([&] { return gated_forward(x, gates, alpha, start, state, final_state, keep_states, given(callers)); });
    return result({got.h, got.last, got.kept});
}

py::object scan_gated_bwd(const Tensor& x, const Tensor& gates, const Tensor& alpha, const Tensor& start, const Tensor& states,
                          const Tensor& grad_h, const OptTensor& grad_state_, bool want_alpha, bool want_state,
                          const OptTensor& callers) {
    const Tensor grad_state = given(grad_state_);
    check_tapes(x, gates, alpha, start);
    check_state(x, grad_state, "grad_state must be float32 [B,d]");
    type_if(!is(states, at::kFloat, {x.size(0), kept_states(x.size(1)), x.size(2)}), "states must be float32 [B,ceil(T/64),d]");
    type_if(grad_h.scalar_type() != x.scalar_type() || grad_h.sizes() != x.sizes(), "grad_h must be [B,T,d] of x's dtype");
    check_places({&x, &gates, &alpha, &start, &states, &grad_h, &grad_state});
    const variable_list g = unlocked([&] {
        return gated_backward(x, gates, alpha, start, states, grad_h, grad_state, want_alpha, want_state, given(callers));
    });
    return py::make_tuple(g[0], g[1], g[2], g[3]);
}

Tensor gated_step(const Tensor& x, const Tensor& gates, const Tensor& alpha, const Tensor& state, const OptTensor& start_) {
    const Tensor start = given(start_);
    value_if(x.dim() != 2, "x must be [B,d]");
    check_gates(x, gates, alpha);
    type_if(start.defined() && !is(start, at::kByte, {x.size(0)}), "start must be uint8 [B]");
    check_state(x, state, "state must be float32 [B,d]");
    refuse_tangents({&x, &gates, &alpha, &state});
    if (at::GradMode::is_enabled() &&
        (x.requires_grad() || gates.requires_grad() || alpha.requires_grad() || state.requires_grad()))
        throw std::runtime_error("gated_step has no gradient: call it under torch.no_grad(), or gated_scan() on tapes of one step");
    check_places({&x, &gates, &alpha, &start, &state});
    const py::gil_scoped_release free;
    Tensor h = at::empty_like(x);
    launch("memoroid_gated_step", memoroid_gated_step, x, ptr(x), ptr(gates), floats(alpha), (const uint8_t*)ptr(start),
           floats(state), ptr(h), x.size(0), x.size(1), dtype_of(x));
    // a graph that has saved the state refuses its backward pass
    if (!state.is_inference()) state.unsafeGetTensorImpl()->bump_version();
    return h;
}

Tensor drop_rows(const Tensor& x, double p, const OptTensor& rng_, int64_t site, const OptTensor& residual_) {
    const Tensor rng = given(rng_), residual = given(residual_);
    check_rows(x, residual, p, rng, site);
    check_places({&x, &residual, &rng});
    return unlocked([&] { return drop(x, p, rng, site, residual); });
}

py::object norm_rows(const Tensor& x, const OptTensor& weight_, const OptTensor& bias_, double eps, const OptTensor& residual_,
                     double p, const OptTensor& rng_, int64_t site, bool keep_stats) {
    const Tensor weight = given(weight_), bias = given(bias_), residual = given(residual_), rng = given(rng_);
    check_rows(x, residual, p, rng, site);
    check_weights(x, weight, bias);
    check_places({&x, &residual, &weight, &bias, &rng});
    const Normed got = unlocked([&] { return norm_forward(x, weight, bias, eps, residual, p, rng, site, keep_stats); });
    return result({got.y, got.s, got.stats});
}

py::object norm_rows_bwd(const Tensor& x, const Tensor& stats, const Tensor& grad_y, const OptTensor& weight_,
                         const OptTensor& residual_, const OptTensor& grad_s_, double p, const OptTensor& rng_, int64_t site,
                         bool want_weights, const OptTensor& callers) {
    const Tensor weight = given(weight_), residual = given(residual_), grad_s = given(grad_s_), rng = given(rng_);
    check_rows(x, residual, p, rng, site);
    check_weights(x, weight, Tensor());
    for (const Tensor* g : {&grad_y, &grad_s})
        type_if(g->defined() && (g->scalar_type() != x.scalar_type() || g->sizes() != x.sizes()),
                "upstream gradients must be like x");
    type_if(stats.scalar_type() != at::kFloat || stats.sizes() != at::IntArrayRef(stats_size(x)), "stats must be float32 [...,2]");
    check_places({&x, &residual, &weight, &rng, &stats, &grad_y, &grad_s});
    const variable_list g = unlocked([&] {
        return norm_backward(x, stats, grad_y, weight, residual, grad_s, p, rng, site, want_weights, want_weights, given(callers));
    });
    return py::make_tuple(g[0], g[1], g[2], g[3]);
}

py::object gated_scan(const Tensor& x, const Tensor& gates, const Tensor& alpha, const Tensor& start, const OptTensor& state,
                      bool final_state) {
    const Tensor s = given(state);
    check_tapes(x, gates, alpha, start);
    check_state(x, s, "state must be float32 [B,d]");
    refuse_tangents({&x, &gates, &alpha, &s});
    check_places({&x, &gates, &alpha, &start, &s});
    if (!in_graph({&x, &gates, &alpha, &s})) {
        const Scanned got = unlocked([&] { return gated_forward(x, gates, alpha, start, s, final_state, false, Tensor()); });
        return result({got.h, got.last});
    }
    return result(unlocked([&] { return GatedScan::apply(x, gates, alpha, start, state, final_state); }));
}

py::object layer_norm(const Tensor& x, const OptTensor& weight, const OptTensor& bias, double eps, const OptTensor& residual,
                      double p, const OptTensor& rng, int64_t site) {
    const Tensor w = given(weight), b = given(bias), res = given(residual), numbers = given(rng);
    check_rows(x, res, p, numbers, site);
    check_weights(x, w, b);
    refuse_tangents({&x, &res, &w, &b});
    check_places({&x, &res, &w, &b, &numbers});
    if (!in_graph({&x, &res, &w, &b})) {
        const Normed got = unlocked([&] { return norm_forward(x, w, b, eps, res, p, numbers, site, false); });
        return result({got.y, got.s});
    }
    return result(unlocked([&] { return LayerNorm::apply(x, weight, bias, eps, residual, p, rng, site); }));
}

Tensor dropout(const Tensor& x, double p, const OptTensor& rng, int64_t site, const OptTensor& residual) {
    const Tensor numbers = given(rng), res = given(residual);
    check_rows(x, res, p, numbers, site);
    refuse_tangents({&x, &res});
    check_places({&x, &res, &numbers});
    if (!in_graph({&x, &res})) return unlocked([&] { return drop(x, p, numbers, site, res); });
    return unlocked([&] { return Dropout::apply(x, p, rng, site, residual); });
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    const py::call_guard<Unrecorded> unrecorded;
    m.def("scan_gated", scan_gated, unrecorded);
    m.def("scan_gated_bwd", scan_gated_bwd, unrecorded);
    m.def("gated_step", gated_step, unrecorded);
    m.def("drop_rows", drop_rows, unrecorded);
    m.def("norm_rows", norm_rows, unrecorded);
    m.def("norm_rows_bwd", norm_rows_bwd, unrecorded);
    m.def("gated_scan", gated_scan, unrecorded);
    m.def("layer_norm", layer_norm, unrecorded);
    m.def("dropout", dropout, unrecorded);
    py::register_local_exception_translator([](std::exception_ptr e) {
        try {
            if (e) std::rethrow_exception(e);
        } catch (const StatusError& s) {
            const py::object type = py::module_::import("paper_2402_09900_amd.binding").attr("MemoroidError");
            const py::object error = type(s.status, s.where);
            PyErr_SetObject(type.ptr(), error.ptr());
        }
    });
}
