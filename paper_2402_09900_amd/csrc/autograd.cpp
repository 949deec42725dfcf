// autograd.cpp -- the differentiable gated recurrence, layer norm and dropout: nodes of
// torch's autograd engine that allocate outputs and call the library (include/memoroid.h).
//
// In C++ because their backward pass runs on a thread of the engine's.  Small layers are bound by
// the host, and Python on two threads costs about twice what it does on one (5997 x 250
// fp32, norm and its gradient: 125 us with Python nodes).
// Arguments have been checked by the binding (binding.py), gradients by the engine.
#include <torch/extension.h>

#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>

#include "memoroid.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::Function;
using torch::autograd::variable_list;
using OptTensor = std::optional<Tensor>;

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
Tensor given(const OptTensor& t) { return t.has_value() ? *t : Tensor(); }
Tensor dense(const Tensor& t) { return t.defined() ? t.contiguous() : t; }
int dtype_of(const Tensor& t) { return t.scalar_type() == at::kBFloat16 ? MEMOROID_BF16 : MEMOROID_F32; }
Tensor new_floats(const Tensor& like, at::IntArrayRef size) { return at::empty(size, like.options().dtype(at::kFloat)); }

// fn(args..., stream) on `like`'s device and that device's current stream
template <class F, class... A>
void launch(const char* name, F fn, const Tensor& like, A... args) {
    const c10::OptionalDeviceGuard guard(like.device());
    const int st = fn(args..., (void*)c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(like.device().index()).stream());
    if (st != MEMOROID_OK) throw StatusError(name, st);
}
// A call's own workspace: (tensor that holds it)
Tensor workspace(const Tensor& like, size_t bytes) {
    return at::empty({(int64_t)std::max<size_t>(bytes, 256)}, like.options().dtype(at::kByte));
}

// Gradients here have none of their own: where the engine builds a graph of them, this
// stands in it and refuses to be differentiated.
struct Once : Function<Once> {
    static Tensor forward(AutogradContext*, const Tensor& t) { return t.detach(); }
    static variable_list backward(AutogradContext*, variable_list) {
        throw std::runtime_error("trying to differentiate twice a function that has one derivative");
    }
};
template <class F>
variable_list once(F&& f) {
    if (!at::GradMode::is_enabled()) return f();
    variable_list got;
    {
        const at::NoGradGuard off;
        got = f();
    }
    for (Tensor& t : got)
        if (t.defined()) t = Once::apply(t.detach().requires_grad_());
    return got;
}

// ------------------------------------------------------- gated recurrence

struct GatedScan : Function<GatedScan> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& gates, const Tensor& alpha,
                                 const Tensor& start, const OptTensor& state_, bool final_state) {
        const int64_t B = x.size(0), T = x.size(1), d = x.size(2);
        const Tensor state = given(state_);
        Tensor h = at::empty_like(x), last;
        if (final_state) last = new_floats(x, {B, d});
        const Tensor kept = new_floats(x, {B, (T + MEMOROID_GATED_STATE_STEPS - 1) / MEMOROID_GATED_STATE_STEPS, d});
        if (T == 0 && final_state) {                         // no step: the state stays
            if (state.defined()) last.copy_(state);
            else last.zero_();
        }
        const int dt = dtype_of(x);
        const size_t bytes = memoroid_scan_gated_workspace_bytes(B, T, d, dt);
        const Tensor ws = workspace(x, bytes);
        launch("memoroid_scan_gated", memoroid_scan_gated, x, ptr(x), ptr(gates), floats(alpha), (const uint8_t*)ptr(start),
               floats(state), ptr(h), floats(last), floats(kept), B, T, d, dt, ptr(ws), (size_t)ws.numel());
        ctx->save_for_backward({x, gates, alpha, start, kept});
        ctx->saved_data["state"] = state.defined();
        ctx->set_materialize_grads(false);
        return final_state ? variable_list{h, last} : variable_list{h};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        return once([&] {
            const variable_list saved = ctx->get_saved_variables();
            const Tensor &x = saved[0], &gates = saved[1], &alpha = saved[2], &start = saved[3], &kept = saved[4];
            const int64_t B = x.size(0), T = x.size(1), d = x.size(2);
            const Tensor gh = grads[0].defined() ? grads[0].contiguous() : at::zeros_like(x);
            const Tensor gl = grads.size() > 1 ? dense(grads[1]) : Tensor();
            const bool has_state = ctx->saved_data["state"].toBool();
            Tensor gx = at::empty_like(x), gg = at::empty_like(gates), ga, gs;
            if (ctx->needs_input_grad(2)) ga = at::empty_like(alpha);
            if (has_state && ctx->needs_input_grad(4)) gs = new_floats(x, {B, d});
            if (B == 0 || T == 0) {                          // no step: the state stays, nothing decays
                if (ga.defined()) ga.zero_();
                if (gs.defined() && gl.defined()) gs.copy_(gl);
                else if (gs.defined()) gs.zero_();
            } else {
                const int dt = dtype_of(x);
                const size_t bytes = memoroid_scan_gated_bwd_workspace_bytes(B, T, d, dt);
                const Tensor ws = workspace(x, bytes);
                launch("memoroid_scan_gated_bwd", memoroid_scan_gated_bwd, x, ptr(x), ptr(gates), floats(alpha),
                       (const uint8_t*)ptr(start), floats(kept), ptr(gh), floats(gl), ptr(gx), ptr(gg), floats(ga),
                       floats(gs), B, T, d, dt, ptr(ws), (size_t)ws.numel());
            }
            return variable_list{gx, gg, ga, Tensor(), gs, Tensor()};
        });
    }
};

// ---------------------------------------------------- layer norm and dropout

struct LayerNorm : Function<LayerNorm> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const OptTensor& weight_, const OptTensor& bias_,
                                 double eps, const OptTensor& residual_, double p, const OptTensor& rng_, int64_t site) {
        const Tensor weight = given(weight_), bias = given(bias_), residual = given(residual_), rng = given(rng_);
        const int64_t d = x.size(-1), n = d ? x.numel() / d : 0;
        Tensor y = at::empty_like(x), s;
        if (residual.defined() || p > 0) s = at::empty_like(x);
        std::vector<int64_t> size = x.sizes().vec();
        size.back() = 2;
        const Tensor stats = new_floats(x, size);
        launch("memoroid_layer_norm", memoroid_layer_norm, x, ptr(x), ptr(residual), floats(weight), floats(bias),
               (const int64_t*)ptr(rng), ptr(y), ptr(s), floats(stats), (float)eps, p, site, n, d, dtype_of(x));
        ctx->save_for_backward({x, weight, residual, p > 0 ? rng : Tensor(), stats});
        ctx->saved_data["p"] = p;
        ctx->saved_data["site"] = site;
        // (bits: weight, bias)
        ctx->saved_data["has"] = (int64_t)(weight.defined() + 2 * bias.defined());
        ctx->set_materialize_grads(false);
        return s.defined() ? variable_list{y, s} : variable_list{y};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        return once([&] {
            const variable_list saved = ctx->get_saved_variables();
            const Tensor &x = saved[0], &weight = saved[1], &residual = saved[2], &rng = saved[3], &stats = saved[4];
            const double p = ctx->saved_data["p"].toDouble();
            const int64_t site = ctx->saved_data["site"].toInt(), has = ctx->saved_data["has"].toInt();
            const int64_t d = x.size(-1), n = d ? x.numel() / d : 0;
            const Tensor gy = grads[0].defined() ? grads[0].contiguous() : at::zeros_like(x);
            const Tensor gs = grads.size() > 1 ? dense(grads[1]) : Tensor();
            Tensor gx = at::empty_like(x), gr, gw, gb, ws;
            if (residual.defined()) gr = p > 0 ? at::empty_like(x) : gx;
            // (tensors that were given are counted: x, weight, bias)
            if ((has & 1) && ctx->needs_input_grad(1)) gw = new_floats(x, {d});
            if ((has & 2) && ctx->needs_input_grad(has & 1 ? 2 : 1)) gb = new_floats(x, {d});
            if (gw.defined() || gb.defined()) {
                if (n == 0) {                                // no rows: sums of nothing
                    if (gw.defined()) gw.zero_();
                    if (gb.defined()) gb.zero_();
                }
                ws = workspace(x, memoroid_layer_norm_bwd_workspace_bytes(n, d));
            }
            launch("memoroid_layer_norm_bwd", memoroid_layer_norm_bwd, x, ptr(x), ptr(residual), floats(weight),
                   (const int64_t*)ptr(rng), floats(stats), ptr(gy), ptr(gs), ptr(gx), p > 0 ? ptr(gr) : nullptr,
                   floats(gw), floats(gb), p, site, n, d, dtype_of(x), ptr(ws), (size_t)(ws.defined() ? ws.numel() : 0));
            return variable_list{gx, gw, gb, Tensor(), gr, Tensor(), Tensor(), Tensor()};
        });
    }
};

Tensor drop(const Tensor& x, double p, const Tensor& rng, int64_t site, const Tensor& residual) {
    const int64_t d = x.size(-1), n = d ? x.numel() / d : 0;
    Tensor out = at::empty_like(x);
    launch("memoroid_dropout", memoroid_dropout, x, ptr(x), ptr(residual), (const int64_t*)ptr(rng), ptr(out), p, site, n, d,
           dtype_of(x));
    return out;
}

struct Dropout : Function<Dropout> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, double p, const OptTensor& rng_, int64_t site,
                          const OptTensor& residual_) {
        const Tensor rng = given(rng_), residual = given(residual_);
        ctx->save_for_backward({p > 0 ? rng : Tensor()});
        ctx->saved_data["p"] = p;
        ctx->saved_data["site"] = site;
        ctx->saved_data["residual"] = residual.defined();
        return drop(x, p, rng, site, residual);
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        return once([&] {
            const variable_list saved = ctx->get_saved_variables();
            const double p = ctx->saved_data["p"].toDouble();
            Tensor gx;
            if (ctx->needs_input_grad(0))
                gx = p > 0 ? drop(grads[0].contiguous(), p, saved[0], ctx->saved_data["site"].toInt(), Tensor()) : grads[0];
            return variable_list{gx, Tensor(), Tensor(), Tensor(),
                                 ctx->saved_data["residual"].toBool() ? grads[0] : Tensor()};
        });
    }
};

py::object result(const variable_list& got) {
    return got.size() == 1 ? py::cast(got[0]) : py::object(py::make_tuple(got[0], got[1]));
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    m.def("gated_scan", [](const Tensor& x, const Tensor& gates, const Tensor& alpha, const Tensor& start,
                           const OptTensor& state, bool final_state) {
        return result(GatedScan::apply(x, gates, alpha, start, state, final_state));
    });
    m.def("layer_norm", [](const Tensor& x, const OptTensor& weight, const OptTensor& bias, double eps,
                           const OptTensor& residual, double p, const OptTensor& rng, int64_t site) {
        return result(LayerNorm::apply(x, weight, bias, eps, residual, p, rng, site));
    });
    m.def("dropout", [](const Tensor& x, double p, const OptTensor& rng, int64_t site, const OptTensor& residual) {
        return Dropout::apply(x, p, rng, site, residual);
    });
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
