// The calls of memory.py and of the preference loss, with their autograd: checks, outputs
// and workspaces from the caching allocator, one call of the library.  From Python, by
// ctypes and a Python autograd function, the same took 12 to 19 us of the host a call and
// 138 us for a scan with its gradient; here 4 to 10 us and 55 to 78 (torch's own layer norm with
// its gradient: 69 to 71, its silu 45).
#include "pictura_tensors.h"

#include <ATen/TracerMode.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/variable.h>

#include "pictura.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

static_assert(sizeof(Sequences) == sizeof(pictura_sequences) && sizeof(Norm) == sizeof(pictura_norm), "the library's structs");

// The library's entries: it is loaded by the Python binding, which hands over their addresses.
struct Entries {
    decltype(&pictura_gated_scan_workspace) scan_workspace;
    decltype(&pictura_gated_scan) scan;
    decltype(&pictura_gated_scan_gradient) scan_gradient;
    decltype(&pictura_gated_step) step;
    decltype(&pictura_rms_norm) norm;
    decltype(&pictura_rms_norm_codes) norm_codes;
    decltype(&pictura_row_values) row_values;
    decltype(&pictura_rms_norm_gradient_workspace) norm_workspace;
    decltype(&pictura_rms_norm_gradient) norm_gradient;
    decltype(&pictura_preference_loss_workspace) preference_workspace;
    decltype(&pictura_preference_loss) preference_loss;
} entries{};

constexpr Py_ssize_t kEntries = sizeof(Entries) / sizeof(void*);

PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != kEntries) {
        PyErr_Format(PyExc_TypeError, "bind: %zd addresses, expected %zd", n, kEntries);
        return nullptr;
    }
    void* at[kEntries];
    for (Py_ssize_t i = 0; i < n; ++i) {
        at[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    memcpy(&entries, at, sizeof(entries));
    Py_RETURN_NONE;
}

// ---- what every call does -----------------------------------------------------------

void on_device(const Tensor& t, const char* name)
{
    if (!t.is_cuda()) refuse(name, ": tensor on ", t.device(), ", expected the HIP device");
}

void* stream_of(const Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

void check(pictura_status st, const char* call)
{
    if (st == PICTURA_OK) return;
    std::ostringstream s;
    s << "pictura status " << st << ": " << call << " failed";
    if (st == PICTURA_EINVAL) throw Refused(s.str());
    throw std::runtime_error(s.str());
}

Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const Tensor& like)
{
    return at::empty(sizes, like.options().dtype(type).requires_grad(false));
}

template <class T>
T* data(const Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }

bool wants_gradient(std::initializer_list<const Tensor*> ts)
{
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor* t : ts)
        if (t && t->requires_grad()) return true;
    return false;
}

// A leaf that an eager graph still holds accumulates on that graph's stream.  A capture
// cannot wait for the default stream: its backward would end the process.
void check_capture(std::initializer_list<std::pair<const Tensor*, const char*>> ts)
{
    if (!ts.begin()->first->is_cuda() || c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None) return;
    for (const auto& [t, name] : ts) {
        if (!t || !t->is_leaf() || !t->requires_grad()) continue;
        const auto held = torch::autograd::impl::try_get_grad_accumulator(*t);
        const auto s = held ? held->stream() : std::nullopt;
        if (s && *s != c10::impl::VirtualGuardImpl(t->device().type()).getStream(t->device()))
            refuse(name, ": a graph recorded on another stream still holds this leaf; drop it before the capture");
    }
}

// What a backward returns can not be differentiated again.  Where a graph of it is wanted,
// it hangs on what it was computed from by a node that raises.
struct Twice : torch::autograd::Node {
    variable_list apply(variable_list&&) override
    {
        throw std::runtime_error("trying to differentiate twice a function of this library, whose gradients have none");
    }
};

variable_list once(const variable_list& from, variable_list out)
{
    if (!at::GradMode::is_enabled()) return out;
    const auto node = std::make_shared<Twice>();
    node->set_next_edges(torch::autograd::collect_next_edges(from));
    for (Tensor& t : out)
        if (t.defined()) torch::autograd::set_history(t, node);
    return out;
}

// The calls are no operators of torch: what records or transforms a program by its operators
// sees only the outputs' allocation, and would take what comes out for a constant.
void check_seen(const char* call)
{
    const char* by = nullptr;
    if (at::tracer::impl::is_dispatch_enabled()) by = "torch.jit.trace";
    else if (c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode)) by = "torch.func";
    else if (c10::impl::TorchDispatchModeTLS::any_modes_set()) by = "a dispatch mode";
    if (by) refuse(call, ": called under ", by, ", which would not see it");
}

// Forward-mode differentiation: a dual tensor need not want a gradient to have a tangent.
void check_tangents(std::initializer_list<std::pair<const Tensor*, const char*>> ts)
{
    if (!c10::AutogradState::get_tls_state().get_fw_grad_mode()) return;
    for (const auto& [t, name] : ts)
        if (t && t->defined() && t->_fw_grad(0).defined()) refuse(name, ": has a tangent, and this call hands on none");
}

// Outputs that have no gradient, of a call that wants one: it is not lost without a word, but
// raises where it would arrive.
struct Refuses : torch::autograd::Node {
    explicit Refuses(const char* what) : what_(what) {}
    variable_list apply(variable_list&&) override { throw std::runtime_error(what_); }
    const char* what_;
};

void refuse_gradient(const char* what, const variable_list& from, const variable_list& out)
{
    const auto node = std::make_shared<Refuses>(what);
    node->set_next_edges(torch::autograd::collect_next_edges(from));
    for (const Tensor& t : out)
        if (t.is_floating_point()) torch::autograd::set_history(t, node);
}

// The gradient of a sum: what arrives, for both terms.
struct SumOfTwo : torch::autograd::Node {
    variable_list apply(variable_list&& grads) override { return {grads[0], grads[0]}; }
};

// f() with what it refuses as a ValueError, and torch's own errors as torch has them.
template <class F>
PyObject* guarded(const char* call, F f)
{
    HANDLE_TH_ERRORS
    if (!entries.scan) {
        PyErr_SetString(PyExc_RuntimeError, "the library's entries are not bound: import memory or policy");
        return nullptr;
    }
    try {
        check_seen(call);
        return f();
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

void arguments(Py_ssize_t got, Py_ssize_t expected, const char* call)
{
    if (got != expected) refuse(call, ": ", got, " arguments, expected ", expected);
}

PyObject* tuple(const variable_list& ts)
{
    PyObject* result = PyTuple_New((Py_ssize_t)ts.size());
    if (!result) return nullptr;
    for (size_t i = 0; i < ts.size(); ++i) {
        PyObject* o = ts[i].defined() ? THPVariable_Wrap(ts[i]) : Py_NewRef(Py_None);
        if (!o) {
            Py_DECREF(result);
            return nullptr;
        }
        PyTuple_SET_ITEM(result, (Py_ssize_t)i, o);
    }
    return result;
}

double number(PyObject* o, const char* name)
{
    if (PyBool_Check(o) || (!PyFloat_Check(o) && !PyLong_Check(o))) refuse(name, ": expected a number");
    const double x = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        refuse(name, ": expected a number within range");
    }
    return x;
}

using Optional = std::optional<Tensor>;

Optional or_none(const Tensor* t) { return t ? Optional(*t) : std::nullopt; }

const Tensor* or_null(const Tensor& t) { return t.defined() ? &t : nullptr; }

const Tensor* or_null(const Optional& t) { return t ? &*t : nullptr; }

// ---- the gated recurrence -----------------------------------------------------------

// [batch, steps, channels] in the order of t's batch and steps.
Tensor like_sequences(const Tensor& t)
{
    if (t.stride(1) > t.stride(0)) return empty({t.size(1), t.size(0), t.size(2)}, t.scalar_type(), t).transpose(0, 1);
    return empty(t.sizes(), t.scalar_type(), t);
}

const pictura_sequences* c(const Sequences& q) { return reinterpret_cast<const pictura_sequences*>(&q); }

Tensor scan_workspace(const Sequences& q, const Tensor& like)
{
    uint64_t bytes = 0;
    check(entries.scan_workspace(c(q), &bytes), "gated_scan_workspace");
    return empty({(int64_t)bytes}, at::kByte, like);
}

variable_list scan(const Tensor& gates, const Tensor& inputs, const Tensor* state, const Tensor* resets, bool save)
{
    const Sequences q = sequences_of(true, gates, inputs, state, resets);
    on_device(gates, "gates");
    const c10::DeviceGuard guard(gates.device());
    const Tensor out = like_sequences(inputs), last = empty({q.batch, q.channels}, at::kFloat, gates);
    Tensor saved;
    if (save) saved = empty({(q.steps + PICTURA_SCAN_STEPS - 1) / PICTURA_SCAN_STEPS, q.batch, q.channels}, at::kFloat, gates);
    const Tensor ws = scan_workspace(q, gates);
    check(entries.scan(c(q), out.data_ptr(), out.stride(0), out.stride(1), data<float>(last), data<float>(saved), ws.data_ptr(),
                       (uint64_t)ws.numel(), stream_of(gates)),
          "gated_scan");
    return {out, last, saved};
}

struct GatedScan : torch::autograd::Function<GatedScan> {
    static variable_list forward(AutogradContext* ctx, const Tensor& gates, const Tensor& inputs, const Optional& state,
                                 const Optional& resets)
    {
        const variable_list r = scan(gates, inputs, or_null(state), or_null(resets), true);
        ctx->save_for_backward({gates, inputs, r[2], resets ? *resets : Tensor()});
        ctx->saved_data["state"] = state && state->requires_grad();
        ctx->set_materialize_grads(false);
        return {r[0], r[1]};
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        const variable_list held = ctx->get_saved_variables();
        const Tensor &gates = held[0], &inputs = held[1], &saved = held[2], &resets = held[3];
        variable_list out(4);
        check_seen("the gradient of gated_scan");
        check_tangents({{&grads[0], "the gradient of out"}, {&grads[1], "the gradient of the state"}});
        {
            const at::AutoGradMode off(false);
            const c10::DeviceGuard guard(gates.device());
            const Sequences q = sequences_of(true, gates, inputs, nullptr, or_null(resets));
            Tensor dout = grads[0], dlast = grads[1];
            if (!dout.defined()) dout = at::zeros({inputs.size(2)}, inputs.options().requires_grad(false)).expand(inputs.sizes());
            else if (dout.is_neg() || (dout.size(2) > 1 && dout.stride(2) != 1))
                dout = dout.resolve_neg().clone(at::MemoryFormat::Contiguous);
            if (dlast.defined()) dlast = dlast.resolve_neg().contiguous();
            const Place dy = place(dout, "the gradient of out", gates, true);
            const uint64_t dl = dlast.defined() ? floats(q, gates, dlast, "the gradient of the state", false) : 0;
            out[0] = like_sequences(gates);
            out[1] = like_sequences(inputs);
            if (ctx->saved_data["state"].toBool()) out[2] = empty({q.batch, q.channels}, at::kFloat, gates);
            const Tensor ws = scan_workspace(q, gates);
            check(entries.scan_gradient(c(q), data<float>(saved), (const void*)dy.at, dy.batch, dy.step, (const float*)dl,
                                        out[0].data_ptr(), out[0].stride(0), out[0].stride(1), out[1].data_ptr(),
                                        out[1].stride(0), out[1].stride(1), data<float>(out[2]), ws.data_ptr(),
                                        (uint64_t)ws.numel(), stream_of(gates)),
                  "gated_scan_gradient");
        }
        return once({gates, inputs, saved, grads[0], grads[1]}, std::move(out));
    }
};

// gated_scan(gates, inputs, state, resets) -> (out, last state)
PyObject* gated_scan(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded("gated_scan", [&]() -> PyObject* {
        arguments(n, 4, "gated_scan");
        const Tensor &gates = given(args[0], "gates"), &inputs = given(args[1], "inputs");
        const Tensor *state = optional(args[2], "state"), *resets = optional(args[3], "resets");
        check_tangents({{&gates, "gates"}, {&inputs, "inputs"}, {state, "state"}});
        if (wants_gradient({&gates, &inputs, state})) {
            check_capture({{&gates, "gates"}, {&inputs, "inputs"}, {state, "state"}});
            return tuple(GatedScan::apply(gates, inputs, or_none(state), or_none(resets)));
        }
        variable_list r = scan(gates, inputs, state, resets, false);
        r.pop_back();
        return tuple(r);
    });
}

// gated_step(gates, inputs, state, resets, out) -> out
PyObject* gated_step(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded("gated_step", [&]() -> PyObject* {
        arguments(n, 5, "gated_step");
        const Tensor &gates = given(args[0], "gates"), &inputs = given(args[1], "inputs"), &state = given(args[2], "state");
        const Sequences q = sequences_of(false, gates, inputs, &state, optional(args[3], "resets"));
        const Tensor* given_out = optional(args[4], "out");
        if (wants_gradient({&gates, &inputs, &state, given_out}))
            refuse("gated_step hands on no gradient: call it under torch.no_grad(), or gated_scan");
        check_tangents({{&gates, "gates"}, {&inputs, "inputs"}, {&state, "state"}, {given_out, "out"}});
        const Place o = given_out ? place(*given_out, "out", gates, false) : Place{};
        if (given_out && !apart(q, o)) refuse("out: strides ", given_out->strides(), ": elements overlap");
        check_step(q, (int64_t)gates.element_size(), o, q.state);
        on_device(gates, "gates");
        const c10::DeviceGuard guard(gates.device());
        const Tensor out = given_out ? *given_out : empty(inputs.sizes(), inputs.scalar_type(), inputs);
        check(entries.step(c(q), out.data_ptr(), out.stride(0), data<float>(state), stream_of(gates)), "gated_step");
        for (const Tensor* t : {&state, given_out})   // (a backward through a graph that saved them is refused)
            if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
        return THPVariable_Wrap(out);
    });
}

// ---- the norm -------------------------------------------------------------------------

const pictura_norm* c(const Norm& q) { return reinterpret_cast<const pictura_norm*>(&q); }

// t [..., width] as rows (a copy where its strides allow no view of them).
Tensor rows_of(const Tensor& t, const char* name)
{
    if (t.dim() < 1) refuse(name, ": expected a torch tensor [..., width], got one without dimensions");
    if (t.layout() != at::kStrided || t.size(-1) < 1)
        refuse(name, ": shape ", t.sizes(), ": expected rows of 1 to ", PICTURA_MAX_NORM, " elements");
    if (t.dim() == 2 && (t.stride(1) == 1 || t.size(1) == 1)) return t;
    const Tensor r = t.reshape({t.numel() / t.size(-1), t.size(-1)});
    return r.stride(1) == 1 || r.size(1) == 1 ? r : r.clone(at::MemoryFormat::Contiguous);
}

Tensor residual_rows(const Tensor* residual, const Tensor& x)
{
    if (!residual) return {};
    if (residual->sizes() != x.sizes()) refuse("residual: shape ", residual->sizes(), ", x has ", x.sizes());
    return rows_of(*residual, "residual");
}

// (out, x + residual, factors), the latter two where they are wanted
variable_list normed(const Tensor& x, const Tensor& weight, const Tensor* residual, double eps, bool save)
{
    const Tensor r = rows_of(x, "x"), res = residual_rows(residual, x);
    const Norm q = norm_of(r, weight, or_null(res), eps);
    on_device(x, "x");
    const c10::DeviceGuard guard(x.device());
    const Tensor out = empty(x.sizes(), x.scalar_type(), x);
    Tensor total, factors;
    if (residual) total = empty(x.sizes(), x.scalar_type(), x);
    if (save) factors = empty({q.rows}, at::kFloat, x);
    check(entries.norm(c(q), data<void>(total), q.width, out.data_ptr(), q.width, data<float>(factors), stream_of(x)), "rms_norm");
    return {out, total, factors};
}

struct RMSNorm : torch::autograd::Function<RMSNorm> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& weight, const Optional& residual, double eps)
    {
        const variable_list r = normed(x, weight, or_null(residual), eps, true);
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({weight, r[2], residual ? r[1] : x});
        if (!residual) return {r[0]};
        return {r[0], r[1]};
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        const variable_list held = ctx->get_saved_variables();
        const Tensor &weight = held[0], &factors = held[1], &total = held[2];
        const Tensor dsum = grads.size() > 1 ? grads[1] : Tensor();
        variable_list out(4);
        if (!grads[0].defined()) {
            out[0] = out[2] = dsum;   // (both undefined without a residual; linear, so nothing is lost)
            return out;
        }
        check_seen("the gradient of rms_norm");
        check_tangents({{&grads[0], "the gradient of y"}, {&dsum, "the gradient of the sum"}});
        {
            const at::AutoGradMode off(false);
            const c10::DeviceGuard guard(total.device());
            const Tensor s = rows_of(total, "x"), dy = rows_of(grads[0].resolve_neg(), "the gradient of y");
            const Tensor ds = dsum.defined() ? rows_of(dsum.resolve_neg(), "the gradient of the sum") : Tensor();
            const Norm q = norm_of(s, weight, nullptr, 0.0);
            std::pair<uint64_t, int64_t> dya = rows_at(dy, "the gradient of y", s, false), dsa{0, 0};
            same_type(dy, "the gradient of y", s);
            if (ds.defined()) {
                same_type(ds, "the gradient of the sum", s);
                dsa = rows_at(ds, "the gradient of the sum", s, false);
            }
            const Tensor dx = empty(total.sizes(), total.scalar_type(), total), dw = empty(weight.sizes(), weight.scalar_type(), weight);
            uint64_t bytes = 0;
            check(entries.norm_workspace(c(q), &bytes), "rms_norm_gradient_workspace");
            const Tensor ws = empty({(int64_t)bytes}, at::kByte, total);
            check(entries.norm_gradient(c(q), data<float>(factors), (const void*)dya.first, dya.second, (const void*)dsa.first,
                                        dsa.second, dx.data_ptr(), q.width, dw.data_ptr(), ws.data_ptr(), bytes, stream_of(total)),
                  "rms_norm_gradient");
            out[0] = dx;
            out[1] = dw;
        }
        out = once({total, weight, grads[0], dsum}, std::move(out));
        if (grads.size() > 1) out[2] = out[0];   // (there is a residual)
        return out;
    }
};

// rms_norm(x, weight, residual, eps) -> y, or (y, x + residual)
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded("rms_norm", [&]() -> PyObject* {
        arguments(n, 4, "rms_norm");
        const Tensor &x = given(args[0], "x"), &weight = given(args[1], "weight");
        const Tensor* residual = optional(args[2], "residual");
        const double eps = number(args[3], "eps");
        check_tangents({{&x, "x"}, {&weight, "weight"}, {residual, "residual"}});
        variable_list r;
        if (wants_gradient({&x, &weight, residual})) {
            check_capture({{&x, "x"}, {&weight, "weight"}, {residual, "residual"}});
            r = RMSNorm::apply(x, weight, or_none(residual), eps);
        } else {
            r = normed(x, weight, residual, eps, false);
            r.pop_back();
        }
        if (!residual) return THPVariable_Wrap(r[0]);
        return tuple(r);
    });
}

int32_t code_kind(const Tensor& t, const char* name)
{
    if (t.scalar_type() != at::kChar && t.scalar_type() != at::kFloat8_e4m3fn)
        refuse(name, ": dtype ", t.scalar_type(), ", expected int8 or float8_e4m3fn");
    return t.scalar_type() == at::kChar ? PICTURA_INT8 : PICTURA_E4M3;
}

// rms_norm_8bit(x, weight, residual, eps, whether e4m3) -> (codes, scales, x + residual or None)
PyObject* rms_norm_8bit(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded("rms_norm_8bit", [&]() -> PyObject* {
        arguments(n, 5, "rms_norm_8bit");
        const Tensor &x = given(args[0], "x"), &weight = given(args[1], "weight");
        const Tensor* residual = optional(args[2], "residual");
        check_tangents({{&x, "x"}, {&weight, "weight"}, {residual, "residual"}});
        const bool wanted = wants_gradient({&x, &weight, residual}), through = wants_gradient({&x, residual});
        if (through) check_capture({{&x, "x"}, {residual, "residual"}});
        const at::AutoGradMode off(false);
        const Tensor r = rows_of(x, "x"), res = residual_rows(residual, x);
        const Norm q = norm_of(r, weight, or_null(res), number(args[3], "eps"));
        on_device(x, "x");
        const c10::DeviceGuard guard(x.device());
        const bool e4m3 = args[4] == Py_True;
        const Tensor codes = empty(x.sizes(), e4m3 ? at::kFloat8_e4m3fn : at::kChar, x);
        const Tensor scales = empty(x.sizes().slice(0, (size_t)x.dim() - 1), at::kFloat, x);
        Tensor total;
        if (residual) total = empty(x.sizes(), x.scalar_type(), x);
        check(entries.norm_codes(c(q), e4m3 ? PICTURA_E4M3 : PICTURA_INT8, data<void>(total), q.width, codes.data_ptr(), q.width,
                                 data<float>(scales), stream_of(x)),
              "rms_norm_codes");
        if (wanted)
            refuse_gradient("rms_norm_8bit: its codes and scales have no gradient: detach them, or call rms_norm",
                            {x, weight, residual ? *residual : Tensor()}, {codes, scales});
        if (residual && through) {   // (the stream that goes on)
            const auto node = std::make_shared<SumOfTwo>();
            node->set_next_edges(torch::autograd::collect_next_edges(x, *residual));
            torch::autograd::set_history(total, node);
        }
        return tuple({codes, scales, total});
    });
}

// row_values(codes, scales, out or None) -> out
PyObject* row_values(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded("row_values", [&]() -> PyObject* {
        arguments(n, 3, "row_values");
        const Tensor &codes = given(args[0], "codes"), &scales = given(args[1], "scales");
        const Tensor* given_out = optional(args[2], "out");
        check_tangents({{&codes, "codes"}, {&scales, "scales"}, {given_out, "out"}});
        const bool wanted = wants_gradient({&codes, &scales, given_out});
        if (wanted && given_out) refuse("out: hands on no gradient, and one is wanted: detach the codes and scales");
        const at::AutoGradMode off(false);
        const int32_t kind = code_kind(codes, "codes");
        const Tensor r = rows_of(codes, "codes");
        if (r.size(1) > PICTURA_MAX_NORM || r.size(0) > 0x7FFFFFFF)
            refuse("codes: shape ", codes.sizes(), ": rows of 1 to ", PICTURA_MAX_NORM, " elements, fewer than 2^31 of them");
        const auto [at, stride] = rows_at(r, "codes", r, false);
        strided(scales, "scales", codes.device());
        if (scales.scalar_type() != at::kFloat || scales.sizes() != codes.sizes().slice(0, (size_t)codes.dim() - 1) ||
            !scales.is_contiguous())
            refuse("scales: ", scales.scalar_type(), " ", scales.sizes(), ", expected contiguous float32, one for each row of ",
                   codes.sizes());
        if (given_out) {
            strided(*given_out, "out", codes.device());
            if (given_out->scalar_type() != at::kFloat) refuse("out: dtype ", given_out->scalar_type(), ", expected float32");
            if (given_out->sizes() != codes.sizes() || !given_out->is_contiguous())
                refuse("out: expected a contiguous tensor of shape ", codes.sizes());
            using namespace pictura;
            const Region y = region(given_out->data_ptr(), r.size(0), r.size(1) * 4, r.size(1) * 4);
            if (overlap(y, region((const void*)at, r.size(0), r.size(1), stride))) refuse("out: overlaps the codes");
            if (overlap(y, region(scales.data_ptr(), r.size(0), 4, 4))) refuse("out: overlaps the scales");
        }
        on_device(codes, "codes");
        const c10::DeviceGuard guard(codes.device());
        const Tensor out = given_out ? *given_out : empty(codes.sizes(), at::kFloat, codes);
        check(entries.row_values((const void*)at, stride, data<float>(scales), kind, r.size(0), (int32_t)r.size(1), data<float>(out),
                                 r.size(1), stream_of(codes)),
              "row_values");
        if (wanted) refuse_gradient("the values of 8-bit codes have no gradient: detach the codes and scales", {codes, scales}, {out});
        if (given_out && !out.is_inference()) out.unsafeGetTensorImpl()->bump_version();
        return THPVariable_Wrap(out);
    });
}

// ---- the preference loss --------------------------------------------------------------

struct Preferences {
    Tensor actions, offsets, ref, weights, mask;
    double beta, smoothing, denominator;
    bool average;
};

// [rows, columns] with contiguous rows that do not overlap -> elements between them
int64_t matrix(const Tensor& t, const char* name)
{
    if (t.is_neg()) refuse(name, ": a lazily negated tensor");
    if (t.layout() != at::kStrided || (t.size(1) > 1 && t.stride(1) != 1) || (t.size(0) > 1 && t.stride(0) < t.size(1)))
        refuse(name, ": strides ", t.strides(), ": a row has to be contiguous, and apart from the next");
    return t.size(0) > 1 ? t.stride(0) : t.size(1);
}

void* vector(const Tensor& t, const char* name, at::ScalarType type, int64_t count, const Tensor& like)
{
    if (!t.defined()) return nullptr;
    if (t.device() != like.device()) refuse(name, ": tensor on ", t.device(), ", the logits are on ", like.device());
    if (t.scalar_type() != type) refuse(name, ": dtype ", t.scalar_type(), ", expected ", type);
    if (t.dim() != 1 || t.size(0) != count) refuse(name, ": shape ", t.sizes(), ", expected [", count, "]");
    if (t.layout() != at::kStrided || !t.is_contiguous() || t.is_neg()) refuse(name, ": tensor is not contiguous");
    return t.data_ptr();
}

// (stats, dlogits, ratios)
variable_list preferred(const Tensor& logits, const Preferences& p)
{
    pictura_logits l{};
    l.dtype = dtype_code(logits, "logits");
    if (logits.dim() != 2 || logits.size(1) < 1 || logits.size(1) > PICTURA_MAX_ACTIONS || logits.size(0) > 0x7FFFFFFF)
        refuse("logits: shape ", logits.sizes(), ", expected [rows, actions]: 1 to ", PICTURA_MAX_ACTIONS,
               " actions, fewer than 2^31 rows");
    l.stride = matrix(logits, "logits");
    l.rows = logits.size(0);
    l.actions = (int32_t)logits.size(1);
    l.data = logits.data_ptr();
    if (p.mask.defined()) {
        const Tensor& m = p.mask;
        if (m.device() != logits.device()) refuse("mask: tensor on ", m.device(), ", the logits are on ", logits.device());
        if (m.scalar_type() != at::kBool && m.scalar_type() != at::kByte) refuse("mask: dtype ", m.scalar_type(), ", expected bool or uint8");
        const bool one = m.dim() == 1 || (m.dim() == 2 && (m.size(0) == 1 || m.stride(0) == 0));
        if ((m.dim() != 1 && m.dim() != 2) || m.size(-1) != l.actions || (m.dim() == 2 && m.size(0) != 1 && m.size(0) != l.rows))
            refuse("mask: shape ", m.sizes(), ", expected [", l.rows, ", ", l.actions, "] or one row for all");
        if (one) {
            if (m.layout() != at::kStrided || (l.actions > 1 && m.stride(-1) != 1)) refuse("mask: strides ", m.strides(), ", expected contiguous rows");
        } else {
            l.mask_stride = matrix(m, "mask");
        }
        l.mask = static_cast<const uint8_t*>(m.data_ptr());
    }
    const Tensor& o = p.offsets;
    if (o.dim() != 1 || o.size(0) % 2 == 0) refuse("offsets: shape ", o.sizes(), ", expected [2 pairs + 1]");
    pictura_preferences q{};
    q.pairs = o.size(0) / 2;
    q.actions = (const int64_t*)vector(p.actions, "actions", at::kLong, l.rows, logits);
    q.offsets = (const int64_t*)vector(o, "offsets", at::kLong, 2 * q.pairs + 1, logits);
    q.ref_logp = (const float*)vector(p.ref, "ref_logp", at::kFloat, l.rows, logits);
    q.weights = (const float*)vector(p.weights, "weights", at::kFloat, q.pairs, logits);
    if (!(p.beta > 0 && p.beta < 3e38) || (float)p.beta == 0.0f) refuse("beta: ", p.beta, ", expected a number within range");
    if (!(p.smoothing >= 0 && (float)p.smoothing < 1.0f)) refuse("smoothing: ", p.smoothing, ", expected a number within range");
    if (!(p.denominator >= 0 && p.denominator < 3e38) || (p.denominator > 0 && (float)p.denominator == 0.0f)) refuse("denominator: ", p.denominator, ", expected a number within range");
    q.beta = (float)p.beta;
    q.smoothing = (float)p.smoothing;
    q.denominator = (float)p.denominator;
    q.average = p.average;
    uint64_t bytes = 0;
    if (entries.preference_workspace(l.rows, l.actions, q.pairs, &bytes) != PICTURA_OK)
        refuse("offsets: ", q.pairs, " pairs, expected 2^23 at most");
    on_device(logits, "logits");
    const c10::DeviceGuard guard(logits.device());
    const Tensor stats = empty({PICTURA_PREFERENCE_STATS}, at::kFloat, logits), ratios = empty({2 * q.pairs}, at::kFloat, logits);
    const Tensor dlogits = empty(logits.sizes(), logits.scalar_type(), logits), ws = empty({(int64_t)bytes}, at::kByte, logits);
    check(entries.preference_loss(&l, &q, ws.data_ptr(), bytes, data<float>(stats), data<float>(ratios), dlogits.data_ptr(), l.actions,
                                  stream_of(logits)),
          "preference_loss");
    return {stats, dlogits, ratios};
}

struct PreferenceLoss : torch::autograd::Function<PreferenceLoss> {
    static variable_list forward(AutogradContext* ctx, const Tensor& logits, const Preferences& p)
    {
        // (float16's range is too short for a gradient that a loss scale has yet to lift)
        const bool half = logits.scalar_type() == at::kHalf;
        const variable_list r = preferred(half ? logits.to(at::kFloat) : logits, p);
        ctx->save_for_backward({r[1]});
        ctx->saved_data["half"] = half;
        const Tensor loss = r[0].select(0, 0).clone();
        ctx->mark_non_differentiable({r[0], r[2]});
        ctx->set_materialize_grads(false);
        return {loss, r[0], r[2]};
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        variable_list out(2);
        if (grads[0].defined()) {
            const at::AutoGradMode off(false);
            const Tensor dlogits = ctx->get_saved_variables()[0];
            const bool half = ctx->saved_data["half"].toBool();
            if (dlogits.scalar_type() == at::kFloat) {
                out[0] = dlogits.mul(grads[0]);
                if (half) out[0] = out[0].to(at::kHalf);
            } else {   // (the product in fp32: a loss scale may be beyond what the type holds.  bfloat16 is rounded
                       // before it too, half a step more: its range loses nothing, and fp32 takes twice the memory)
                out[0] = at::empty_like(dlogits);
                at::mul_out(out[0], dlogits.to(at::kFloat), grads[0]);
            }
        }
        return once({grads[0]}, std::move(out));   // (the logits are not kept for this)
    }
};

bool truth(PyObject* o, const char* name)
{
    const int is = PyObject_IsTrue(o);
    if (is < 0) {
        PyErr_Clear();
        refuse(name, ": ", Py_TYPE(o)->tp_name, ", expected a bool");
    }
    return is == 1;
}

Preferences preferences(PyObject* const* args)
{
    auto or_undefined = [](const Tensor* t) { return t ? *t : Tensor(); };
    return Preferences{given(args[1], "actions"), given(args[2], "offsets"), or_undefined(optional(args[3], "ref_logp")),
                       or_undefined(optional(args[4], "weights")), or_undefined(optional(args[5], "mask")),
                       number(args[6], "beta"), number(args[7], "smoothing"), number(args[9], "denominator"),
                       truth(args[8], "average")};
}

// preference_gradient(logits, actions, offsets, ref_logp, weights, mask, beta, smoothing,
// average, denominator) -> (stats, dlogits, ratios)
PyObject* preference_gradient(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded("preference_gradient", [&]() -> PyObject* {
        arguments(n, 10, "preference_gradient");
        const at::AutoGradMode off(false);
        const Tensor& logits = given(args[0], "logits");
        const Preferences p = preferences(args);
        check_tangents({{&logits, "logits"}, {or_null(p.ref), "ref_logp"}, {or_null(p.weights), "weights"}});
        return tuple(preferred(logits, p));
    });
}

// preference_loss(the same) -> (loss, stats, ratios)
PyObject* preference_loss(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded("preference_loss", [&]() -> PyObject* {
        arguments(n, 10, "preference_loss");
        const Tensor& logits = given(args[0], "logits");
        const Preferences p = preferences(args);
        check_tangents({{&logits, "logits"}, {or_null(p.ref), "ref_logp"}, {or_null(p.weights), "weights"}});
        if (wants_gradient({or_null(p.ref)})) refuse("ref_logp: wants a gradient, and there is no gradient of it: detach it");
        if (wants_gradient({or_null(p.weights)})) refuse("weights: want a gradient, and there is no gradient of them: detach them");
        if (wants_gradient({&logits})) check_capture({{&logits, "logits"}});
        return tuple(PreferenceLoss::apply(logits, p));
    });
}

}  // namespace

#define CALL(name, text) {#name, (PyCFunction)(void (*)())name, METH_FASTCALL, text}

PyMethodDef pictura_calls[] = {CALL(bind, "The library's entries."),
                               CALL(gated_scan, "Gated recurrence over sequences."),
                               CALL(gated_step, "One step of it in place."),
                               CALL(rms_norm, "Root-mean-square norm of rows."),
                               CALL(rms_norm_8bit, "The same with an output in 8 bits."),
                               CALL(row_values, "What 8-bit rows stand for."),
                               CALL(preference_gradient, "Preference loss and its gradient."),
                               CALL(preference_loss, "Preference loss for autograd."),
                               {nullptr, nullptr, 0, nullptr}};
