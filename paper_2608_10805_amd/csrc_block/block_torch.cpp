// Native host path of the layer norm, the scaled residual and AdamW: the same
// checks, allocations and library calls as paper_2608_10805_amd.binding,
// .autograd and .optim make, without the Python interpreter (a step of 600
// tensors took 2.1 ms of host time there).
//
// Every function takes the plain case alone (dense GPU tensors that fit the
// problem, nothing tracing, transforming or overriding torch functions) and
// answers None or False to any other; the caller then goes through Python,
// which converts, raises or traces. The library's entry points come in as
// addresses (init), so this module links to torch only.
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/extension.h>

#include "wtconv.h"

namespace {

using at::Tensor;
using torch::autograd::Node;
using torch::autograd::SavedVariable;
using torch::autograd::variable_list;
using OptTensor = std::optional<Tensor>;

decltype(&wtconv_layer_norm_forward) norm_forward = nullptr;
decltype(&wtconv_layer_norm_backward_workspace_bytes) norm_bytes = nullptr;
decltype(&wtconv_layer_norm_backward) norm_backward = nullptr;
decltype(&wtconv_scaled_residual_forward) residual_forward = nullptr;
decltype(&wtconv_scaled_residual_backward_workspace_bytes) residual_bytes = nullptr;
decltype(&wtconv_scaled_residual_backward) residual_backward = nullptr;
decltype(&wtconv_adamw_step) adamw_fn = nullptr;
decltype(&wtconv_adamw_moments) moments_fn = nullptr;
PyObject* python_norm = nullptr;      // autograd._norm_backward
PyObject* python_residual = nullptr;  // autograd._residual_backward
PyTypeObject* parameter_type = nullptr;

struct Refused {
};  // the library refused the call

// A strided GPU tensor without wrappers (functorch, subclasses with a dispatch
// of their own) and without a forward-mode tangent.
bool plain(const Tensor& t, c10::Device dev, bool tangents = true)
{
    static const c10::DispatchKeySet wrapped(
        {c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::FuncTorchBatched,
         c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize, c10::DispatchKey::Conjugate,
         c10::DispatchKey::Negative, c10::DispatchKey::ZeroTensor});
    return t.defined() && t.is_cuda() && t.device() == dev && t.layout() == at::kStrided &&
           !t.key_set().has_any(wrapped) && !(tangents && t._fw_grad(0).defined());
}

bool vector_of(const OptTensor& t, c10::Device dev, int64_t n)
{
    return !t || (plain(*t, dev) && t->is_contiguous() && t->scalar_type() == at::kFloat && t->dim() == 1 &&
                  t->size(0) == n);
}

bool modes_active()
{
    const auto tls = c10::impl::tls_local_dispatch_key_set().included_;
    return at::impl::torch_function_mode_enabled() || torch::jit::tracer::isTracing() ||
           c10::impl::TorchDispatchModeTLS::any_modes_set() ||
           tls.has(c10::DispatchKey::FuncTorchDynamicLayerFrontMode) || tls.has(c10::DispatchKey::Functionalize);
}

// A torch.Tensor or torch.nn.Parameter itself: other subclasses may override
// torch functions without a dispatch key that shows it.
bool exact_tensor(py::handle t)
{
    return Py_TYPE(t.ptr()) == reinterpret_cast<PyTypeObject*>(THPVariableClass) || Py_TYPE(t.ptr()) == parameter_type;
}

// The argument as a tensor, or nothing for None; false for anything else.
bool optional_tensor(py::handle t, OptTensor& out)
{
    if (t.is_none()) return true;
    if (!exact_tensor(t)) return false;
    out = THPVariable_Unpack(t.ptr());
    return true;
}

bool type_of(const Tensor& t, wtconv_dtype& d)
{
    switch (t.scalar_type()) {
        case at::kFloat: d = WTCONV_F32; return true;
        case at::kBFloat16: d = WTCONV_BF16; return true;
        case at::kHalf: d = WTCONV_F16; return true;
        default: return false;
    }
}

// Elements from one row (the last dimension) to the next; 0 where the rows do
// not lie at one distance from each other.
int64_t row_stride(const Tensor& t)
{
    const auto sizes = t.sizes(), strides = t.strides();
    const int64_t d = t.dim(), C = sizes[d - 1];
    if (C > 1 && strides[d - 1] != 1) return 0;
    int64_t stride = 0, rows = 0;
    for (int64_t i = d - 2; i >= 0; --i) {
        if (sizes[i] == 1) continue;
        if (!rows) {
            stride = strides[i];
            rows = sizes[i];
        } else if (strides[i] != stride * rows) {
            return 0;
        } else {
            rows *= sizes[i];
        }
    }
    if (!rows) return C;
    return stride >= C ? stride : 0;
}

const float* ptr(const OptTensor& t) { return t ? t->const_data_ptr<float>() : nullptr; }

hipStream_t stream_of(const Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()); }

Tensor floats(at::IntArrayRef sizes, const Tensor& like) { return at::empty(sizes, like.options().dtype(at::kFloat)); }

Tensor bytes(size_t n, const Tensor& like) { return at::empty({(int64_t)n}, like.options().dtype(at::kByte)); }

variable_list from_python(PyObject* fn, py::tuple args)
{
    try {
        const py::object r = py::reinterpret_borrow<py::object>(fn)(*args);
        variable_list out;
        for (const py::handle& t : py::reinterpret_borrow<py::tuple>(r))
            out.push_back(t.is_none() ? Tensor() : t.cast<Tensor>());
        return out;
    } catch (py::error_already_set& e) {  // as the autograd engine hands Python errors on
        e.restore();
        python_error err;
        err.persist();
        throw python_error(std::move(err));
    }
}

// Whether a backward has to go through Python: its gradients will be
// differentiated, which is refused there. They depend on dy and on every saved
// tensor that trains.
bool twice(const Tensor& dy, const OptTensor& a, const OptTensor& b)
{
    return at::GradMode::is_enabled() && (dy.requires_grad() || (a && a->requires_grad()) || (b && b->requires_grad()));
}

// ----------------------------------------------------------------------------
// layer norm
// ----------------------------------------------------------------------------

struct NormArguments {
    double eps;
    int64_t in, out;  // the channels' dimension of x and of y, 1 or -1
};

bool describe(const Tensor& x, const NormArguments& a, wtconv_norm_desc& d)
{
    if (!x.defined() || !x.is_cuda() || x.dim() < 2 || !plain(x, x.device()) || x.numel() == 0 || !type_of(x, d.dtype))
        return false;
    if (!(a.in == 1 && (a.out == 1 || a.out == -1)) && !(a.in == -1 && a.out == -1)) return false;
    const int64_t C = x.size(a.in == 1 ? 1 : x.dim() - 1);
    if (C > WTCONV_MAX_CHANNELS) return false;
    d.in = a.in == 1 ? WTCONV_PLANES : WTCONV_ROWS;
    d.out = a.out == 1 ? WTCONV_PLANES : WTCONV_ROWS;
    d.B = x.size(0);
    d.C = (int)C;
    d.S = x.numel() / (d.B * C);
    d.x_stride = d.dy_stride = 0;
    d.eps = a.eps;
    if (a.in == 1) return x.is_contiguous();
    d.x_stride = row_stride(x);
    return d.x_stride != 0;
}

std::vector<int64_t> out_sizes(const Tensor& x, const NormArguments& a)
{
    std::vector<int64_t> s = x.sizes().vec();
    if (a.in != a.out) {
        s.push_back(s[1]);
        s.erase(s.begin() + 1);
    }
    return s;
}

Tensor norm(const Tensor& x, const OptTensor& w, const OptTensor& b, const NormArguments& a, Tensor* stats)
{
    wtconv_norm_desc d;
    TORCH_CHECK(describe(x, a, d), "layer_norm: the arguments changed");
    const c10::DeviceGuard guard(x.device());
    Tensor y = at::empty(out_sizes(x, a), x.options());
    float *mean = nullptr, *rstd = nullptr;
    if (stats) {
        *stats = floats({2, d.B * d.S}, x);
        mean = stats->mutable_data_ptr<float>();
        rstd = mean + d.B * d.S;
    }
    if (norm_forward(&d, x.const_data_ptr(), ptr(w), ptr(b), y.mutable_data_ptr(), mean, rstd, stream_of(x)) !=
        WTCONV_OK)
        throw Refused();
    return y;
}

// The saved tensors' and edges' own class rather than torch::autograd::Function:
// no list of arguments is taken apart and nothing is kept by name.
struct NormNode : public Node {
    SavedVariable x_, stats_, w_;
    NormArguments args;
    bool has_w = false, released = false;

    std::string name() const override { return "WTConvLayerNorm"; }
    void release_variables() override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        x_.reset_data();
        stats_.reset_data();
        w_.reset_data();
        released = true;
    }

    variable_list apply(variable_list&& grads) override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        TORCH_CHECK(!released, torch::autograd::ERR_BACKWARD_TWICE);
        variable_list out(3);
        Tensor dy = grads[0];
        if (!dy.defined()) return out;
        const Tensor x = x_.unpack(), stats = stats_.unpack();
        OptTensor w;
        if (has_w) w = w_.unpack();
        const bool need_dx = task_should_compute_output(0), need_dw = task_should_compute_output(1),
                   need_db = task_should_compute_output(2);
        wtconv_norm_desc d;
        const bool ok = !twice(dy, x, w) && describe(x, args, d) && plain(stats, x.device()) && stats.is_contiguous() &&
                        stats.scalar_type() == at::kFloat && stats.numel() == 2 * d.B * d.S &&
                        vector_of(w, x.device(), d.C) && plain(dy, x.device()) &&
                        dy.scalar_type() == x.scalar_type() && dy.sizes() == at::IntArrayRef(out_sizes(x, args));
        if (ok) {
            const c10::DeviceGuard guard(x.device());
            if (args.out == 1) {
                dy = dy.contiguous();
            } else if (!(d.dy_stride = row_stride(dy))) {
                dy = dy.contiguous();
                d.dy_stride = 0;
            }
            if (need_dx) out[0] = at::empty(x.sizes(), x.options());
            if (need_dw) out[1] = floats({d.C}, x);
            if (need_db) out[2] = floats({d.C}, x);
            const size_t n = need_dw || need_db ? norm_bytes(&d) : 0;
            const Tensor ws = n ? bytes(n, x) : Tensor();
            const float* mean = stats.const_data_ptr<float>();
            if (norm_backward(&d, dy.const_data_ptr(), x.const_data_ptr(), mean, mean + d.B * d.S, ptr(w),
                              need_dx ? out[0].mutable_data_ptr() : nullptr,
                              need_dw ? out[1].mutable_data_ptr<float>() : nullptr,
                              need_db ? out[2].mutable_data_ptr<float>() : nullptr,
                              n ? ws.mutable_data_ptr() : nullptr, n, stream_of(x)) == WTCONV_OK)
                return out;
        }
        py::gil_scoped_acquire gil;
        return from_python(python_norm,
                           py::make_tuple(py::make_tuple(args.eps, args.in, args.out, need_dx, need_dw, need_db),
                                          grads[0], x, stats.select(0, 0), stats.select(0, 1), w));
    }
};

Tensor norm_with_grad(const Tensor& x, const OptTensor& w, const OptTensor& b, const NormArguments& a)
{
    Tensor stats;
    Tensor y = norm(x, w, b, a, &stats);
    std::shared_ptr<NormNode> node(new NormNode(), torch::autograd::deleteNode);
    node->set_next_edges(torch::autograd::collect_next_edges(x, w ? *w : Tensor(), b ? *b : Tensor()));
    node->x_ = SavedVariable(x, false);
    node->stats_ = SavedVariable(stats, false);
    if (w) node->w_ = SavedVariable(*w, false);
    node->has_w = (bool)w;
    node->args = a;
    torch::autograd::set_history(y, node);
    return y;
}

py::object layer_norm(py::handle x, py::handle weight, py::handle bias, py::handle eps, py::handle in, py::handle out)
{
    if (!norm_forward || modes_active() || !exact_tensor(x)) return py::none();
    OptTensor w, b;
    if (!optional_tensor(weight, w) || !optional_tensor(bias, b)) return py::none();
    if (!PyFloat_CheckExact(eps.ptr()) || !PyLong_CheckExact(in.ptr()) || !PyLong_CheckExact(out.ptr()))
        return py::none();
    const Tensor& xt = THPVariable_Unpack(x.ptr());
    const NormArguments a = {PyFloat_AS_DOUBLE(eps.ptr()), PyLong_AsLong(in.ptr()), PyLong_AsLong(out.ptr())};
    wtconv_norm_desc d;
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return py::none();
    }
    if (!describe(xt, a, d) || !vector_of(w, xt.device(), d.C) || !vector_of(b, xt.device(), d.C)) return py::none();
    const bool grad = at::GradMode::is_enabled() &&
                      (xt.requires_grad() || (w && w->requires_grad()) || (b && b->requires_grad()));
    Tensor y;
    try {
        py::gil_scoped_release no_gil;
        y = grad ? norm_with_grad(xt, w, b, a) : norm(xt, w, b, a, nullptr);
    } catch (const Refused&) {
        return py::none();  // the Python path raises the library's error
    }
    return py::cast(y);
}

// ----------------------------------------------------------------------------
// scaled residual
// ----------------------------------------------------------------------------

bool describe(const Tensor& x, wtconv_residual_desc& d)
{
    if (!x.defined() || !x.is_cuda() || x.dim() < 2 || !plain(x, x.device()) || !x.is_contiguous() ||
        x.numel() == 0 || !type_of(x, d.dtype) || x.size(1) > WTCONV_MAX_CHANNELS)
        return false;
    d.B = x.size(0);
    d.C = (int)x.size(1);
    d.S = x.numel() / (d.B * d.C);
    return true;
}

// [B, ..., C] for planes [B, C, ...]
std::vector<int64_t> rows_sizes(const Tensor& x)
{
    std::vector<int64_t> s = x.sizes().vec();
    s.push_back(s[1]);
    s.erase(s.begin() + 1);
    return s;
}

bool rows_of(const Tensor& z, const Tensor& x)
{
    return plain(z, x.device()) && z.is_contiguous() && z.scalar_type() == x.scalar_type() &&
           z.sizes() == at::IntArrayRef(rows_sizes(x));
}

Tensor residual(const Tensor& x, const Tensor& z, const OptTensor& gamma, const OptTensor& keep)
{
    wtconv_residual_desc d;
    TORCH_CHECK(describe(x, d), "scaled_residual: the arguments changed");
    const c10::DeviceGuard guard(x.device());
    Tensor y = at::empty(x.sizes(), x.options());
    if (residual_forward(&d, x.const_data_ptr(), z.const_data_ptr(), ptr(gamma), ptr(keep), y.mutable_data_ptr(),
                         stream_of(x)) != WTCONV_OK)
        throw Refused();
    return y;
}

struct ResidualNode : public Node {
    SavedVariable z_, gamma_, keep_;
    bool has_z = false, has_gamma = false, has_keep = false, released = false;

    std::string name() const override { return "WTConvScaledResidual"; }
    void release_variables() override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        z_.reset_data();
        gamma_.reset_data();
        keep_.reset_data();
        released = true;
    }

    variable_list apply(variable_list&& grads) override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        TORCH_CHECK(!released, torch::autograd::ERR_BACKWARD_TWICE);
        variable_list out(3);
        if (!grads[0].defined()) return out;
        OptTensor z, gamma, keep;
        if (has_z) z = z_.unpack();
        if (has_gamma) gamma = gamma_.unpack();
        if (has_keep) keep = keep_.unpack();
        const bool need_dx = task_should_compute_output(0), need_dz = task_should_compute_output(1),
                   need_dg = z && task_should_compute_output(2);
        const bool second = twice(grads[0], z, gamma);
        const Tensor dy = second ? grads[0] : grads[0].contiguous();
        wtconv_residual_desc d;
        if (!second && describe(dy, d) && vector_of(gamma, dy.device(), d.C) && vector_of(keep, dy.device(), d.B) &&
            (!need_dg || rows_of(*z, dy))) {
            const c10::DeviceGuard guard(dy.device());
            if (need_dx) out[0] = dy;
            if (need_dz) out[1] = at::empty(rows_sizes(dy), dy.options());
            if (need_dg) out[2] = floats({d.C}, dy);
            const size_t n = need_dg ? residual_bytes(&d) : 0;
            const Tensor ws = n ? bytes(n, dy) : Tensor();
            if (residual_backward(&d, dy.const_data_ptr(), need_dg ? z->const_data_ptr() : nullptr, ptr(gamma),
                                  ptr(keep), need_dz ? out[1].mutable_data_ptr() : nullptr,
                                  need_dg ? out[2].mutable_data_ptr<float>() : nullptr,
                                  n ? ws.mutable_data_ptr() : nullptr, n, stream_of(dy)) == WTCONV_OK)
                return out;
        }
        py::gil_scoped_acquire gil;
        return from_python(python_residual,
                           py::make_tuple(py::make_tuple(need_dx, need_dz, need_dg), grads[0], z, gamma, keep));
    }
};

Tensor residual_with_grad(const Tensor& x, const Tensor& z, const OptTensor& gamma, const OptTensor& keep)
{
    Tensor y = residual(x, z, gamma, keep);
    std::shared_ptr<ResidualNode> node(new ResidualNode(), torch::autograd::deleteNode);
    node->set_next_edges(torch::autograd::collect_next_edges(x, z, gamma ? *gamma : Tensor()));
    // z is needed for the gradient of gamma alone
    node->has_z = gamma && gamma->requires_grad();
    if (node->has_z) node->z_ = SavedVariable(z, false);
    node->has_gamma = (bool)gamma;
    if (gamma) node->gamma_ = SavedVariable(*gamma, false);
    node->has_keep = (bool)keep;
    if (keep) node->keep_ = SavedVariable(*keep, false);
    torch::autograd::set_history(y, node);
    return y;
}

py::object scaled_residual(py::handle x, py::handle z, py::handle gamma, py::handle keep)
{
    if (!residual_forward || modes_active() || !exact_tensor(x) || !exact_tensor(z)) return py::none();
    OptTensor g, k;
    if (!optional_tensor(gamma, g) || !optional_tensor(keep, k)) return py::none();
    const Tensor &xt = THPVariable_Unpack(x.ptr()), &zt = THPVariable_Unpack(z.ptr());
    wtconv_residual_desc d;
    if (!describe(xt, d) || !rows_of(zt, xt) || !vector_of(g, xt.device(), d.C) || !vector_of(k, xt.device(), d.B) ||
        (k && k->requires_grad()))
        return py::none();
    const bool grad = at::GradMode::is_enabled() &&
                      (xt.requires_grad() || zt.requires_grad() || (g && g->requires_grad()));
    Tensor y;
    try {
        py::gil_scoped_release no_gil;
        y = grad ? residual_with_grad(xt, zt, g, k) : residual(xt, zt, g, k);
    } catch (const Refused&) {
        return py::none();
    }
    return py::cast(y);
}

// ----------------------------------------------------------------------------
// AdamW
// ----------------------------------------------------------------------------

// What stays the same of a parameter group from step to step.
struct Group {
    std::vector<Tensor> params;
    std::vector<int64_t> offsets, numel;
    std::vector<std::vector<int64_t>> orders;  // of the parameters' memory, as optim._order() has them
    Tensor steps, m, v;                        // steps: int64 on the host
    OptTensor ms, vs;

    Group(std::vector<Tensor> params_, std::vector<int64_t> offsets_, std::vector<int64_t> numel_,
          std::vector<std::vector<int64_t>> orders_, Tensor steps_, Tensor m_, Tensor v_, OptTensor ms_, OptTensor vs_)
        : params(std::move(params_)), offsets(std::move(offsets_)), numel(std::move(numel_)),
          orders(std::move(orders_)), steps(std::move(steps_)), m(std::move(m_)), v(std::move(v_)),
          ms(std::move(ms_)), vs(std::move(vs_))
    {
    }

    // Whether parameter i still lies in memory as its moments do.
    bool in_order(size_t i, const Tensor& p) const
    {
        const std::vector<int64_t>& order = orders[i];
        if (order.empty()) return p.is_contiguous();
        if (order.size() != (size_t)p.dim() || p.is_contiguous()) return false;
        for (size_t d = 0; d < order.size(); ++d)
            if (order[d] != (p.size((int64_t)d) > 1 ? p.stride((int64_t)d) : 0)) return false;
        return true;
    }
};

uint32_t mix(uint32_t x)
{
    x = (x ^ (x >> 15)) * 0x85EBCA6Bu;
    x = (x ^ (x >> 13)) * 0xC2B2AE35u;
    return x ^ (x >> 16);
}

// optim.rounding_key()
uint32_t rounding_key(uint64_t seed, int64_t step, uint32_t group)
{
    return mix(group * 0x9E3779B1u + mix((uint32_t)seed * 0x9E3779B1u + (uint32_t)step * 0x9E3779B9u));
}

struct Call {
    std::vector<wtconv_adamw_group> groups;
    std::vector<wtconv_adamw_tensor> tensors;
};

// One step of every parameter that has a gradient. plans: null for a group of no
// parameters. hyper: (lr, beta1, beta2, eps, weight_decay) of each group. False,
// with nothing done, where one of them is not the plain case.
bool adamw_step(const std::vector<Group*>& plans, py::sequence params, const std::vector<std::array<double, 5>>& hyper,
                int bits, uint64_t seed, py::handle scale)
{
    if (!adamw_fn || modes_active() || plans.size() != hyper.size() || params.size() != plans.size()) return false;
    Call calls[3];  // by type
    std::vector<std::pair<int64_t*, const Tensor*>> taken;
    std::optional<c10::Device> dev;
    for (size_t gi = 0; gi < plans.size(); ++gi) {
        PyObject* list = params[gi].ptr();
        if (!plans[gi] && PyList_CheckExact(list) && PyList_GET_SIZE(list) == 0) continue;
        if (!plans[gi]) return false;
        const Group& q = *plans[gi];
        if (!PyList_CheckExact(list) || (size_t)PyList_GET_SIZE(list) != q.numel.size()) return false;
        int64_t* steps = q.steps.mutable_data_ptr<int64_t>();
        int64_t place_step[3] = {-1, -1, -1};  // the step of the call's last group, if it is of this parameter group
        for (size_t i = 0; i < q.numel.size(); ++i) {
            const py::handle h = PyList_GET_ITEM(list, i);
            if (!exact_tensor(h)) return false;
            const Tensor& p = THPVariable_Unpack(h.ptr());
            if (!p.is_same(q.params[i])) return false;
            const Tensor& g = p.grad();
            if (!g.defined()) continue;
            wtconv_dtype type;
            if (!plain(p, q.m.device(), false) || !plain(g, q.m.device(), false) || !type_of(p, type) ||
                g.scalar_type() != p.scalar_type() || p.numel() != q.numel[i] || g.sizes() != p.sizes() ||
                g.strides() != p.strides() || !q.in_order(i, p) || p.is_inference())
                return false;
            if (dev && *dev != p.device()) return false;
            dev = p.device();
            taken.emplace_back(steps + i, &p);
            if (!q.numel[i]) continue;  // (a group of nothing else has no buffers)
            Call& c = calls[type];
            const int64_t step = steps[i] + 1;
            if (place_step[type] != step) {
                place_step[type] = step;
                wtconv_adamw_group o;
                std::tie(o.lr, o.beta1, o.beta2, o.eps, o.weight_decay) =
                    std::make_tuple(hyper[gi][0], hyper[gi][1], hyper[gi][2], hyper[gi][3], hyper[gi][4]);
                o.step = step;
                o.key = rounding_key(seed, step, (uint32_t)gi);
                o.exp_avg = q.m.mutable_data_ptr();
                o.exp_avg_sq = q.v.mutable_data_ptr();
                o.exp_avg_scale = q.ms ? q.ms->mutable_data_ptr<uint8_t>() : nullptr;
                o.exp_avg_sq_scale = q.vs ? q.vs->mutable_data_ptr<uint8_t>() : nullptr;
                c.groups.push_back(o);
            }
            c.tensors.push_back({p.mutable_data_ptr(), g.const_data_ptr(), q.numel[i], q.offsets[i],
                                 (int)c.groups.size() - 1});
        }
    }
    if (!dev) return true;
    OptTensor s;
    if (!optional_tensor(scale, s)) return false;
    if (s && (!plain(*s, *dev) || s->scalar_type() != at::kFloat || s->numel() != 1)) return false;
    const c10::DeviceGuard guard(*dev);
    const hipStream_t stream = c10::hip::getCurrentHIPStream(dev->index());
    bool first = true;
    for (int type = 0; type < 3; ++type) {
        const Call& c = calls[type];
        if (c.tensors.empty()) continue;
        const wtconv_status st =
            adamw_fn((int)c.groups.size(), c.groups.data(), (int)c.tensors.size(), c.tensors.data(),
                     (wtconv_dtype)type, bits, ptr(s), stream);
        if (st != WTCONV_OK) {
            if (first) return false;  // refused before any launch: the Python path raises the library's error
            TORCH_CHECK(false, "wtconv_adamw_step: status ", (int)st);
        }
        first = false;
    }
    for (const auto& [step, p] : taken) {
        ++*step;
        p->unsafeGetTensorImpl()->bump_version();
    }
    return true;
}

// The values of a group's 8-bit moments, or None.
py::object adamw_moments(const Group& q, at::ScalarType type)
{
    wtconv_dtype d;
    if (!moments_fn || !q.ms || !q.vs || modes_active()) return py::none();
    const c10::DeviceGuard guard(q.m.device());
    const auto options = q.m.options().dtype(type);
    Tensor m = at::empty(q.m.sizes(), options), v = at::empty(q.m.sizes(), options);
    if (!type_of(m, d) ||
        moments_fn(q.m.numel(), q.m.const_data_ptr<uint8_t>(), q.ms->const_data_ptr<uint8_t>(),
                   q.v.const_data_ptr<uint8_t>(), q.vs->const_data_ptr<uint8_t>(), m.mutable_data_ptr(),
                   v.mutable_data_ptr(), d, stream_of(m)) != WTCONV_OK)
        return py::none();
    return py::make_tuple(m, v);
}

void init(const std::vector<uintptr_t>& fns, py::object norm_py, py::object residual_py)
{
    TORCH_CHECK(fns.size() == 8, "init takes the addresses of eight entry points");
    norm_forward = reinterpret_cast<decltype(norm_forward)>(fns[0]);
    norm_bytes = reinterpret_cast<decltype(norm_bytes)>(fns[1]);
    norm_backward = reinterpret_cast<decltype(norm_backward)>(fns[2]);
    residual_forward = reinterpret_cast<decltype(residual_forward)>(fns[3]);
    residual_bytes = reinterpret_cast<decltype(residual_bytes)>(fns[4]);
    residual_backward = reinterpret_cast<decltype(residual_backward)>(fns[5]);
    adamw_fn = reinterpret_cast<decltype(adamw_fn)>(fns[6]);
    moments_fn = reinterpret_cast<decltype(moments_fn)>(fns[7]);
    py::object parameter = py::module_::import("torch.nn").attr("Parameter");
    parameter_type = reinterpret_cast<PyTypeObject*>(parameter.release().ptr());
    Py_XDECREF(python_norm);
    Py_XDECREF(python_residual);
    python_norm = norm_py.release().ptr();  // for the life of the process
    python_residual = residual_py.release().ptr();
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m)
{
    py::class_<Group>(m, "AdamWGroup")
        .def(py::init<std::vector<Tensor>, std::vector<int64_t>, std::vector<int64_t>, std::vector<std::vector<int64_t>>,
                      Tensor, Tensor, Tensor, OptTensor, OptTensor>());
    m.def("init", &init);
    m.def("layer_norm", &layer_norm);
    m.def("scaled_residual", &scaled_residual);
    m.def("adamw_step", &adamw_step);
    m.def("adamw_moments", &adamw_moments);
}
