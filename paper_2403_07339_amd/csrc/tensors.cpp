// The argument marshalling of the calls whose host time counts, in C++: a norm of a few rows takes the GPU five microseconds, an optimiser's
// step takes six lists of hundreds of tensors, and as lines of Python their checks, allocations and addresses took 10 and 165 us more than
// the launches.  What is checked and what is raised is the binding's: ValueError for tensors that do not fit, the binding's own error for a code that
// the library returns.  No arithmetic, no GPU code; the library's functions come as addresses from the binding, which has loaded it.
#include <Python.h>
#include <ATen/ATen.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <optional>
#include <stdexcept>
#include <string>
#include <vector>

#include "../../include/imunpack.h"

namespace {
PyObject *g_error = nullptr;  // the binding's error class, called with (code, where)
decltype(&imunpack_rmsnorm) g_rmsnorm = nullptr;
decltype(&imunpack_rmsnorm_quantize) g_rmsnorm_quantize = nullptr;
decltype(&imunpack_rmsnorm_backward_workspace) g_rmsnorm_backward_workspace = nullptr;
decltype(&imunpack_rmsnorm_backward) g_rmsnorm_backward = nullptr;
decltype(&imunpack_adamw) g_adamw = nullptr;
decltype(&imunpack_xent_workspace) g_xent_workspace = nullptr;
decltype(&imunpack_xent) g_xent = nullptr;
decltype(&imunpack_xent_rescale) g_xent_rescale = nullptr;

struct Refused : std::runtime_error {  // becomes a ValueError
    using std::runtime_error::runtime_error;
};
struct Raised {};                      // a Python error is set already

void check(int code, const char *where) {
    if (code == IMUNPACK_OK) return;
    if (PyObject *e = PyObject_CallFunction(g_error, "is", code, where)) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Raised();
}
void need(bool ok, const char *what) {
    if (!ok) throw Refused(what);
}

const at::Tensor &tensor(PyObject *o, const char *what) {
    if (!THPVariable_Check(o)) throw Refused(std::string(what) + ": not a tensor");
    return THPVariable_Unpack(o);
}
at::Tensor maybe(PyObject *o, const char *what) { return o == Py_None ? at::Tensor() : tensor(o, what); }
double number(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}
long long whole(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}
bool truth(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised();
    return v != 0;
}
void *address(PyObject *o) {
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Raised();
    return p;
}
void *data(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
PyObject *wrap(const at::Tensor &t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
template <size_t N>
PyObject *wrapped(const std::array<at::Tensor, N> &ts) {
    PyObject *r = PyTuple_New(N);
    if (!r) throw Raised();
    for (size_t k = 0; k < N; ++k) {
        PyObject *o = wrap(ts[k]);
        if (!o) {
            Py_DECREF(r);
            throw Raised();
        }
        PyTuple_SET_ITEM(r, k, o);
    }
    return r;
}

// A kernel reads and writes one GPU's memory, and the stream that it is given is the current GPU's.
bool beside(const at::Tensor &t, const at::Tensor &x) { return !t.defined() || t.device() == x.device(); }
void need_current(const at::Device &device) { need(device == c10::impl::getDeviceGuardImpl(at::kCUDA)->getDevice(), "tensors of a GPU that is not the current one"); }

// IMUNPACK_F32, IMUNPACK_BF16 or a refusal.
int type_of(const at::Tensor &t, const char *what) {
    if (t.scalar_type() == at::kFloat) return IMUNPACK_F32;
    if (t.scalar_type() == at::kBFloat16) return IMUNPACK_BF16;
    throw Refused(std::string(what) + ": fp32 or bfloat16");
}
// A tensor as rows of d elements with unit stride, a pitch apart; laid out anew where its strides are others.
struct Rows {
    at::Tensor t;
    int64_t pitch = 0;
    void *p = nullptr;
};
Rows spread(const at::Tensor &t, int64_t d) {
    Rows r;
    r.pitch = d;
    if (!t.defined()) return r;
    r.t = t;
    if (!t.is_contiguous()) {
        if (t.dim() != 2) r.t = t.reshape({-1, d});
        if ((r.t.stride(1) != 1 && d > 1) || (r.t.size(0) > 1 && r.t.stride(0) < d)) r.t = r.t.contiguous();
        r.pitch = r.t.size(0) > 1 ? r.t.stride(0) : d;
    }
    r.p = r.t.data_ptr();
    return r;
}
at::Tensor dense_like(const at::Tensor &t, at::ScalarType type) { return at::empty(t.sizes(), t.options().dtype(type).requires_grad(false)); }

struct Norm {  // the arguments that every norm takes, checked
    int64_t d;
    int type, weight_type;
};
Norm norm_arguments(const at::Tensor &x, const at::Tensor &weight, const at::Tensor &residual) {
    need(x.is_cuda() && weight.is_cuda(), "rmsnorm takes fp32 or bfloat16 device tensors");
    need(x.dim() >= 1, "rmsnorm: x has no dimension");
    const Norm n = {x.size(-1), type_of(x, "rmsnorm: x"), type_of(weight, "rmsnorm: weight")};
    need(weight.dim() == 1 && weight.size(0) == n.d && weight.is_contiguous(), "rmsnorm: weight is one dense row like x's");
    need(beside(weight, x) && beside(residual, x), "rmsnorm: tensors of different devices");
    need(!residual.defined() || (residual.is_cuda() && residual.scalar_type() == x.scalar_type() && residual.sizes() == x.sizes()), "rmsnorm: residual must be like x");
    return n;
}
at::Tensor per_row(const at::Tensor &x) { return at::empty(x.sizes().slice(0, x.dim() - 1), x.options().dtype(at::kFloat).requires_grad(false)); }

PyObject *rmsnorm(PyObject *const *a) {  // x, weight, eps, residual, stream -> y, h, rstd
    const at::Tensor &x = tensor(a[0], "rmsnorm: x"), &weight = tensor(a[1], "rmsnorm: weight");
    const at::Tensor residual = maybe(a[3], "rmsnorm: residual");
    const Norm n = norm_arguments(x, weight, residual);
    need_current(x.device());
    const Rows rx = spread(x, n.d), rr = spread(residual, n.d);
    const at::Tensor y = dense_like(x, x.scalar_type()), h = residual.defined() ? dense_like(x, x.scalar_type()) : x, rstd = per_row(x);
    check(g_rmsnorm(rx.p, rx.pitch, rr.p, rr.pitch, weight.data_ptr(), rstd.numel(), n.d, n.type, n.weight_type, (float)number(a[2]), y.data_ptr(), n.d,
                    residual.defined() ? h.data_ptr() : nullptr, n.d, (float *)rstd.data_ptr(), address(a[4])), "imunpack_rmsnorm");
    return wrapped<3>({y, h, rstd});
}

PyObject *rmsnorm_quantize(PyObject *const *a) {  // x, weight, eps, b, residual, want_values, stream -> q, scale, h, values
    const at::Tensor &x = tensor(a[0], "rmsnorm: x"), &weight = tensor(a[1], "rmsnorm: weight");
    const at::Tensor residual = maybe(a[4], "rmsnorm: residual");
    const Norm n = norm_arguments(x, weight, residual);
    need_current(x.device());
    const Rows rx = spread(x, n.d), rr = spread(residual, n.d);
    const at::Tensor q = dense_like(x, at::kChar), scale = per_row(x), h = residual.defined() ? dense_like(x, x.scalar_type()) : x;
    const at::Tensor values = truth(a[5]) ? dense_like(x, x.scalar_type()) : at::Tensor();
    check(g_rmsnorm_quantize(rx.p, rx.pitch, rr.p, rr.pitch, weight.data_ptr(), scale.numel(), n.d, n.type, n.weight_type, (float)number(a[2]), (int)whole(a[3]),
                             (int8_t *)q.data_ptr(), n.d, (float *)scale.data_ptr(), data(values), n.d, residual.defined() ? h.data_ptr() : nullptr, n.d,
                             address(a[6])), "imunpack_rmsnorm_quantize");
    return wrapped<4>({q, scale, h, values});
}

PyObject *rmsnorm_backward(PyObject *const *a) {  // gy, x, residual, gh, weight, rstd, want_weight, stream -> gx, gweight
    const at::Tensor &gy = tensor(a[0], "rmsnorm: gy"), &x = tensor(a[1], "rmsnorm: x"), &weight = tensor(a[4], "rmsnorm: weight"), &rstd = tensor(a[5], "rmsnorm: rstd");
    const at::Tensor residual = maybe(a[2], "rmsnorm: residual"), gh = maybe(a[3], "rmsnorm: gh");
    const Norm n = norm_arguments(x, weight, residual);
    auto like = [&](const at::Tensor &t) { return t.is_cuda() && t.scalar_type() == x.scalar_type() && t.sizes() == x.sizes(); };
    need(like(gy) && (!gh.defined() || like(gh)), "rmsnorm: h, gy and gh must be like x");
    need(rstd.is_cuda() && rstd.scalar_type() == at::kFloat && rstd.is_contiguous() && rstd.sizes() == x.sizes().slice(0, x.dim() - 1),
         "rmsnorm: saved must be what imunpack_rmsnorm returned");
    need(beside(gy, x) && beside(gh, x) && beside(rstd, x), "rmsnorm: tensors of different devices");
    need_current(x.device());
    const Rows rg = spread(gy, n.d), rx = spread(x, n.d), rr = spread(residual, n.d), rh = spread(gh, n.d);
    const int64_t rows = rstd.numel();
    const at::Tensor gx = dense_like(x, x.scalar_type());
    at::Tensor gw, ws;
    size_t bytes = 0;
    if (truth(a[6])) {
        gw = dense_like(weight, weight.scalar_type());
        check(g_rmsnorm_backward_workspace(rows, n.d, n.type, &bytes), "imunpack_rmsnorm_backward_workspace");
        ws = at::empty({(int64_t)bytes}, x.options().dtype(at::kByte).requires_grad(false));
    }
    check(g_rmsnorm_backward(rg.p, rg.pitch, rx.p, rx.pitch, rr.p, rr.pitch, rh.p, rh.pitch, weight.data_ptr(), (const float *)rstd.data_ptr(), rows, n.d, n.type,
                             n.weight_type, gx.data_ptr(), n.d, data(gw), data(ws), bytes, address(a[7])), "imunpack_rmsnorm_backward");
    return wrapped<2>({gx, gw});
}

// What can be iterated over, as a list that holds its tensors until the call is over (an iterator may be all that does).
struct Listed {
    PyObject *o;
    explicit Listed(PyObject *list) : o(PySequence_Fast(list, "adamw takes lists of tensors")) {
        if (!o) throw Raised();
    }
    Listed(const Listed &) = delete;
    ~Listed() { Py_DECREF(o); }
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(o); }
    const at::Tensor &operator()(Py_ssize_t k, const char *what) const { return tensor(PySequence_Fast_GET_ITEM(o, k), what); }
};
// The addresses of a list of dense tensors of one type, of given sizes, on one GPU.
std::vector<void *> table(const Listed &list, at::ScalarType type, const std::vector<int64_t> &sizes, const at::Device &device, const char *what) {
    const Py_ssize_t n = list.size();
    if ((size_t)n != sizes.size()) throw Refused("adamw: lists of different lengths");
    std::vector<void *> at(n);
    for (Py_ssize_t k = 0; k < n; ++k) {
        const at::Tensor &t = list(k, what);
        if (t.scalar_type() != type || t.device() != device || !t.is_contiguous() || t.numel() != sizes[k])
            throw Refused(std::string("adamw: ") + what + ": a tensor of the wrong type, size, device or layout");
        at[k] = t.data_ptr();
    }
    return at;
}

PyObject *adamw(PyObject *const *a) {  // params, grads, exp_avg, exp_avg_sq, m_scales, v_scales, copies, lr, beta1, beta2, eps, decay, step, seed, stream
    const bool eight = a[4] != Py_None, copied = a[6] != Py_None;
    const Listed params(a[0]), grads(a[1]), exp_avg(a[2]), exp_avg_sq(a[3]);
    std::vector<int64_t> numel, held, blocks;
    at::Device device(at::kCPU);
    const Py_ssize_t n = params.size();
    for (Py_ssize_t k = 0; k < n; ++k) {
        const at::Tensor &t = params(k, "adamw: params");
        if (k == 0) device = t.device();
        numel.push_back(t.numel());
        blocks.push_back((t.numel() + IMUNPACK_ADAMW_BLOCK - 1) / IMUNPACK_ADAMW_BLOCK);
        held.push_back(eight ? blocks.back() * IMUNPACK_ADAMW_BLOCK : t.numel());
    }
    need(eight == (a[5] != Py_None), "adamw: scales for both states or for none");
    const at::ScalarType state = eight ? at::kFloat8_e4m3fn : at::kFloat;
    at::ScalarType gtype = at::kFloat;
    if (n > 0) {
        need(device.is_cuda(), "adamw takes device tensors");
        need(grads.size() == n, "adamw: lists of different lengths");
        gtype = grads(0, "adamw: grads").scalar_type();
        need(gtype == at::kFloat || gtype == at::kBFloat16, "adamw: gradients are fp32 or bfloat16 tensors");
    }
    const auto p = table(params, at::kFloat, numel, device, "params"), g = table(grads, gtype, numel, device, "grads");
    const auto m = table(exp_avg, state, held, device, "exp_avg"), v = table(exp_avg_sq, state, held, device, "exp_avg_sq");
    std::vector<void *> ms, vs, copies;
    std::optional<Listed> m_scales, v_scales, copy_list;
    if (eight) {
        ms = table(m_scales.emplace(a[4]), at::kFloat, blocks, device, "m_scales");
        vs = table(v_scales.emplace(a[5]), at::kFloat, blocks, device, "v_scales");
    }
    if (copied) copies = table(copy_list.emplace(a[6]), at::kBFloat16, numel, device, "copies");
    if (n > 0) need_current(device);
    check(g_adamw(n, (float *const *)p.data(), g.data(), m.data(), v.data(), eight ? (float *const *)ms.data() : nullptr, eight ? (float *const *)vs.data() : nullptr,
                  copied ? copies.data() : nullptr, numel.data(), gtype == at::kFloat ? IMUNPACK_F32 : IMUNPACK_BF16, eight ? 8 : 32, number(a[7]), number(a[8]),
                  number(a[9]), number(a[10]), number(a[11]), whole(a[12]), (uint32_t)whole(a[13]), address(a[14])), "imunpack_adamw");
    Py_RETURN_NONE;
}

struct Xent {  // the arguments that the loss and its gradients take, checked
    at::Tensor x, w, target;
    int64_t d, vocab, rows;
    int type;
};
Xent xent_arguments(PyObject *const *a) {  // x, w, target
    Xent n = {tensor(a[0], "xent: x"), tensor(a[1], "xent: W"), tensor(a[2], "xent: target"), 0, 0, 0, 0};
    n.type = type_of(n.x, "xent: x");
    need(n.w.scalar_type() == n.x.scalar_type() && n.x.is_cuda() && n.w.is_cuda(), "xent takes x and W as device tensors, both fp32 or both bfloat16");
    need(n.w.dim() == 2 && n.x.dim() >= 1 && n.x.size(-1) == n.w.size(1), "xent: x and W have no product x W^T");
    need(n.target.scalar_type() == at::kLong && n.target.is_cuda() && n.target.sizes() == n.x.sizes().slice(0, n.x.dim() - 1), "xent: target is an int64 device tensor of x's leading shape");
    need(beside(n.w, n.x) && beside(n.target, n.x), "xent: tensors of different devices");
    n.d = n.w.size(1);
    n.vocab = n.w.size(0);
    n.rows = n.target.numel();
    return n;
}
// One call of the library: the loss, where it is wanted, and the gradients of x and W that are.
PyObject *xent(PyObject *const *a) {  // x, w, target, ignore_index, how, want_loss, grad, want_x, want_w, stream -> loss, gx, gw
    const Xent n = xent_arguments(a);
    const int how = (int)whole(a[4]);
    const at::Tensor grad = maybe(a[6], "xent: grad"), target = n.target.contiguous();
    need(beside(grad, n.x), "xent: tensors of different devices");
    need_current(n.x.device());
    const Rows x = spread(n.x, n.d), w = spread(n.w, n.d);
    const at::TensorOptions floats = n.x.options().dtype(at::kFloat).requires_grad(false);
    const at::Tensor loss = !truth(a[5]) ? at::Tensor() : how == IMUNPACK_NONE ? at::empty(n.target.sizes(), floats) : at::empty({}, floats);
    const at::Tensor gx = truth(a[7]) ? dense_like(n.x, n.x.scalar_type()) : at::Tensor(), gw = truth(a[8]) ? dense_like(n.w, n.w.scalar_type()) : at::Tensor();
    size_t bytes = 0;
    check(g_xent_workspace(w.p, w.pitch, n.rows, n.d, n.vocab, n.type, gx.defined() || gw.defined(), &bytes), "imunpack_xent_workspace");
    const at::Tensor workspace = at::empty({(int64_t)bytes}, floats.dtype(at::kByte));
    check(g_xent(x.p, x.pitch, w.p, w.pitch, (const int64_t *)target.data_ptr(), n.rows, n.d, n.vocab, n.type, whole(a[3]), how, (float *)data(loss), (const float *)data(grad),
                 data(gx), n.d, data(gw), n.d, workspace.data_ptr(), bytes, address(a[9])), "imunpack_xent");
    return wrapped<3>({loss, gx, gw});
}

PyObject *xent_rescale(PyObject *const *a) {  // x, w, target, grad, gx, gw, stream: gx and gw (either may be None) times grad, in place
    const Xent n = xent_arguments(a);
    const at::Tensor &grad = tensor(a[3], "xent: grad");
    const at::Tensor gx = maybe(a[4], "xent: gx"), gw = maybe(a[5], "xent: gw");
    need(beside(grad, n.x) && beside(gx, n.x) && beside(gw, n.x), "xent: tensors of different devices");
    need_current(n.x.device());
    check(g_xent_rescale((const float *)grad.data_ptr(), data(gx), gx.defined() ? gx.numel() : 0, data(gw), gw.defined() ? gw.numel() : 0, n.type, address(a[6])),
          "imunpack_xent_rescale");
    Py_RETURN_NONE;
}

PyObject *bind(PyObject *const *a) {  // error class, then the addresses of the library's functions
    Py_INCREF(a[0]);
    Py_XDECREF(g_error);
    g_error = a[0];
    g_rmsnorm = (decltype(g_rmsnorm))address(a[1]);
    g_rmsnorm_quantize = (decltype(g_rmsnorm_quantize))address(a[2]);
    g_rmsnorm_backward_workspace = (decltype(g_rmsnorm_backward_workspace))address(a[3]);
    g_rmsnorm_backward = (decltype(g_rmsnorm_backward))address(a[4]);
    g_adamw = (decltype(g_adamw))address(a[5]);
    g_xent_workspace = (decltype(g_xent_workspace))address(a[6]);
    g_xent = (decltype(g_xent))address(a[7]);
    g_xent_rescale = (decltype(g_xent_rescale))address(a[8]);
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        need(n == N, "wrong number of arguments");
        return F(args);
    } catch (const Raised &) {
    } catch (const Refused &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception &e) {  // torch's own (memory, a view that cannot be)
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyMethodDef method(const char *name) {
    return {name, (PyCFunction)(void (*)(void))entry<F, N>, METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {method<bind, 9>("bind"), method<rmsnorm, 5>("rmsnorm"), method<rmsnorm_quantize, 7>("rmsnorm_quantize"),
                           method<rmsnorm_backward, 8>("rmsnorm_backward"), method<adamw, 15>("adamw"),
                           method<xent, 10>("xent"), method<xent_rescale, 7>("xent_rescale"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_tensors", "Argument marshalling of the calls whose host time counts.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};
}  // namespace

PyMODINIT_FUNC PyInit__tensors(void) { return PyModule_Create(&g_module); }
