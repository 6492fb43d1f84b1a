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
decltype(&imunpack_block8_quantize) g_block8_quantize = nullptr;
decltype(&imunpack_block8_turn) g_block8_turn = nullptr;
decltype(&imunpack_block8_values) g_block8_values = nullptr;
decltype(&imunpack_block8_gemm_workspace) g_block8_gemm_workspace = nullptr;
decltype(&imunpack_block8_gemm) g_block8_gemm = nullptr;
decltype(&imunpack_act8) g_act8 = nullptr;
decltype(&imunpack_act8_backward) g_act8_backward = nullptr;
decltype(&imunpack_logprobs_workspace) g_logprobs_workspace = nullptr;
decltype(&imunpack_logprobs) g_logprobs = nullptr;
decltype(&imunpack_logprobs_backward) g_logprobs_backward = nullptr;
decltype(&imunpack_block8_many) g_block8_many = nullptr;
decltype(&imunpack_column_sums_workspace) g_column_sums_workspace = nullptr;
decltype(&imunpack_column_sums) g_column_sums = nullptr;

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

// A tensor in 8 bits: codes over whole blocks and a power of two (a byte) for every row and block.
constexpr int64_t kBlock = IMUNPACK_BLOCK8;
int64_t whole_of(int64_t n, int64_t of) { return (n + of - 1) / of * of; }
struct Eight {
    at::Tensor codes, scales;
    int64_t cols = 0, ldc = 0, lds = 0;
    int format = 0;
    void *c() const { return data(codes); }
    void *s() const { return data(scales); }
    int64_t rows() const { return codes.size(0); }
};
int format_of(at::ScalarType t, const char *what) {
    if (t == at::kFloat8_e4m3fn) return IMUNPACK_E4M3;
    if (t == at::kFloat8_e5m2) return IMUNPACK_E5M2;
    throw Refused(std::string(what) + ": codes are float8_e4m3fn or float8_e5m2");
}
Eight eight(PyObject *codes, PyObject *scales, PyObject *cols, const char *what) {
    Eight e = {tensor(codes, what), tensor(scales, what), whole(cols)};
    const at::Tensor &c = e.codes, &s = e.scales;
    e.format = format_of(c.scalar_type(), what);
    auto dense = [](const at::Tensor &t, int64_t least) {
        return t.is_cuda() && t.dim() == 2 && t.size(1) >= least && (t.stride(1) == 1 || t.size(1) == 1) && (t.size(0) <= 1 || (t.stride(0) >= t.size(1) && t.stride(0) % 16 == 0)) &&
               (uintptr_t)t.data_ptr() % 16 == 0;
    };
    if (e.cols < 1 || s.scalar_type() != at::kFloat8_e8m0fnu || !dense(c, whole_of(e.cols, kBlock)) || !dense(s, whole_of((e.cols + kBlock - 1) / kBlock, 16)) || s.size(0) != c.size(0) ||
        !beside(s, c))
        throw Refused(std::string(what) + ": not a tensor in 8 bits as imunpack_block8_quantize lays it out");
    e.ldc = c.size(0) > 1 ? c.stride(0) : whole_of(c.size(1), 16);
    e.lds = s.size(0) > 1 ? s.stride(0) : whole_of(s.size(1), 16);
    return e;
}
Eight new_eight(int64_t rows, int64_t cols, at::ScalarType type, const at::Tensor &like) {
    Eight e;
    e.cols = cols, e.ldc = whole_of(cols, kBlock), e.lds = whole_of(e.ldc / kBlock, 16);
    e.codes = at::empty({rows, e.ldc}, like.options().dtype(type).requires_grad(false));
    e.scales = at::empty({rows, e.lds}, like.options().dtype(at::kFloat8_e8m0fnu).requires_grad(false));
    return e;
}
int64_t rows_of(const at::Tensor &x, int64_t cols) { return cols ? x.numel() / cols : 0; }

PyObject *block8_quantize(PyObject *const *a) {  // x, e5m2, square, lying, turned, stream -> codes, scales, turned codes, turned scales
    const at::Tensor &x = tensor(a[0], "block8: x");
    const int type = type_of(x, "block8: x"), format = truth(a[1]) ? IMUNPACK_E5M2 : IMUNPACK_E4M3;
    need(x.is_cuda() && x.dim() >= 1 && x.size(-1) >= 1, "block8: x is a device tensor with columns");
    need_current(x.device());
    const int64_t cols = x.size(-1), rows = rows_of(x, cols);
    const Rows r = spread(x, cols);
    const at::ScalarType code = format == IMUNPACK_E5M2 ? at::kFloat8_e5m2 : at::kFloat8_e4m3fn;
    Eight q, t;
    if (truth(a[3])) q = new_eight(rows, cols, code, x);
    if (truth(a[4])) {
        need(rows >= 1, "block8: a tensor without rows cannot be turned");
        t = new_eight(cols, rows, code, x);
    }
    check(g_block8_quantize(r.p, r.pitch, rows, cols, type, format, truth(a[2]), q.c(), q.ldc, q.s(), q.lds, t.c(), t.ldc, t.s(), t.lds, address(a[5])), "imunpack_block8_quantize");
    return wrapped<4>({q.codes, q.scales, t.codes, t.scales});
}

PyObject *block8_turn(PyObject *const *a) {  // codes, scales, cols, stream -> codes, scales
    const Eight q = eight(a[0], a[1], a[2], "block8: x");
    need(q.rows() >= 1, "block8: a tensor without rows cannot be turned");
    need_current(q.codes.device());
    const Eight t = new_eight(q.cols, q.rows(), q.codes.scalar_type(), q.codes);
    check(g_block8_turn(q.c(), q.ldc, q.s(), q.lds, q.rows(), q.cols, q.format, t.c(), t.ldc, t.s(), t.lds, address(a[3])), "imunpack_block8_turn");
    return wrapped<2>({t.codes, t.scales});
}

PyObject *block8_many(PyObject *const *a) {  // jobs (tuples of x or codes, scales or None, cols of codes, square, lying, turned), e5m2, stream -> codes, scales, turned codes, turned scales of each
    need(PyTuple_Check(a[0]) && PyTuple_GET_SIZE(a[0]) >= 1 && PyTuple_GET_SIZE(a[0]) <= IMUNPACK_BLOCK8_MANY, "block8: one to four tensors at a time");
    const int count = (int)PyTuple_GET_SIZE(a[0]), format = truth(a[1]) ? IMUNPACK_E5M2 : IMUNPACK_E4M3;
    const at::ScalarType code = format == IMUNPACK_E5M2 ? at::kFloat8_e5m2 : at::kFloat8_e4m3fn;
    imunpack_block8_job jobs[IMUNPACK_BLOCK8_MANY] = {};
    Eight q[IMUNPACK_BLOCK8_MANY], t[IMUNPACK_BLOCK8_MANY], from[IMUNPACK_BLOCK8_MANY];
    Rows r[IMUNPACK_BLOCK8_MANY];
    at::Tensor first;
    for (int k = 0; k < count; ++k) {
        PyObject *const job = PyTuple_GET_ITEM(a[0], k);
        need(PyTuple_Check(job) && PyTuple_GET_SIZE(job) == 6, "block8: a tensor comes with how it is wanted");
        PyObject *const *p = ((PyTupleObject *)job)->ob_item;
        imunpack_block8_job &j = jobs[k];
        const at::Tensor &x = tensor(p[0], "block8: x");
        if (k == 0) first = x;
        need(beside(x, first), "block8: tensors of different devices");
        const bool lying = truth(p[4]), turned = truth(p[5]);
        if (p[1] != Py_None) {
            from[k] = eight(p[0], p[1], p[2], "block8: x");
            need(from[k].format == format && turned && !lying, "block8: a tensor in 8 bits is turned, in its own format");
            j.x = from[k].c(), j.ldx = from[k].ldc, j.x_scales = from[k].s(), j.ldxs = from[k].lds, j.rows = from[k].rows(), j.cols = from[k].cols;
        } else {
            j.dtype = type_of(x, "block8: x");
            need(x.is_cuda() && x.dim() >= 1 && x.size(-1) >= 1 && (lying || turned), "block8: x is a device tensor with columns, wanted as it lies, turned or both");
            j.cols = x.size(-1), j.rows = rows_of(x, j.cols), j.square = truth(p[3]);
            r[k] = spread(x, j.cols);
            j.x = r[k].p, j.ldx = r[k].pitch;
        }
        if (k == 0) need_current(x.device());
        if (lying) {
            q[k] = new_eight(j.rows, j.cols, code, x);
            j.codes = q[k].c(), j.ldc = q[k].ldc, j.scales = q[k].s(), j.lds = q[k].lds;
        }
        if (turned) {
            need(j.rows >= 1, "block8: a tensor without rows cannot be turned");
            t[k] = new_eight(j.cols, j.rows, code, x);
            j.turned = t[k].c(), j.ldt = t[k].ldc, j.turned_scales = t[k].s(), j.ldts = t[k].lds;
        }
    }
    check(g_block8_many(count, jobs, format, address(a[2])), "imunpack_block8_many");
    std::array<at::Tensor, 4 * IMUNPACK_BLOCK8_MANY> all;
    for (int k = 0; k < count; ++k) all[4 * k] = q[k].codes, all[4 * k + 1] = q[k].scales, all[4 * k + 2] = t[k].codes, all[4 * k + 3] = t[k].scales;
    return wrapped<4 * IMUNPACK_BLOCK8_MANY>(all);
}

PyObject *block8_values(PyObject *const *a) {  // codes, scales, cols, bf16, stream -> values
    const Eight q = eight(a[0], a[1], a[2], "block8: x");
    need_current(q.codes.device());
    const bool half = truth(a[3]);
    const at::Tensor out = at::empty({q.rows(), q.cols}, q.codes.options().dtype(half ? at::kBFloat16 : at::kFloat));
    check(g_block8_values(q.c(), q.ldc, q.s(), q.lds, q.rows(), q.cols, q.format, out.data_ptr(), q.cols, half ? IMUNPACK_BF16 : IMUNPACK_F32, address(a[4])), "imunpack_block8_values");
    return wrap(out);
}

PyObject *block8_gemm(PyObject *const *a) {  // codes, scales of A, codes, scales of B, cols of A, of B, bf16, bias, stream -> out
    const Eight x = eight(a[0], a[1], a[4], "block8_gemm: A"), w = eight(a[2], a[3], a[5], "block8_gemm: B");
    const at::Tensor bias = maybe(a[7], "block8_gemm: bias");
    need(x.cols == w.cols, "block8_gemm: A and B have no product A B^T");
    need(beside(w.codes, x.codes) && beside(bias, x.codes), "block8_gemm: tensors of different devices");
    need(!bias.defined() || (bias.scalar_type() == at::kFloat && bias.is_contiguous() && bias.dim() == 1 && bias.size(0) == w.rows()), "block8_gemm: bias is fp32, one for each row of B");
    need_current(x.codes.device());
    const int64_t m = x.rows(), n = w.rows();
    const int type = truth(a[6]) ? IMUNPACK_BF16 : IMUNPACK_F32;
    const at::Tensor out = at::empty({m, n}, x.codes.options().dtype(type == IMUNPACK_BF16 ? at::kBFloat16 : at::kFloat));
    size_t bytes = 0;
    check(g_block8_gemm_workspace(m, n, x.cols, type, &bytes), "imunpack_block8_gemm_workspace");
    at::Tensor workspace;
    if (bytes) workspace = at::empty({(int64_t)bytes}, x.codes.options().dtype(at::kByte));
    check(g_block8_gemm(x.c(), x.ldc, x.s(), x.lds, x.format, w.c(), w.ldc, w.s(), w.lds, w.format, m, n, x.cols, (const float *)data(bias), out.data_ptr(), n, type,
                        data(workspace), bytes, address(a[8])), "imunpack_block8_gemm");
    return wrap(out);
}

PyObject *act8(PyObject *const *a) {  // u, act, gated, quantize, keep, want_y, stream -> y, codes, scales, kept codes, scales, kept2 codes, scales
    const at::Tensor &u = tensor(a[0], "act8: u");
    const int type = type_of(u, "act8: u"), act = (int)whole(a[1]);
    const bool gated = truth(a[2]), keep = truth(a[4]);
    need(u.is_cuda() && u.dim() >= 1 && u.size(-1) >= 1 && (!gated || u.size(-1) % 2 == 0), "act8: u is a device tensor with columns, twice as many where it is gated");
    need_current(u.device());
    const int64_t wide = u.size(-1), cols = gated ? wide / 2 : wide, rows = rows_of(u, wide);
    const Rows r = spread(u, wide);
    auto shape = u.sizes().vec();
    shape.back() = cols;
    Eight q, k, k2;
    at::Tensor y;
    if (truth(a[5])) y = at::empty(shape, u.options().requires_grad(false));
    if (truth(a[3])) q = new_eight(rows, cols, at::kFloat8_e4m3fn, u);
    if (keep) k = new_eight(rows, cols, at::kFloat8_e4m3fn, u);
    if (keep && gated) k2 = new_eight(rows, cols, at::kFloat8_e4m3fn, u);
    check(g_act8(r.p, r.pitch, rows, cols, type, act, gated, data(y), cols, q.c(), q.ldc, q.s(), q.lds, k.c(), k2.c(), k.ldc, k.s(), k2.s(), k.lds, address(a[6])), "imunpack_act8");
    return wrapped<7>({y, q.codes, q.scales, k.codes, k.scales, k2.codes, k2.scales});
}

PyObject *act8_backward(PyObject *const *a) {  // g, act, kept codes, scales, kept2 codes, scales (None: not gated), cols, stream -> gu
    const at::Tensor &g = tensor(a[0], "act8: g");
    const int type = type_of(g, "act8: g");
    const bool gated = a[4] != Py_None;
    const Eight k = eight(a[2], a[3], a[6], "act8: kept"), k2 = gated ? eight(a[4], a[5], a[6], "act8: kept") : Eight();
    const int64_t cols = k.cols, rows = k.rows();
    need(g.is_cuda() && g.dim() >= 1 && g.size(-1) == cols && g.numel() == rows * cols, "act8: g is shaped like y");
    need(k.format == IMUNPACK_E4M3 && (!gated || (k2.format == IMUNPACK_E4M3 && k2.rows() == rows && k2.ldc == k.ldc && k2.lds == k.lds)), "act8: kept must be what imunpack_act8 returned");
    need(beside(k.codes, g) && beside(k2.codes, g), "act8: tensors of different devices");
    need_current(g.device());
    const Rows r = spread(g, cols);
    auto shape = g.sizes().vec();
    shape.back() = gated ? 2 * cols : cols;
    const at::Tensor gu = at::empty(shape, g.options().requires_grad(false));
    check(g_act8_backward(r.p, r.pitch, rows, cols, type, (int)whole(a[1]), gated, k.c(), k2.c(), k.ldc, k.s(), k2.s(), k.lds, gu.data_ptr(), shape.back(), address(a[7])),
          "imunpack_act8_backward");
    return wrap(gu);
}

PyObject *column_sums(PyObject *const *a) {  // x, stream -> sums
    const at::Tensor &x = tensor(a[0], "column_sums: x");
    const int type = type_of(x, "column_sums: x");
    need(x.is_cuda() && x.dim() >= 1 && x.size(-1) >= 1, "column_sums: x is a device tensor with columns");
    need_current(x.device());
    const int64_t cols = x.size(-1), rows = rows_of(x, cols);
    const Rows r = spread(x, cols);
    const at::Tensor out = at::empty({cols}, x.options().dtype(at::kFloat).requires_grad(false));
    size_t bytes = 0;
    check(g_column_sums_workspace(rows, cols, type, &bytes), "imunpack_column_sums_workspace");
    at::Tensor workspace;
    if (bytes) workspace = at::empty({(int64_t)bytes}, x.options().dtype(at::kByte).requires_grad(false));
    check(g_column_sums(r.p, r.pitch, rows, cols, type, (float *)out.data_ptr(), data(workspace), bytes, address(a[1])), "imunpack_column_sums");
    return wrap(out);
}

struct Logprobs {  // the arguments that log probabilities and their gradients take, checked
    at::Tensor logits, tokens;
    int64_t vocab, rows, count;
    int type;
};
Logprobs logprobs_arguments(PyObject *const *a) {  // logits, tokens (None: none)
    Logprobs n = {tensor(a[0], "logprobs: logits"), maybe(a[1], "logprobs: tokens"), 0, 0, 0, 0};
    n.type = type_of(n.logits, "logprobs: logits");
    need(n.logits.is_cuda() && n.logits.dim() >= 1 && n.logits.size(-1) >= 1, "logprobs: logits are a device tensor with columns");
    n.vocab = n.logits.size(-1);
    n.rows = rows_of(n.logits, n.vocab);
    if (n.tokens.defined()) {
        const auto lead = n.logits.sizes().slice(0, n.logits.dim() - 1), given = n.tokens.sizes();
        const bool one = given == lead, some = given.size() == lead.size() + 1 && given.slice(0, lead.size()) == lead;
        need(n.tokens.is_cuda() && n.tokens.scalar_type() == at::kLong && (one || some), "logprobs: tokens are an int64 device tensor of the logits' leading shape, or with some to a row behind it");
        need(beside(n.tokens, n.logits), "logprobs: tensors of different devices");
        n.count = one ? 1 : given.back();
        n.tokens = n.tokens.contiguous();
    }
    need_current(n.logits.device());
    return n;
}
PyObject *logprobs(PyObject *const *a) {  // logits, tokens, ignore_index, top, want_entropy, stream -> logp, lse, stats, entropy, top_logp, top_index
    const Logprobs n = logprobs_arguments(a);
    const int64_t top = whole(a[3]);
    need(top >= 0 && top <= IMUNPACK_LOGPROBS_TOP && top <= n.vocab, "logprobs: top is 0 to 64 and no more than there are logits");
    const Rows l = spread(n.logits, n.vocab);
    const at::TensorOptions floats = n.logits.options().dtype(at::kFloat).requires_grad(false);
    const auto lead = n.logits.sizes().slice(0, n.logits.dim() - 1);
    auto shape = lead.vec();
    shape.push_back(top);
    const at::Tensor logp = n.tokens.defined() ? at::empty(n.tokens.sizes(), floats) : at::Tensor(), lse = at::empty(lead, floats), stats = at::empty({n.rows, 2}, floats), entropy = truth(a[4]) ? at::empty(lead, floats) : at::Tensor();
    const at::Tensor top_logp = top ? at::empty(shape, floats) : at::Tensor(), top_index = top ? at::empty(shape, floats.dtype(at::kLong)) : at::Tensor();
    size_t bytes = 0;
    check(g_logprobs_workspace(n.rows, n.vocab, n.count, top, n.type, &bytes), "imunpack_logprobs_workspace");
    at::Tensor workspace;
    if (bytes) workspace = at::empty({(int64_t)bytes}, floats.dtype(at::kByte));
    check(g_logprobs(l.p, l.pitch, n.rows, n.vocab, n.type, (const int64_t *)data(n.tokens), n.count, whole(a[2]), top, (float *)data(logp), (float *)data(lse), (float *)data(stats),
                     (float *)data(entropy), (float *)data(top_logp), (int64_t *)data(top_index), data(workspace), bytes, address(a[5])), "imunpack_logprobs");
    return wrapped<6>({logp, lse, stats, entropy, top_logp, top_index});
}
PyObject *logprobs_backward(PyObject *const *a) {  // logits, tokens, ignore_index, top_index, stats, entropy, g_logp, g_entropy, g_top, stream -> gl
    const Logprobs n = logprobs_arguments(a);
    const at::Tensor index = maybe(a[3], "logprobs: top_index"), stats = tensor(a[4], "logprobs: saved"), entropy = maybe(a[5], "logprobs: saved"), gp = maybe(a[6], "logprobs: g_logp"),
                     gh = maybe(a[7], "logprobs: g_entropy"), gt = maybe(a[8], "logprobs: g_top");
    auto floats = [&](const at::Tensor &t, int64_t each) {
        return !t.defined() || (t.is_cuda() && t.scalar_type() == at::kFloat && t.is_contiguous() && t.numel() == n.rows * each && beside(t, n.logits));
    };
    const int64_t top = index.defined() ? index.size(-1) : 0;
    need(floats(stats, 2) && floats(entropy, 1) && (!index.defined() || (index.is_cuda() && index.scalar_type() == at::kLong && index.is_contiguous() && index.numel() == n.rows * top && beside(index, n.logits))),
         "logprobs: saved must be what imunpack_logprobs returned");
    need(floats(gp, n.count) && floats(gh, 1) && floats(gt, top), "logprobs: gradients are fp32 device tensors shaped like what they belong to");
    need((!gp.defined() || n.tokens.defined()) && (!gh.defined() || entropy.defined()) && (!gt.defined() || index.defined()), "logprobs: a gradient of something that was not asked for");
    const Rows l = spread(n.logits, n.vocab);
    const at::Tensor gl = dense_like(n.logits, n.logits.scalar_type());
    check(g_logprobs_backward(l.p, l.pitch, n.rows, n.vocab, n.type, (const int64_t *)data(n.tokens), n.count, whole(a[2]), top, (const int64_t *)data(index), (const float *)data(stats),
                              (const float *)data(entropy), (const float *)data(gp), (const float *)data(gh), (const float *)data(gt), gl.data_ptr(), n.vocab, address(a[9])),
          "imunpack_logprobs_backward");
    return wrap(gl);
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
    g_block8_quantize = (decltype(g_block8_quantize))address(a[9]);
    g_block8_turn = (decltype(g_block8_turn))address(a[10]);
    g_block8_values = (decltype(g_block8_values))address(a[11]);
    g_block8_gemm_workspace = (decltype(g_block8_gemm_workspace))address(a[12]);
    g_block8_gemm = (decltype(g_block8_gemm))address(a[13]);
    g_act8 = (decltype(g_act8))address(a[14]);
    g_act8_backward = (decltype(g_act8_backward))address(a[15]);
    g_logprobs_workspace = (decltype(g_logprobs_workspace))address(a[16]);
    g_logprobs = (decltype(g_logprobs))address(a[17]);
    g_logprobs_backward = (decltype(g_logprobs_backward))address(a[18]);
    g_column_sums_workspace = (decltype(g_column_sums_workspace))address(a[19]);
    g_column_sums = (decltype(g_column_sums))address(a[20]);
    g_block8_many = (decltype(g_block8_many))address(a[21]);
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
PyMethodDef g_methods[] = {method<bind, 22>("bind"), method<rmsnorm, 5>("rmsnorm"), method<rmsnorm_quantize, 7>("rmsnorm_quantize"),
                           method<rmsnorm_backward, 8>("rmsnorm_backward"), method<adamw, 15>("adamw"),
                           method<xent, 10>("xent"), method<xent_rescale, 7>("xent_rescale"),
                           method<block8_quantize, 6>("block8_quantize"), method<block8_turn, 4>("block8_turn"), method<block8_values, 5>("block8_values"),
                           method<block8_gemm, 9>("block8_gemm"), method<act8, 7>("act8"), method<act8_backward, 8>("act8_backward"), method<logprobs, 6>("logprobs"),
                           method<logprobs_backward, 10>("logprobs_backward"), method<column_sums, 2>("column_sums"), method<block8_many, 3>("block8_many"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_tensors", "Argument marshalling of the calls whose host time counts.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};
}  // namespace

PyMODINIT_FUNC PyInit__tensors(void) { return PyModule_Create(&g_module); }
