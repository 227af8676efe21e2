// CPython extension behind binding.py: argument checks, output allocation and the call into the C ABI in native code.
//
// A decode step or a short prompt spends a few microseconds on the GPU; marshalling its arguments through ctypes and checking
// them in Python took longer than that (decode step, B = 1: 12 us per call from Python, host-bound).  Each function here
// handles the calls whose arguments pass its checks and returns the outputs.  For anything else it does not call the library and
// returns None, and binding.py runs its checked path, which names the argument that is wrong.  A status of the library is raised
// here: the call may have launched kernels that update state in place, so it must not be made a second time.
//
// The operators around the core (norm, projection, linear attention) have no second path: their functions name the argument that is
// wrong themselves, and run on the device that their tensors live on.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "rglru.h"

namespace {

struct ParamsHandle {
    rglru_params_t p;
    int32_t H, D, io;
    at::ScalarType dtype;
    c10::Device device;
};
const char *const HANDLE = "rglru.params";

// A tensor argument or None; `bad` is set for anything else.
const at::Tensor *tensor_arg(PyObject *o, bool &bad) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) { bad = true; return nullptr; }
    return &THPVariable_Unpack(o);
}
// Absent, or contiguous with this shape, dtype and device
bool fits(const at::Tensor *t, at::IntArrayRef shape, at::ScalarType dtype, c10::Device dev) {
    return t == nullptr || (t->scalar_type() == dtype && t->device() == dev && t->sizes() == shape && t->is_contiguous());
}
void *ptr(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType dtype, c10::Device dev) {
    return at::Tensor(at::detail::empty_cuda(shape, dtype, dev, std::nullopt));
}
void *current_stream() { return (void *)c10::cuda::getCurrentCUDAStream().stream(); }
PyObject *wrap(const at::Tensor &t) { return THPVariable_Wrap(t); }

// binding.py's exception type for a status of the library, RglruError(code, where)
PyObject *error_type = nullptr;
PyObject *raise_status(int32_t rc, const char *where) {
    PyObject *e = PyObject_CallFunction(error_type ? error_type : PyExc_RuntimeError, "is", (int)rc, where);
    if (e) { PyErr_SetObject((PyObject *)Py_TYPE(e), e); Py_DECREF(e); }
    return nullptr;
}
PyObject *set_error_type(PyObject *, PyObject *type) {
    Py_INCREF(type);
    Py_XSETREF(error_type, type);
    Py_RETURN_NONE;
}

// Workspace of the call: the caller's, or scratch of this call (the library needs no particular contents)
struct Workspace {
    at::Tensor own;
    void *p = nullptr;
    size_t n = 0;
    bool take(const at::Tensor *given, const rglru_shape_t &s, int op, c10::Device dev) {
        if (given) { p = given->data_ptr(); n = (size_t)given->numel(); return true; }
        n = rglru_workspace_bytes(&s, op);
        if (n == 0) return false;
        own = fresh({(int64_t)n}, at::kByte, dev);
        p = own.data_ptr();
        return true;
    }
};

// The call into the library without the interpreter lock: a launch can block (a full queue, a first use that loads code), and other
// Python threads go on meanwhile.  The tensors stay alive: the caller's arguments hold them.
template <typename F> int32_t unlocked(F &&call) {
    int32_t rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}

struct Call {
    const ParamsHandle *h = nullptr;
    rglru_shape_t s{};
    bool begin(PyObject *handle, PyObject *c, PyObject *flags, const at::Tensor *x, int dims) {
        h = (const ParamsHandle *)PyCapsule_GetPointer(handle, HANDLE);
        if (!h) { PyErr_Clear(); return false; }
        if (!x || x->dim() != dims || x->scalar_type() != h->dtype || x->device() != h->device || !x->is_contiguous()) return false;
        if (!h->device.is_cuda() || x->size(dims - 1) != h->D) return false;
        for (int i = 0; i < dims; ++i)
            if (x->size(i) > INT32_MAX) return false;
        const double cv = PyFloat_AsDouble(c);
        const unsigned long fv = PyLong_AsUnsignedLong(flags);
        if (PyErr_Occurred()) { PyErr_Clear(); return false; }
        s.B = (int32_t)x->size(0); s.T = dims == 3 ? (int32_t)x->size(1) : 1; s.D = h->D; s.H = h->H;
        s.io = h->io; s.c = (float)cv; s.flags = (uint32_t)fv;
        return true;
    }
};

// params_handle(conv_w, conv_b, W_a, b_a, W_x, b_x, lam) of tensors that binding.Params has checked and keeps alive
PyObject *params_handle(PyObject *, PyObject *const *a, Py_ssize_t n) {
    bool bad = n != 7;
    const at::Tensor *t[7] = {};
    for (int i = 0; !bad && i < 7; ++i) t[i] = tensor_arg(a[i], bad);
    if (bad || !t[0] || !t[2] || !t[3] || !t[4] || !t[5] || !t[6] || t[2]->dim() != 3 || t[0]->dim() != 2) Py_RETURN_NONE;
    ParamsHandle *h = new ParamsHandle{{ptr(t[0]), (const float *)ptr(t[1]), ptr(t[2]), (const float *)ptr(t[3]), ptr(t[4]), (const float *)ptr(t[5]),
                                        (const float *)ptr(t[6])},
                                       (int32_t)t[2]->size(0), (int32_t)t[0]->size(1),
                                       t[0]->scalar_type() == at::kBFloat16 ? (int32_t)RGLRU_BF16 : (int32_t)RGLRU_F32, t[0]->scalar_type(), t[0]->device()};
    PyObject *cap = PyCapsule_New(h, HANDLE, [](PyObject *c) { delete (ParamsHandle *)PyCapsule_GetPointer(c, HANDLE); });
    if (!cap) delete h;
    return cap;
}

// prefill(handle, x, h0, conv_state_in, c, flags, y, h_T, conv_state_out, workspace, gate_branch, a_prod) -> (y, h_T, conv_state_out)
PyObject *prefill(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    bool bad = false;
    const at::Tensor *x = tensor_arg(a[1], bad), *h0 = tensor_arg(a[2], bad), *cs = tensor_arg(a[3], bad), *y = tensor_arg(a[6], bad),
                     *hT = tensor_arg(a[7], bad), *cso = tensor_arg(a[8], bad), *ws = tensor_arg(a[9], bad), *gb = tensor_arg(a[10], bad),
                     *ap = tensor_arg(a[11], bad);
    Call k;
    if (bad || !k.begin(a[0], a[4], a[5], x, 3)) Py_RETURN_NONE;
    const c10::Device dev = k.h->device;
    const at::ScalarType io = k.h->dtype;
    const int64_t B = k.s.B, T = k.s.T, D = k.s.D;
    if (!fits(h0, {B, D}, at::kFloat, dev) || !fits(cs, {B, 3, D}, io, dev) || !fits(y, {B, T, D}, io, dev) || !fits(hT, {B, D}, at::kFloat, dev) ||
        !fits(cso, {B, 3, D}, io, dev) || !fits(gb, {B, T, D}, io, dev) || !fits(ap, {B, D}, at::kFloat, dev))
        Py_RETURN_NONE;
    const at::Tensor yt = y ? *y : fresh({B, T, D}, io, dev), ht = hT ? *hT : fresh({B, D}, at::kFloat, dev), ct = cso ? *cso : fresh({B, 3, D}, io, dev);
    Workspace w;
    if (!w.take(ws, k.s, RGLRU_OP_PREFILL, dev)) Py_RETURN_NONE;
    const rglru_prefill_extras_t ex{ptr(gb), (float *)ptr(ap)};
    void *const st = current_stream();
    const int32_t rc = unlocked([&] {
        return rglru_prefill_ex(&k.s, &k.h->p, ptr(x), (const float *)ptr(h0), ptr(cs), yt.data_ptr(), (float *)ht.data_ptr(), ct.data_ptr(),
                                gb || ap ? &ex : nullptr, w.p, w.n, st);
    });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_prefill");
    PyObject *out = PyTuple_New(3);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, wrap(yt)); PyTuple_SET_ITEM(out, 1, wrap(ht)); PyTuple_SET_ITEM(out, 2, wrap(ct));
    return out;
    END_HANDLE_TH_ERRORS
}

// decode_step(handle, x, h, conv_state, c, flags, y, workspace) -> y
PyObject *decode_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 8) Py_RETURN_NONE;
    bool bad = false;
    const at::Tensor *x = tensor_arg(a[1], bad), *h = tensor_arg(a[2], bad), *cs = tensor_arg(a[3], bad), *y = tensor_arg(a[6], bad), *ws = tensor_arg(a[7], bad);
    Call k;
    if (bad || !h || !cs || !k.begin(a[0], a[4], a[5], x, 2)) Py_RETURN_NONE;
    const c10::Device dev = k.h->device;
    const at::ScalarType io = k.h->dtype;
    const int64_t B = k.s.B, D = k.s.D;
    if (!fits(h, {B, D}, at::kFloat, dev) || !fits(cs, {B, 3, D}, io, dev) || !fits(y, {B, D}, io, dev)) Py_RETURN_NONE;
    const at::Tensor yt = y ? *y : fresh({B, D}, io, dev);
    Workspace w;
    if (!w.take(ws, k.s, RGLRU_OP_DECODE, dev)) Py_RETURN_NONE;
    void *const st = current_stream();
    const int32_t rc = unlocked([&] { return rglru_decode_step(&k.s, &k.h->p, ptr(x), (float *)ptr(h), ptr(cs), yt.data_ptr(), w.p, w.n, st); });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_decode_step");
    if (y) { Py_INCREF(a[6]); return a[6]; }
    return wrap(yt);
    END_HANDLE_TH_ERRORS
}

// backward(handle, x, dy, h0, conv_state_in, y, c, flags, workspace, dh_T, dconv_state_out, state_grads) -> dict of gradients
PyObject *backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    bool bad = false;
    const at::Tensor *x = tensor_arg(a[1], bad), *dy = tensor_arg(a[2], bad), *h0 = tensor_arg(a[3], bad), *cs = tensor_arg(a[4], bad), *y = tensor_arg(a[5], bad),
                     *ws = tensor_arg(a[8], bad), *dhT = tensor_arg(a[9], bad), *dcs = tensor_arg(a[10], bad);
    const int want_state = PyObject_IsTrue(a[11]);
    Call k;
    if (bad || want_state < 0 || !dy || !k.begin(a[0], a[6], a[7], x, 3)) { PyErr_Clear(); Py_RETURN_NONE; }
    const c10::Device dev = k.h->device;
    const at::ScalarType io = k.h->dtype;
    const int64_t B = k.s.B, T = k.s.T, D = k.s.D, H = k.s.H, Dh = D / H;
    if (!fits(dy, {B, T, D}, io, dev) || !fits(h0, {B, D}, at::kFloat, dev) || !fits(cs, {B, 3, D}, io, dev) || !fits(y, {B, T, D}, io, dev) ||
        !fits(dhT, {B, D}, at::kFloat, dev) || !fits(dcs, {B, 3, D}, io, dev))
        Py_RETURN_NONE;
    Workspace w;
    if (!w.take(ws, k.s, RGLRU_OP_BACKWARD, dev)) Py_RETURN_NONE;
    const char *const names[10] = {"x", "conv_w", "conv_b", "W_a", "b_a", "W_x", "b_x", "lam", "h0", "conv_state"};
    const int count = want_state ? 10 : 8;
    at::Tensor g[10] = {fresh({B, T, D}, io, dev), fresh({4, D}, at::kFloat, dev), fresh({D}, at::kFloat, dev), fresh({H, Dh, Dh}, at::kFloat, dev),
                        fresh({D}, at::kFloat, dev), fresh({H, Dh, Dh}, at::kFloat, dev), fresh({D}, at::kFloat, dev), fresh({D}, at::kFloat, dev)};
    if (want_state) { g[8] = fresh({B, D}, at::kFloat, dev); g[9] = fresh({B, 3, D}, io, dev); }
    const rglru_state_grads_t sg{(const float *)ptr(dhT), ptr(dcs), want_state ? (float *)g[8].data_ptr() : nullptr, want_state ? g[9].data_ptr() : nullptr};
    auto f = [&](int i) { return (float *)g[i].data_ptr(); };
    void *const st = current_stream();
    const int32_t rc = unlocked([&] {
        return rglru_backward(&k.s, &k.h->p, ptr(x), (const float *)ptr(h0), ptr(cs), ptr(y), ptr(dy), g[0].data_ptr(), f(1), f(2), f(3), f(4), f(5), f(6), f(7),
                              want_state || dhT || dcs ? &sg : nullptr, w.p, w.n, st);
    });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_backward");
    PyObject *out = PyDict_New();
    if (!out) return nullptr;
    for (int i = 0; i < count; ++i) {
        PyObject *t = wrap(g[i]);
        PyDict_SetItemString(out, names[i], t);
        Py_DECREF(t);
    }
    return out;
    END_HANDLE_TH_ERRORS
}

// ---- the operators around the core
const at::Tensor *optional(PyObject *o, const char *name) {
    if (o == Py_None) return nullptr;
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, ": expected a tensor or None");
    return &THPVariable_Unpack(o);
}
const at::Tensor &required(PyObject *o, const char *name) {
    const at::Tensor *t = optional(o, name);
    TORCH_CHECK_TYPE(t, name, ": expected a tensor");
    return *t;
}
int32_t io_code(const at::Tensor &t, const char *name) {
    TORCH_CHECK_TYPE(t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16, name, ": io dtype must be float32 or bfloat16, got ", t.scalar_type());
    TORCH_CHECK_VALUE(t.is_cuda(), name, ": expected a CUDA tensor (there is no CPU fallback)");
    return t.scalar_type() == at::kBFloat16 ? (int32_t)RGLRU_BF16 : (int32_t)RGLRU_F32;
}
void check(const at::Tensor *t, const char *name, at::IntArrayRef shape, at::ScalarType dtype, c10::Device dev) {
    TORCH_CHECK_VALUE(fits(t, shape, dtype, dev), name, ": expected contiguous ", dtype, " tensor of shape ", shape, " on ", dev, ", got ", t->scalar_type(), " ",
                      t->sizes(), " with strides ", t->strides(), " on ", t->device());
}
double number(PyObject *o, const char *name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); TORCH_CHECK_TYPE(false, name, ": expected a number"); }
    return v;
}
int64_t integer(PyObject *o, const char *name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); TORCH_CHECK_TYPE(false, name, ": expected an integer"); }
    return v;
}
bool truth(PyObject *o, const char *name) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) { PyErr_Clear(); TORCH_CHECK_TYPE(false, name, ": expected True or False"); }
    return v != 0;
}
int32_t int32_size(int64_t v, const char *name) {
    TORCH_CHECK_VALUE(v <= INT32_MAX, name, " is too large: ", v);
    return (int32_t)v;
}
void arguments(Py_ssize_t n, Py_ssize_t want) { TORCH_CHECK_TYPE(n == want, "expected ", want, " arguments, got ", n); }
// The caller's workspace, or scratch of this call
struct Scratch {
    at::Tensor own;
    void *p = nullptr;
    size_t n = 0;
    Scratch(const at::Tensor *given, size_t need, c10::Device dev) {
        if (given) {
            TORCH_CHECK_VALUE(given->scalar_type() == at::kByte && given->device() == dev && given->is_contiguous(), "workspace: expected a contiguous uint8 tensor on ", dev);
            p = given->data_ptr(); n = (size_t)given->numel();
        } else if (need) {
            own = fresh({(int64_t)need}, at::kByte, dev);
            p = own.data_ptr(); n = need;
        }
    }
};
void *stream_of(c10::Device dev) { return (void *)c10::cuda::getCurrentCUDAStream(dev.index()).stream(); }
PyObject *gradients(std::initializer_list<std::pair<const char *, const at::Tensor *>> g) {
    PyObject *out = PyDict_New();
    if (!out) return nullptr;
    for (const auto &[name, t] : g) {
        if (!t->defined()) continue;
        PyObject *v = wrap(*t);
        PyDict_SetItemString(out, name, v);
        Py_DECREF(v);
    }
    return out;
}

rglru_norm_shape_t norm_shape(const at::Tensor &x, bool center, double eps) {
    const int32_t io = io_code(x, "x");
    TORCH_CHECK_VALUE(x.dim() >= 1 && x.is_contiguous(), "x: expected a contiguous tensor of at least one dimension");
    const int64_t N = x.size(-1);
    return {N ? x.numel() / N : 0, int32_size(N, "the last dimension of x"), io, center, (float)eps};
}

// layer_norm(x, weight, bias, eps, center, stats, y) -> y, or (y, mean or None, rstd)
PyObject *layer_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 7);
    const at::Tensor &x = required(a[0], "x");
    const at::Tensor *w = optional(a[1], "weight"), *b = optional(a[2], "bias"), *y = optional(a[6], "y");
    const bool center = truth(a[4], "center"), stats = truth(a[5], "stats");
    const rglru_norm_shape_t s = norm_shape(x, center, number(a[3], "eps"));
    const c10::Device dev = x.device();
    check(w, "weight", {s.N}, at::kFloat, dev); check(b, "bias", {s.N}, at::kFloat, dev); check(y, "y", x.sizes(), x.scalar_type(), dev);
    c10::cuda::CUDAGuard guard(dev);
    const at::Tensor out = y ? *y : fresh(x.sizes(), x.scalar_type(), dev);
    const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
    at::Tensor mean, rstd;
    if (stats) rstd = fresh(lead, at::kFloat, dev);
    if (stats && center) mean = fresh(lead, at::kFloat, dev);
    void *const st = stream_of(dev);
    const int32_t rc = unlocked([&] {
        return rglru_layer_norm(&s, x.data_ptr(), (const float *)ptr(w), (const float *)ptr(b), out.data_ptr(), mean.defined() ? (float *)mean.data_ptr() : nullptr,
                                stats ? (float *)rstd.data_ptr() : nullptr, st);
    });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_layer_norm");
    if (!stats) return wrap(out);
    PyObject *tuple = PyTuple_New(3);
    if (!tuple) return nullptr;
    PyTuple_SET_ITEM(tuple, 0, wrap(out));
    if (center) PyTuple_SET_ITEM(tuple, 1, wrap(mean));
    else { Py_INCREF(Py_None); PyTuple_SET_ITEM(tuple, 1, Py_None); }
    PyTuple_SET_ITEM(tuple, 2, wrap(rstd));
    return tuple;
    END_HANDLE_TH_ERRORS
}

// layer_norm_backward(dy, x, rstd, mean, weight, param_grads, dx, workspace) -> dict of gradients
PyObject *layer_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 8);
    const at::Tensor &dy = required(a[0], "dy"), &x = required(a[1], "x"), &rstd = required(a[2], "rstd");
    const at::Tensor *mean = optional(a[3], "mean"), *w = optional(a[4], "weight"), *given = optional(a[6], "dx"), *ws = optional(a[7], "workspace");
    const bool sums = truth(a[5], "param_grads");
    const rglru_norm_shape_t s = norm_shape(x, mean != nullptr, 0.0);
    const c10::Device dev = x.device();
    const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
    check(&dy, "dy", x.sizes(), x.scalar_type(), dev); check(&rstd, "rstd", lead, at::kFloat, dev); check(mean, "mean", lead, at::kFloat, dev);
    check(w, "weight", {s.N}, at::kFloat, dev); check(given, "dx", x.sizes(), x.scalar_type(), dev);
    c10::cuda::CUDAGuard guard(dev);
    const at::Tensor dx = given ? *given : fresh(x.sizes(), x.scalar_type(), dev);
    at::Tensor dw, db;
    if (sums) { dw = fresh({s.N}, at::kFloat, dev); db = fresh({s.N}, at::kFloat, dev); }
    const Scratch scratch(ws, sums ? rglru_layer_norm_workspace_bytes(&s) : 0, dev);
    void *const st = stream_of(dev);
    const int32_t rc = unlocked([&] {
        return rglru_layer_norm_backward(&s, dy.data_ptr(), x.data_ptr(), (const float *)ptr(mean), (const float *)rstd.data_ptr(), (const float *)ptr(w), dx.data_ptr(),
                                         sums ? (float *)dw.data_ptr() : nullptr, sums ? (float *)db.data_ptr() : nullptr, scratch.p, scratch.n, st);
    });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_layer_norm_backward");
    return gradients({{"x", &dx}, {"weight", &dw}, {"bias", &db}});
    END_HANDLE_TH_ERRORS
}

rglru_linear_shape_t linear_shape(const at::Tensor &rows, const char *rows_name, int64_t width, const at::Tensor &weight, int64_t activation, int64_t flags) {
    const int32_t io = io_code(weight, "weight");
    TORCH_CHECK_VALUE(weight.dim() == 2, "weight: expected [outputs, inputs], got ", weight.sizes());
    TORCH_CHECK_VALUE(rows.dim() >= 1 && rows.size(-1) == width, rows_name, ": expected a last dimension of ", width, ", got ", rows.sizes());
    check(&weight, "weight", weight.sizes(), weight.scalar_type(), weight.device());
    check(&rows, rows_name, rows.sizes(), weight.scalar_type(), weight.device());
    TORCH_CHECK_VALUE(flags >= 0 && flags <= UINT32_MAX, "flags: out of range");
    return {width ? rows.numel() / width : 0, int32_size(weight.size(1), "inputs"), int32_size(weight.size(0), "outputs"), io, (int32_t)activation, (uint32_t)flags};
}
c10::SmallVector<int64_t, 6> with_last(at::IntArrayRef sizes, int64_t last) {
    c10::SmallVector<int64_t, 6> v(sizes.begin(), sizes.end());
    v.back() = last;
    return v;
}

// linear(x, weight, bias, activation, residual, y, keep_preact, flags, workspace) -> y, or (y, preact)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 9);
    const at::Tensor &x = required(a[0], "x"), &w = required(a[1], "weight");
    const at::Tensor *b = optional(a[2], "bias"), *res = optional(a[4], "residual"), *y = optional(a[5], "y"), *ws = optional(a[8], "workspace");
    const bool keep = truth(a[6], "keep_preact");
    TORCH_CHECK_VALUE(w.dim() == 2, "weight: expected [outputs, inputs], got ", w.sizes());
    const rglru_linear_shape_t s = linear_shape(x, "x", w.size(1), w, integer(a[3], "activation"), integer(a[7], "flags"));
    const c10::Device dev = w.device();
    const at::ScalarType io = w.scalar_type();
    const auto shape = with_last(x.sizes(), s.N);
    check(b, "bias", {s.N}, at::kFloat, dev); check(res, "residual", shape, io, dev); check(y, "y", shape, io, dev);
    c10::cuda::CUDAGuard guard(dev);
    const at::Tensor out = y ? *y : fresh(shape, io, dev);
    at::Tensor pre;
    if (keep) pre = fresh(shape, io, dev);
    const Scratch scratch(ws, rglru_linear_workspace_bytes(&s, RGLRU_OP_PREFILL), dev);
    void *const st = stream_of(dev);
    const int32_t rc = unlocked([&] {
        return rglru_linear(&s, x.data_ptr(), w.data_ptr(), (const float *)ptr(b), ptr(res), out.data_ptr(), keep ? pre.data_ptr() : nullptr, scratch.p, scratch.n, st);
    });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_linear");
    if (!keep) return wrap(out);
    PyObject *tuple = PyTuple_New(2);
    if (!tuple) return nullptr;
    PyTuple_SET_ITEM(tuple, 0, wrap(out)); PyTuple_SET_ITEM(tuple, 1, wrap(pre));
    return tuple;
    END_HANDLE_TH_ERRORS
}

// linear_backward(dy, x, weight, preact, activation, want_x, want_weight, want_bias, flags, workspace) -> dict of gradients
PyObject *linear_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 10);
    const at::Tensor &dy = required(a[0], "dy"), &x = required(a[1], "x"), &w = required(a[2], "weight");
    const at::Tensor *pre = optional(a[3], "preact"), *ws = optional(a[9], "workspace");
    const bool wx = PyObject_IsTrue(a[5]) > 0, ww = PyObject_IsTrue(a[6]) > 0, wb = PyObject_IsTrue(a[7]) > 0;
    TORCH_CHECK_VALUE(w.dim() == 2, "weight: expected [outputs, inputs], got ", w.sizes());
    const rglru_linear_shape_t s = linear_shape(x, "x", w.size(1), w, integer(a[4], "activation"), integer(a[8], "flags"));
    const c10::Device dev = w.device();
    const at::ScalarType io = w.scalar_type();
    const auto shape = with_last(x.sizes(), s.N);
    TORCH_CHECK_VALUE(s.activation == RGLRU_ACT_NONE || pre, "preact: the backward through an activation needs what linear(..., keep_preact=True) returned");
    check(&dy, "dy", shape, io, dev); check(pre, "preact", shape, io, dev);
    c10::cuda::CUDAGuard guard(dev);
    at::Tensor dx, dw, db;
    if (wx) dx = fresh(x.sizes(), io, dev);
    if (ww) dw = fresh(w.sizes(), io, dev);
    if (wb) db = fresh({s.N}, at::kFloat, dev);
    const Scratch scratch(ws, rglru_linear_workspace_bytes(&s, RGLRU_OP_BACKWARD), dev);
    void *const st = stream_of(dev);
    const int32_t rc = unlocked([&] {
        return rglru_linear_backward(&s, dy.data_ptr(), x.data_ptr(), w.data_ptr(), ptr(pre), wx ? dx.data_ptr() : nullptr, ww ? dw.data_ptr() : nullptr,
                                     wb ? (float *)db.data_ptr() : nullptr, scratch.p, scratch.n, st);
    });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_linear_backward");
    return gradients({{"x", &dx}, {"weight", &dw}, {"bias", &db}});
    END_HANDLE_TH_ERRORS
}

// [B,T,H,width] with the heads of a token side by side; the distances between tokens and between sequences are free
rglru_stride_t token_strides(const at::Tensor &t, const char *name, int64_t B, int64_t T, int64_t H, int64_t width, at::ScalarType io, c10::Device dev) {
    TORCH_CHECK_VALUE(t.dim() == 4 && t.size(0) == B && t.size(1) == T && t.size(2) == H && t.size(3) == width && t.scalar_type() == io && t.device() == dev,
                      name, ": expected ", io, " tensor of shape [", B, ", ", T, ", ", H, ", ", width, "] on ", dev, ", got ", t.scalar_type(), " ", t.sizes(), " on ", t.device());
    const int64_t row = H * width, token = T == 1 ? row : t.stride(1), batch = B == 1 ? (T - 1) * token + row : t.stride(0);
    TORCH_CHECK_VALUE((width == 1 || t.stride(3) == 1) && (H == 1 || t.stride(2) == width) && token >= row && batch >= row,
                      name, ": the heads of a token have to lie side by side and no token over another, got strides ", t.strides());
    return {token, batch};
}
rglru_linear_attention_shape_t mix_shape(const at::Tensor &q, const at::Tensor &v, int dims, PyObject *scale, int64_t flags) {
    const int32_t io = io_code(q, "q");
    TORCH_CHECK_VALUE(q.dim() == dims && v.dim() == dims, "q, v: expected ", dims, " dimensions, got ", q.sizes(), " and ", v.sizes());
    TORCH_CHECK_VALUE(flags >= 0 && flags <= UINT32_MAX, "flags: out of range");
    rglru_linear_attention_shape_t s{};
    s.B = int32_size(q.size(0), "sequences"); s.T = dims == 4 ? int32_size(q.size(1), "tokens") : 1; s.H = int32_size(q.size(dims - 2), "heads");
    s.dk = int32_size(q.size(dims - 1), "the width of q"); s.dv = int32_size(v.size(dims - 1), "the width of v");
    s.io = io; s.flags = (uint32_t)flags;
    s.scale = scale == Py_None ? (float)(1.0 / std::sqrt((double)std::max(s.dk, 1))) : (float)number(scale, "scale");
    return s;
}

// linear_attention_prefill(q, k, v, log_decay, s0, scale, o, s_T, flags, workspace) -> (o, s_T)
PyObject *linear_attention_prefill(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 10);
    const at::Tensor &q = required(a[0], "q"), &k = required(a[1], "k"), &v = required(a[2], "v"), &decay = required(a[3], "log_decay");
    const at::Tensor *s0 = optional(a[4], "s0"), *o = optional(a[6], "o"), *sT = optional(a[7], "s_T"), *ws = optional(a[9], "workspace");
    const rglru_linear_attention_shape_t s = mix_shape(q, v, 4, a[5], integer(a[8], "flags"));
    const c10::Device dev = q.device();
    const at::ScalarType io = q.scalar_type();
    rglru_linear_attention_strides_t st{};
    st.q = token_strides(q, "q", s.B, s.T, s.H, s.dk, io, dev);
    st.k = token_strides(k, "k", s.B, s.T, s.H, s.dk, io, dev);
    st.v = token_strides(v, "v", s.B, s.T, s.H, s.dv, io, dev);
    if (o) st.o = token_strides(*o, "o", s.B, s.T, s.H, s.dv, io, dev);
    check(&decay, "log_decay", {s.H}, at::kFloat, dev);
    check(s0, "s0", {s.B, s.H, s.dk, s.dv}, at::kFloat, dev); check(sT, "s_T", {s.B, s.H, s.dk, s.dv}, at::kFloat, dev);
    c10::cuda::CUDAGuard guard(dev);
    const at::Tensor ot = o ? *o : fresh({s.B, s.T, s.H, s.dv}, io, dev), stt = sT ? *sT : fresh({s.B, s.H, s.dk, s.dv}, at::kFloat, dev);
    const Scratch scratch(ws, rglru_linear_attention_workspace_bytes(&s, RGLRU_OP_PREFILL), dev);
    void *const stream = stream_of(dev);
    const int32_t rc = unlocked([&] {
        return rglru_linear_attention_prefill(&s, &st, q.data_ptr(), k.data_ptr(), v.data_ptr(), (const float *)decay.data_ptr(), (const float *)ptr(s0), ot.data_ptr(),
                                              (float *)stt.data_ptr(), scratch.p, scratch.n, stream);
    });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_linear_attention_prefill");
    PyObject *tuple = PyTuple_New(2);
    if (!tuple) return nullptr;
    PyTuple_SET_ITEM(tuple, 0, wrap(ot)); PyTuple_SET_ITEM(tuple, 1, wrap(stt));
    return tuple;
    END_HANDLE_TH_ERRORS
}

// linear_attention_decode_step(q, k, v, log_decay, s, scale, o) -> o
PyObject *linear_attention_decode_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 7);
    const at::Tensor &q = required(a[0], "q"), &k = required(a[1], "k"), &v = required(a[2], "v"), &decay = required(a[3], "log_decay"), &state = required(a[4], "s");
    const at::Tensor *o = optional(a[6], "o");
    const rglru_linear_attention_shape_t s = mix_shape(q, v, 3, a[5], 0);
    const c10::Device dev = q.device();
    const at::ScalarType io = q.scalar_type();
    check(&q, "q", {s.B, s.H, s.dk}, io, dev); check(&k, "k", {s.B, s.H, s.dk}, io, dev); check(&v, "v", {s.B, s.H, s.dv}, io, dev);
    check(&decay, "log_decay", {s.H}, at::kFloat, dev); check(&state, "s", {s.B, s.H, s.dk, s.dv}, at::kFloat, dev); check(o, "o", {s.B, s.H, s.dv}, io, dev);
    c10::cuda::CUDAGuard guard(dev);
    const at::Tensor ot = o ? *o : fresh({s.B, s.H, s.dv}, io, dev);
    void *const stream = stream_of(dev);
    const int32_t rc = unlocked([&] {
        return rglru_linear_attention_decode_step(&s, q.data_ptr(), k.data_ptr(), v.data_ptr(), (const float *)decay.data_ptr(), (float *)state.data_ptr(), ot.data_ptr(),
                                                  stream);
    });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_linear_attention_decode_step");
    return wrap(ot);
    END_HANDLE_TH_ERRORS
}

// linear_attention_backward(q, k, v, log_decay, do, s0, ds_T, scale, state_grads, dq, dk, dv, flags, workspace) -> dict of gradients
PyObject *linear_attention_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 14);
    const at::Tensor &q = required(a[0], "q"), &k = required(a[1], "k"), &v = required(a[2], "v"), &decay = required(a[3], "log_decay"), &dout = required(a[4], "do");
    const at::Tensor *s0 = optional(a[5], "s0"), *dsT = optional(a[6], "ds_T"), *gq = optional(a[9], "dq"), *gk = optional(a[10], "dk"), *gv = optional(a[11], "dv"),
                     *ws = optional(a[13], "workspace");
    const bool want_state = truth(a[8], "state_grads");
    const rglru_linear_attention_shape_t s = mix_shape(q, v, 4, a[7], integer(a[12], "flags"));
    const c10::Device dev = q.device();
    const at::ScalarType io = q.scalar_type();
    rglru_linear_attention_strides_t st{};
    st.q = token_strides(q, "q", s.B, s.T, s.H, s.dk, io, dev);
    st.k = token_strides(k, "k", s.B, s.T, s.H, s.dk, io, dev);
    st.v = token_strides(v, "v", s.B, s.T, s.H, s.dv, io, dev);
    st.o = token_strides(dout, "do", s.B, s.T, s.H, s.dv, io, dev);
    if (gq) st.dq = token_strides(*gq, "dq", s.B, s.T, s.H, s.dk, io, dev);
    if (gk) st.dk = token_strides(*gk, "dk", s.B, s.T, s.H, s.dk, io, dev);
    if (gv) st.dv = token_strides(*gv, "dv", s.B, s.T, s.H, s.dv, io, dev);
    check(&decay, "log_decay", {s.H}, at::kFloat, dev);
    check(s0, "s0", {s.B, s.H, s.dk, s.dv}, at::kFloat, dev); check(dsT, "ds_T", {s.B, s.H, s.dk, s.dv}, at::kFloat, dev);
    c10::cuda::CUDAGuard guard(dev);
    const at::Tensor dq = gq ? *gq : fresh({s.B, s.T, s.H, s.dk}, io, dev), dk = gk ? *gk : fresh({s.B, s.T, s.H, s.dk}, io, dev),
                     dv = gv ? *gv : fresh({s.B, s.T, s.H, s.dv}, io, dev);
    at::Tensor ds0;
    if (want_state) ds0 = fresh({s.B, s.H, s.dk, s.dv}, at::kFloat, dev);
    const Scratch scratch(ws, rglru_linear_attention_workspace_bytes(&s, RGLRU_OP_BACKWARD), dev);
    void *const stream = stream_of(dev);
    const int32_t rc = unlocked([&] {
        return rglru_linear_attention_backward(&s, &st, q.data_ptr(), k.data_ptr(), v.data_ptr(), (const float *)decay.data_ptr(), (const float *)ptr(s0), dout.data_ptr(),
                                               (const float *)ptr(dsT), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), want_state ? (float *)ds0.data_ptr() : nullptr,
                                               scratch.p, scratch.n, stream);
    });
    if (rc != RGLRU_OK) return raise_status(rc, "rglru_linear_attention_backward");
    return gradients({{"q", &dq}, {"k", &dk}, {"v", &dv}, {"s0", &ds0}});
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"set_error_type", set_error_type, METH_O, nullptr},
    {"params_handle", (PyCFunction)(void (*)(void))params_handle, METH_FASTCALL, nullptr},
    {"prefill", (PyCFunction)(void (*)(void))prefill, METH_FASTCALL, nullptr},
    {"decode_step", (PyCFunction)(void (*)(void))decode_step, METH_FASTCALL, nullptr},
    {"backward", (PyCFunction)(void (*)(void))backward, METH_FASTCALL, nullptr},
    {"layer_norm", (PyCFunction)(void (*)(void))layer_norm, METH_FASTCALL, nullptr},
    {"layer_norm_backward", (PyCFunction)(void (*)(void))layer_norm_backward, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
    {"linear_backward", (PyCFunction)(void (*)(void))linear_backward, METH_FASTCALL, nullptr},
    {"linear_attention_prefill", (PyCFunction)(void (*)(void))linear_attention_prefill, METH_FASTCALL, nullptr},
    {"linear_attention_decode_step", (PyCFunction)(void (*)(void))linear_attention_decode_step, METH_FASTCALL, nullptr},
    {"linear_attention_backward", (PyCFunction)(void (*)(void))linear_attention_backward, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host(void) { return PyModule_Create(&module); }
