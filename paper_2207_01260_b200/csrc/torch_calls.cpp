// The operators' calls as programs make them most of the time (tensors that are in order, results allocated by the call, the current stream), without
// the interpreter between the checks: what a small call costs is spent on the host.  A function here checks its tensors, allocates the results and calls the C
// ABI; where anything is not in order, or the library refuses, it returns None, and binding.py goes through the same steps itself and says what is wrong.  Where
// the library fails on the way (CUDA), part of the work may be under way: that is raised here, and nothing is tried again.
// (us a call of a 7x7x352 image's group norm: 12.7 by binding.py's own steps, 5.8 here.)
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstring>
#include <utility>
#include <vector>

#include "cprune.h"

namespace {

// the library's functions, handed over by binding.py (which loads the library)
struct Library {
    decltype(&cprune_padded_channels) padded_channels;
    decltype(&cprune_group_norm_workspace_bytes) group_norm_workspace_bytes;
    decltype(&cprune_group_norm) group_norm;
    decltype(&cprune_group_norm_backward) group_norm_backward;
    decltype(&cprune_gradient_workspace_bytes) gradient_workspace_bytes;
    decltype(&cprune_clip_gradients) clip_gradients;
    decltype(&cprune_mx_quantize) mx_quantize;
    decltype(&cprune_mx_fc_workspace_bytes) mx_fc_workspace_bytes;
    decltype(&cprune_mx_fc) mx_fc;
} lib;

using Dims = c10::ArrayRef<int64_t>;

// A tensor argument: `in_order` when it is None, or of this type and shape, contiguous and on the current device
struct Argument {
    const at::Tensor *t = nullptr;
    bool in_order = true;
    explicit Argument(PyObject *o) {
        if (o == Py_None) return;
        if (THPVariable_Check(o)) t = &THPVariable_Unpack(o);
        else in_order = false;
    }
    bool is(at::ScalarType type, Dims shape, c10::DeviceIndex device) const {
        return in_order && (!t || (t->is_cuda() && t->device().index() == device && t->scalar_type() == type && t->sizes() == shape && t->is_contiguous()));
    }
    bool given(at::ScalarType type, Dims shape, c10::DeviceIndex device) const { return t && is(type, shape, device); }
    void *address() const { return t ? t->data_ptr() : nullptr; }
};

int library_type(at::ScalarType t) { return t == at::kBFloat16 ? CPRUNE_TYPE_BF16 : t == at::kFloat ? CPRUNE_TYPE_F32 : -1; }

// Runs f without the interpreter's lock, so that a launch that has to wait holds up nobody else (an exception takes the lock back first)
template <typename F> cprune_status call(F f) {
    struct Unlocked {
        PyThreadState *state = PyEval_SaveThread();
        ~Unlocked() { PyEval_RestoreThread(state); }
    } unlocked;
    return f();
}
PyObject *none() {
    PyErr_Clear();
    Py_RETURN_NONE;
}
PyObject *raise_for;                    // binding.py's function that raises for a status

// What a call returns that has not succeeded: None where its arguments were refused (nothing is under way), else an exception
PyObject *failed(cprune_status s, const char *where) {
    if (s == CPRUNE_ERR_INVALID_ARG || s == CPRUNE_ERR_UNSUPPORTED || s == CPRUNE_ERR_WORKSPACE_TOO_SMALL) return none();
    PyObject *r = PyObject_CallFunction(raise_for, "is", (int)s, where);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, where);
    return nullptr;
}
PyObject *pack(std::initializer_list<PyObject *> items) {
    PyObject *r = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject *o : items) PyTuple_SET_ITEM(r, i++, o);
    return r;
}
PyObject *no_object() { Py_RETURN_NONE; }
void *stream() { return (void *)c10::cuda::getCurrentCUDAStream().stream(); }
at::Tensor bytes_like(const at::Tensor &t, size_t n) { return n ? at::empty({(int64_t)n}, t.options().dtype(at::kByte)) : at::Tensor(); }

// (no C++ exception may leave through the interpreter: out of memory, for one, is told by the other way's allocation)
template <typename F> PyObject *guarded(F f) {
    try {
        return f();
    } catch (...) {
        return none();
    }
}

// an integer argument; anything else, or one that an int does not hold, is an error
int as_int(PyObject *o) {
    const long v = PyLong_AsLong(o);
    if (v != (int)v && !PyErr_Occurred()) PyErr_SetString(PyExc_OverflowError, "not an int");
    return (int)v;
}

// x, dtype and geometry of an activation [N, H, W, channels in memory]
struct Activation {
    Argument x;
    int type = -1;
    c10::DeviceIndex device = -1;
    Activation(PyObject *o, int C, size_t dims) : x(o) {
        if (!x.t || !x.t->is_cuda()) return;
        device = c10::cuda::current_device();
        const int t = library_type(x.t->scalar_type());
        const auto s = x.t->sizes();
        if (t < 0 || (dims && s.size() != dims) || s.empty() || C < 1 || C > (1 << 24) || x.t->device().index() != device || !x.t->is_contiguous()) return;
        for (auto n : s)
            if (n > 0x7fffffff) return;
        if (s.back() == (t == CPRUNE_TYPE_BF16 ? lib.padded_channels(C) : C)) type = t;
    }
};

// group_norm(x, C, groups, gamma, beta, eps, activation, residual) -> (y, stats)
PyObject *group_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 8) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const int C = as_int(a[1]), groups = as_int(a[2]), act = as_int(a[6]);
        const double eps = PyFloat_AsDouble(a[5]);
        if (PyErr_Occurred()) return none();
        const Activation v(a[0], C, 4);
        const Argument gamma(a[3]), beta(a[4]), res(a[7]);
        const int64_t channels[1] = {C};
        if (v.type < 0 || groups < 1 || !gamma.is(at::kFloat, channels, v.device) || !beta.is(at::kFloat, channels, v.device) ||
            !res.is(v.x.t->scalar_type(), v.x.t->sizes(), v.device)) return none();
        const at::Tensor &x = *v.x.t;
        const int N = (int)x.size(0), H = (int)x.size(1), W = (int)x.size(2);
        const size_t need = lib.group_norm_workspace_bytes(v.type, N, H, W, C, groups, 0);
        at::Tensor y = at::empty(x.sizes(), x.options()), stats = at::empty({N, groups, 2}, x.options().dtype(at::kFloat)), work = bytes_like(x, need);
        const cprune_status st = call([&] {
            return lib.group_norm(x.data_ptr(), v.type, N, H, W, C, groups, (const float *)gamma.address(), (const float *)beta.address(), (float)eps, act, res.address(),
                                  y.data_ptr(), (float *)stats.data_ptr(), need ? work.data_ptr() : nullptr, need, stream());
        });
        if (st != CPRUNE_OK) return failed(st, "cprune_group_norm");
        return pack({THPVariable_Wrap(y), THPVariable_Wrap(stats)});
    });
}

// group_norm_backward(dy, x, C, groups, stats, gamma, beta, activation, residual) -> (dx, dgamma, dbeta, dresidual)
PyObject *group_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const int C = as_int(a[2]), groups = as_int(a[3]), act = as_int(a[7]);
        if (PyErr_Occurred()) return none();
        const Activation v(a[1], C, 4);
        const Argument dy(a[0]), stats(a[4]), gamma(a[5]), beta(a[6]), res(a[8]);
        if (v.type < 0 || groups < 1) return none();
        const at::Tensor &x = *v.x.t;
        const int64_t channels[1] = {C}, kept[3] = {x.size(0), groups, 2};
        if (!dy.given(x.scalar_type(), x.sizes(), v.device) || !stats.given(at::kFloat, kept, v.device) || !gamma.is(at::kFloat, channels, v.device) ||
            !beta.is(at::kFloat, channels, v.device) || !res.is(x.scalar_type(), x.sizes(), v.device)) return none();
        const int N = (int)x.size(0), H = (int)x.size(1), W = (int)x.size(2);
        const size_t need = lib.group_norm_workspace_bytes(v.type, N, H, W, C, groups, 1);
        const auto f32 = x.options().dtype(at::kFloat);
        at::Tensor dx = at::empty(x.sizes(), x.options()), dgamma = at::empty({C}, f32), dbeta = at::empty({C}, f32), work = bytes_like(x, need), dres;
        if (res.t) dres = at::empty(x.sizes(), x.options());
        const cprune_status st = call([&] {
            return lib.group_norm_backward(dy.address(), x.data_ptr(), v.type, N, H, W, C, groups, (const float *)stats.address(), (const float *)gamma.address(),
                                           (const float *)beta.address(), act, res.address(), dx.data_ptr(), (float *)dgamma.data_ptr(), (float *)dbeta.data_ptr(),
                                           res.t ? dres.data_ptr() : nullptr, need ? work.data_ptr() : nullptr, need, stream());
        });
        if (st != CPRUNE_OK) return failed(st, "cprune_group_norm_backward");
        return pack({THPVariable_Wrap(dx), THPVariable_Wrap(dgamma), THPVariable_Wrap(dbeta), res.t ? THPVariable_Wrap(dres) : no_object()});
    });
}

// Addresses, counts and types of a list of gradients; whether all are in order (by themselves)
struct GradientList {
    std::vector<void *> addresses;
    std::vector<unsigned long long> counts;
    std::vector<int> types;
    bool read(PyObject *list, c10::DeviceIndex device) {
        if (!PyList_Check(list) && !PyTuple_Check(list)) return false;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
        addresses.reserve(n);
        counts.reserve(n);
        types.reserve(n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            const Argument g(PySequence_Fast_GET_ITEM(list, i));
            if (!g.t || !g.t->is_cuda() || g.t->device().index() != device || !g.t->is_contiguous()) return false;
            const int type = library_type(g.t->scalar_type());
            if (type < 0) return false;
            addresses.push_back(g.t->data_ptr());
            counts.push_back((unsigned long long)g.t->numel());
            types.push_back(type);
        }
        return true;
    }
};

// Whether tensors of the list share memory, with one another or with results that are not in their own place
bool overlap(const GradientList &g, const GradientList *out) {
    std::vector<std::pair<uintptr_t, uintptr_t>> runs;
    runs.reserve(2 * g.addresses.size());
    for (size_t i = 0; i < g.addresses.size(); ++i) {
        if (!g.counts[i]) continue;
        const uintptr_t bytes = g.counts[i] * (g.types[i] == CPRUNE_TYPE_BF16 ? 2 : 4), at = (uintptr_t)g.addresses[i];
        runs.emplace_back(at, at + bytes);
        if (out && out->addresses[i] != g.addresses[i]) runs.emplace_back((uintptr_t)out->addresses[i], (uintptr_t)out->addresses[i] + bytes);
    }
    std::sort(runs.begin(), runs.end());
    for (size_t i = 1; i < runs.size(); ++i)
        if (runs[i].first < runs[i - 1].second) return true;
    return false;
}

// clip_gradients(grads, max_norm, out) -> norm
PyObject *clip_gradients(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 3) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const double max_norm = PyFloat_AsDouble(a[1]);
        if (PyErr_Occurred()) return none();
        const c10::DeviceIndex device = c10::cuda::current_device();
        GradientList g, o;
        if (!g.read(a[0], device) || g.addresses.empty()) return none();
        if (a[2] != Py_None && (!o.read(a[2], device) || o.counts != g.counts || o.types != g.types)) return none();
        if (overlap(g, a[2] != Py_None ? &o : nullptr)) return none();
        const int count = (int)g.addresses.size();
        const size_t need = lib.gradient_workspace_bytes(count);
        const auto like = at::TensorOptions().device(at::kCUDA, device);
        at::Tensor norm = at::empty({1}, like.dtype(at::kFloat)), work = at::empty({(int64_t)need}, like.dtype(at::kByte));
        const cprune_status st = call([&] {
            return lib.clip_gradients(g.addresses.data(), g.counts.data(), g.types.data(), count, (float)max_norm, a[2] != Py_None ? o.addresses.data() : nullptr,
                                      (float *)norm.data_ptr(), work.data_ptr(), need, stream());
        });
        if (st != CPRUNE_OK) return failed(st, "cprune_clip_gradients");
        return THPVariable_Wrap(norm);
    });
}

int64_t rows_of(const at::Tensor &x) {
    int64_t rows = 1;
    for (size_t i = 0; i + 1 < x.sizes().size(); ++i) rows *= x.size(i);
    return rows;
}

// mx_quantize(x, C, values) -> (codes, scales, values or None)
PyObject *mx_quantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 3) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const int C = as_int(a[1]);
        if (PyErr_Occurred()) return none();
        const Activation v(a[0], C, 0);
        if (v.type < 0) return none();
        const at::Tensor &x = *v.x.t;
        const int64_t rows = rows_of(x), blocks = (C + 31) / 32;
        const auto u8 = x.options().dtype(at::kByte);
        const bool with_values = a[2] == Py_True;
        at::Tensor codes = at::empty({rows, blocks * 16}, u8), scales = at::empty({(rows + 127) / 128, (blocks + 3) / 4, 32, 4, 4}, u8), values;
        if (with_values) values = at::empty(x.sizes(), x.options());
        const cprune_status st = call([&] {
            return lib.mx_quantize(x.data_ptr(), v.type, (size_t)rows, C, codes.data_ptr(), scales.data_ptr(), with_values ? values.data_ptr() : nullptr, stream());
        });
        if (st != CPRUNE_OK) return failed(st, "cprune_mx_quantize");
        return pack({THPVariable_Wrap(codes), THPVariable_Wrap(scales), with_values ? THPVariable_Wrap(values) : no_object()});
    });
}

// mx_fc(x, in, codes, scales, b_packed, out, activation, residual, out_f32) -> y
PyObject *mx_fc(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const int in = as_int(a[1]), out = as_int(a[5]), act = as_int(a[6]), f32 = PyObject_IsTrue(a[8]);
        if (PyErr_Occurred() || out < 1 || out > (1 << 24)) return none();
        const Activation v(a[0], in, 0);
        if (v.type != CPRUNE_TYPE_BF16) return none();
        const at::Tensor &x = *v.x.t;
        const Argument codes(a[2]), scales(a[3]), bias(a[4]), res(a[7]);
        const int64_t rows = rows_of(x), blocks = (in + 31) / 32, out_pad = lib.padded_channels(out);
        const int64_t shape_c[2] = {out, blocks * 16}, shape_s[5] = {(out + 127) / 128, (blocks + 3) / 4, 32, 4, 4}, shape_b[1] = {out_pad};
        std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = out_pad;
        if (!codes.given(at::kByte, shape_c, v.device) || !scales.given(at::kByte, shape_s, v.device) || !bias.given(at::kFloat, shape_b, v.device) ||
            !res.is(at::kBFloat16, shape, v.device)) return none();
        if (f32) shape.back() = out;
        const size_t need = lib.mx_fc_workspace_bytes((size_t)rows, in, out);
        at::Tensor y = at::empty(shape, x.options().dtype(f32 ? at::kFloat : at::kBFloat16)), work = bytes_like(x, need);
        const cprune_status st = call([&] {
            return lib.mx_fc(x.data_ptr(), (size_t)rows, in, codes.address(), scales.address(), (const float *)bias.address(), out, act, res.address(), f32, y.data_ptr(),
                             need ? work.data_ptr() : nullptr, need, stream());
        });
        if (st != CPRUNE_OK) return failed(st, "cprune_mx_fc");
        return THPVariable_Wrap(y);
    });
}

// load(function that raises for a status, addresses of the library's functions in the order of `Library`)
PyObject *load(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 1 + (Py_ssize_t)(sizeof(Library) / sizeof(void *))) {
        PyErr_SetString(PyExc_TypeError, "load: a function that raises, the library's functions, one by one");
        return nullptr;
    }
    void *f[sizeof(Library) / sizeof(void *)];
    for (Py_ssize_t i = 1; i < n; ++i)
        if (!(f[i - 1] = PyLong_AsVoidPtr(a[i]))) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "load: a function without an address");
            return nullptr;
        }
    std::memcpy(&lib, f, sizeof(Library));
    Py_INCREF(a[0]);
    Py_XDECREF(raise_for);
    raise_for = a[0];
    Py_RETURN_NONE;
}

#define CALL(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(load), CALL(group_norm), CALL(group_norm_backward), CALL(clip_gradients), CALL(mx_quantize), CALL(mx_fc), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods};

}  // namespace

// (build.py looks for this text in the built file)
PyMODINIT_FUNC PyInit__torch_calls() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built", BUILT_FOR) < 0) Py_CLEAR(m);
    return m;
}
