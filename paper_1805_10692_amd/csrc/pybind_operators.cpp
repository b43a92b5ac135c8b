// The operators beside a projection as native functions of the binding (_cerops): rms_norm, rms_norm_backward, adapter_matmul, adapter_backward,
// grad_norm, grad_clip.
//
// A call takes up to eight tensors and a decode step's call lasts some microseconds on the GPU.  Read through their Python attributes, a
// tensor's shape, strides, type, device and address cost 0.6 us (torch makes a new object for each); torch's C++ interface gives them in some
// nanoseconds.  The entry points' addresses are handed over by binding.py when it has loaded the library (`bind`).
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>
#include <vector>

#include "../../include/cer.h"

namespace {

using NormFn = decltype(&rms_norm);
using NormBackwardFn = decltype(&rms_norm_backward);
using AdapterFn = decltype(&adapter_matmul);
using AdapterBackwardFn = decltype(&adapter_backward);
using NormOfFn = decltype(&grad_norm);
using ClipFn = decltype(&grad_clip);
struct {
    NormFn norm;
    NormBackwardFn norm_backward;
    AdapterFn adapter;
    AdapterBackwardFn adapter_backward;
    NormOfFn grad_norm;
    ClipFn grad_clip;
} g_fn = {};

PyObject* g_check = nullptr;       // binding._check(rc, name): raises for an error code
PyObject* g_get_device = nullptr;  // torch._C._cuda_getDevice, ._cuda_getCurrentRawStream
PyObject* g_raw_stream = nullptr;
PyObject* s_cuda_stream = nullptr;
constexpr int kInt32 = 100;  // beside CER_TYPE_*

bool fail(const char* what, const char* why) {
    PyErr_Format(PyExc_ValueError, "%s %s", what, why);
    return false;
}

// The arguments of a call by position and name, nullptr where not given (or None).
struct Signature {
    const char* name;
    int required, count;
    const char* const* names;
};
bool take(const Signature& f, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames, PyObject** a) {
    for (int i = 0; i < f.count; ++i) a[i] = nullptr;
    if (nargs > f.count) {
        PyErr_Format(PyExc_TypeError, "%s() takes at most %d positional arguments but %zd were given", f.name, f.count, nargs);
        return false;
    }
    for (Py_ssize_t i = 0; i < nargs; ++i) a[i] = args[i];
    const Py_ssize_t nkw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    for (Py_ssize_t k = 0; k < nkw; ++k) {
        PyObject* name = PyTuple_GET_ITEM(kwnames, k);
        int i = 0;
        while (i < f.count && PyUnicode_CompareWithASCIIString(name, f.names[i]) != 0) ++i;
        if (i == f.count) {
            PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", f.name, name);
            return false;
        }
        if (a[i]) {
            PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%s'", f.name, f.names[i]);
            return false;
        }
        a[i] = args[nargs + k];
    }
    for (int i = 0; i < f.count; ++i) {
        if (a[i] == Py_None) a[i] = nullptr;
        if (!a[i] && i < f.required) {
            PyErr_Format(PyExc_TypeError, "%s() missing required argument '%s'", f.name, f.names[i]);
            return false;
        }
    }
    return true;
}

const at::Tensor* tensor_of(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a torch tensor", what);
        return nullptr;
    }
    const at::Tensor* t = &THPVariable_Unpack(o);
    if (t->layout() == at::kStrided) return t;
    fail(what, "must be a dense tensor");
    return nullptr;
}
int type_of(const at::Tensor& t) {  // -1: another one
    switch (t.scalar_type()) {
        case at::kFloat: return CER_TYPE_F32;
        case at::kBFloat16: return CER_TYPE_BF16;
        case at::kHalf: return CER_TYPE_F16;
        case at::kFloat8_e4m3fn: return CER_TYPE_F8;
        case at::kInt: return kInt32;
        default: return -1;
    }
}

// All tensors of a call: in device memory, on the current device.  The stream is asked for when there has been one (torch has initialised the
// device then).
struct Device {
    long current = -1;
    bool has(const at::Tensor& t, const char* what) {
        if (!t.is_cuda()) return fail(what, "must be in device memory");
        if (current < 0) {
            PyObject* v = PyObject_CallNoArgs(g_get_device);
            if (!v) return false;
            current = PyLong_AsLong(v);
            Py_DECREF(v);
            if (current == -1 && PyErr_Occurred()) return false;
        }
        if (t.get_device() != current) return fail(what, "is on another device than the current one");
        return true;
    }
    // None: the current torch stream of the current device; an int; or an object with .cuda_stream.
    bool stream(PyObject* s, void** out) {
        PyObject* v;
        if (!s) {
            PyObject* device = PyLong_FromLong(current);
            v = device ? PyObject_CallOneArg(g_raw_stream, device) : nullptr;
            Py_XDECREF(device);
        } else if (PyLong_Check(s)) {
            Py_INCREF(s);
            v = s;
        } else {
            v = PyObject_GetAttr(s, s_cuda_stream);
        }
        if (!v) return false;
        *out = PyLong_AsVoidPtr(v);
        Py_DECREF(v);
        return *out || !PyErr_Occurred();
    }
};

// (tokens, features), either dimension contiguous.  *tokens, *features: -1 takes the tensor's, else they have to be.
bool tokens_of(PyObject* o, const char* what, Device& dev, cer_tokens_t* out, int64_t* tokens, int64_t* features) {
    const at::Tensor* t = tensor_of(o, what);
    if (!t || !dev.has(*t, what)) return false;
    if (t->dim() != 2) return fail(what, "must have 2 dimensions");
    const int type = type_of(*t);
    if (type < 0 || type == kInt32) return fail(what, "must be float32, bfloat16, float16 or float8_e4m3fn");
    const int64_t size[2] = {t->sizes()[0], t->sizes()[1]}, stride[2] = {t->strides()[0], t->strides()[1]};
    if (*tokens < 0) *tokens = size[0];
    if (*features < 0) *features = size[1];
    if (size[0] != *tokens || size[1] != *features) return fail(what, "has another shape than the other arguments ask for");
    out->type = type;
    if (stride[1] == 1 || size[1] <= 1) {
        out->order = CER_ORDER_ROWS;
        out->ld = stride[0];
    } else if (stride[0] == 1 || size[0] <= 1) {
        out->order = CER_ORDER_COLUMNS;
        out->ld = stride[1];
    } else {
        return fail(what, "must have one contiguous dimension");
    }
    if (size[0] <= 1 && out->order == CER_ORDER_ROWS) out->ld = size[1];  // not used: one token
    if (size[0] == 0 || size[1] == 0) out->ld = 0;
    out->data = t->data_ptr();
    return true;
}
// A single token's or feature's order is both of them: the one that the call's other matrices have.
void same_order(cer_tokens_t* m, const cer_tokens_t& as, int64_t tokens, int64_t features) {
    if (!m->data || m->order == as.order) return;
    if (tokens == 1 && m->order == CER_ORDER_ROWS) {  // rows with features side by side: columns of one token, ld 1
        m->order = CER_ORDER_COLUMNS;
        m->ld = 1;
    } else if (features == 1 && m->order == CER_ORDER_COLUMNS) {
        m->order = CER_ORDER_ROWS;
        m->ld = 1;
    } else if (tokens == 1 && m->order == CER_ORDER_COLUMNS && m->ld == 1) {
        m->order = CER_ORDER_ROWS;
        m->ld = features;
    } else if (features == 1 && m->order == CER_ORDER_ROWS && m->ld == 1) {
        m->order = CER_ORDER_COLUMNS;
        m->ld = tokens;
    }
}

// A contiguous tensor of `numbers` elements (-1: any number) of a type (-1: any of the three floating ones, told in *type).
bool flat_of(PyObject* o, const char* what, Device& dev, int type, int64_t numbers, void** out, int* type_out = nullptr, int64_t* numbers_out = nullptr) {
    const at::Tensor* t = tensor_of(o, what);
    if (!t || !dev.has(*t, what)) return false;
    const int have = type_of(*t);
    if (type >= 0 ? have != type : (have != CER_TYPE_F32 && have != CER_TYPE_BF16 && have != CER_TYPE_F16))
        return fail(what, type == kInt32 ? "must be int32" : type == CER_TYPE_F32 ? "must be float32" : "must be float32, bfloat16 or float16");
    if (!t->is_contiguous()) return fail(what, "must be contiguous");
    if (numbers >= 0 && t->numel() != numbers) return fail(what, "has another number of elements than the other arguments ask for");
    if (type_out) *type_out = have;
    if (numbers_out) *numbers_out = t->numel();
    *out = t->data_ptr();
    return true;
}

template <class Fn, class... Args>
PyObject* call(Fn fn, const char* name, Args... args) {
    if (!fn) return PyErr_Format(PyExc_RuntimeError, "%s is not bound", name);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(args...);
    Py_END_ALLOW_THREADS
    if (rc != 0) {
        PyObject* r = PyObject_CallFunction(g_check, "is", rc, name);
        if (!r) return nullptr;
        Py_DECREF(r);
    }
    Py_RETURN_NONE;
}

PyObject* py_rms_norm(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"X", "Y", "weight", "residual", "sum", "eps", "scale", "rstd", "stream"};
    enum { X, Y, kWeight, kResidual, kSum, kEps, kScale, kRstd, kStream, kCount };
    static const Signature f = {"rms_norm", 2, kCount, names};
    PyObject* a[kCount];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void* stream;
    Device dev;
    int64_t tokens = -1, n = -1;
    cer_tokens_t x{}, y{}, r{}, sum{};
    if (!tokens_of(a[X], "X", dev, &x, &tokens, &n) || !tokens_of(a[Y], "Y", dev, &y, &tokens, &n)) return nullptr;
    if (a[kResidual] && !tokens_of(a[kResidual], "residual", dev, &r, &tokens, &n)) return nullptr;
    if (a[kSum] && !tokens_of(a[kSum], "sum", dev, &sum, &tokens, &n)) return nullptr;
    same_order(&r, x, tokens, n);
    same_order(&sum, x, tokens, n);
    void *weight = nullptr, *scale = nullptr, *rstd = nullptr;
    int weight_type = CER_TYPE_F32;
    if (a[kWeight] && !flat_of(a[kWeight], "weight", dev, -1, n, &weight, &weight_type)) return nullptr;
    if (a[kScale] && !flat_of(a[kScale], "scale", dev, CER_TYPE_F32, tokens, &scale)) return nullptr;
    if (a[kRstd] && !flat_of(a[kRstd], "rstd", dev, CER_TYPE_F32, tokens, &rstd)) return nullptr;
    const double eps = a[kEps] ? PyFloat_AsDouble(a[kEps]) : 1e-6;
    if (eps == -1.0 && PyErr_Occurred()) return nullptr;
    if (!dev.stream(a[kStream], &stream)) return nullptr;
    return call(g_fn.norm, f.name, &x, &r, &sum, &y, tokens, n, weight, weight_type, (float)eps, static_cast<float*>(scale), static_cast<float*>(rstd), stream);
}

PyObject* py_rms_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"dY", "H", "rstd", "dX", "weight", "dsum", "dweight", "stream"};
    enum { kDY, H, kRstd, kDX, kWeight, kDSum, kDWeight, kStream, kCount };
    static const Signature f = {"rms_norm_backward", 4, kCount, names};
    PyObject* a[kCount];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void* stream;
    Device dev;
    int64_t tokens = -1, n = -1;
    cer_tokens_t dy{}, h{}, dsum{}, dx{};
    if (!tokens_of(a[kDY], "dY", dev, &dy, &tokens, &n) || !tokens_of(a[H], "H", dev, &h, &tokens, &n) || !tokens_of(a[kDX], "dX", dev, &dx, &tokens, &n)) return nullptr;
    if (a[kDSum] && !tokens_of(a[kDSum], "dsum", dev, &dsum, &tokens, &n)) return nullptr;
    if (h.order == CER_ORDER_COLUMNS) same_order(&h, dy, tokens, n);
    if (dy.order == CER_ORDER_ROWS) same_order(&dy, h, tokens, n);
    same_order(&dx, h, tokens, n);
    same_order(&dsum, h, tokens, n);
    void *rstd = nullptr, *weight = nullptr, *dweight = nullptr;
    int weight_type = CER_TYPE_F32;
    if (!flat_of(a[kRstd], "rstd", dev, CER_TYPE_F32, tokens, &rstd)) return nullptr;
    if (a[kWeight] && !flat_of(a[kWeight], "weight", dev, -1, n, &weight, &weight_type)) return nullptr;
    if (a[kDWeight] && !flat_of(a[kDWeight], "dweight", dev, CER_TYPE_F32, n, &dweight)) return nullptr;
    if (!dev.stream(a[kStream], &stream)) return nullptr;
    return call(g_fn.norm_backward, f.name, &dy, &h, &dsum, &dx, tokens, n, static_cast<float*>(rstd), weight, weight_type, static_cast<float*>(dweight), stream);
}

// A (adapters, rank, in), B (adapters, out, rank), scales, ranks, index
bool adapters_of(PyObject* a, PyObject* b, PyObject* scales, PyObject* ranks, Device& dev, cer_adapters_t* w) {
    const at::Tensor *A = tensor_of(a, "A"), *B = A ? tensor_of(b, "B") : nullptr;
    if (!B || !dev.has(*A, "A") || !dev.has(*B, "B")) return false;
    const int type = type_of(*A);
    if (type != CER_TYPE_F32 && type != CER_TYPE_BF16 && type != CER_TYPE_F16) return fail("A", "must be float32, bfloat16 or float16");
    if (type_of(*B) != type) return fail("B", "must have A's type");
    if (A->dim() != 3 || B->dim() != 3) return fail("A, B", "must have 3 dimensions");
    const auto sa = A->sizes(), ta = A->strides(), sb = B->sizes(), tb = B->strides();
    if (sb[0] != sa[0] || sb[2] != sa[1]) return fail("B", "must have A's number of adapters and rank: A (adapters, rank, in), B (adapters, out, rank)");
    if ((ta[2] != 1 && sa[2] > 1) || (tb[2] != 1 && sb[2] > 1)) return fail("A, B", "must have contiguous rows");
    void *ps = nullptr, *pr = nullptr;
    if (scales && !flat_of(scales, "scales", dev, CER_TYPE_F32, sa[0], &ps)) return false;
    if (ranks && !flat_of(ranks, "ranks", dev, kInt32, sa[0], &pr)) return false;
    *w = {A->data_ptr(), B->data_ptr(), static_cast<float*>(ps), static_cast<int32_t*>(pr), sa[0], sa[1], sa[2], sb[1], ta[0], ta[1], tb[0], tb[1], type};
    return true;
}

PyObject* py_adapter_matmul(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"A", "B", "index", "X", "Y", "scales", "ranks", "base", "hidden", "workspace", "stream"};
    enum { A, B, kIndex, X, Y, kScales, kRanks, kBase, kHidden, kWorkspace, kStream, kCount };
    static const Signature f = {"adapter_matmul", 5, kCount, names};
    PyObject* a[kCount];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void* stream;
    Device dev;
    cer_adapters_t w;
    if (!adapters_of(a[A], a[B], a[kScales], a[kRanks], dev, &w)) return nullptr;
    int64_t tokens = -1;
    cer_tokens_t x{}, y{}, base{};
    if (!tokens_of(a[X], "X", dev, &x, &tokens, &w.in) || !tokens_of(a[Y], "Y", dev, &y, &tokens, &w.out)) return nullptr;
    if (a[kBase] && !tokens_of(a[kBase], "base", dev, &base, &tokens, &w.out)) return nullptr;
    same_order(&y, x, tokens, w.out);
    same_order(&x, y, tokens, w.in);
    same_order(&base, y, tokens, w.out);
    void *index, *hidden = nullptr, *workspace = nullptr;
    int64_t room = 0;
    if (!flat_of(a[kIndex], "index", dev, kInt32, tokens, &index)) return nullptr;
    if (a[kHidden] && !flat_of(a[kHidden], "hidden", dev, CER_TYPE_F32, tokens * w.rank, &hidden)) return nullptr;
    if (a[kWorkspace] && !flat_of(a[kWorkspace], "workspace", dev, CER_TYPE_F32, -1, &workspace, nullptr, &room)) return nullptr;
    if (!dev.stream(a[kStream], &stream)) return nullptr;
    return call(g_fn.adapter, f.name, &w, static_cast<const int32_t*>(index), tokens, &x, &base, &y, static_cast<float*>(hidden), workspace, room * 4, stream);
}

PyObject* py_adapter_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"A", "B", "index", "dY", "X", "hidden", "scales", "ranks", "base", "dX", "dA", "dB", "stream"};
    enum { A, B, kIndex, kDY, X, kHidden, kScales, kRanks, kBase, kDX, kDA, kDB, kStream, kCount };
    static const Signature f = {"adapter_backward", 6, kCount, names};
    PyObject* a[kCount];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void* stream;
    Device dev;
    cer_adapters_t w;
    if (!adapters_of(a[A], a[B], a[kScales], a[kRanks], dev, &w)) return nullptr;
    int64_t tokens = -1;
    cer_tokens_t dy{}, x{}, base{}, dx{};
    if (!tokens_of(a[kDY], "dY", dev, &dy, &tokens, &w.out) || !tokens_of(a[X], "X", dev, &x, &tokens, &w.in)) return nullptr;
    if (a[kBase] && !tokens_of(a[kBase], "base", dev, &base, &tokens, &w.in)) return nullptr;
    if (a[kDX] && !tokens_of(a[kDX], "dX", dev, &dx, &tokens, &w.in)) return nullptr;
    same_order(&x, dy, tokens, w.in);
    same_order(&dy, x, tokens, w.out);
    same_order(&dx, x, tokens, w.in);
    same_order(&base, x, tokens, w.in);
    void *index, *hidden = nullptr, *dA = nullptr, *dB = nullptr;
    if (!flat_of(a[kIndex], "index", dev, kInt32, tokens, &index)) return nullptr;
    if (!flat_of(a[kHidden], "hidden", dev, CER_TYPE_F32, tokens * w.rank, &hidden)) return nullptr;
    if (a[kDA] && !flat_of(a[kDA], "dA", dev, CER_TYPE_F32, w.adapters * w.rank * w.in, &dA)) return nullptr;
    if (a[kDB] && !flat_of(a[kDB], "dB", dev, CER_TYPE_F32, w.adapters * w.rank * w.out, &dB)) return nullptr;
    if (!dev.stream(a[kStream], &stream)) return nullptr;
    return call(g_fn.adapter_backward, f.name, &w, static_cast<const int32_t*>(index), tokens, &dy, &x, static_cast<const float*>(hidden), &base, &dx,
                static_cast<float*>(dA), static_cast<float*>(dB), stream);
}

// A list or tuple of tensors; outs: as many of the same types and lengths, or nullptr (in place).
bool gradients_of(PyObject* grads, PyObject* outs, Device& dev, std::vector<cer_gradient_t>* list) {
    PyObject* g = PySequence_Fast(grads, "grads must be a sequence of tensors");
    if (!g) return false;
    PyObject* o = outs ? PySequence_Fast(outs, "outs must be a sequence of tensors") : nullptr;
    bool ok = !outs || o;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(g);
    if (ok && o && PySequence_Fast_GET_SIZE(o) != n) ok = fail("outs", "must have as many tensors as grads");
    if (ok) {
        try {
            list->resize((size_t)n);
        } catch (...) {
            PyErr_NoMemory();
            ok = false;
        }
    }
    for (Py_ssize_t i = 0; i < n && ok; ++i) {
        cer_gradient_t& e = (*list)[(size_t)i];
        void* p = nullptr;
        int type = 0;
        ok = flat_of(PySequence_Fast_GET_ITEM(g, i), "a gradient", dev, -1, -1, &p, &type, &e.numbers);
        e.grad = e.out = p;
        e.type = type;
        if (ok && o) ok = flat_of(PySequence_Fast_GET_ITEM(o, i), "an output", dev, type, e.numbers, &e.out);
    }
    Py_DECREF(g);
    Py_XDECREF(o);
    return ok;
}

PyObject* py_grad_norm(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"grads", "norm", "stream"};
    static const Signature f = {"grad_norm", 2, 3, names};
    PyObject* a[3];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void *stream, *norm;
    Device dev;
    std::vector<cer_gradient_t> list;
    if (!gradients_of(a[0], nullptr, dev, &list) || !flat_of(a[1], "norm", dev, CER_TYPE_F32, 1, &norm) || !dev.stream(a[2], &stream)) return nullptr;
    return call(g_fn.grad_norm, f.name, list.data(), (int64_t)list.size(), static_cast<float*>(norm), stream);
}

PyObject* py_grad_clip(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"grads", "max_norm", "norm", "outs", "stream"};
    static const Signature f = {"grad_clip", 3, 5, names};
    PyObject* a[5];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void *stream, *norm;
    Device dev;
    std::vector<cer_gradient_t> list;
    if (!gradients_of(a[0], a[3], dev, &list) || !flat_of(a[2], "norm", dev, CER_TYPE_F32, 1, &norm) || !dev.stream(a[4], &stream)) return nullptr;
    const double most = PyFloat_AsDouble(a[1]);
    if (most == -1.0 && PyErr_Occurred()) return nullptr;
    return call(g_fn.grad_clip, f.name, list.data(), (int64_t)list.size(), (float)most, static_cast<float*>(norm), stream);
}

// setup(check): binding.py's function
PyObject* setup(PyObject*, PyObject* check) {
    Py_INCREF(check);
    Py_XSETREF(g_check, check);
    Py_RETURN_NONE;
}

// bind(addresses): where the loaded library has the operators, in the order of g_fn
PyObject* bind(PyObject*, PyObject* args) {
    unsigned long long at[6];
    if (!PyArg_ParseTuple(args, "KKKKKK", &at[0], &at[1], &at[2], &at[3], &at[4], &at[5])) return nullptr;
    g_fn = {reinterpret_cast<NormFn>((uintptr_t)at[0]),    reinterpret_cast<NormBackwardFn>((uintptr_t)at[1]),
            reinterpret_cast<AdapterFn>((uintptr_t)at[2]), reinterpret_cast<AdapterBackwardFn>((uintptr_t)at[3]),
            reinterpret_cast<NormOfFn>((uintptr_t)at[4]),  reinterpret_cast<ClipFn>((uintptr_t)at[5])};
    Py_RETURN_NONE;
}

using Entry = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t, PyObject*);
template <Entry kEntry>  // torch's interface may throw; nothing does through the interpreter
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    try {
        return kEntry(self, args, nargs, kwnames);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

#define CER_OPERATOR(name, fn, text) \
    {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(guarded<fn>)), METH_FASTCALL | METH_KEYWORDS, text}

PyMethodDef g_methods[] = {
    CER_OPERATOR("rms_norm", py_rms_norm, "rms_norm(X, Y, weight=None, residual=None, sum=None, eps=1e-6, scale=None, rstd=None, stream=None)\n--\n\n"),
    CER_OPERATOR("rms_norm_backward", py_rms_norm_backward, "rms_norm_backward(dY, H, rstd, dX, weight=None, dsum=None, dweight=None, stream=None)\n--\n\n"),
    CER_OPERATOR("adapter_matmul", py_adapter_matmul,
                 "adapter_matmul(A, B, index, X, Y, scales=None, ranks=None, base=None, hidden=None, workspace=None, stream=None)\n--\n\n"),
    CER_OPERATOR("adapter_backward", py_adapter_backward,
                 "adapter_backward(A, B, index, dY, X, hidden, scales=None, ranks=None, base=None, dX=None, dA=None, dB=None, stream=None)\n--\n\n"),
    CER_OPERATOR("grad_norm", py_grad_norm, "grad_norm(grads, norm, stream=None)\n--\n\n"),
    CER_OPERATOR("grad_clip", py_grad_clip, "grad_clip(grads, max_norm, norm, outs=None, stream=None)\n--\n\n"),
    {"setup", setup, METH_O, nullptr},
    {"bind", bind, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_cerops", "Native operator calls of the binding.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cerops(void) {
    PyObject* c = PyImport_ImportModule("torch._C");
    if (!c) return nullptr;
    g_get_device = PyObject_GetAttrString(c, "_cuda_getDevice");
    g_raw_stream = g_get_device ? PyObject_GetAttrString(c, "_cuda_getCurrentRawStream") : nullptr;
    Py_DECREF(c);
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    return g_raw_stream && s_cuda_stream ? PyModule_Create(&g_module) : nullptr;
}
