// The operators beside a projection as native functions of the binding (_cerops): rms_norm, rms_norm_backward, adapter_matmul, adapter_backward,
// grad_norm, grad_clip; and those of a block around projections: linear_matmul, linear_backward, block_norm, block_norm_backward, dropout_add.
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
using LinearFn = decltype(&linear_matmul);
using LinearBackwardFn = decltype(&linear_backward);
using BlockFn = decltype(&block_norm);
using BlockBackwardFn = decltype(&block_norm_backward);
using DropoutFn = decltype(&dropout_add);
struct {
    NormFn norm;
    NormBackwardFn norm_backward;
    AdapterFn adapter;
    AdapterBackwardFn adapter_backward;
    NormOfFn grad_norm;
    ClipFn grad_clip;
    LinearFn linear;
    LinearBackwardFn linear_backward;
    BlockFn block;
    BlockBackwardFn block_backward;
    DropoutFn dropout;
} g_fn = {};

PyObject* g_check = nullptr;       // binding._check(rc, name): raises for an error code
PyObject* g_get_device = nullptr;  // torch._C._cuda_getDevice, ._cuda_getCurrentRawStream
PyObject* g_raw_stream = nullptr;
PyObject* s_cuda_stream = nullptr;
constexpr int kInt32 = 100, kInt64 = 101;  // beside CER_TYPE_*

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
        case at::kLong: return kInt64;
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
    if (type < 0 || type >= kInt32) return fail(what, "must be float32, bfloat16, float16 or float8_e4m3fn");
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
        return fail(what, type == kInt32 ? "must be int32" : type == kInt64 ? "must be int64" : type == CER_TYPE_F32 ? "must be float32" : "must be float32, bfloat16 or float16");
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

// ---- operators of a block around projections
// (out, in), rows contiguous
bool weights_of(PyObject* o, const char* what, Device& dev, const void** at, int64_t* ld, int* type, int64_t* out, int64_t* in) {
    const at::Tensor* t = tensor_of(o, what);
    if (!t || !dev.has(*t, what)) return false;
    if (t->dim() != 2) return fail(what, "must have 2 dimensions");
    const int have = type_of(*t);
    if (have != CER_TYPE_F32 && have != CER_TYPE_BF16 && have != CER_TYPE_F16) return fail(what, "must be float32, bfloat16 or float16");
    if (*type >= 0 && have != *type) return fail(what, "must have W's type");
    const auto size = t->sizes(), stride = t->strides();
    if (*out < 0) *out = size[0], *in = size[1];
    if (size[0] != *out || size[1] != *in) return fail(what, "must have W's shape");
    if (stride[1] != 1 && size[1] > 1) return fail(what, "must have contiguous rows");
    *type = have;
    *ld = size[0] > 1 ? stride[0] : size[1];
    *at = t->data_ptr();
    return true;
}
bool activation_of(PyObject* o, int* kind) {
    static const char* const names[] = {"none", "relu", "gelu", "gelu_tanh", "silu"};
    *kind = CER_ACTIVATION_NONE;
    if (!o) return true;
    if (PyUnicode_Check(o))
        for (int k = 0; k < 5; ++k)
            if (PyUnicode_CompareWithASCIIString(o, names[k]) == 0) {
                *kind = k;
                return true;
            }
    return fail("activation", "must be 'none', 'relu', 'gelu', 'gelu_tanh' or 'silu'");
}
bool number_of(PyObject* o, double otherwise, double* v) {
    *v = o ? PyFloat_AsDouble(o) : otherwise;
    return *v != -1.0 || !PyErr_Occurred();
}
// Any number of fp32 numbers, or nothing.
struct Workspace {
    void* at = nullptr;
    int64_t numbers = 0;
    bool of(PyObject* o, Device& dev) { return !o || flat_of(o, "workspace", dev, CER_TYPE_F32, -1, &at, nullptr, &numbers); }
};
// Matrices that a call wants in one order.  A single token's or feature's order is both, as long as its numbers lie side by side: those that have a choice follow one that has
// none -- one of several tokens and features, or one whose numbers lie apart (a token of a batch in columns, a feature of one in rows).
template <int kMany>
void one_order(cer_tokens_t* const (&m)[kMany], const int64_t (&features)[kMany], int64_t tokens) {
    const cer_tokens_t rows{nullptr, 0, 0, CER_ORDER_ROWS}, *lead = &rows;
    for (int k = kMany; k-- > 0;) {
        const bool token = tokens == 1, feature = features[k] == 1, apart = m[k]->ld != 1 && (token ? m[k]->order == CER_ORDER_COLUMNS : feature && m[k]->order == CER_ORDER_ROWS);
        if (m[k]->data && ((!token && !feature) || apart)) lead = m[k];
    }
    const cer_tokens_t as = *lead;
    for (int k = 0; k < kMany; ++k) same_order(m[k], as, tokens, features[k]);
}

PyObject* py_linear_matmul(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"W", "X", "Y", "bias", "residual", "activation", "pre", "workspace", "stream"};
    enum { W, X, Y, kBias, kResidual, kActivation, kPre, kWorkspace, kStream, kCount };
    static const Signature f = {"linear_matmul", 3, kCount, names};
    PyObject* a[kCount];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void* stream;
    Device dev;
    const void* w;
    int64_t ldw, out = -1, in = -1, tokens = -1;
    int type = -1, bias_type = CER_TYPE_F32, kind;
    if (!weights_of(a[W], "W", dev, &w, &ldw, &type, &out, &in)) return nullptr;
    cer_tokens_t x{}, y{}, r{}, pre{};
    if (!tokens_of(a[X], "X", dev, &x, &tokens, &in) || !tokens_of(a[Y], "Y", dev, &y, &tokens, &out)) return nullptr;
    if (a[kResidual] && !tokens_of(a[kResidual], "residual", dev, &r, &tokens, &out)) return nullptr;
    if (a[kPre] && !tokens_of(a[kPre], "pre", dev, &pre, &tokens, &out)) return nullptr;
    one_order<4>({&x, &y, &r, &pre}, {in, out, out, out}, tokens);
    void* bias = nullptr;
    if (a[kBias] && !flat_of(a[kBias], "bias", dev, -1, out, &bias, &bias_type)) return nullptr;
    Workspace work;
    if (!activation_of(a[kActivation], &kind) || !work.of(a[kWorkspace], dev) || !dev.stream(a[kStream], &stream)) return nullptr;
    return call(g_fn.linear, f.name, w, ldw, type, tokens, in, out, &x, &y, static_cast<const void*>(bias), bias_type, &r, kind, &pre, work.at, work.numbers * 4, stream);
}

PyObject* py_linear_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"W", "dY", "X", "activation", "pre", "base", "dX", "dW", "dbias", "workspace", "stream"};
    enum { W, kDY, X, kActivation, kPre, kBase, kDX, kDW, kDBias, kWorkspace, kStream, kCount };
    static const Signature f = {"linear_backward", 2, kCount, names};
    PyObject* a[kCount];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void* stream;
    Device dev;
    const void *w, *dw = nullptr;
    int64_t ldw, lddw = 0, out = -1, in = -1, tokens = -1;
    int type = -1, kind;
    if (!weights_of(a[W], "W", dev, &w, &ldw, &type, &out, &in)) return nullptr;
    cer_tokens_t dy{}, x{}, pre{}, base{}, dx{};
    if (!tokens_of(a[kDY], "dY", dev, &dy, &tokens, &out)) return nullptr;
    if (a[X] && !tokens_of(a[X], "X", dev, &x, &tokens, &in)) return nullptr;
    if (a[kPre] && !tokens_of(a[kPre], "pre", dev, &pre, &tokens, &out)) return nullptr;
    if (a[kBase] && !tokens_of(a[kBase], "base", dev, &base, &tokens, &in)) return nullptr;
    if (a[kDX] && !tokens_of(a[kDX], "dX", dev, &dx, &tokens, &in)) return nullptr;
    one_order<5>({&dy, &x, &pre, &base, &dx}, {out, in, out, in, in}, tokens);
    if (a[kDW] && !weights_of(a[kDW], "dW", dev, &dw, &lddw, &type, &out, &in)) return nullptr;
    void* dbias = nullptr;
    if (a[kDBias] && !flat_of(a[kDBias], "dbias", dev, CER_TYPE_F32, out, &dbias)) return nullptr;
    Workspace work;
    if (!activation_of(a[kActivation], &kind) || !work.of(a[kWorkspace], dev) || !dev.stream(a[kStream], &stream)) return nullptr;
    return call(g_fn.linear_backward, f.name, w, ldw, type, tokens, in, out, &dy, &x, kind, &pre, &base, &dx, const_cast<void*>(dw), lddw, static_cast<float*>(dbias), work.at,
                work.numbers * 4, stream);
}

// gate: (n,) of any type, or (tokens, n)
struct Gate {
    cer_tokens_t each{};
    void* vector = nullptr;
    int type = CER_TYPE_F32;
    bool of(PyObject* o, const char* what, Device& dev, int only, int64_t tokens, int64_t n) {
        if (!o) return true;
        const at::Tensor* t = tensor_of(o, what);
        if (!t) return false;
        if (t->dim() == 1) return flat_of(o, what, dev, only, n, &vector, &type);
        if (!tokens_of(o, what, dev, &each, &tokens, &n)) return false;
        rows(&each, tokens, n);
        return true;
    }
    static void rows(cer_tokens_t* m, int64_t tokens, int64_t n) { same_order(m, cer_tokens_t{nullptr, 0, 0, CER_ORDER_ROWS}, tokens, n); }
};

PyObject* py_block_norm(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"X", "F", "H", "Y", "gate", "post_weight", "pre_weight", "scale", "eps", "post", "rstd_post", "rstd_pre", "workspace", "stream"};
    enum { X, F, H, Y, kGate, kPostWeight, kPreWeight, kScale, kEps, kPost, kRstdPost, kRstdPre, kWorkspace, kStream, kCount };
    static const Signature f = {"block_norm", 4, kCount, names};
    PyObject* a[kCount];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void* stream;
    Device dev;
    int64_t tokens = -1, n = -1;
    cer_tokens_t x{}, o{}, h{}, y{};
    if (!tokens_of(a[X], "X", dev, &x, &tokens, &n) || !tokens_of(a[F], "F", dev, &o, &tokens, &n) || !tokens_of(a[H], "H", dev, &h, &tokens, &n) ||
        !tokens_of(a[Y], "Y", dev, &y, &tokens, &n))
        return nullptr;
    for (cer_tokens_t* m : {&x, &h, &o, &y}) Gate::rows(m, tokens, n);
    Gate gate;
    if (!gate.of(a[kGate], "gate", dev, -1, tokens, n)) return nullptr;
    void *post_weight = nullptr, *pre_weight = nullptr, *rstd_post = nullptr, *rstd_pre = nullptr;
    int post_type = CER_TYPE_F32, pre_type = CER_TYPE_F32;
    if (a[kPostWeight] && !flat_of(a[kPostWeight], "post_weight", dev, -1, n, &post_weight, &post_type)) return nullptr;
    if (a[kPreWeight] && !flat_of(a[kPreWeight], "pre_weight", dev, -1, n, &pre_weight, &pre_type)) return nullptr;
    if (a[kRstdPost] && !flat_of(a[kRstdPost], "rstd_post", dev, CER_TYPE_F32, tokens, &rstd_post)) return nullptr;
    if (a[kRstdPre] && !flat_of(a[kRstdPre], "rstd_pre", dev, CER_TYPE_F32, tokens, &rstd_pre)) return nullptr;
    double scale, eps;
    if (!number_of(a[kScale], 1.0, &scale) || !number_of(a[kEps], 1e-6, &eps)) return nullptr;
    const int post = a[kPost] ? PyObject_IsTrue(a[kPost]) : 1;
    Workspace work;
    if (post < 0 || !work.of(a[kWorkspace], dev) || !dev.stream(a[kStream], &stream)) return nullptr;
    return call(g_fn.block, f.name, &x, &o, &h, &y, tokens, n, &gate.each, static_cast<const void*>(gate.vector), gate.type, static_cast<const void*>(post_weight), post_type,
                static_cast<const void*>(pre_weight), pre_type, (float)scale, (float)eps, post, static_cast<float*>(rstd_post), static_cast<float*>(rstd_pre), work.at,
                work.numbers * 4, stream);
}

PyObject* py_block_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"dY", "H", "F", "rstd_pre", "dX", "dF", "rstd_post", "gate", "post_weight", "pre_weight", "scale", "dsum", "dgate", "dpost_weight", "dpre_weight",
                                        "workspace", "stream"};
    enum { kDY, H, F, kRstdPre, kDX, kDF, kRstdPost, kGate, kPostWeight, kPreWeight, kScale, kDSum, kDGate, kDPostWeight, kDPreWeight, kWorkspace, kStream, kCount };
    static const Signature f = {"block_norm_backward", 6, kCount, names};
    PyObject* a[kCount];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void* stream;
    Device dev;
    int64_t tokens = -1, n = -1;
    cer_tokens_t dy{}, h{}, o{}, dx{}, df{}, dsum{};
    if (!tokens_of(a[kDY], "dY", dev, &dy, &tokens, &n) || !tokens_of(a[H], "H", dev, &h, &tokens, &n) || !tokens_of(a[F], "F", dev, &o, &tokens, &n) ||
        !tokens_of(a[kDX], "dX", dev, &dx, &tokens, &n) || !tokens_of(a[kDF], "dF", dev, &df, &tokens, &n))
        return nullptr;
    if (a[kDSum] && !tokens_of(a[kDSum], "dsum", dev, &dsum, &tokens, &n)) return nullptr;
    for (cer_tokens_t* m : {&dy, &h, &dx, &dsum}) Gate::rows(m, tokens, n);
    one_order<2>({&o, &df}, {n, n}, tokens);
    Gate gate, dgate;
    if (!gate.of(a[kGate], "gate", dev, -1, tokens, n) || !dgate.of(a[kDGate], "dgate", dev, CER_TYPE_F32, tokens, n)) return nullptr;
    if (a[kDGate] && (!dgate.vector) != (!gate.vector)) return fail("dgate", "must have gate's shape"), nullptr;
    void *rstd_pre = nullptr, *rstd_post = nullptr, *post_weight = nullptr, *pre_weight = nullptr, *dpost = nullptr, *dpre = nullptr;
    int post_type = CER_TYPE_F32, pre_type = CER_TYPE_F32;
    if (!flat_of(a[kRstdPre], "rstd_pre", dev, CER_TYPE_F32, tokens, &rstd_pre)) return nullptr;
    if (a[kRstdPost] && !flat_of(a[kRstdPost], "rstd_post", dev, CER_TYPE_F32, tokens, &rstd_post)) return nullptr;
    if (a[kPostWeight] && !flat_of(a[kPostWeight], "post_weight", dev, -1, n, &post_weight, &post_type)) return nullptr;
    if (a[kPreWeight] && !flat_of(a[kPreWeight], "pre_weight", dev, -1, n, &pre_weight, &pre_type)) return nullptr;
    if (a[kDPostWeight] && !flat_of(a[kDPostWeight], "dpost_weight", dev, CER_TYPE_F32, n, &dpost)) return nullptr;
    if (a[kDPreWeight] && !flat_of(a[kDPreWeight], "dpre_weight", dev, CER_TYPE_F32, n, &dpre)) return nullptr;
    double scale;
    Workspace work;
    if (!number_of(a[kScale], 1.0, &scale) || !work.of(a[kWorkspace], dev) || !dev.stream(a[kStream], &stream)) return nullptr;
    return call(g_fn.block_backward, f.name, &dy, &h, &o, static_cast<const float*>(rstd_pre), static_cast<const float*>(rstd_post), &dx, &df, tokens, n, &gate.each,
                static_cast<const void*>(gate.vector), gate.type, static_cast<const void*>(post_weight), post_type, static_cast<const void*>(pre_weight), pre_type, (float)scale, &dsum,
                &dgate.each, static_cast<float*>(dgate.vector), static_cast<float*>(dpost), static_cast<float*>(dpre), work.at, work.numbers * 4, stream);
}

PyObject* py_dropout_add(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static const char* const names[] = {"X", "Y", "key", "p", "residual", "call", "stream"};
    enum { X, Y, kKey, P, kResidual, kCall, kStream, kCount };
    static const Signature f = {"dropout_add", 4, kCount, names};
    PyObject* a[kCount];
    if (!take(f, args, nargs, kwnames, a)) return nullptr;
    void *stream, *key;
    Device dev;
    int64_t tokens = -1, n = -1;
    cer_tokens_t x{}, y{}, r{};
    if (!tokens_of(a[X], "X", dev, &x, &tokens, &n) || !tokens_of(a[Y], "Y", dev, &y, &tokens, &n)) return nullptr;
    if (a[kResidual] && !tokens_of(a[kResidual], "residual", dev, &r, &tokens, &n)) return nullptr;
    one_order<3>({&x, &y, &r}, {n, n, n}, tokens);
    if (!flat_of(a[kKey], "key", dev, kInt64, 2, &key)) return nullptr;
    double p;
    if (!number_of(a[P], 0.0, &p)) return nullptr;
    const long long which = a[kCall] ? PyLong_AsLongLong(a[kCall]) : 0;
    if ((which == -1 && PyErr_Occurred()) || !dev.stream(a[kStream], &stream)) return nullptr;
    return call(g_fn.dropout, f.name, &x, &r, &y, tokens, n, static_cast<const int64_t*>(key), p, (int64_t)which, stream);
}

// setup(check): binding.py's function
PyObject* setup(PyObject*, PyObject* check) {
    Py_INCREF(check);
    Py_XSETREF(g_check, check);
    Py_RETURN_NONE;
}

// bind(addresses): where the loaded library has the operators, in the order of g_fn
PyObject* bind(PyObject*, PyObject* args) {
    unsigned long long at[11];
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKK", &at[0], &at[1], &at[2], &at[3], &at[4], &at[5], &at[6], &at[7], &at[8], &at[9], &at[10])) return nullptr;
    g_fn = {reinterpret_cast<NormFn>((uintptr_t)at[0]),    reinterpret_cast<NormBackwardFn>((uintptr_t)at[1]),
            reinterpret_cast<AdapterFn>((uintptr_t)at[2]), reinterpret_cast<AdapterBackwardFn>((uintptr_t)at[3]),
            reinterpret_cast<NormOfFn>((uintptr_t)at[4]),  reinterpret_cast<ClipFn>((uintptr_t)at[5]),
            reinterpret_cast<LinearFn>((uintptr_t)at[6]),  reinterpret_cast<LinearBackwardFn>((uintptr_t)at[7]),
            reinterpret_cast<BlockFn>((uintptr_t)at[8]),   reinterpret_cast<BlockBackwardFn>((uintptr_t)at[9]),
            reinterpret_cast<DropoutFn>((uintptr_t)at[10])};
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
    CER_OPERATOR("linear_matmul", py_linear_matmul, "linear_matmul(W, X, Y, bias=None, residual=None, activation='none', pre=None, workspace=None, stream=None)\n--\n\n"),
    CER_OPERATOR("linear_backward", py_linear_backward,
                 "linear_backward(W, dY, X=None, activation='none', pre=None, base=None, dX=None, dW=None, dbias=None, workspace=None, stream=None)\n--\n\n"),
    CER_OPERATOR("block_norm", py_block_norm,
                 "block_norm(X, F, H, Y, gate=None, post_weight=None, pre_weight=None, scale=1.0, eps=1e-6, post=True, rstd_post=None, rstd_pre=None, workspace=None, "
                 "stream=None)\n--\n\n"),
    CER_OPERATOR("block_norm_backward", py_block_norm_backward,
                 "block_norm_backward(dY, H, F, rstd_pre, dX, dF, rstd_post=None, gate=None, post_weight=None, pre_weight=None, scale=1.0, dsum=None, dgate=None, "
                 "dpost_weight=None, dpre_weight=None, workspace=None, stream=None)\n--\n\n"),
    CER_OPERATOR("dropout_add", py_dropout_add, "dropout_add(X, Y, key, p, residual=None, call=0, stream=None)\n--\n\n"),
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
