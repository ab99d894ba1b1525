// What the native calls of the Python binding share: one call's view of its arguments, its result, and what a status comes to.
#pragma once
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/sp24.h"

namespace {

// One call's view of its arguments; ok turns false with the first that is not as documented.
struct Call {
    PyObject* const* args;
    bool ok;

    const at::Tensor* tensor(int i)
    {
        PyObject* o = args[i];
        if (!ok || !THPVariable_Check(o)) return fail();
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda()) return fail();
        return &t;
    }
    const at::Tensor* fail()
    {
        ok = false;
        return nullptr;
    }
    bool none(int i) const { return args[i] == Py_None; }
    void require(bool cond) { ok = ok && cond; }

    // two-dimensional, unit stride along a row (the stride of a dimension of size 1 means nothing)
    const at::Tensor* rowmajor(int i)
    {
        const at::Tensor* t = tensor(i);
        if (!ok || t->dim() != 2 || (t->stride(1) != 1 && t->size(1) > 1)) return fail();
        return t;
    }
    // contiguous, any shape
    const at::Tensor* contiguous(int i)
    {
        const at::Tensor* t = tensor(i);
        if (!ok || !t->is_contiguous()) return fail();
        return t;
    }
    bool text_is(int i, const char* s)
    {
        PyObject* o = args[i];
        return PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, s) == 0;
    }
    sp24_layout layout(int i)
    {
        if (text_is(i, "tiled")) return SP24_LAYOUT_TILED;
        require(text_is(i, "canonical"));
        return SP24_LAYOUT_CANONICAL;
    }
    sp24_border border(int i)
    {
        if (text_is(i, "k")) return SP24_B_KMAJOR;
        require(text_is(i, "n"));
        return SP24_B_NMAJOR;
    }
    at::ScalarType dtype(int i)
    {
        if (!THPDtype_Check(args[i])) {
            ok = false;
            return at::kFloat;
        }
        return reinterpret_cast<THPDtype*>(args[i])->scalar_type;
    }
    int64_t integer(int i)
    {
        if (!PyLong_Check(args[i])) {
            ok = false;
            return 0;
        }
        const long long v = PyLong_AsLongLong(args[i]);
        if (v == -1 && PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return v;
    }
    float real(int i)
    {
        const double v = PyFloat_AsDouble(args[i]);
        if (v == -1.0 && PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return (float)v;
    }
    int truth(int i)
    {
        const int v = PyObject_IsTrue(args[i]);
        if (v < 0) {
            PyErr_Clear();
            ok = false;
        }
        return v > 0;
    }
    // a pair of integers
    void pair(int i, int& a, int& b)
    {
        PyObject* o = args[i];
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2 || !PyLong_Check(PyTuple_GET_ITEM(o, 0)) || !PyLong_Check(PyTuple_GET_ITEM(o, 1))) {
            ok = false;
            return;
        }
        const long x = PyLong_AsLong(PyTuple_GET_ITEM(o, 0)), y = PyLong_AsLong(PyTuple_GET_ITEM(o, 1));
        if (PyErr_Occurred()) {                        // past a long
            PyErr_Clear();
            ok = false;
        }
        require(x >= 0 && x <= 4096 && y >= 0 && y <= 4096);
        a = (int)x;
        b = (int)y;
    }
    // float32 vector with one entry per row
    const float* row_vector(int i, int64_t M)
    {
        const at::Tensor* t = contiguous(i);
        if (!ok) return nullptr;
        require(t->scalar_type() == at::kFloat && t->numel() == M);
        return static_cast<const float*>(t->data_ptr());
    }
};

sp24_dtype type_of(at::ScalarType t, bool& ok)
{
    switch (t) {
    case at::kHalf: return SP24_F16;
    case at::kBFloat16: return SP24_BF16;
    case at::kChar: return SP24_I8;
    case at::kFloat: return SP24_F32;
    case at::kInt: return SP24_I32;
    case at::kFloat8_e4m3fn: return SP24_F8;
    default: ok = false; return SP24_F32;
    }
}

bool is_input(at::ScalarType t) { return t == at::kHalf || t == at::kBFloat16 || t == at::kChar || t == at::kFloat8_e4m3fn; }

// leading dimension of a row-major matrix; a single row may carry any stride
int64_t ld(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1)); }

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

// New memory comes by way of torch's dispatcher only where that does more than allocate: where a dispatch mode is to see it, and where new memory is to be filled
// (torch.use_deterministic_algorithms).  Past it 0.47 us for 0.70, where a launch takes 2.7 (routing of 16 tokens a call 5.8 -> 4.8).
inline bool by_dispatcher()
{
    const auto& context = at::globalContext();
    return c10::impl::dispatch_mode_enabled() || (context.deterministicAlgorithms() && context.deterministicFillUninitializedMemory());
}
inline at::Tensor make(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like)
{
    if (by_dispatcher()) return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
    return at::Tensor(at::detail::empty_cuda(shape, type, like.device(), c10::nullopt));
}
// rows x columns with rows of `pitch`
inline at::Tensor make_pitched(int64_t rows, int64_t columns, int64_t pitch, at::ScalarType type, const at::Tensor& like)
{
    if (pitch == columns) return make({rows, columns}, type, like);
    if (by_dispatcher()) return make({rows, pitch}, type, like).narrow(1, 0, columns);
    const int64_t shape[2] = {rows, columns}, strides[2] = {pitch, 1};
    return at::Tensor(at::detail::empty_strided_cuda(shape, strides, type, like.device()));
}

// The result: a new tensor, or the caller's (argument i), which must have exactly the result's shape and type.
struct Result {
    at::Tensor fresh;
    const at::Tensor* t = nullptr;
    PyObject* given = nullptr;
    Result(Call& c, int i, at::IntArrayRef shape, at::ScalarType type, const at::Tensor* like)
    {
        if (!c.ok) return;
        if (c.none(i)) {
            fresh = make(shape, type, *like);
            t = &fresh;
            return;
        }
        t = c.rowmajor(i);
        if (!c.ok) return;
        c.require(t->sizes() == shape && t->scalar_type() == type);
        given = c.args[i];
    }
    PyObject* object()
    {
        if (given) {
            Py_INCREF(given);
            return given;
        }
        return THPVariable_Wrap(std::move(fresh));
    }
};

template <typename F>
sp24_status without_gil(F&& f)
{
    PyThreadState* state = PyEval_SaveThread();
    const sp24_status s = f();
    PyEval_RestoreThread(state);
    return s;
}

inline PyObject* not_handled() { Py_RETURN_NONE; }

// What a status other than SP24_OK comes to.  (module: this one, which holds sp24.py's exception as Sp24Error.)
PyObject* refused(PyObject* module, sp24_status s, const char* where)
{
    if (s != SP24_ERR_LAUNCH) return not_handled();
    PyObject* type = PyObject_GetAttrString(module, "Sp24Error");
    if (!type) return nullptr;
    if (PyObject* error = PyObject_CallFunction(type, "is", (int)s, where)) {
        PyErr_SetObject(type, error);
        Py_DECREF(error);
    }
    Py_DECREF(type);
    return nullptr;
}

// No exception of torch's (an allocation that fails) crosses into the interpreter: the Python code meets it again.
using Fn = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
template <Fn F>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n)
{
    try {
        return F(self, args, n);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

#define SP24_METHOD(name, ...) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(static_cast<Fn>(guarded<__VA_ARGS__>))), METH_FASTCALL, nullptr}

} // namespace

// the operators around the products (host_layers.cpp)
extern PyMethodDef sp24_layer_methods[];
