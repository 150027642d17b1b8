// Argument marshalling for binding.py: addresses, strides and sizes of tensors, and the C ABI's calls with plain Python
// numbers as arguments.  A small pass is bounded by what the host does between two launches: through ctypes and tensor
// attributes a call of 30 arguments over six matrices took 14 us, so 3.
//
// Only torch.Tensor itself (and Parameter) is read here; anything else (a table in host memory, a subclass, a tensor without
// memory of its own under a transform) goes to the Python functions that binding.py registers, which decide and raise as before.
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <tuple>
#include <utility>

#include "gas.h"

namespace {

PyObject* slow_mat = nullptr;      // binding._mat_any
PyObject* slow_size = nullptr;     // binding._size_any
PyObject* slow_ptr = nullptr;      // binding._ptr_any

const at::Tensor* plain(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.unsafeGetTensorImpl()->has_storage() ||
        t.unsafeGetTensorImpl()->key_set().has(c10::DispatchKey::Python) || t.unsafeGetTensorImpl()->is_python_dispatch())
        return nullptr;
    const at::DeviceType d = t.device().type();
    return d == at::kCUDA || d == at::kCPU ? &t : nullptr;
}

// Whether t is a matrix with contiguous rows; its row stride as the C ABI takes it.
bool matrix(const at::Tensor& t, int64_t* ld) {
    if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) return false;
    *ld = t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
    return true;
}

PyObject* mat(PyObject*, PyObject* o) {
    try {
        int64_t ld;
        const at::Tensor* t = plain(o);
        if (t && matrix(*t, &ld)) {
            PyObject* out = PyTuple_New(2);
            if (!out) return nullptr;
            PyTuple_SET_ITEM(out, 0, PyLong_FromVoidPtr(t->data_ptr()));
            PyTuple_SET_ITEM(out, 1, PyLong_FromLongLong(ld));
            return out;
        }
    } catch (...) {
    }
    return PyObject_CallOneArg(slow_mat, o);
}

// (pointer, row stride, rows, columns, dtype code) of a matrix of the feature types
PyObject* size(PyObject*, PyObject* o) {
    try {
        int64_t ld;
        const at::Tensor* t = plain(o);
        const at::ScalarType s = t ? t->scalar_type() : at::kDouble;
        if (t && (s == at::kFloat || s == at::kBFloat16) && matrix(*t, &ld)) {
            PyObject* out = PyTuple_New(5);
            if (!out) return nullptr;
            PyTuple_SET_ITEM(out, 0, PyLong_FromVoidPtr(t->data_ptr()));
            PyTuple_SET_ITEM(out, 1, PyLong_FromLongLong(ld));
            PyTuple_SET_ITEM(out, 2, PyLong_FromLongLong(t->size(0)));
            PyTuple_SET_ITEM(out, 3, PyLong_FromLongLong(t->size(1)));
            PyTuple_SET_ITEM(out, 4, PyLong_FromLong(s == at::kFloat ? GAS_F32 : GAS_BF16));
            return out;
        }
    } catch (...) {
    }
    return PyObject_CallOneArg(slow_size, o);
}

// ptr(t, dtype=None): the address of a contiguous tensor (of that type), 0 for None
PyObject* ptr(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n >= 1 && n <= 2) {
        if (args[0] == Py_None) return PyLong_FromLong(0);
        try {
            const at::Tensor* t = plain(args[0]);
            const bool any = n == 1 || args[1] == Py_None;
            if (t && (any || (THPDtype_Check(args[1]) && reinterpret_cast<THPDtype*>(args[1])->scalar_type == t->scalar_type())) &&
                t->is_contiguous())
                return PyLong_FromVoidPtr(t->data_ptr());
        } catch (...) {
        }
    }
    return PyObject_Vectorcall(slow_ptr, args, n, nullptr);
}

// tensors(list): addresses, elements (int64 each) and dtype codes (int32) of contiguous tensors of the feature types, as bytes; None
// if any of them is something else, which the Python function decides about
PyObject* tensors(PyObject*, PyObject* o) {
    PyObject* list = PySequence_Fast(o, "a list of tensors");
    if (!list) return nullptr;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
    PyObject* at = PyBytes_FromStringAndSize(nullptr, n * 8);
    PyObject* count = PyBytes_FromStringAndSize(nullptr, n * 8);
    PyObject* code = PyBytes_FromStringAndSize(nullptr, n * 4);
    bool ok = at && count && code;
    Py_ssize_t i = 0;
    try {
        for (; ok && i < n; ++i) {
            const at::Tensor* t = plain(PySequence_Fast_GET_ITEM(list, i));
            const at::ScalarType s = t ? t->scalar_type() : at::kDouble;
            if (!t || (s != at::kFloat && s != at::kBFloat16) || !t->is_contiguous()) break;
            const int64_t address = (int64_t)(uintptr_t)t->data_ptr(), elements = t->numel();
            const int32_t c = s == at::kFloat ? GAS_F32 : GAS_BF16;
            memcpy(PyBytes_AS_STRING(at) + 8 * i, &address, 8);
            memcpy(PyBytes_AS_STRING(count) + 8 * i, &elements, 8);
            memcpy(PyBytes_AS_STRING(code) + 4 * i, &c, 4);
        }
    } catch (...) {
    }
    Py_DECREF(list);
    PyObject* out = nullptr;
    if (ok && i == n) {
        out = PyTuple_Pack(3, at, count, code);
    } else if (ok) {
        Py_INCREF(Py_None);
        out = Py_None;
    }
    Py_XDECREF(at);
    Py_XDECREF(count);
    Py_XDECREF(code);
    return out;
}

// floats(list): numbers as float32 in bytes
PyObject* floats(PyObject*, PyObject* o) {
    PyObject* list = PySequence_Fast(o, "a list of numbers");
    if (!list) return nullptr;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
    PyObject* out = PyBytes_FromStringAndSize(nullptr, n * 4);
    for (Py_ssize_t i = 0; out && i < n; ++i) {
        const double v = PyFloat_AsDouble(PySequence_Fast_GET_ITEM(list, i));
        if (v == -1.0 && PyErr_Occurred()) Py_CLEAR(out);
        else {
            const float f = (float)v;
            memcpy(PyBytes_AS_STRING(out) + 4 * i, &f, 4);
        }
    }
    Py_DECREF(list);
    return out;
}

// alike(like, t, ...): (rows, columns, dtype code, address and row stride of t, ...) of matrices of the feature types and of like's sizes and
// type, 0 and 0 for None.  None if any of them is something else, which the Python function decides about
PyObject* alike(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        int64_t ld;
        const at::Tensor* like = n > 0 ? plain(args[0]) : nullptr;
        const at::ScalarType s = like ? like->scalar_type() : at::kDouble;
        if (like && (s == at::kFloat || s == at::kBFloat16) && matrix(*like, &ld)) {
            PyObject* out = PyTuple_New(3 + 2 * (n - 1));
            if (!out) return nullptr;
            PyTuple_SET_ITEM(out, 0, PyLong_FromLongLong(like->size(0)));
            PyTuple_SET_ITEM(out, 1, PyLong_FromLongLong(like->size(1)));
            PyTuple_SET_ITEM(out, 2, PyLong_FromLong(s == at::kFloat ? GAS_F32 : GAS_BF16));
            for (Py_ssize_t i = 1; i < n; ++i) {
                const at::Tensor* t = args[i] == Py_None ? nullptr : plain(args[i]);
                if (args[i] != Py_None && (!t || t->scalar_type() != s || !matrix(*t, &ld) || t->size(0) != like->size(0) || t->size(1) != like->size(1))) {
                    Py_DECREF(out);
                    Py_RETURN_NONE;
                }
                PyTuple_SET_ITEM(out, 2 * i + 1, PyLong_FromVoidPtr(t ? t->data_ptr() : nullptr));
                PyTuple_SET_ITEM(out, 2 * i + 2, PyLong_FromLongLong(t ? ld : 0));
            }
            return out;
        }
    } catch (...) {
    }
    Py_RETURN_NONE;
}

// vectors(width, v, ...): addresses of contiguous float32 tensors of `width` elements, 0 for None; None if any of them is something else
PyObject* vectors(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        const long long width = n > 0 ? PyLong_AsLongLong(args[0]) : -1;
        if (width == -1 && PyErr_Occurred()) return nullptr;
        PyObject* out = PyTuple_New(n > 0 ? n - 1 : 0);
        if (!out) return nullptr;
        for (Py_ssize_t i = 1; i < n; ++i) {
            const at::Tensor* t = args[i] == Py_None ? nullptr : plain(args[i]);
            if (args[i] != Py_None && (!t || t->scalar_type() != at::kFloat || t->numel() != width || !t->is_contiguous())) {
                Py_DECREF(out);
                Py_RETURN_NONE;
            }
            PyTuple_SET_ITEM(out, i - 1, PyLong_FromVoidPtr(t ? t->data_ptr() : nullptr));
        }
        return out;
    } catch (...) {
    }
    Py_RETURN_NONE;
}

// ---- calls
// A pointer argument: an address, None, a ctypes array (its memory) or a ctypes pointer (its value).
bool get(PyObject* o, uintptr_t* out) {
    if (PyLong_Check(o)) {
        *out = (uintptr_t)PyLong_AsUnsignedLongLong(o);
        return !(*out == (uintptr_t)-1 && PyErr_Occurred());
    }
    if (o == Py_None) {
        *out = 0;
        return true;
    }
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_FORMAT | PyBUF_ND) != 0) return false;
    const bool ok = view.ndim > 0 || view.itemsize == (Py_ssize_t)sizeof(void*);
    if (ok) *out = view.ndim > 0 ? (uintptr_t)view.buf : *(uintptr_t*)view.buf;
    PyBuffer_Release(&view);             // the argument's reference is the caller's and outlives the call
    if (!ok) PyErr_SetString(PyExc_TypeError, "expected an address");
    return ok;
}

template <class T>
bool convert(PyObject* o, T* out) {
    if constexpr (std::is_pointer_v<T>) {
        uintptr_t p;
        if (!get(o, &p)) return false;
        *out = reinterpret_cast<T>(p);
    } else if constexpr (std::is_floating_point_v<T>) {
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) return false;
        *out = (T)v;
    } else {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) return false;
        *out = (T)v;
        if ((long long)*out != v) {
            PyErr_SetString(PyExc_OverflowError, "an argument does not fit its type");
            return false;
        }
    }
    return true;
}

template <auto Fn, class R, class... A, size_t... I>
PyObject* invoke(R (*)(A...), PyObject* const* args, std::index_sequence<I...>) {
    std::tuple<A...> v;
    if (!(convert(args[I], &std::get<I>(v)) && ...)) return nullptr;
    PyThreadState* state = PyEval_SaveThread();          // a launch may wait for room in its queue
    const R r = std::apply(Fn, v);
    PyEval_RestoreThread(state);
    return PyLong_FromLongLong((long long)r);
}

template <class R, class... A>
constexpr size_t arity(R (*)(A...)) { return sizeof...(A); }

template <auto Fn>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr size_t want = arity(Fn);
    if (n != (Py_ssize_t)want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, the call takes %zu", n, want);
        return nullptr;
    }
    return invoke<Fn>(Fn, args, std::make_index_sequence<want>{});
}

PyObject* set_slow(PyObject*, PyObject* args) {
    PyObject *m, *s, *p;
    if (!PyArg_ParseTuple(args, "OOO", &m, &s, &p)) return nullptr;
    Py_INCREF(m); Py_INCREF(s); Py_INCREF(p);
    Py_XDECREF(slow_mat); Py_XDECREF(slow_size); Py_XDECREF(slow_ptr);
    slow_mat = m; slow_size = s; slow_ptr = p;
    Py_RETURN_NONE;
}

#define GAS_CALL(name) {#name, (PyCFunction)(void (*)())call<&name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"mat", mat, METH_O, nullptr},
    {"size", size, METH_O, nullptr},
    {"ptr", (PyCFunction)(void (*)())ptr, METH_FASTCALL, nullptr},
    {"tensors", tensors, METH_O, nullptr},
    {"floats", floats, METH_O, nullptr},
    {"alike", (PyCFunction)(void (*)())alike, METH_FASTCALL, nullptr},
    {"vectors", (PyCFunction)(void (*)())vectors, METH_FASTCALL, nullptr},
    {"set_slow", set_slow, METH_VARARGS, nullptr},
    GAS_CALL(gas_pull), GAS_CALL(gas_push), GAS_CALL(gas_pull_host), GAS_CALL(gas_push_host), GAS_CALL(gas_gcn_norm),
    GAS_CALL(gas_spmm), GAS_CALL(gas_spmm_hist), GAS_CALL(gas_spmm_table), GAS_CALL(gas_fuse_sources), GAS_CALL(gas_spmm_t),
    GAS_CALL(gas_spmm_t_relu), GAS_CALL(gas_linear), GAS_CALL(gas_linear_in_order), GAS_CALL(gas_linear_push), GAS_CALL(gas_mlp2), GAS_CALL(gas_mlp2_push),
    GAS_CALL(gas_mlp2_keep), GAS_CALL(gas_spmm_linear), GAS_CALL(gas_spmm_t_relu_linear), GAS_CALL(gas_spmm_linear_layers),
    GAS_CALL(gas_spmm_t_relu_linear_layers), GAS_CALL(gas_relu_bwd), GAS_CALL(gas_linear_bwd_input),
    GAS_CALL(gas_linear_bwd_input_add), GAS_CALL(gas_linear_bwd_weight), GAS_CALL(gas_linear_bwd_weight_workspace),
    GAS_CALL(gas_linear_bwd_weights), GAS_CALL(gas_linear_bwd_weights_workspace), GAS_CALL(gas_softmax_xent),
    GAS_CALL(gas_sgd_step), GAS_CALL(gas_sgd_steps), GAS_CALL(gas_axpy), GAS_CALL(gas_row_dot),
    GAS_CALL(gas_pna_aggregate_own), GAS_CALL(gas_pna_aggregate_bwd_bounded), GAS_CALL(gas_pna_aggregate_bwd_workspace),
    GAS_CALL(gas_pna_groups), GAS_CALL(gas_pna_groups_workspace), GAS_CALL(gas_pna_linear), GAS_CALL(gas_pna_linear_workspace),
    GAS_CALL(gas_pna_linear_bwd_input), GAS_CALL(gas_pna_linear_bwd_weight), GAS_CALL(gas_pna_linear_bwd_weight_workspace),
    GAS_CALL(gas_residual_norm), GAS_CALL(gas_residual_norm_bwd), GAS_CALL(gas_residual_norm_bwd_workspace), GAS_CALL(gas_residual_norm_bwd_typed_workspace), GAS_CALL(gas_sq_norms),
    GAS_CALL(gas_sq_norms_workspace), GAS_CALL(gas_adamw_elements), GAS_CALL(gas_adamw_steps), GAS_CALL(gas_adamw_unpack),
    GAS_CALL(gas_linear_xent), GAS_CALL(gas_linear_xent_bwd), GAS_CALL(gas_linear_distill), GAS_CALL(gas_linear_distill_bwd), GAS_CALL(gas_linear_top),
    GAS_CALL(gas_linear_xent_workspace), GAS_CALL(gas_linear_xent_bwd_workspace), GAS_CALL(gas_linear_distill_workspace),
    GAS_CALL(gas_linear_distill_bwd_workspace), GAS_CALL(gas_linear_top_workspace),
    GAS_CALL(gas_gat_aggregate_push), GAS_CALL(gas_gat_aggregate_bwd_bounded), GAS_CALL(gas_gat_aggregate_bwd_heads_workspace),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch and the interpreter whose layouts were compiled in (_build.built_for); binding.py compares it with those it runs in.
PyMODINIT_FUNC PyInit__marshal() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", GAS_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
