// What a checked call costs the host beyond its launch, in native code: the checks of a tensor argument (dev) and the call
// of a C-ABI entry point with converted arguments (one function per entry point).  binding.py builds the argument tuples.
//
// A tensor that passes every check gives its address; anything else gives None and binding.py repeats the checks in Python,
// which raises the error with the argument's name.  In Python a tensor's checks take 0.6 us and the conversion of the
// step's 19 arguments by ctypes 1.7 us; here 0.1 us and 0.2 us.
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <tuple>
#include <type_traits>
#include <utility>

#include "ragged.h"

namespace {

// dtype: None, a torch.dtype or a tuple of them
bool dtype_is(PyObject* want, at::ScalarType have) {
    if (THPDtype_Check(want)) return reinterpret_cast<THPDtype*>(want)->scalar_type == have;
    if (!PyTuple_Check(want)) return false;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(want); ++i) {
        PyObject* one = PyTuple_GET_ITEM(want, i);
        if (THPDtype_Check(one) && reinterpret_cast<THPDtype*>(one)->scalar_type == have) return true;
    }
    return false;
}

// shape: None or a tuple of integers
bool shape_is(PyObject* want, c10::IntArrayRef have) {
    if (!PyTuple_Check(want) || PyTuple_GET_SIZE(want) != static_cast<Py_ssize_t>(have.size())) return false;
    for (size_t i = 0; i < have.size(); ++i) {
        PyObject* one = PyTuple_GET_ITEM(want, i);
        if (!PyLong_CheckExact(one)) return false;
        int overflow = 0;
        if (PyLong_AsLongLongAndOverflow(one, &overflow) != have[i] || overflow != 0) return false;
    }
    return true;
}

// dev(tensor, dtype, shape) -> address of a contiguous GPU tensor of that type and shape, or None.  Only plain tensors: a
// subclass may have its own idea of its attributes.
PyObject* dev(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "dev takes a tensor, a dtype and a shape");
        return nullptr;
    }
    if (!THPVariable_CheckExact(args[0])) Py_RETURN_NONE;
    try {
        const at::Tensor& t = THPVariable_Unpack(args[0]);
        if (!t.is_cuda() || !t.is_contiguous()) Py_RETURN_NONE;
        if (args[1] != Py_None && !dtype_is(args[1], t.scalar_type())) Py_RETURN_NONE;
        if (args[2] != Py_None && !shape_is(args[2], t.sizes())) Py_RETURN_NONE;
        return PyLong_FromVoidPtr(t.data_ptr());
    } catch (...) {                                            // a tensor without storage of its own (tracing, vmap)
        Py_RETURN_NONE;
    }
}

// rows(tensor, dtype, shape) -> (address, elements between tokens) of a [rows, H, D] GPU view of that type and shape whose [H, D] block is
// contiguous inside a token, or None.  With fewer than two tokens the distance is at least one row.
PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "rows takes a tensor, a dtype and a shape");
        return nullptr;
    }
    if (!THPVariable_CheckExact(args[0])) Py_RETURN_NONE;
    try {
        const at::Tensor& t = THPVariable_Unpack(args[0]);
        if (!t.is_cuda() || t.dim() != 3 || t.stride(2) != 1 || t.stride(1) != t.size(2)) Py_RETURN_NONE;
        if (args[1] != Py_None && !dtype_is(args[1], t.scalar_type())) Py_RETURN_NONE;
        if (args[2] != Py_None && !shape_is(args[2], t.sizes())) Py_RETURN_NONE;
        const int64_t row = t.size(1) * t.size(2), stride = t.size(0) > 1 || t.stride(0) > row ? t.stride(0) : row;
        PyObject* const out = PyTuple_New(2);
        if (!out) return nullptr;
        PyTuple_SET_ITEM(out, 0, PyLong_FromVoidPtr(t.data_ptr()));
        PyTuple_SET_ITEM(out, 1, PyLong_FromLongLong(stride));
        return out;
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// here(device, tensor or None, ...) -> whether all tensors are on that device
PyObject* here(PyObject*, PyObject* const* args, Py_ssize_t n) {
    const long device = n > 0 ? PyLong_AsLong(args[0]) : -1;
    if (PyErr_Occurred()) return nullptr;
    for (Py_ssize_t i = 1; i < n; ++i) {
        if (args[i] == Py_None) continue;
        if (!THPVariable_Check(args[i]) || THPVariable_Unpack(args[i]).device().index() != device) Py_RETURN_FALSE;
    }
    Py_RETURN_TRUE;
}

// Memory of an argument: n rows of len bytes, step bytes apart.
struct Memory {
    const char* at;
    int64_t n, step, len;
    const char* end() const { return at + (n - 1) * step + len; }
};
Memory memory_of(const at::Tensor& t, int64_t most) {
    const int64_t size = static_cast<int64_t>(t.element_size());
    Memory m{static_cast<const char*>(t.data_ptr()), t.numel() == 0 ? 0 : 1, 0, t.numel() * size};
    if (m.n && !t.is_contiguous()) {
        m.len = size;
        for (int64_t d = 1; d < t.dim(); ++d) m.len += (t.size(d) - 1) * t.stride(d) * size;
        m.n = t.size(0);
        m.step = t.stride(0) * size;
        if (m.n > 1 && m.step < m.len) m = Memory{m.at, 1, 0, (m.n - 1) * m.step + m.len};       // (rows that run into each other: as one)
    }
    if (m.len > most) m.len = most;
    return m;
}
// Whether any byte is in both.  Rows at different distances whose ranges meet count as overlapping.
bool overlap(Memory a, Memory b) {
    if (a.n == 0 || b.n == 0) return false;
    if (b.at < a.at) std::swap(a, b);
    if (b.at >= a.end()) return false;
    if (a.n == 1 || (b.n > 1 && a.step != b.step)) return true;
    const int64_t behind = (b.at - a.at) % a.step;             // of the first of b, behind the start of a row of a
    return behind < a.len || behind + b.len > a.step;
}

// placed(device, written, argument, ...) -> 0; 1: an argument is not on that device; 2: one of the first `written` shares memory with another.
// Arguments are tensors, None, or (tensor, bytes) where only its first bytes are used.
PyObject* placed(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr Py_ssize_t kMost = 16;
    const long device = n > 1 ? PyLong_AsLong(args[0]) : -1, written = n > 1 ? PyLong_AsLong(args[1]) : -1;
    if (PyErr_Occurred()) return nullptr;
    if (n < 2 || n - 2 > kMost) {
        PyErr_SetString(PyExc_TypeError, "placed takes a device, a count and up to 16 arguments");
        return nullptr;
    }
    try {
        Memory memory[kMost];
        for (Py_ssize_t i = 0; i < n - 2; ++i) {
            PyObject* one = args[i + 2];
            memory[i] = Memory{nullptr, 0, 0, 0};
            if (one == Py_None) continue;
            int64_t most = INT64_MAX;
            if (PyTuple_Check(one) && PyTuple_GET_SIZE(one) == 2) {
                most = PyLong_AsLongLong(PyTuple_GET_ITEM(one, 1));
                if (PyErr_Occurred()) return nullptr;
                one = PyTuple_GET_ITEM(one, 0);
            }
            if (!THPVariable_Check(one) || THPVariable_Unpack(one).device().index() != device) return PyLong_FromLong(1);
            memory[i] = memory_of(THPVariable_Unpack(one), most);
        }
        for (Py_ssize_t i = 0; i < written && i < n - 2; ++i)
            for (Py_ssize_t j = i + 1; j < n - 2; ++j)
                if (overlap(memory[i], memory[j])) return PyLong_FromLong(2);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    return PyLong_FromLong(0);
}

template <typename T>
bool convert(PyObject* o, T& out) {
    if constexpr (std::is_pointer_v<T>) {
        if (o == Py_None) { out = nullptr; return true; }
        out = reinterpret_cast<T>(PyLong_AsVoidPtr(o));
    } else if constexpr (std::is_floating_point_v<T>) {
        out = static_cast<T>(PyFloat_AsDouble(o));
    } else {
        if (!PyLong_Check(o)) { PyErr_SetString(PyExc_TypeError, "an integer is required"); return false; }
        out = static_cast<T>(PyLong_AsUnsignedLongLongMask(o));
    }
    return !PyErr_Occurred();
}

template <typename... A, size_t... I>
PyObject* invoke(int (*fn)(A...), PyObject* const* args, std::index_sequence<I...>) {
    std::tuple<A...> v;
    if (!(convert(args[I], std::get<I>(v)) && ...)) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = fn(std::get<I>(v)...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}
template <typename... A>
PyObject* invoke(int (*fn)(A...), PyObject* const* args, Py_ssize_t n) {
    if (n != static_cast<Py_ssize_t>(sizeof...(A))) {
        PyErr_Format(PyExc_TypeError, "%zd arguments given, %zd expected", n, static_cast<Py_ssize_t>(sizeof...(A)));
        return nullptr;
    }
    return invoke(fn, args, std::make_index_sequence<sizeof...(A)>{});
}
template <auto Fn>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) { return invoke(Fn, args, n); }

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<&name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"dev", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&dev)), METH_FASTCALL, nullptr},
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&rows)), METH_FASTCALL, nullptr},
    {"placed", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&placed)), METH_FASTCALL, nullptr},
    {"here", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&here)), METH_FASTCALL, nullptr},
    ENTRY(ragged_pack), ENTRY(ragged_attn), ENTRY(ragged_attn_strided), ENTRY(ragged_attn_checked), ENTRY(ragged_attn_padded),
    ENTRY(ragged_unpack), ENTRY(ragged_repack), ENTRY(ragged_cls_extract), ENTRY(ragged_pack_attn_unpack), ENTRY(ragged_linear),
    ENTRY(ragged_layernorm), ENTRY(ragged_token_scores_l2), ENTRY(ragged_keep_topk), ENTRY(ragged_noop),
    ENTRY(ragged_rope), ENTRY(ragged_rope_frequencies), ENTRY(ragged_attn_lse), ENTRY(ragged_attn_backward), ENTRY(ragged_layernorm_backward),
    ENTRY(ragged_grad_plan), ENTRY(ragged_grad_clip),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ragged_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ragged_marshal() { return PyModule_Create(&module); }
