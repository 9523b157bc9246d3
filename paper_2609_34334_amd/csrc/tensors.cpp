// _tensors: reads lists of torch tensors for the Python binding.  An AdamW
// step over 150 tensors of six lists asks 900 tensors for five properties
// each; asked from Python that took 0.23 ms, here 0.01.
//
// read(name, tensors, dtype, device): the tensors' addresses as bytes (native
// 64-bit words), once all are contiguous tensors of `dtype` on the GPU number
// `device` (-1: not on a GPU).  TypeError or ValueError, naming the list,
// otherwise.
// table(device, *columns): lists of one length side by side, as bytes of eight
// words a tensor (hoccl_adamw_tensor_t): the addresses, in the columns' order,
// and last the number of elements.  A column is None (zeros) or (name,
// tensors, dtype, n): a tensor of it has an n-th of the first column's
// elements, rounded up.  Checked like read().
// rows(name, tensors, columns): their first sizes as bytes, once all have two
// dimensions, the second of `columns`; ValueError otherwise.
// wrote(*lists): the tensors of the lists (None: of none) have been written
// through their addresses: their versions go on, as after torch's own writes,
// so that a backward pass over a graph that saved one of them is refused.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <vector>

namespace {

// f(i, tensor) of every tensor of a list or tuple; false where f is, or with
// an error set.
template <typename F>
bool each(PyObject *seq, F &&f) {
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject *o = PySequence_Fast_GET_ITEM(seq, i);
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_TypeError, "a list of tensors is needed");
            return false;
        }
        if (!f(i, THPVariable_Unpack(o))) return false;
    }
    return true;
}

// Runs f; a C++ exception becomes a Python one.
template <typename F>
PyObject *guarded(F &&f) {
    try {
        return f();
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unexpected C++ exception");
    }
    return nullptr;
}

// Bytes of a 64-bit word a tensor, which f(i, tensor, word) fills; f returns
// false with an error set.
template <typename F>
PyObject *words(PyObject *list, F &&f) {
    PyObject *seq = PySequence_Fast(list, "a list of tensors is needed");
    if (!seq) return nullptr;
    PyObject *out = PyBytes_FromStringAndSize(nullptr, 8 * PySequence_Fast_GET_SIZE(seq));
    PyObject *done = !out ? nullptr : guarded([&]() -> PyObject * {
        const bool fine = each(seq, [&](Py_ssize_t i, const at::Tensor &t) {
            int64_t word;
            if (!f(i, t, word)) return false;
            std::memcpy(PyBytes_AS_STRING(out) + 8 * i, &word, 8);
            return true;
        });
        return fine ? out : nullptr;
    });
    Py_DECREF(seq);
    if (!done) Py_XDECREF(out);
    return done;
}

// The address of tensor i of the list `name`; false with an error set where it
// is not a contiguous one of `dtype` on `device`.
bool address(const char *name, Py_ssize_t i, const at::Tensor &t, PyObject *dtype, int device, int64_t &word) {
    if (t.scalar_type() != reinterpret_cast<THPDtype *>(dtype)->scalar_type) {
        PyErr_Format(PyExc_TypeError, "%s[%zd] must be %S", name, i, dtype);
        return false;
    }
    if ((t.is_cuda() ? (int)t.get_device() : -1) != device) {
        PyErr_Format(PyExc_ValueError, "%s[%zd]: all buffers must live on the same GPU", name, i);
        return false;
    }
    if (!t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s[%zd]: buffers must be contiguous", name, i);
        return false;
    }
    word = (int64_t)(uintptr_t)t.mutable_data_ptr();
    return true;
}

PyObject *read(PyObject *, PyObject *args) {
    const char *name;
    PyObject *list, *dtype;
    int device;
    if (!PyArg_ParseTuple(args, "sOO!i", &name, &list, (PyTypeObject *)&THPDtypeType, &dtype, &device)) return nullptr;
    return words(list, [&](Py_ssize_t i, const at::Tensor &t, int64_t &word) {
        return address(name, i, t, dtype, device, word);
    });
}

// One column of the table; the first makes it, with the numbers of elements.
bool column(PyObject *spec, int c, int device, std::vector<int64_t> &out) {
    const char *name;
    PyObject *list, *dtype;
    long long per;
    if (!PyArg_ParseTuple(spec, "sOO!L", &name, &list, (PyTypeObject *)&THPDtypeType, &dtype, &per)) return false;
    PyObject *seq = PySequence_Fast(list, "a list of tensors is needed");
    if (!seq) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    bool fine = true;
    if (c == 0) {
        out.assign(8 * n, 0);
    } else if ((size_t)n * 8 != out.size()) {
        PyErr_Format(PyExc_ValueError, "%s has %zd tensors, not %zd", name, n, (Py_ssize_t)out.size() / 8);
        fine = false;
    }
    fine = fine && each(seq, [&](Py_ssize_t i, const at::Tensor &t) {
        int64_t *row = &out[8 * i];
        if (c == 0) row[7] = t.numel();
        if (!address(name, i, t, dtype, device, row[c])) return false;
        const int64_t want = (row[7] + per - 1) / per;
        if (t.numel() == want) return true;
        PyErr_Format(PyExc_ValueError, "%s[%zd] has %lld elements, not %lld", name, i, (long long)t.numel(),
                     (long long)want);
        return false;
    });
    Py_DECREF(seq);
    return fine;
}

PyObject *table(PyObject *, PyObject *args) {
    return guarded([&]() -> PyObject * {
        const Py_ssize_t n = PyTuple_GET_SIZE(args);
        const long device = n ? PyLong_AsLong(PyTuple_GET_ITEM(args, 0)) : -1;
        if (device == -1 && PyErr_Occurred()) return nullptr;
        if (n < 2 || n > 8) {
            PyErr_SetString(PyExc_TypeError, "table(device, *columns) takes one to seven columns");
            return nullptr;
        }
        std::vector<int64_t> out;
        for (Py_ssize_t c = 0; c + 1 < n; ++c) {
            PyObject *spec = PyTuple_GET_ITEM(args, c + 1);
            if (c > 0 && spec == Py_None) continue;
            if (!PyTuple_Check(spec)) {
                PyErr_SetString(PyExc_TypeError, "a column is (name, tensors, dtype, n)");
                return nullptr;
            }
            if (!column(spec, (int)c, (int)device, out)) return nullptr;
        }
        return PyBytes_FromStringAndSize((const char *)out.data(), (Py_ssize_t)(out.size() * 8));
    });
}

PyObject *rows(PyObject *, PyObject *args) {
    const char *name;
    PyObject *list;
    Py_ssize_t columns;
    if (!PyArg_ParseTuple(args, "sOn", &name, &list, &columns)) return nullptr;
    return words(list, [&](Py_ssize_t i, const at::Tensor &t, int64_t &word) {
        if (t.dim() != 2 || t.size(1) != columns) {
            PyErr_Format(PyExc_ValueError, "%s[%zd] must have the shape [tokens, %zd]", name, i, columns);
            return false;
        }
        word = t.size(0);
        return true;
    });
}

PyObject *wrote(PyObject *, PyObject *args) {
    return guarded([&]() -> PyObject * {
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(args); ++i) {
            if (PyTuple_GET_ITEM(args, i) == Py_None) continue;
            PyObject *seq = PySequence_Fast(PyTuple_GET_ITEM(args, i), "a list of tensors is needed");
            if (!seq) return nullptr;
            // Views share their version; of neighbours that do, one is enough
            // (150 shards of five flat buffers each: 7 us, 2 so).
            const c10::VariableVersion *last = nullptr;
            const bool fine = each(seq, [&](Py_ssize_t, const at::Tensor &t) {
                at::TensorImpl *impl = t.unsafeGetTensorImpl();
                const c10::VariableVersion &version = impl->version_counter();
                if (!version.enabled()) return true;  // of inference mode
                if (!last || std::memcmp((const void *)last, (const void *)&version, sizeof version)) impl->bump_version();
                last = &version;
                return true;
            });
            Py_DECREF(seq);
            if (!fine) return nullptr;
        }
        Py_RETURN_NONE;
    });
}

PyMethodDef methods[] = {{"read", (PyCFunction)read, METH_VARARGS, nullptr},
                         {"table", (PyCFunction)table, METH_VARARGS, nullptr},
                         {"rows", (PyCFunction)rows, METH_VARARGS, nullptr},
                         {"wrote", (PyCFunction)wrote, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
