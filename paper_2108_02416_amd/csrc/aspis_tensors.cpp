// aspis_tensors.cpp -- the Python module _tensors: where the tensors of a
// list are and how they are laid out, in one call.  The list calls look at
// this every time, and four questions a tensor through Python take longer
// than the kernels of a short list (62 tensors: 7.3 us).
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <vector>

namespace {

// state(list of tensors) -> bytes: of every tensor the address, number of
// elements, type and contiguity, and of one that is not contiguous its sizes
// and strides.
PyObject *state(PyObject *, PyObject *arg) {
    if (!PyList_Check(arg)) {
        PyErr_SetString(PyExc_TypeError, "state() takes a list of tensors");
        return nullptr;
    }
    try {
        const Py_ssize_t n = PyList_GET_SIZE(arg);
        std::vector<int64_t> words;
        words.reserve(3 * (size_t)n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            PyObject *item = PyList_GET_ITEM(arg, i);
            if (!THPVariable_Check(item)) {
                PyErr_SetString(PyExc_TypeError, "state() takes a list of tensors");
                return nullptr;
            }
            const at::Tensor &t = THPVariable_Unpack(item);
            const bool contiguous = t.is_contiguous();
            words.push_back((int64_t)(intptr_t)t.data_ptr());
            words.push_back(t.numel());
            words.push_back((int64_t)t.scalar_type() * 2 + contiguous);
            if (contiguous) continue;
            words.push_back(t.dim());
            for (int64_t size : t.sizes()) words.push_back(size);
            for (int64_t stride : t.strides()) words.push_back(stride);
        }
        return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(words.data()),
                                         (Py_ssize_t)(words.size() * sizeof(int64_t)));
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyMethodDef methods[] = {
    {"state", state, METH_O, "Where a list's tensors are and how they are laid out, as bytes."},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
