// aspis_tensors.cpp -- the Python module _tensors: what the norm, clipping
// and update calls ask of torch tensors every time, in one call each.  Asked
// attribute by attribute through Python it takes longer than a small call's
// kernels (four questions of 62 tensors: 7.3 us; a buffer's checks: 0.7 us).
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <vector>

namespace {

// state(list of tensors) -> bytes: of every tensor the address, number of
// elements, type, contiguity and whether it is a negated view (its memory
// holds the opposite of its values), and of one that is not contiguous its
// sizes and strides.
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
            words.push_back((int64_t)t.scalar_type() * 4 + t.is_neg() * 2 + contiguous);
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

// buffer(x, dtype, n, device index) -> the address of x, or None unless x is
// a contiguous tensor of this type on this GPU with at least n elements.
PyObject *buffer(PyObject *, PyObject *const *args, Py_ssize_t count) {
    if (count != 4 || !THPDtype_Check(args[1])) {
        PyErr_SetString(PyExc_TypeError, "buffer() takes an object, a dtype, a size and an index");
        return nullptr;
    }
    const long long n = PyLong_AsLongLong(args[2]);
    const long index = PyLong_AsLong(args[3]);
    if (PyErr_Occurred()) return nullptr;
    if (!THPVariable_Check(args[0])) Py_RETURN_NONE;
    try {
        const at::Tensor &t = THPVariable_Unpack(args[0]);
        if (!t.is_cuda() || t.layout() != at::kStrided || t.get_device() != index ||
            t.numel() < n || !t.is_contiguous() || t.is_neg() ||
            t.scalar_type() != reinterpret_cast<THPDtype *>(args[1])->scalar_type)
            Py_RETURN_NONE;
        return PyLong_FromUnsignedLongLong((unsigned long long)(uintptr_t)t.data_ptr());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// rows(x) -> (rows, d, d, type code of aspis.h) of a contiguous GPU tensor
// [..., d] of a type the kernels take, or None.
PyObject *rows(PyObject *, PyObject *arg) {
    if (!THPVariable_Check(arg)) Py_RETURN_NONE;
    try {
        const at::Tensor &t = THPVariable_Unpack(arg);
        if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() < 1 || t.numel() == 0 ||
            !t.is_contiguous() || t.is_neg())
            Py_RETURN_NONE;
        int code = 0;
        switch (t.scalar_type()) {
            case at::kFloat: code = 0; break;
            case at::kBFloat16: code = 1; break;
            case at::kHalf: code = 2; break;
            default: Py_RETURN_NONE;
        }
        const long long d = t.size(-1);
        return Py_BuildValue("LLLi", (long long)t.numel() / d, d, d, code);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// The spans of memory of a list's tensors that are not empty: their first and
// past-the-end addresses in pairs, by the first, then the largest end.
struct Spans {
    const uint64_t *at;
    Py_ssize_t n;
    uint64_t first() const { return at[0]; }
    uint64_t end() const { return at[2 * n]; }
};

// Whether no span of one list overlaps one of the other (spans of the same
// list may): in order of their starts, none starts before the furthest end
// so far of the other list.
bool apart(const Spans &a, const Spans &b) {
    if (a.n == 0 || b.n == 0 || a.end() <= b.first() || b.end() <= a.first()) return true;
    uint64_t end_a = 0, end_b = 0;
    for (Py_ssize_t i = 0, j = 0; i < a.n || j < b.n;) {
        const bool from_a = j == b.n || (i < a.n && a.at[2 * i] <= b.at[2 * j]);
        const uint64_t *span = from_a ? a.at + 2 * i++ : b.at + 2 * j++;
        if (span[0] < (from_a ? end_b : end_a)) return false;
        uint64_t &end = from_a ? end_a : end_b;
        if (span[1] > end) end = span[1];
    }
    return true;
}

// apart(spans, spans, ...) -> whether the lists' tensors share no memory.
PyObject *apart_py(PyObject *, PyObject *const *args, Py_ssize_t count) {
    constexpr Py_ssize_t kMost = 8, kWord = sizeof(uint64_t);
    Spans lists[kMost];
    if (count > kMost) {
        PyErr_SetString(PyExc_TypeError, "apart() takes up to 8 lists' spans");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < count; ++i) {
        if (!PyBytes_Check(args[i]) || PyBytes_GET_SIZE(args[i]) % (2 * kWord) != kWord) {
            PyErr_SetString(PyExc_TypeError, "apart() takes spans as bytes");
            return nullptr;
        }
        // (a bytes object's data is aligned to 8)
        lists[i] = {reinterpret_cast<const uint64_t *>(PyBytes_AS_STRING(args[i])),
                    PyBytes_GET_SIZE(args[i]) / (2 * kWord)};
        for (Py_ssize_t j = 0; j < i; ++j)
            if (!apart(lists[i], lists[j])) Py_RETURN_FALSE;
    }
    Py_RETURN_TRUE;
}

PyMethodDef methods[] = {
    {"apart", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(apart_py)),
     METH_FASTCALL, "Whether lists of spans share no memory."},
    {"rows", rows, METH_O, "Rows, length, distance and type code of a contiguous GPU tensor."},
    {"buffer", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(buffer)), METH_FASTCALL,
     "The address of a contiguous GPU tensor of a type and size, or None."},
    {"state", state, METH_O, "Where a list's tensors are and how they are laid out, as bytes."},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
