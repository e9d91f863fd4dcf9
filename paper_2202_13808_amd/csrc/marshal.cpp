// What a call over hundreds of tensors has to know of each of them, in one pass: address, number of elements, type, device,
// whether it is contiguous.  Asked for from Python, each of these costs 70 ns a tensor; twenty of them for a step over 150
// tensors took 150 us of host time, longer than the step's kernels.  Only reads the tensors; the kernels stay behind the C ABI.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>
#include <vector>

namespace {

// the codes of layers.py: dropit_dtype for the first two
int32_t type_code(c10::ScalarType t)
{
    switch (t) {
    case c10::ScalarType::Float: return 0;
    case c10::ScalarType::BFloat16: return 1;
    case c10::ScalarType::Byte: return 2;
    case c10::ScalarType::Short: return 3;
    default: return -1;
    }
}

// describe(tensors) -> (addresses, numels, types, type, device, contiguous): bytes of int64, int64 and int32, one entry a
// tensor; the one type and device of all of them, -2 where they differ, -1 where it is another type or the host
PyObject *describe(PyObject *, PyObject *sequence)
{
    PyObject *fast = PySequence_Fast(sequence, "a sequence of tensors");
    if (fast == nullptr) return nullptr;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
    PyObject **items = PySequence_Fast_ITEMS(fast);
    PyObject *result = nullptr;
    try {
        std::vector<int64_t> address(n), numel(n);
        std::vector<int32_t> type(n);
        int one_type = -2, one_device = -2, contiguous = 1;
        bool tensors = true;
        for (Py_ssize_t i = 0; i < n; ++i) {
            if (!THPVariable_Check(items[i])) {
                PyErr_Format(PyExc_TypeError, "expected tensors, got %s", Py_TYPE(items[i])->tp_name);
                tensors = false;
                break;
            }
            const at::Tensor &t = THPVariable_Unpack(items[i]);
            const int device = t.is_cuda() ? int(t.get_device()) : -1;
            const bool plain = t.layout() == c10::kStrided && t.is_contiguous();
            address[i] = plain ? int64_t(reinterpret_cast<uintptr_t>(t.const_data_ptr())) : 0;
            numel[i] = t.numel();
            type[i] = type_code(t.scalar_type());
            contiguous &= plain;
            one_type = i == 0 ? type[i] : one_type == type[i] ? one_type : -2;
            one_device = i == 0 ? device : one_device == device ? one_device : -2;
        }
        if (tensors) {
            auto bytes = [&](const void *p, size_t each) { return PyBytes_FromStringAndSize(static_cast<const char *>(p), Py_ssize_t(n * each)); };
            result = Py_BuildValue("(NNNiiO)", bytes(address.data(), 8), bytes(numel.data(), 8), bytes(type.data(), 4), one_type, one_device,
                                   contiguous ? Py_True : Py_False);
        }
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "a tensor could not be read");
    }
    Py_DECREF(fast);
    return result;
}

PyMethodDef methods[] = {{"describe", describe, METH_O, "addresses, element counts, types, device and contiguity of a sequence of tensors"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
