// bundle_module.cpp -- Python module `_bundle`: a list of label tensors -> the dash_labels that a call takes.  Host code; part of the
// binding, not of libdash.so.  (Asking 12 tensors of a bundle for address and stride from Python takes 6 us, as long as a small layer.)
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <string.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/dash.h"

// describe(tensors, address, n_elem): fills the dash_labels at `address`; a None leaves its residue empty
static PyObject* describe(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 3 || !PyList_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "describe(list of tensors, address, n_elem)");
        return nullptr;
    }
    dash_labels* const to = (dash_labels*)PyLong_AsVoidPtr(args[1]);
    if (!to && PyErr_Occurred()) return nullptr;
    const long long n_elem = PyLong_AsLongLong(args[2]);
    if (n_elem == -1 && PyErr_Occurred()) return nullptr;
    const Py_ssize_t n = PyList_GET_SIZE(args[0]);
    if (!to || n > DASH_MAX_PRIMES) {
        PyErr_SetString(PyExc_IndexError, "more tensors than a bundle holds");
        return nullptr;
    }
    try {
        memset(to, 0, sizeof(*to));
        for (Py_ssize_t i = 0; i < n; i++) {
            PyObject* const item = PyList_GET_ITEM(args[0], i);
            if (item == Py_None) continue;
            if (!THPVariable_Check(item)) {
                PyErr_SetString(PyExc_TypeError, "a bundle holds tensors");
                return nullptr;
            }
            const at::Tensor& t = THPVariable_Unpack(item);
            to->data[i] = t.data_ptr();
            to->chunk_stride[i] = t.stride(0);
        }
        to->n_elem = n_elem;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"describe", (PyCFunction)(void (*)(void))describe, METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bundle", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
PyMODINIT_FUNC PyInit__bundle() { return PyModule_Create(&module); }
