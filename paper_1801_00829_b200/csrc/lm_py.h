// The calls of lm.py, for the table of the CPython extension (training_py.cpp).
#pragma once

namespace fo_py {

PyObject *head_norm_impl(PyObject *const *a);
PyObject *head_norm_grad_impl(PyObject *const *a);
PyObject *scan_impl(PyObject *const *a);
PyObject *scan_grad_impl(PyObject *const *a);
PyObject *distill_impl(PyObject *const *a);
PyObject *distill_grad_impl(PyObject *const *a);

}  // namespace fo_py
