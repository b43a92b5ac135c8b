// What the two sources of the binding's native module share.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

namespace cerpy {

// None: the current torch stream of the current device; an int; or an object with .cuda_stream.  false: a Python error is set.
bool stream_pointer(PyObject* s, void** out);
// The current device's number, by torch's own path once torch has initialised it; -1: not known (no torch, or not initialised), -2: error.
long current_device();
// Raises CerError for a code other than 0.
bool raise_unless_ok(int rc, const char* name);
// Loads the library (binding.lib), which binds the entry points' addresses.
bool load_library();

extern PyMethodDef operator_methods[];  // pybind_operators.cpp
bool setup_operators();

}  // namespace cerpy
