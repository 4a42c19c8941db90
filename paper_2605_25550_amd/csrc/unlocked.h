// A compiled call of the binding: gather(arguments) may throw and own things, and returns what makes the C
// call; that is made without the interpreter's lock, as ctypes makes it, and its status returned.  None: the
// arguments did not fit (gather threw), or the call ended by an exception.
#pragma once
#include <Python.h>

#include <optional>
#include <type_traits>

template <auto gather>
PyObject* unlocked_call(PyObject*, PyObject* const* v, Py_ssize_t n) {
  using Call = decltype(gather(v, n));
  // PyEval_RestoreThread does not return to a thread that finds the interpreter at its end: it ends the thread,
  // which unwinds its stack.  A destructor or a catch around it would end the process instead.
  static_assert(std::is_trivially_destructible_v<Call>, "nothing is alive around PyEval_RestoreThread");
  std::optional<Call> call;
  try {
    call.emplace(gather(v, n));
  } catch (...) {
    Py_RETURN_NONE;
  }
  long status = 0;
  bool done = true;
  PyThreadState* state = PyEval_SaveThread();
  try {
    status = (long)(*call)();
  } catch (...) {
    done = false;
  }
  PyEval_RestoreThread(state);
  if (!done) Py_RETURN_NONE;
  return PyLong_FromLong(status);
}
