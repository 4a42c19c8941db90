"""Compiled calls that are on their way in daemon threads while the interpreter ends: each thread ends, the process goes on
to its exit status."""
import os
import subprocess
import sys
import sysconfig

import pytest

from paper_2605_25550_amd import build as B

# A call of C code takes 0.3 s in a daemon thread; the main module is cleared, which takes 0.6 s.
ENDS = """
class Late:
    def __del__(self, nap=time.sleep):
        nap(0.6)
        print("late", flush=True)


_late = Late()
threading.Thread(target=call, args=args, daemon=True).start()
time.sleep(0.05)
"""


def ends_well(code):
    r = subprocess.run([sys.executable, "-c", "import sys, threading, time\n" + code + ENDS], cwd=B.ROOT, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and "late" in r.stdout, (r.returncode, r.stdout, r.stderr[-2000:])


def test_a_call_without_the_lock(tmp_path):
    (tmp_path / "napping.cpp").write_text("""
#include <unistd.h>
#include "unlocked.h"
static auto nap(PyObject* const* v, Py_ssize_t n) {
  if (n != 1) throw 1;
  const long us = PyLong_AsLong(v[0]);
  return [=] { if (us < 0) throw 2; return usleep(us); };
}
static PyMethodDef methods[] = {{"nap", (PyCFunction)(void*)unlocked_call<nap>, METH_FASTCALL, nullptr}, {}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "napping", nullptr, -1, methods};
PyMODINIT_FUNC PyInit_napping(void) { return PyModule_Create(&module); }
""")
    subprocess.run(["g++", "-O2", "-fPIC", "-shared", "-std=c++17", "-Wall", "-I", B.CSRC, "-I", sysconfig.get_paths()["include"],
                    "napping.cpp", "-o", "napping.so"], cwd=tmp_path, check=True)
    come = f"sys.path.insert(0, {str(tmp_path)!r})\nimport napping\n"
    ends_well(come + "call, args = napping.nap, (300000,)\n")
    r = subprocess.run([sys.executable, "-c", "import sys\n" + come + "print(napping.nap(), napping.nap(-1), napping.nap(10))"],
                       capture_output=True, text=True)
    assert r.stdout.split() == ["None", "None", "0"]  # no fit, an exception, a status


@pytest.mark.gpu
def test_an_operators_call():
    """A function that sleeps stands in for the library's: as long as the rows that it is given say."""
    ends_well("""
import ctypes
import torch
import paper_2605_25550_amd as dm
dm.lib()
if dm._CALLS is None:
    raise SystemExit("the compiled calls are not built")
usleep = ctypes.cast(ctypes.CDLL(None).usleep, ctypes.c_void_p).value
dm._CALLS.bind(dm.LinearShape, dm.QkShape, usleep, usleep, usleep, usleep)
args = (torch.zeros(300000, 32, device="cuda"), torch.zeros(300000 * 16, dtype=torch.uint8, device="cuda"),
        torch.zeros(300000 * 8, dtype=torch.uint8, device="cuda"))
call = dm._CALLS.quantize_fp4
assert call(args[0][:10], args[1][:160], args[2][:80]) == 0
""")
