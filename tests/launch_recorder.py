"""Records what the library asks of the runtime, without a GPU: a small shared object stands in for the runtime's calls in a
child process, which loads the built library behind it and runs a piece of Python there."""

import json
import os
import shutil
import subprocess
import sys
import textwrap

import pytest

from paper_2605_17862_amd import binding as fb

SOURCE = r"""
#include <stddef.h>
#include <string.h>
typedef struct { unsigned x, y, z; } dim3;
enum { MOST = 4096, BYTES = 4096 };
const void* launched[MOST];
unsigned grids[MOST];
char arguments[MOST][BYTES];      /* of the first argument, as many bytes as asked for */
const void* attributes[MOST];
int launches, attribute_calls, argument_bytes;

int hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t lds, void* stream) {
  (void)block; (void)lds; (void)stream;
  if (launches == MOST) return 1;
  launched[launches] = f;
  grids[launches] = grid.x;
  memcpy(arguments[launches], args[0], argument_bytes);
  ++launches;
  return 0;
}
/* (what a launch passes through on its way; the runtime's own refuse without a device) */
static dim3 next_grid, next_block;
static size_t next_lds;
static void* next_stream;
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, void* stream) {
  next_grid = grid; next_block = block; next_lds = lds; next_stream = stream;
  return 0;
}
int __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, void** stream) {
  *grid = next_grid; *block = next_block; *lds = next_lds; *stream = next_stream;
  return 0;
}
int hipFuncSetAttribute(const void* f, int what, int value) {
  (void)what; (void)value;
  if (attribute_calls == MOST) return 1;
  attributes[attribute_calls++] = f;
  return 0;
}
int hipGetDevice(int* device) { *device = 0; return 0; }
int hipGetLastError(void) { return 0; }
int hipDeviceGetAttribute(int* value, int what, int device) { (void)what; (void)device; *value = 256; return 0; }
"""

# what a child starts with: lib (the library), rec (the recorder), P = c_void_p and the names of ctypes
PROLOGUE = """
import ctypes, json, sys
from ctypes import *
rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
P = c_void_p
def count(name):
    return c_int.in_dll(rec, name).value
"""


def recorded(tmp_path, code):
    """What `code` leaves in `result`."""
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    fb.load_library()                                       # (fails loudly where it is not built)
    src, so = tmp_path / "recorder.c", tmp_path / "recorder.so"
    src.write_text(SOURCE)
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", str(src), "-o", str(so)], check=True, capture_output=True)
    child = PROLOGUE + textwrap.dedent(code) + "\nprint(json.dumps(result))\n"
    out = subprocess.run([sys.executable, "-c", child, str(so), os.path.abspath(fb.library_path())], check=True, capture_output=True, text=True)
    return json.loads(out.stdout.splitlines()[-1])
