"""The heads that a workgroup of an append takes (csrc/page_layout.h), compiled for the tests with 256 compute units."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "page_layout.h"
namespace qcf { int compute_unit_count() { return 256; } }
extern "C" int heads(const qcf_layer_desc* L, const qcf_page_cache* c, int B, long long rows) {
  return qcf::pages::append_heads(*L, *c, qcf::pages::append_units(*c, B, rows));
}
"""


@functools.lru_cache(None)
def library():
    folder = tempfile.mkdtemp()
    src, so = os.path.join(folder, "rules.cpp"), os.path.join(folder, "rules.so")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2604_08585_amd", "csrc"), src, "-o", so], check=True)
    lib = C.CDLL(so)
    lib.heads.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_longlong]
    return lib


def heads(desc, cache, B, rows):
    return library().heads(C.addressof(desc), C.addressof(getattr(cache, "desc", cache)), B, rows)
