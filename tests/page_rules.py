"""The division of the attention over pages (csrc/page_layout.h), compiled for the tests with 256 compute units."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "page_layout.h"
namespace qcf { int compute_unit_count() { return 256; } }
using namespace qcf::pages;
extern "C" void division(const qcf_layer_desc* L, const qcf_page_cache* c, int B, int n_q, int n_keep, long long* out) {
  const Division d = divide(*L, *c, B, n_q, n_keep);
  const long long v[] = {d.contexts, d.rows, d.row_tiles, d.row_blocks, d.inner, d.slots, d.least, d.pad, d.whole, divides(d),
                         (long long)parts(d), (long long)workspace(*L, d), part_rows(d)};
  for (int i = 0; i < 13; ++i) out[i] = v[i];
}
extern "C" long long grains(long long tokens) { return grains_of(tokens); }
extern "C" long long range_grains(long long total, int slots, int least) { return range_of(total, slots, least); }
"""
NAMES = ("contexts", "rows", "row_tiles", "row_blocks", "inner", "slots", "least", "pad", "whole", "divides", "parts", "workspace", "part_rows")


@functools.lru_cache(None)
def library():
    folder = tempfile.mkdtemp()
    src, so = os.path.join(folder, "rules.cpp"), os.path.join(folder, "rules.so")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2604_08585_amd", "csrc"), src, "-o", so], check=True)
    lib = C.CDLL(so)
    lib.grains.restype = lib.range_grains.restype = C.c_longlong
    lib.grains.argtypes = [C.c_longlong]
    lib.range_grains.argtypes = [C.c_longlong, C.c_int, C.c_int]
    return lib


def division(desc, cache, B, n_q, n_keep):
    """How a call's contexts are divided; cache: a PageCache or its descriptor."""
    out = (C.c_longlong * len(NAMES))()
    library().division(C.byref(desc), C.byref(getattr(cache, "desc", cache)), B, n_q, n_keep, out)
    return dict(zip(NAMES, out))
