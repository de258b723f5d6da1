"""How calls over 8-bit pages divide their work (csrc/page_layout.h, compiled for the tests with 256 compute units)."""
import ctypes as C
import functools
import itertools
import os
import subprocess
import tempfile

import pytest

from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd.inputs import LayerShape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "page_layout.h"
namespace qcf { int compute_unit_count() { return 256; } }
using namespace qcf::pages;
extern "C" void division(const qcf_layer_desc* L, const qcf_page_cache* c, int B, int n_q, int n_keep, long long* out) {
  const Division d = divide(*L, *c, B, n_q, n_keep, 1);
  const long long v[] = {d.contexts, d.rows, d.row_tiles, d.row_blocks, d.inner, d.heads, d.slots, d.least, d.whole, divides(d), (long long)parts(d),
                         (long long)workspace(*L, d), part_rows(d), at_once(L->head_dim, d.row_tiles, true)};
  for (int i = 0; i < 14; ++i) out[i] = v[i];
}
"""
NAMES = ("contexts", "rows", "row_tiles", "row_blocks", "inner", "heads", "slots", "least", "whole", "divides", "parts", "workspace", "part_rows", "at_once")


@functools.lru_cache(None)
def library():
    folder = tempfile.mkdtemp()
    src, so = os.path.join(folder, "rules.cpp"), os.path.join(folder, "rules.so")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2604_08585_amd", "csrc"), src, "-o", so], check=True)
    return C.CDLL(so)


def division(H, Hkv, D, dtype, B, n_q, tokens, n_keep=0, adjacent=True, page=16):
    desc = qb.make_desc(LayerShape(H * D, H, Hkv, D, 10000.0, dtype))
    strides = (Hkv * D, D) if adjacent else (D, page * D)
    c = qb.PageCacheDesc(4096, 4096, None, 4096, page * Hkv * D, *strides, 1000, page, -(-tokens // page), 0)
    out = (C.c_longlong * len(NAMES))()
    library().division(C.byref(desc), C.byref(c), B, n_q, n_keep, out)
    return dict(zip(NAMES, out))


SHAPES = [(32, 8, 128), (64, 8, 128), (32, 8, 64), (4, 2, 64), (6, 3, 128), (16, 1, 128), (64, 64, 64), (128, 2, 64), (12, 4, 64)]


@pytest.mark.parametrize("H,Hkv,D", SHAPES)
def test_what_a_division_promises(H, Hkv, D):
    for dtype, B, n_q, tokens, keep, adjacent in itertools.product(("bf16", "f32"), (1, 7, 64), (1, 4, 16), (16, 700, 5000, 131072), (0, 9), (True, False)):
        d = division(H, Hkv, D, dtype, B, n_q, tokens, keep, adjacent)
        assert d["inner"] == Hkv * d["row_blocks"] and d["inner"] % d["heads"] == 0 and Hkv % d["heads"] == 0
        assert d["row_blocks"] * 16 * d["row_tiles"] >= d["rows"] > (d["row_blocks"] - 1) * 16 * d["row_tiles"]
        # heads side by side: only where their rows lie next to each other, in kernels that there are
        assert d["heads"] in (1, 256 // D) and (d["heads"] == 1 or (adjacent and not keep and d["row_tiles"] == 1))
        # as many workgroups as the GPU holds at once, or one range
        assert d["slots"] == 1 or d["slots"] * d["inner"] // d["heads"] <= d["at_once"] * 256
        assert d["parts"] == 2 * d["slots"] * d["inner"] * d["part_rows"]
        assert d["workspace"] == (d["parts"] * (D + 2) * 4 if d["divides"] else 0)
        assert not (d["whole"] and d["divides"]) and not (d["whole"] and d["row_tiles"] > 1)


def test_heads_side_by_side_where_there_is_much_to_read():
    assert division(32, 8, 128, "bf16", 64, 1, 12288)["heads"] == 2 and division(32, 8, 64, "bf16", 64, 1, 12288)["heads"] == 4
    assert division(32, 8, 128, "bf16", 64, 1, 12288, adjacent=False)["heads"] == 1
    assert division(32, 8, 128, "bf16", 1, 1, 30000)["heads"] == 1 and division(32, 8, 128, "bf16", 1, 1, 131072)["heads"] == 2
    assert division(6, 3, 128, "bf16", 64, 1, 131072)["heads"] == 1                                # (three heads: no pairs)


@pytest.mark.parametrize("dtype,D,workgroups,longest", [("bf16", 64, 1, 1400), ("f32", 64, 1, 704), ("bf16", 64, 64, 1728), ("bf16", 64, 192, 3294), ("f32", 64, 192, 1647),
                                                        ("bf16", 128, 192, 3294), ("bf16", 64, 512, 3072), ("bf16", 128, 264, 1024), ("f32", 128, 512, 512)])
def test_whole_contexts_up_to_a_number_of_tokens(dtype, D, workgroups, longest):
    B = max(1, workgroups // 8)
    shape = (32, 8, D) if workgroups >= 8 else (4, 1, D)
    assert division(*shape, dtype, B, 1, longest - 64, adjacent=False)["whole"] and not division(*shape, dtype, B, 1, longest + 64, adjacent=False)["whole"]


def test_whole_contexts_of_several_rows_and_of_heads_side_by_side():
    for adjacent, B, longest in ((False, 64, 3072), (True, 64, 1024), (True, 32, 4096)):
        below, above = (division(32, 8, 128, "bf16", B, 4, n, adjacent=adjacent) for n in (longest, longest + 16))
        assert below["heads"] == above["heads"] == 1 + adjacent and below["whole"] and not above["whole"]
    # (kept pages: a row of its own, whatever their number)
    assert division(32, 8, 128, "bf16", 16, 4, 5000, n_keep=64)["whole"] and not division(32, 8, 128, "bf16", 16, 4, 5000, n_keep=65)["whole"]
    for D, B, longest in ((64, 32, 2048), (64, 64, 1024)):
        below, above = division(32, 8, D, "bf16", B, 1, longest), division(32, 8, D, "bf16", B, 1, longest + 16)
        assert below["heads"] == above["heads"] == 4 and below["whole"] and not above["whole"]
    assert division(32, 8, 128, "bf16", 64, 1, 1000)["heads"] == 2 and not division(32, 8, 128, "bf16", 64, 1, 1000)["whole"]


def test_two_tiles_of_rows_where_there_is_much_to_read():
    assert division(64, 8, 128, "bf16", 8, 4, 6016)["row_tiles"] == 1 and division(64, 8, 128, "bf16", 64, 4, 12288)["row_tiles"] == 2
    assert division(32, 8, 64, "bf16", 8, 8, 6016)["row_tiles"] == 2 and division(32, 8, 128, "bf16", 64, 4, 12288)["row_tiles"] == 1
