"""Host side of the paged calls (qcf_pages.h): the struct that crosses the boundary, refusals, empty work."""
import ctypes as C
import os
import re
import subprocess
import types

import pytest
import torch

from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd import pipeline
from paper_2604_08585_amd.inputs import LayerShape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000                      # aligned, never dereferenced: validation fails before any launch


def _desc(**kw):
    base = dict(d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, rope_base=10000.0, dtype="f32")
    base.update(kw)
    return qb.make_desc(LayerShape(**base))


def _cache(**kw):
    c = qb.PageCacheDesc(FAKE, FAKE, FAKE, FAKE, 16 * 128, 128, 64, 10, 16, 5, 0)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def _append(lib, d, c, B=1, q=FAKE, qs=256, k=FAKE, ks=128, v=FAKE, vs=128, off=FAKE, rows=4, lens=FAKE, pos=None, out=FAKE):
    return lib.qcf_page_append(C.byref(d), C.byref(c) if c else None, B, q, qs, k, ks, v, vs, off, rows, lens, pos, out, None)


def _select(lib, d, c, B=1, n_q=1, q=FAKE, seen=FAKE, keep=4, first=1, last=1, pages=FAKE, ws=FAKE, have=1 << 30):
    return lib.qcf_page_select(C.byref(d), C.byref(c), B, n_q, q, seen, keep, first, last, pages, ws, have, None)


def _attn(lib, d, c, B=1, n_q=1, q=FAKE, seen=FAKE, pages=None, keep=0, o=FAKE, lse=None, ws=FAKE, have=1 << 40):
    return lib.qcf_page_attn(C.byref(d), C.byref(c), B, n_q, q, seen, pages, keep, o, lse, ws, have, None)


def test_header_and_binding_agree(tmp_path):
    text = open(os.path.join(ROOT, "include", "qcf_pages.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(qcf_[a-z_]+)\s*\(", text))) == sorted(qb.PAGES_EXPORTS)
    for name in qb.PAGES_EXPORTS:
        assert hasattr(qb.load_library(), name)
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "qcf_pages.h"\nint main(void) { typedef qcf_page_cache P; '
                   'printf("%zu %zu %zu %zu", sizeof(P), offsetof(P, table), offsetof(P, head_stride), offsetof(P, max_pages)); }')
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "size")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "size")], capture_output=True, text=True, check=True).stdout.split()]
    P = qb.PageCacheDesc
    assert got == [C.sizeof(P), P.table.offset, P.head_stride.offset, P.max_pages.offset]


@pytest.mark.parametrize("change,status,word", [
    (dict(page_size=8), 2, b"page_size"), (dict(page_size=48), 2, b"page_size"), (dict(page_size=512), 2, b"page_size"),
    (dict(n_pages=0), 1, b"n_pages"), (dict(max_pages=0), 1, b"max_pages"), (dict(max_pages=1 << 27), 2, b"2^30"),
    (dict(reserved=1), 1, b"reserved"), (dict(slot_stride=124), 1, b"multiples of 8"), (dict(slot_stride=56), 1, b"strides"),
    (dict(head_stride=0), 1, b"strides"), (dict(slot_stride=120), 1, b"overlap"), (dict(page_stride=16 * 128 - 8), 1, b"page_stride"),
    (dict(page_stride=1 << 32), 1, b"page_stride"), (dict(slot_stride=1 << 25, page_stride=1 << 30), 1, b"strides"),
    (dict(k=None), 1, b"cache k"), (dict(v=FAKE + 8), 1, b"cache v"), (dict(table=None), 1, b"table")])
def test_caches_that_no_call_takes(change, status, word):
    lib = qb.load_library()
    d, c = _desc(), _cache(**change)
    for call in (_append, _select, _attn):
        assert call(lib, d, c) == status and word in lib.qcf_last_error(), call


def test_other_refusals():
    lib = qb.load_library()
    d, c = _desc(), _cache()
    assert _append(lib, d, None) == 1 and b"NULL" in lib.qcf_last_error()
    assert _append(lib, _desc(head_dim=96), c) == 2
    for kw, word in [(dict(B=-1), b"negative"), (dict(rows=-1), b"negative"), (dict(k=None), b"k is"), (dict(v=FAKE + 4), b"v is"),
                     (dict(off=None), b"row_off"), (dict(lens=None), b"len_dev"), (dict(ks=120), b"k_stride"), (dict(vs=132), b"v_stride"),
                     (dict(qs=248), b"q_stride"), (dict(q=None), b"both"), (dict(out=None), b"both"), (dict(out=FAKE + 4), b"q_out"),
                     (dict(qs=264), b"dense"), (dict(pos=FAKE + 1), b"pos_dev")]:
        assert _append(lib, d, c, **kw) == 1 and word in lib.qcf_last_error(), kw
    assert _append(lib, d, c, B=65536) == 2 and _append(lib, d, c, rows=(1 << 30) + 1) == 2
    for kw, word in [(dict(B=-1), b"negative"), (dict(first=3, last=2), b"n_keep"), (dict(first=-1), b"negative"), (dict(q=None), b"q is"),
                     (dict(seen=None), b"seen"), (dict(pages=None), b"pages")]:
        assert _select(lib, d, c, **kw) == 1 and word in lib.qcf_last_error(), kw
    assert _select(lib, d, _cache(bounds=None)) == 1 and b"bounds" in lib.qcf_last_error()
    assert _select(lib, d, c, n_q=17) == 2 and _select(lib, d, c, keep=1 << 27) == 2
    need = lib.qcf_page_select_workspace_bytes(C.byref(d), C.byref(c), 2, 3, 4)
    assert need >= 2 * 3 * 2 * 5 * 4
    assert _select(lib, d, c, B=2, n_q=3, have=need - 1) == 3 and _select(lib, d, c, B=2, n_q=3, ws=None) == 3
    for kw, word in [(dict(n_q=-1), b"negative"), (dict(pages=FAKE), b"n_keep"), (dict(keep=3), b"n_keep"), (dict(q=FAKE + 2), b"q is"),
                     (dict(seen=None), b"seen"), (dict(o=None), b"o_out"), (dict(lse=FAKE + 2), b"lse")]:
        assert _attn(lib, d, c, **kw) == 1 and word in lib.qcf_last_error(), kw
    assert _attn(lib, d, c, n_q=17) == 2 and _attn(lib, d, c, B=65536) == 2


def test_empty_work_is_ok_and_launches_nothing():
    lib = qb.load_library()
    d, c = _desc(), _cache()
    assert _append(lib, d, c, rows=0, k=None) == 0 and _append(lib, d, c, B=0, off=None) == 0
    assert _select(lib, d, c, B=0, q=None) == 0 and _select(lib, d, c, keep=0, first=0, last=0, pages=None) == 0
    assert _attn(lib, d, c, n_q=0, o=None) == 0 and _attn(lib, d, c, B=0) == 0
    assert lib.qcf_page_attn_workspace_bytes(C.byref(d), C.byref(c), 0, 1, 0) == 0


def test_binding_refuses_what_it_cannot_describe():
    pool = torch.zeros(3, 16, 2, 64)
    table = torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(qb.QcfError):
        qb.page_cache(pool, pool, None, table)                      # not on a GPU
    with pytest.raises(qb.QcfError):
        qb.page_cache(pool, pool[:2], None, table)
    with pytest.raises(qb.QcfError):
        qb.page_cache(pool.transpose(2, 3), pool.transpose(2, 3), None, table)
    with pytest.raises(qb.QcfError):
        qb._rows(torch.zeros(4, 2, 64).transpose(0, 1))
    cache = qb.PageCache(_cache(), (pool, pool, None, table))
    with pytest.raises(qb.QcfError, match="2 requests, 1 rows"):
        cache.of(2)
    with pytest.raises(qb.QcfError, match="n_keep"):
        qb.qcf_page_attn(_desc(), cache, 1, 1, pool, table, torch.zeros(1, 1, 2, 3, dtype=torch.int32), 4, pool, None)


@pytest.mark.parametrize("x,w,dtype", [((7, 256), (512, 256), torch.float32), ((6, 255), (512, 255), torch.float32),
                                       ((6, 256), (256, 512), torch.float32), ((6, 256), (512, 256), torch.bfloat16)])
def test_a_step_refuses_rows_weights_and_types_that_do_not_fit(x, w, dtype):
    P = types.SimpleNamespace(desc=_desc(), B=2, new=3, qkv=torch.zeros(6, 512))
    with pytest.raises(ValueError, match="2 requests of 3 rows of 256"):
        pipeline.decode_step(P, torch.zeros(x, dtype=dtype), torch.zeros(w))
