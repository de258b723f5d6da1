"""Host side of the calls over 8-bit pages and of eviction (qcf_pages8.h, qcf_evict.h): exports, refusals, empty work, the binding."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd.inputs import LayerShape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000                      # aligned, never dereferenced: validation fails before any launch
H, HKV, D, PAGES, B, NEW, KEEP, ROWS, WIDTH = 4, 2, 64, 5, 3, 2, 4, 7, 5
I32, I64, F32, BF16, E4M3 = torch.int32, torch.int64, torch.float32, torch.bfloat16, torch.float8_e4m3fn


def _desc(**kw):
    return qb.make_desc(LayerShape(**{**dict(d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, rope_base=10000.0, dtype="f32"), **kw}))


def _raw(**kw):
    c = qb.PageCacheDesc(FAKE, FAKE, FAKE, FAKE, 16 * 128, 128, 64, 10, 16, 5, 0)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def _append(d, c, B=1, sc=FAKE, q=FAKE, qs=256, k=FAKE, ks=128, v=FAKE, vs=128, off=FAKE, rows=4, lens=FAKE, pos=None, out=FAKE):
    return qb.load_library().qcf_page8_append(C.byref(d), C.byref(c) if c else None, sc, B, q, qs, k, ks, v, vs, off, rows, lens, pos, out, None)


def _attn(d, c, B=1, sc=FAKE, n_q=1, q=FAKE, seen=FAKE, pages=None, keep=0, o=FAKE, lse=None, ws=FAKE, have=1 << 40):
    return qb.load_library().qcf_page8_attn(C.byref(d), C.byref(c), sc, B, n_q, q, seen, pages, keep, o, lse, ws, have, None)


def _weigh(d, c, B=1, sc=FAKE, n_q=1, q=FAKE, seen=FAKE, lse=FAKE, old=None, alpha=1.0, beta=1.0, w=FAKE):
    return qb.load_library().qcf_page_weigh(C.byref(d), C.byref(c), sc, B, n_q, q, seen, lse, old, alpha, beta, w, None)


def _evict(d, c, B=1, sc=FAKE, lens=FAKE, w=FAKE, keep=4, first=1, last=1, to=None, to_sc=FAKE, kept=FAKE, to_w=None, to_len=FAKE, ws=FAKE, have=1 << 50):
    return qb.load_library().qcf_page_evict(C.byref(d), C.byref(c), sc, B, lens, w, keep, first, last, C.byref(to or _raw()), to_sc, kept, to_w,
                                            to_len, ws, have, None)


def _said():
    return qb.load_library().qcf_last_error()


@pytest.mark.parametrize("header,names", [("qcf_pages8.h", qb.PAGES8_EXPORTS), ("qcf_evict.h", qb.EVICT_EXPORTS)])
def test_header_and_binding_agree(header, names):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(qcf_[a-z0-9_]+)\s*\(", text))) == sorted(names)
    assert all(hasattr(qb.load_library(), n) for n in names)


@pytest.mark.parametrize("change,status,word", [
    (dict(page_size=8), 2, b"page_size"), (dict(n_pages=0), 1, b"n_pages"), (dict(max_pages=1 << 27), 2, b"2^30"), (dict(reserved=1), 1, b"reserved"),
    (dict(slot_stride=120), 1, b"overlap"), (dict(page_stride=1 << 32), 1, b"page_stride"), (dict(k=None), 1, b"cache k"),
    (dict(v=FAKE + 8), 1, b"cache v"), (dict(table=None), 1, b"table"), (dict(slot_stride=136, page_stride=16 * 136), 1, b"multiples of 16"),
    (dict(page_stride=16 * 128 + 8), 1, b"multiples of 16")])
def test_caches_that_no_call_takes(change, status, word):
    d, c = _desc(), _raw(**change)
    for call in (_append, _attn, _weigh, _evict):
        assert call(d, c) == status and word in _said(), call
    if b"16" not in word:
        assert _evict(d, _raw(), to=c) == status and word in _said()
    else:
        assert _evict(d, _raw(), to=c) == 1 and word in _said()


def test_other_refusals():
    d, c = _desc(), _raw()
    assert _append(d, None) == 1 and _append(_desc(head_dim=96), c) == 2
    for kw, word in [(dict(B=-1), b"negative"), (dict(rows=-1), b"negative"), (dict(k=None), b"k is"), (dict(off=None), b"row_off"),
                     (dict(ks=120), b"k_stride"), (dict(q=None), b"both"), (dict(qs=264), b"dense"), (dict(sc=None), b"scales"),
                     (dict(sc=FAKE + 2), b"scales"), (dict(pos=FAKE + 1), b"pos_dev")]:
        assert _append(d, c, **kw) == 1 and word in _said(), kw
    assert _append(d, c, B=65536) == 2 and _append(d, c, rows=(1 << 30) + 1) == 2
    for kw, word in [(dict(n_q=-1), b"negative"), (dict(pages=FAKE), b"n_keep"), (dict(keep=3), b"n_keep"), (dict(q=FAKE + 2), b"q is"),
                     (dict(seen=None), b"seen"), (dict(o=None), b"o_out"), (dict(sc=None), b"scales")]:
        assert _attn(d, c, **kw) == 1 and word in _said(), kw
    assert _attn(d, c, n_q=17) == 2 and _attn(d, _raw(max_pages=1 << 16), have=16) == 3
    for kw, word in [(dict(n_q=-1), b"negative"), (dict(q=None), b"q is"), (dict(seen=None), b"seen"), (dict(lse=None), b"lse"),
                     (dict(old=FAKE + 1), b"old"), (dict(w=None), b"weights"), (dict(w=FAKE + 4), b"weights"), (dict(alpha=float("nan")), b"finite"),
                     (dict(beta=float("inf")), b"finite"), (dict(sc=FAKE + 1), b"scales")]:
        assert _weigh(d, c, **kw) == 1 and word in _said(), kw
    assert _weigh(d, c, n_q=17) == 2 and _weigh(d, c, B=65536) == 2
    for kw, word in [(dict(B=-1), b"negative"), (dict(keep=0), b"positive"), (dict(first=3, last=2), b"n_keep"),
                     (dict(first=-1), b"negative"), (dict(sc=None), b"both"), (dict(to_sc=None), b"both"), (dict(lens=None), b"len_dev"),
                     (dict(w=None), b"weights"), (dict(kept=None), b"kept"), (dict(to_len=None), b"to_len"), (dict(to_w=FAKE), b"other memory"),
                     (dict(to_w=FAKE + 4), b"to_weights")]:
        assert _evict(d, c, **kw) == 1 and word in _said(), kw
    assert _evict(d, c, B=65536) == 2
    for call in (_append, _attn, _weigh, _evict):
        assert call(d, _raw(n_pages=1 << 29)) == 2 and b"2^31 scales" in _said(), call
    long = _raw(max_pages=1 << 16)
    need = qb.load_library().qcf_page_evict_workspace_bytes(C.byref(d), C.byref(long), 3, 4)
    assert need > 0 and _evict(d, long, B=3, have=need - 1) == 3 and _evict(d, long, B=3, ws=None) == 3
    assert qb.load_library().qcf_page_evict_workspace_bytes(C.byref(d), C.byref(c), 3, 4) == 0


def test_launches_of_more_than_2_to_the_32_threads_are_refused():
    wide = _raw(max_pages=1 << 26, n_pages=1 << 26)
    assert _append(_desc(n_q_heads=1, n_kv_heads=1), _raw(slot_stride=64), rows=1 << 30, ks=64, vs=64, q=None, out=None) == 2 and b"too many rows" in _said()
    assert _evict(_desc(), wide, B=64, keep=1 << 30, to=wide) == 2 and b"too many rows" in _said()
    d = _desc(n_q_heads=128, n_kv_heads=128)
    c = _raw(slot_stride=128 * 64, page_stride=16 * 128 * 64)
    assert _evict(d, c, B=65535, to=c) == 2 and b"too many rows" in _said()


def test_empty_work_is_ok_and_launches_nothing():
    d, c = _desc(), _raw()
    assert _append(d, c, rows=0, k=None) == 0 and _append(d, c, B=0, off=None) == 0
    assert _attn(d, c, n_q=0, o=None) == 0 and _attn(d, c, B=0) == 0
    assert _weigh(d, c, n_q=0, w=None) == 0 and _weigh(d, c, B=0) == 0 and _evict(d, c, B=0, kept=None) == 0
    assert qb.load_library().qcf_page8_attn_workspace_bytes(C.byref(d), C.byref(c), 0, 1, 0) == 0


# ------------------------------------------------------------------ the binding: refused for its device once everything else fits

def _z(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype)


def _cache(dtype=F32, heads=HKV, d=D, eight=True, width=WIDTH):
    pool = torch.zeros(PAGES, 16, heads, d, dtype=torch.uint8).view(E4M3) if eight else _z(PAGES, 16, heads, d, dtype=dtype)
    c = qb.PageCacheDesc(4096, 4096, 4096, 4096, 16 * heads * d, heads * d, d, PAGES, 16, width, 0)
    tensors = (pool, pool, None, torch.zeros(B, width, dtype=I32))
    return qb.Page8Cache(c, tensors, _z(PAGES, heads, 2, 1), dtype) if eight else qb.PageCache(c, tensors)


def _b_append(cache=None, desc=None, **kw):
    a = dict(q=_z(ROWS, H, D), k=_z(ROWS, HKV, D), v=_z(ROWS, HKV, D), row_off=_z(B + 1, dtype=I64), total_rows=ROWS, lens=_z(B, dtype=I32),
             pos=_z(ROWS, dtype=I32), q_out=_z(ROWS, H, D))
    qb.qcf_page8_append(desc or _desc(), cache or _cache(), B, **{**a, **kw})


def _b_attn(cache=None, desc=None, **kw):
    a = dict(q=_z(B, NEW, H, D), seen=_z(B, NEW, dtype=I32), pages=_z(B, NEW, HKV, KEEP, dtype=I32), n_keep=KEEP, o_out=_z(B, NEW, H, D),
             lse_out=_z(B, NEW, H), workspace=_z(1 << 16, dtype=torch.uint8))
    qb.qcf_page8_attn(desc or _desc(), cache or _cache(), B, NEW, **{**a, **kw})


def _b_weigh(cache=None, desc=None, **kw):
    a = dict(q=_z(B, NEW, H, D), seen=_z(B, NEW, dtype=I32), lse=_z(B, NEW, H), old=_z(B, dtype=I32), alpha=1.0, beta=1.0,
             weights=_z(B, HKV, 16 * WIDTH))
    qb.qcf_page_weigh(desc or _desc(), cache or _cache(), B, NEW, **{**a, **kw})


def _b_evict(cache=None, desc=None, **kw):
    a = dict(lens=_z(B, dtype=I32), weights=_z(B, HKV, 16 * WIDTH), n_keep=KEEP, n_first=1, n_last=1, to=_cache(width=2), kept=_z(B, HKV, KEEP, dtype=I32),
             to_weights=_z(B, HKV, 32), to_lens=_z(B, dtype=I32))
    qb.qcf_page_evict(desc or _desc(), cache or _cache(), B, **{**a, **kw})


@pytest.mark.parametrize("call,kw", [
    (_b_append, {}), (_b_attn, {}), (_b_weigh, {}), (_b_evict, {}), (_b_append, dict(q=None, q_out=None, pos=None)), (_b_attn, dict(pages=None, n_keep=0)),
    (_b_weigh, dict(old=None)), (_b_evict, dict(to_weights=None)), (_b_weigh, dict(weights=_z(B + 2, HKV, 16 * WIDTH))),
    (_b_weigh, dict(cache=_cache(eight=False))), (_b_evict, dict(cache=_cache(eight=False), to=_cache(eight=False, width=2)))])
def test_what_fits_is_only_refused_for_its_device(call, kw):
    with pytest.raises(qb.QcfError, match="current device"):
        call(**kw)


@pytest.mark.parametrize("call,kw", [
    (_b_append, dict(k=_z(ROWS, HKV, D, dtype=BF16))), (_b_append, dict(k=_z(ROWS - 1, HKV, D))), (_b_append, dict(lens=_z(B, dtype=I64))),
    (_b_append, dict(cache=_cache(dtype=BF16))), (_b_append, dict(cache=_cache(heads=4))), (_b_append, dict(cache=_cache(eight=False))),
    (_b_append, dict(q_out=_z(ROWS, H, D - 1))), (_b_attn, dict(seen=_z(B * NEW - 1, dtype=I32))), (_b_attn, dict(n_keep=KEEP + 1)),
    (_b_attn, dict(o_out=_z(B, NEW, H, D, dtype=BF16))), (_b_attn, dict(cache=_cache(eight=False))), (_b_attn, dict(lse_out=_z(B, NEW, H - 1))),
    (_b_weigh, dict(weights=_z(B, HKV, 16 * WIDTH - 16))), (_b_weigh, dict(weights=_z(B - 1, HKV, 16 * WIDTH))), (_b_weigh, dict(lse=_z(B, NEW, H - 1))),
    (_b_weigh, dict(old=_z(B, dtype=I64))), (_b_weigh, dict(weights=_z(B, HKV, 16 * WIDTH, dtype=BF16))), (_b_weigh, dict(q=_z(B, NEW, H, D, dtype=BF16))),
    (_b_evict, dict(kept=_z(B, HKV, KEEP + 1, dtype=I32))), (_b_evict, dict(kept=_z(B - 1, HKV, KEEP, dtype=I32))), (_b_evict, dict(to=_cache(eight=False))),
    (_b_evict, dict(to=_cache(heads=1))), (_b_evict, dict(to_weights=_z(B, HKV, 48))), (_b_evict, dict(lens=_z(B - 1, dtype=I32))),
    (_b_evict, dict(to=_cache(dtype=BF16)))])
def test_tensors_that_do_not_hold_what_a_call_reads_or_writes(call, kw):
    with pytest.raises(qb.QcfError) as e:
        call(**kw)
    assert "current device" not in str(e.value)


def test_calls_for_pages_of_the_layers_type_refuse_8_bit_pages():
    c, d = _cache(), _desc()
    with pytest.raises(qb.QcfError, match="8-bit"):
        qb.qcf_page_append(d, c, B, None, _z(ROWS, HKV, D), _z(ROWS, HKV, D), _z(B + 1, dtype=I64), ROWS, _z(B, dtype=I32), None, None)
    with pytest.raises(qb.QcfError, match="8-bit"):
        qb.qcf_page_attn(d, c, B, 1, _z(B, 1, H, D), _z(B, dtype=I32), None, 0, _z(B, 1, H, D), None, _z(16))
    with pytest.raises(qb.QcfError, match="current device"):                     # (selection reads bounds alone)
        qb.qcf_page_select(d, c, B, 1, _z(B, 1, H, D), _z(B, dtype=I32), KEEP, 1, 1, _z(B, 1, HKV, KEEP, dtype=I32), _z(1 << 12))


def test_binding_refuses_what_it_cannot_describe():
    pool, table = torch.zeros(3, 16, 2, 64, dtype=torch.uint8).view(E4M3), torch.zeros(1, 2, dtype=I32)
    sc = _z(3, 2, 2, 1)
    for args in [(pool, pool, sc, None, table, torch.float16), (pool.view(torch.uint8), pool.view(torch.uint8), sc, None, table, F32),
                 (pool, pool[:2], sc, None, table, F32), (pool, pool, sc, None, table, F32)]:          # (the last: not on a GPU)
        with pytest.raises(qb.QcfError):
            qb.page8_cache(*args)
