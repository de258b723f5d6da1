"""Paged calls of more rows than a launch has threads for are refused on the host, before anything is launched."""
import ctypes as C

from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd.inputs import LayerShape

FAKE = 0x1000                      # aligned, never dereferenced
REFUSED = 2                        # QCF_ERR_UNSUPPORTED


def _desc(H, Hkv):
    return qb.make_desc(LayerShape(H * 64, H, Hkv, 64, 10000.0, "bf16"))


def _cache(Hkv, width, page=16):
    return qb.PageCacheDesc(FAKE, FAKE, FAKE, FAKE, page * Hkv * 64, Hkv * 64, 64, 10, page, width, 0)


def test_launches_of_more_than_2_to_the_32_threads_are_refused():
    lib = qb.load_library()
    # 65535 requests of 16 rows, 8 KV heads: 8.4 million workgroups of 1024 threads choose pages
    d, c = _desc(8, 8), _cache(8, 4)
    assert lib.qcf_page_select(C.byref(d), C.byref(c), 65535, 16, FAKE, FAKE, 2, 0, 0, FAKE, FAKE, 1 << 40, None) == REFUSED
    assert b"too many rows" in lib.qcf_last_error()
    # 16.8 million of 512 threads attend to lists
    d, c = _desc(16, 16), _cache(16, 4)
    assert lib.qcf_page_attn(C.byref(d), C.byref(c), 65535, 16, FAKE, FAKE, FAKE, 2, FAKE, None, FAKE, 1 << 40, None) == REFUSED
    assert b"too many rows" in lib.qcf_last_error()
    # 67 million pages get rows, 1 head to a workgroup
    d, c = _desc(1, 1), _cache(1, 4)
    assert lib.qcf_page_append(C.byref(d), C.byref(c), 1, None, 0, FAKE, 64, FAKE, 64, FAKE, 1 << 30, FAKE, None, None, None) == REFUSED
    assert b"too many rows" in lib.qcf_last_error()
