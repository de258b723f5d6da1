"""The rule by which contexts are taken whole (csrc/page_layout.h) takes the faster form where the two were measured well apart."""
import pytest

import page_rules
from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd.inputs import LayerShape


@pytest.mark.parametrize("dtype,H,Hkv,D,B,tokens,whole", [
    # us whole and divided: 21.4 23.5, 17.6 20.6, 48.1 42.1, 15.3 10.3, 16.0 13.4, 40.0 42.7
    ("bf16", 32, 8, 128, 16, 1536, 1), ("bf16", 32, 8, 128, 16, 1024, 1), ("bf16", 32, 8, 128, 16, 4096, 0), ("bf16", 32, 8, 128, 1, 1024, 0),
    ("bf16", 32, 8, 128, 8, 1024, 0), ("bf16", 32, 8, 128, 64, 1024, 1),
    # 21.5 24.0, 20.5 22.1, 11.0 12.9, 16.3 11.1, 15.9 10.5, 20.6 27.1
    ("bf16", 64, 8, 128, 16, 1536, 1), ("bf16", 32, 32, 128, 4, 1536, 1), ("bf16", 32, 8, 64, 2, 1024, 1), ("bf16", 32, 8, 64, 2, 2048, 0),
    ("f32", 4, 2, 64, 2, 1024, 0), ("f32", 32, 8, 128, 16, 512, 1)])
def test_whole_where_it_was_faster(dtype, H, Hkv, D, B, tokens, whole):
    desc = qb.make_desc(LayerShape(H * D, H, Hkv, D, 10000.0, dtype))
    cache = qb.PageCacheDesc(4096, 4096, None, 4096, 16 * Hkv * D, Hkv * D, D, 1 << 20, 16, tokens // 16, 0)
    assert page_rules.division(desc, cache, B, 1, 0)["whole"] == whole
