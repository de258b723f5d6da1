"""The rule by which an append's workgroups take several KV heads (csrc/page_layout.h), on the CPU."""
import pytest

import append_rules
from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd.inputs import LayerShape


def _heads(dtype, Hkv, D, page, B, rows):
    desc = qb.make_desc(LayerShape(Hkv * D, Hkv, Hkv, D, 10000.0, dtype))
    return append_rules.heads(desc, qb.PageCacheDesc(4096, 4096, None, 4096, page * Hkv * D, Hkv * D, D, 100, page, 10, 0), B, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_heads_divide_and_fill_a_wave_at_most(dtype, D):
    vectors = D // 2 // (8 if dtype == "bf16" else 4)
    seen = set()
    for Hkv in (1, 2, 3, 6, 8, 16, 64, 1024):
        for page in (16, 32, 64, 128, 256):
            for B in (1, 8, 70, 300, 65535):
                for rows in (1, 100, 5000, 100000, 1 << 30):
                    h = _heads(dtype, Hkv, D, page, B, rows)
                    assert h >= 1 and Hkv % h == 0 and h & (h - 1) == 0 and h * vectors <= 64
                    seen.add(h)
    assert max(seen) == 64 // vectors


def test_heads_by_hand():
    assert _heads("bf16", 8, 128, 16, 8, 8) == 1                       # a step of eight requests: 16 units
    assert _heads("bf16", 8, 128, 16, 256, 256) == 8                   # of 256: 528 units
    assert _heads("bf16", 8, 128, 16, 16, 32000) == 8                  # 2032 units, eight workgroups to a compute unit
    assert _heads("bf16", 8, 128, 16, 4, 12000) == 4                   # 758 units: not three workgroups to a compute unit
    assert _heads("bf16", 8, 128, 256, 100, 100 * 256) == 4            # 300 units of 256 rows: two workgroups to a compute unit
    assert _heads("bf16", 8, 128, 128, 100, 100 * 128) == 8
