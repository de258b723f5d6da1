"""Division of the attention over pages (csrc/page_layout.h), on the CPU: every grain of every context in one range, every part in a
place of its own, and the workspace that is reported."""
import ctypes as C
import random

import pytest

import page_rules
from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd.inputs import LayerShape


def _cache(Hkv, D, page, width):
    return qb.PageCacheDesc(4096, 4096, None, 4096, page * Hkv * D, Hkv * D, D, 1 << 20, page, width, 0)


def _ranges(d, tokens):
    """Ranges as the kernels form them: lists of (context, first grain, grains of it, part or None), one for each range."""
    lib = page_rules.library()
    grains = [lib.grains(t) for t in tokens]
    pad, rooms, apart = d["pad"], [g + d["pad"] for g in grains], False
    if len(tokens) <= 64:
        up = [-(-g // d["least"]) * d["least"] for g in grains]
        if sum(up) <= d["least"] * d["slots"]:
            pad, rooms, apart = 0, up, True
    size = lib.range_grains(sum(rooms), d["slots"], d["least"])
    out, starts, at = [[] for _ in range(d["slots"])], [], 0
    for x, (g, room) in enumerate(zip(grains, rooms)):
        starts.append(at + pad)
        for r in range(at // size, (at + room - 1) // size + 1):
            assert r < d["slots"]
            g0, g1 = max(r * size - starts[x], 0), min((r + 1) * size - starts[x], g)
            if g1 > g0:
                out[r].append((x, g0, g1 - g0, None if g1 - g0 == g else 2 * r + (g0 == 0)))
        at += room
    if apart:
        assert all(len(r) <= 1 for r in out)
    return grains, starts, size, out


@pytest.mark.parametrize("dtype,H,Hkv,D", [("bf16", 32, 8, 128), ("bf16", 64, 8, 128), ("bf16", 64, 64, 64), ("f32", 4, 2, 64), ("bf16", 1024, 1, 128),
                                          ("f32", 1024, 1024, 128)])
def test_every_grain_has_one_place(dtype, H, Hkv, D):
    rng = random.Random(1)
    desc = qb.make_desc(LayerShape(H * D, H, Hkv, D, 10000.0, dtype))
    lib = qb.load_library()
    divided = 0
    for _ in range(400):
        page = rng.choice([16, 32, 64, 128, 256])
        width = int(2 ** rng.uniform(0, 13))
        B, n_q = int(2 ** rng.uniform(0, 8)), rng.choice([1, 1, 2, 5, 16])
        keep = rng.choice([0, 0, 1, 7, 300])
        c = _cache(Hkv, D, page, width)
        d = page_rules.division(desc, c, B, n_q, keep)
        assert d["workspace"] == lib.qcf_page_attn_workspace_bytes(C.byref(desc), C.byref(c), B, n_q, keep)
        assert d["row_blocks"] * 16 * d["row_tiles"] >= d["rows"] and d["part_rows"] <= 16 * d["row_tiles"]
        if d["whole"]:
            assert not d["workspace"]
            continue
        divided += 1
        longest = min(keep, width) * page if keep else width * page
        kind = rng.random()
        tokens = [0 if kind < 0.1 else longest if kind < 0.3 else rng.randint(0, longest) if kind < 0.7 else min(longest, rng.randint(0, 200))
                  for _ in range(d["contexts"])]
        grains, starts, size, out = _ranges(d, tokens)
        have, parts = [0] * len(tokens), {}
        for r, pieces in enumerate(out):
            for x, g0, n, part in pieces:
                assert g0 == have[x]                              # in order, without a gap
                have[x] += n
                if part is not None:
                    assert part not in parts and part < 2 * d["slots"] and d["divides"]
                    parts[part] = x
        assert have == grains
        # the joining launch finds the parts of a context again from its first grain
        for x, g in enumerate(grains):
            first, last = starts[x] // size, (starts[x] + g - 1) // size
            if last > first:
                assert [parts[2 * r + (r == first)] for r in range(first, last + 1)] == [x] * (last - first + 1)
        if d["divides"]:
            assert d["workspace"] >= 2 * d["slots"] * d["inner"] * d["part_rows"] * (D + 2) * 4
    assert divided > 50 or Hkv == 1024


def test_short_contexts_are_taken_whole_by_the_rule():
    desc = qb.make_desc(LayerShape(4096, 32, 8, 128, 10000.0, "bf16"))
    whole = lambda width, B, **kw: page_rules.division(desc, _cache(8, 128, 16, width), B, kw.get("n_q", 1), kw.get("keep", 0))["whole"]
    assert whole(32, 1) and not whole(64, 1)                          # 512 and 1024 tokens of one request
    assert whole(64, 16) and not whole(128, 16)                       # of 16
    assert whole(128, 64) and not whole(512, 64)
    assert whole(8192, 32, keep=96) and not whole(8192, 1, keep=256)
    assert whole(32, 1, n_q=8) and not whole(32, 64, n_q=8)           # 32 rows: two tiles of rows to a workgroup where there is much to read
