"""Appends whose workgroups take several KV heads: shared factors, the queries of several groups, bounds joined over all their lanes,
pages of more rows than a workgroup keeps factors for.  Tolerances as in test_gpu_pages.py."""
import numpy as np
import pytest

import append_rules
from gpu_util import to_np
from test_gpu_pages import Paged, _append, _check_append, shape

pytestmark = pytest.mark.gpu

CASES = [
    # dtype, H, Hkv, D, style, page, order, requests, heads to a workgroup
    ("bf16", 16, 8, 128, 0, 16, "token", 130, 8), ("bf16", 16, 8, 128, 1, 128, "head", 130, 8), ("bf16", 24, 8, 128, 0, 64, "token", 129, 8),
    ("bf16", 8, 4, 128, 1, 32, "token", 130, 4), ("f32", 8, 4, 128, 1, 16, "token", 130, 4), ("f32", 4, 4, 128, 0, 128, "head", 130, 4),
    ("f32", 16, 8, 64, 0, 128, "token", 130, 8), ("bf16", 32, 16, 64, 0, 32, "head", 130, 16), ("bf16", 8, 4, 64, 1, 256, "token", 260, 4),
    ("bf16", 16, 8, 128, 0, 16, "token", 380, 4), ("f32", 6, 6, 64, 1, 64, "token", 70, 2), ("bf16", 16, 8, 128, 1, 16, "token", 34, 2)]


@pytest.mark.parametrize("rotated", [True, False])
@pytest.mark.parametrize("case", CASES)
def test_append_of_several_heads_to_a_workgroup(case, rotated):
    dtype, H, Hkv, D, style, page, order, B, heads = case
    rng = np.random.default_rng(81)
    # mostly a row or two behind what a request holds; some requests begin anew, and some get whole pages and part of one
    lens = rng.integers(0, 2 * page, B).tolist()
    new = rng.integers(0, 3, B).tolist()
    for i, n in enumerate([page + 3, 2 * page, 2 * page + page // 2 + 1, page]):
        new[17 * i % B], lens[17 * i % B] = n, [0, page, 5, page - 1][i]
    p = Paged(rng, shape(H, Hkv, D, dtype, style), page, [a + b for a, b in zip(lens, new)], order)
    assert append_rules.heads(p.desc, p.cache, B, sum(new) + 2) == heads          # (two rows of padding behind the last)
    pools, q64, q_out, largest = _append(p, rng, lens, new, rotated)
    got_k, got_b = _check_append(p, pools, q64, q_out, largest, rotated)
    for b, (held, n) in enumerate(zip(lens, new)):
        for pg in range(held // page, -(-(held + n) // page)) if n else ():
            t0, t1 = max(held, pg * page), min(held + n, (pg + 1) * page)
            at = p.table[b, pg]
            rows = got_k[at, t0 - pg * page:t1 - pg * page]
            lo, hi = rows.min(0), rows.max(0)
            if t0 % page:
                lo, hi = np.minimum(lo, p.bounds[at, :, 0]), np.maximum(hi, p.bounds[at, :, 1])
            assert np.array_equal(got_b[at, :, 0], lo) and np.array_equal(got_b[at, :, 1], hi), (b, pg)
