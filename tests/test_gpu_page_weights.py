"""Attention over pages: what its softmax weights hold.

Two tokens with logits of 0 and -x and values of 1 and -1: the output is (1 - w) / (1 + w) with w = exp(-x), about x / 2, so an error
of w comes out whole beside a result that is thousands of times smaller.  Derived bound: a stored result is off by half a step, 2^-8
(bf16) or 2^-24 (f32) of its value; a weight by 2^-22 for its exponential, 2^-24 for each of the roundings of its logit and of the four
sums that it goes through, which the output halves: 2^-22 in all.  A weight of 16 bits would be off by up to 2^-17, the output by 2^-18."""
import math

import numpy as np
import pytest
import torch

from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd import inputs
import page_rules
from gpu_util import DEV, i32, to_np

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.mark.parametrize("mode", ["one", "drafts", "list"])
@pytest.mark.parametrize("dtype,G,D,width", [
    ("bf16", 16, 128, 2), ("bf16", 16, 64, 2), ("f32", 16, 64, 2), ("bf16", 16, 128, 4096), ("bf16", 8, 64, 4096), ("f32", 8, 128, 4096),
    ("bf16", 24, 128, 65536), ("bf16", 24, 64, 65536)])       # (whole contexts, ranges, two tiles of rows)
def test_weights_hold_a_float(dtype, G, D, width, mode):
    rng = np.random.default_rng(41)
    n_q = 3 if mode == "drafts" else 1
    sh = inputs.LayerShape(G * D, G, 1, D, 10000.0, dtype)
    dt = inputs.torch_dtype(dtype)
    # x = q . k / sqrt(d) between 2^-12 and 2^-10
    q = np.zeros((1, n_q, G, D), dtype=np.float32)
    q[..., 5] = inputs.round_to_dtype((2.0 ** rng.uniform(-12, -10, (1, n_q, G)) * math.sqrt(D)).astype(np.float32), dtype)
    k, v = np.zeros((2, 16, 1, D), dtype=np.float32), np.zeros((2, 16, 1, D), dtype=np.float32)
    k[1, 1, 0, 5], v[1, 0], v[1, 1] = -1.0, 1.0, -1.0
    dev = lambda a: torch.from_numpy(a).to(device=DEV, dtype=dt)
    table = np.full((1, width), -1, dtype=np.int32)
    table[0, 0] = 1
    kd, vd = dev(k), dev(v)
    cache, desc = qb.page_cache(kd, vd, None, i32(table)), qb.make_desc(sh)
    keep = min(width, 3000) if mode == "list" else 0
    rule = page_rules.division(desc, cache, 1, n_q, keep)
    assert rule["whole"] == (width == 2) and rule["row_tiles"] == (2 if width == 65536 and mode != "list" else rule["row_tiles"])
    pages = np.full((1, n_q, 1, keep), -1, dtype=np.int32)
    pages[..., :1] = 0
    o, lse = torch.empty(1, n_q, G, D, dtype=dt, device=DEV), torch.empty(1, n_q, G, device=DEV)
    print("weights", dtype, G, D, width, mode, flush=True)
    qb.qcf_page_attn(desc, cache, 1, n_q, dev(q), i32([[2] * n_q]), i32(pages) if keep else None, keep, o, lse)
    torch.cuda.synchronize()
    x = q[..., 5].astype(np.float64) / math.sqrt(D)
    ref = np.tanh(x / 2)[..., None]                            # (1 - w) / (1 + w)
    off = np.abs(to_np(o) - ref)
    print("worst, of the bound:", (off / (HALF_STEP[dtype] * ref + 2.0 ** -22)).max(), flush=True)
    assert np.all(off <= HALF_STEP[dtype] * ref + 2.0 ** -22)
    assert np.all(np.abs(to_np(lse) - np.log1p(np.exp(-x))) <= 2.0 ** -22)
