"""Attention over 8-bit pages: what its softmax weights hold.

Two tokens with logits of 0 and -x and values of 1 and -1: the output is (1 - w) / (1 + w) with w = exp(-x), about x / 2, so an error
of w comes out whole beside a result that is thousands of times smaller.  Codes and scales are exact (powers of two).  Derived bound: a
stored result is off by half a step, 2^-8 (bf16) or 2^-24 (f32) of its value; a weight by 2^-22 for its exponential, 2^-24 for each of the
roundings of its logit and of the four sums that it goes through, which the output halves: 2^-22 in all.  A weight of 16 bits would be off
by up to 2^-17, the output by 2^-18."""
import math

import numpy as np
import pytest
import torch

from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd import inputs
import test_page8_layout as rules
from gpu_pages8 import E4M3, HALF_STEP, shape
from gpu_util import DEV, i32, to_np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["one", "drafts", "list"])
@pytest.mark.parametrize("dtype,G,Hkv,D,width", [
    # whole contexts, ranges, heads side by side, two tiles of rows
    ("bf16", 16, 1, 128, 2), ("bf16", 16, 1, 64, 2), ("f32", 16, 1, 64, 2), ("bf16", 16, 1, 128, 4096), ("bf16", 8, 1, 64, 4096), ("f32", 8, 1, 128, 4096),
    ("bf16", 5, 2, 128, 16384), ("bf16", 5, 4, 64, 16384), ("f32", 5, 2, 128, 16384), ("bf16", 24, 1, 128, 65536), ("bf16", 24, 1, 64, 65536)])
def test_weights_hold_a_float(dtype, G, Hkv, D, width, mode):
    rng = np.random.default_rng(61)
    n_q = 3 if mode == "drafts" else 1
    H, keep = G * Hkv, min(width, 3000) if mode == "list" else 0
    rule = rules.division(H, Hkv, D, dtype, 1, n_q, 16 * width, keep)
    assert rule["whole"] == (width == 2)
    if mode != "list":
        assert rule["heads"] == (256 // D if width == 16384 else 1) and rule["row_tiles"] == (2 if width == 65536 else rule["row_tiles"])
    sh = shape(H, Hkv, D, dtype)
    dt = inputs.torch_dtype(dtype)
    # x = q . k / sqrt(d) between 2^-12 and 2^-10
    q = np.zeros((1, n_q, H, D), dtype=np.float32)
    q[..., 5] = inputs.round_to_dtype((2.0 ** rng.uniform(-12, -10, (1, n_q, H)) * math.sqrt(D)).astype(np.float32), dtype)
    k, v = torch.zeros(2, 16, Hkv, D), torch.zeros(2, 16, Hkv, D)
    k[1, 1, :, 5], v[1, 0], v[1, 1] = -2.0, 8.0, -8.0
    scales = torch.ones(2, Hkv, 2, 1)
    scales[:, :, 0], scales[:, :, 1] = 0.5, 0.125
    kd, vd = (x.to(E4M3).view(torch.uint8).to(DEV).view(E4M3) for x in (k, v))
    table = np.full((1, width), -1, dtype=np.int32)
    table[0, 0] = 1
    cache, desc = qb.page8_cache(kd, vd, scales.to(DEV), None, i32(table), dt), qb.make_desc(sh)
    pages = np.full((1, n_q, Hkv, keep), -1, dtype=np.int32)
    pages[..., :1] = 0
    o, lse = torch.empty(1, n_q, H, D, dtype=dt, device=DEV), torch.empty(1, n_q, H, device=DEV)
    print("weights of 8-bit pages", dtype, G, Hkv, D, width, mode, flush=True)
    qb.qcf_page8_attn(desc, cache, 1, n_q, torch.from_numpy(q).to(device=DEV, dtype=dt), i32([[2] * n_q]), i32(pages) if keep else None, keep, o, lse)
    torch.cuda.synchronize()
    x = q[..., 5].astype(np.float64) / math.sqrt(D)
    ref = np.tanh(x / 2)[..., None]                            # (1 - w) / (1 + w)
    off = np.abs(to_np(o) - ref)
    print("worst, of the bound:", (off / (HALF_STEP[dtype] * ref + 2.0 ** -22)).max(), flush=True)
    assert np.all(off <= HALF_STEP[dtype] * ref + 2.0 ** -22)
    assert np.all(np.abs(to_np(lse) - np.log1p(np.exp(-x))) <= 2.0 ** -22)
