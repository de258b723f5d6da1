"""Attention, weights and evictions over 8-bit pages whose scales are the least and the largest that an append stores, 2^-100 and 2^92.

Powers of two change no bit, and queries are scaled so that logits are ordinary ones."""
import math

import numpy as np
import pytest
import torch

from oracle import qcf_oracle as orc
from paper_2604_08585_amd import binding as qb
from gpu_pages8 import HALF_STEP, Paged8, normal, say, shape
from gpu_util import DEV, i32, i64, to_np

pytestmark = pytest.mark.gpu

LEAST, MOST = 2.0 ** -100, 2.0 ** 92


def _outputs(p, seen, q, w):
    B, n_q = seen.shape
    o, lse = torch.empty_like(q), torch.empty(B, n_q, p.sh.n_q_heads, device=DEV)
    qb.qcf_page8_attn(p.desc, p.cache, B, n_q, q, i32(seen), None, 0, o, lse)
    qb.qcf_page_weigh(p.desc, p.cache, B, n_q, q, i32(seen), lse, None, 0.0, 1.0, w)
    torch.cuda.synchronize()
    return o, lse, w


@pytest.mark.parametrize("width", [None, 8192])               # (whole contexts, ranges)
@pytest.mark.parametrize("dtype,D,n_q", [("bf16", 128, 1), ("bf16", 64, 3), ("f32", 128, 2), ("f32", 64, 1)])
@pytest.mark.parametrize("keys,values", [(MOST, MOST), (LEAST, LEAST), (LEAST, MOST), (MOST, LEAST)])
def test_the_least_and_the_largest_scales(dtype, D, n_q, keys, values, width):
    """The bits of ordinary scales, times the scale: queries take the inverse of the keys' scale."""
    rng = np.random.default_rng(82)
    seen = np.array([[700 - n_q + 1 + i for i in range(n_q)], [33] * n_q, [1] * n_q], dtype=np.int32)
    p = Paged8(rng, shape(8, 2, D, dtype), 16, [700, 33, 1], width=width, bounds=False)
    p.scales[:] = 1.0 / 128                                                     # (codes of up to 448)
    p.upload(bounds=False)
    q = torch.from_numpy(normal(rng, (3, n_q, 8, D), dtype)).to(device=DEV, dtype=p.dt)
    w = torch.zeros(3, 2, p.cache.tokens, device=DEV)
    want = _outputs(p, seen, q, w.clone())
    p.scales[:, :, 0], p.scales[:, :, 1] = keys, values
    p.upload(bounds=False)
    say("scales", dtype, D, keys, values)
    got = _outputs(p, seen, (q.double() / 128 / keys).to(p.dt), w.clone())
    assert torch.isfinite(want[0].float()).all()
    o, ref = got[0].double() / values, want[0].double() * 128
    if values == LEAST and dtype == "bf16":
        # (what a weight's third term has beneath 2^-126 may be lost: 2^-26 of the scale for each of 700 tokens with codes of up to 448)
        assert ((o - ref).abs() <= 2 * HALF_STEP[dtype] * ref.abs() + 700 * 448 * 2.0 ** -26).all()
    else:
        assert torch.equal(o, ref)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_appended_and_evicted_at_both_ends(dtype, D):
    """Elements of 2^100 and of 2^-109 are stored, attended to and moved; blocks that mix both keep the large ones."""
    rng = np.random.default_rng(83)
    sh = shape(4, 2, D, dtype)
    p = Paged8(rng, sh, 16, [64], bounds=False)
    rows = np.exp2(rng.choice([100.0, -109.0], (64, 4 * D))).astype(np.float32) * rng.choice([-1.0, 1.0], (64, 4 * D)).astype(np.float32)
    rows[:16], rows[16:32] = np.copysign(2.0 ** 100, rows[:16]), np.copysign(2.0 ** -109, rows[16:32])
    k, v = (torch.from_numpy(a.reshape(64, 2, D)).to(device=DEV, dtype=p.dt) for a in (rows[:, :2 * D], rows[:, 2 * D:]))
    qb.qcf_page8_append(p.desc, p.cache, 1, None, k, v, i64([0, 64]), 64, i32([0]), None, None)
    torch.cuda.synchronize()
    want = orc.page8_append(p.codes, p.scales, p.bounds, p.table, [0], [0, 64], to_np(k), to_np(v), None, sh.rope_base, 0)
    codes_k, codes_v, scales = p.got()
    used = p.table[0, :4]
    assert np.array_equal(codes_k[used], want[0][0][used]) and np.array_equal(codes_v[used], want[0][1][used]) and np.array_equal(scales[used], want[1][used])
    assert (scales[used[0]] == MOST).all() and (scales[used[1]] == LEAST).all()
    t = Paged8(rng, sh, 16, [40], bounds=False)
    w = torch.from_numpy(rng.random((1, 2, p.cache.tokens)).astype(np.float32)).to(DEV)
    kept, n = torch.empty(1, 2, 40, dtype=torch.int32, device=DEV), i32([64])
    qb.qcf_page_evict(p.desc, p.cache, 1, n, w, 40, 0, 0, t.cache, kept, None, n)
    torch.cuda.synchronize()
    moved, at = t.got(), kept[0].cpu().numpy()
    for which, x in enumerate(orc.page8_values((codes_k, codes_v), scales)):
        for g in range(2):
            src = x[p.table[0, at[g] // 16], at[g] % 16, g]
            for j in range(0, 40, 16):
                s = orc.page8_scale(src[j:j + 16])
                page = t.table[0, j // 16]
                assert moved[2][page, g, which, 0] == s
                assert np.array_equal(moved[which][page, :len(src[j:j + 16]), g], orc.e4m3(src[j:j + 16] / s))
    # a value of 2^100 in every other token, uniform weights: the mean
    q = torch.zeros(1, 1, 4, D, dtype=p.dt, device=DEV)
    o = torch.empty_like(q)
    qb.qcf_page8_attn(p.desc, p.cache, 1, 1, q, i32([[64]]), None, 0, o, None)
    torch.cuda.synchronize()
    v = orc.page8_values((codes_k, codes_v), scales)[1]
    ref = np.concatenate([v[p.table[0, i]] for i in range(4)]).mean(0).repeat(2, 0)
    assert np.all(np.abs(to_np(o)[0, 0] - ref) <= HALF_STEP[dtype] * np.abs(ref) + 2.0 ** -22 * 2.0 ** 100)
