"""8-bit appends whose keys are turned: the codes, scales and bounds that the formula has, in every kernel.

A key turned in 64 bits is at most 2^-41 of its pair off (positions below 2000, angles to 2^-52 of theirs); of a million elements, with middles
between codes at least 2^-4 of them apart, 2^-16 may be expected to lie that close to one, and a scale changes only where a block's largest
element does: all codes and scales are the oracle's.  Queries are turned in 32 bits: (cos, sin) off by 2^-23 each at most, two products and a
sum by 2^-24 each, 2^-21 of the pair in all, then half a step."""
import numpy as np
import pytest
import torch

from oracle import qcf_oracle as orc
from paper_2604_08585_amd import binding as qb
from gpu_pages8 import HALF_STEP, Paged8, normal, say, shape
from gpu_util import DEV, i32, i64, to_np

pytestmark = pytest.mark.gpu


def _append(p, rng, lens, new, rows, pos):
    sh = p.sh
    H, Hkv, D = sh.n_q_heads, sh.n_kv_heads, sh.head_dim
    off = np.concatenate([[0], np.cumsum(new)])
    q, k, v = (a.reshape(len(rows), -1, D) for a in np.split(rows, [H * D, (H + Hkv) * D], axis=1))
    parts = [t.unflatten(1, (-1, D)) for t in torch.from_numpy(rows).to(device=DEV, dtype=p.dt).split([H * D, Hkv * D, Hkv * D], 1)]
    q_out = torch.empty(len(rows), H, D, dtype=p.dt, device=DEV)
    qb.qcf_page8_append(p.desc, p.cache, len(new), *parts, i64(off), len(rows), i32(lens), None if pos is None else i32(pos), q_out)
    torch.cuda.synchronize()
    return off, q, k, v, q_out


@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("bounds", [True, False])             # (a workgroup to a page, or to a block of it)
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("dtype,H,Hkv,D", [("bf16", 8, 8, 128), ("bf16", 8, 8, 64), ("f32", 4, 4, 128), ("f32", 8, 8, 64), ("bf16", 12, 3, 128), ("f32", 2, 1, 64)])
def test_turned_keys_get_the_codes_of_the_formula(dtype, H, Hkv, D, style, bounds, order):
    rng = np.random.default_rng(84)
    page = 32 if Hkv > 4 else 128
    lens, new = [3, 0, 0, 21, 60], [1200, 900, 5, 1, 70]
    p = Paged8(rng, shape(H, Hkv, D, dtype, style), page, [h + n for h, n in zip(lens, new)], order, bounds=bounds)
    rows = normal(rng, (sum(new), (H + 2 * Hkv) * D), dtype)
    pos = np.concatenate([np.arange(n) + h for h, n in zip(lens, new)]).astype(np.int32)
    say("append8, every code", dtype, H, Hkv, D, "style", style, "bounds", bounds, order)
    off, q, k, v, q_out = _append(p, rng, lens, new, rows, pos)
    codes, scales, limits = orc.page8_append(p.codes, p.scales, p.bounds, p.table, lens, off, k, v, pos, p.sh.rope_base, style)
    got_k, got_v, got_s = p.got()
    assert np.array_equal(got_s, scales) and np.array_equal(got_k, codes[0]) and np.array_equal(got_v, codes[1])
    if bounds:
        assert np.array_equal(to_np(p.bd), limits)
    ref = orc.rope_at(q, pos, p.sh.rope_base, style)
    assert np.all(np.abs(to_np(q_out) - ref) <= HALF_STEP[dtype] * np.abs(ref) + 2.0 ** -21 * 2 * np.abs(rows).max())


@pytest.mark.parametrize("dtype,D,page,order", [("bf16", 128, 16, "token"), ("f32", 64, 64, "head"), ("bf16", 64, 256, "token")])
def test_bounds_contain_what_is_stored(dtype, D, page, order):
    """Steps of rows that grow and shrink, whose blocks are rounded again and again: least and largest stored key of a page lie within its
    bounds at all times, and are its bounds where the page was written at once.  (Sizes far enough apart for older tokens to lose bits.)"""
    rng = np.random.default_rng(85)
    sh = shape(4, 2, D, dtype)
    p = Paged8(rng, sh, page, [200, 200], order)
    held, wider = [0, 0], 0
    for step in range(24):
        new = [int(n) for n in rng.integers(0, 14, 2)] if step else [40, 0]
        size = float(2.0 ** rng.uniform(-20, 20))
        rows = normal(rng, (sum(new) + 1, 8 * D), dtype, size)
        pos = np.concatenate([np.arange(n) + h for h, n in zip(held, new)] + [[0]]).astype(np.int32)
        _append(p, rng, held, new, rows, pos if step % 2 else None)
        held = [h + n for h, n in zip(held, new)]
        if max(held) > 186:
            break
        codes_k, _, scales = p.got()
        k, b = orc.page8_values((codes_k, codes_k), scales)[0], to_np(p.bd)
        for r in range(2):
            for i in range(-(-held[r] // page)):
                n = min(page, held[r] - i * page)
                x = k[p.table[r, i], :n]
                for g in range(2):
                    lo, hi = b[p.table[r, i], g]
                    assert np.all(lo <= x[:, g].min(0)) and np.all(hi >= x[:, g].max(0)), (step, r, i, g)
                    wider += int(np.any(lo < x[:, g].min(0)) or np.any(hi > x[:, g].max(0)))
                    if step == 0:
                        assert np.array_equal(lo, x[:, g].min(0)) and np.array_equal(hi, x[:, g].max(0))
    print("pages and heads whose bounds are wider than what is stored:", wider, flush=True)
