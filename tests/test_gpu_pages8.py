"""GPU parity of the calls over 8-bit pages (qcf_pages8.h) against the float64 oracle on identical inputs.

Tolerances, derived.  A code is off by at most half a step: 2^-4 of its value, or 2^-10 of its scale beneath 2^-6.
  values     not computed with before they are rounded: equal.
  keys       a turned element is off by at most slack = 2^-21 (|a| + |b|): (cos, sin) by 2^-23 each at most (a sine of 1 ulp and the
             first-order term), the two products and the sum by 2^-24 each; a code then by half a step of what it stands for and slack; a
             scale only where the largest element lies within slack of the border.
  attention  as for pages of the layer's type (a logit of d products in 32 bits: eps = (d + 4) 2^-24 sum |q k| / sqrt(d), and one more
             rounding each for the two scales; weights by exp(2 eps) and 2^-22; sums of T terms T 2^-24; in bf16 a weight enters its product
             as two terms: cut off after 8 bits, the rest, less than 2^-7 of it, to half a step of 2^-8, so 2^-15 at most; the products of
             both are exact in 32 bits), relative to max |v|.
"""
import math

import numpy as np
import pytest
import torch

from oracle import qcf_oracle as orc
from paper_2604_08585_amd import binding as qb
from gpu_pages8 import E4M3, HALF_STEP, Paged8, normal, say, shape
from gpu_util import DEV, i32, i64, to_np

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ append

APPENDS = [
    # dtype, H, Hkv, D, style, page, order, (held, new) of each request, rotated
    ("bf16", 32, 8, 128, 0, 16, "token", [(0, 1), (15, 1), (16, 1), (777, 1)], True),
    ("bf16", 8, 2, 128, 1, 16, "head", [(5, 40), (0, 0), (31, 2), (16, 16)], True),
    ("bf16", 4, 4, 64, 0, 64, "token", [(45, 131)], True),
    ("bf16", 6, 2, 64, 1, 256, "token", [(0, 300), (250, 7)], True),
    ("bf16", 8, 8, 128, 0, 128, "token", [(0, 257), (3, 1)], False),
    ("bf16", 4, 4, 128, 0, 64, "head", [(0, 2000), (33, 2500), (17, 1500), (64, 3000)], True),       # (workgroups of several heads)
    ("bf16", 6, 3, 64, 1, 32, "token", [(0, 3000), (40, 2500)], True),
    ("f32", 4, 2, 64, 1, 32, "head", [(7, 9), (0, 33), (63, 1)], True),
    ("f32", 16, 1, 128, 0, 16, "token", [(0, 17), (1, 1), (2, 30)], True),
    ("f32", 2, 2, 64, 0, 128, "token", [(100, 100)], False),
    ("f32", 8, 4, 128, 0, 256, "token", [(130, 1500), (0, 2000)], True),
]


def _append(p, rng, lens, new, rotated, far=0, size=1.0, rows=None):
    sh = p.sh
    H, Hkv, D = sh.n_q_heads, sh.n_kv_heads, sh.head_dim
    M = sum(new)
    off = np.concatenate([[0], np.cumsum(new)])
    if rows is None:
        rows = normal(rng, (M + 2, (H + 2 * Hkv) * D), sh.dtype, size)           # two rows behind the last: padding
    q, k, v = (a.reshape(M + 2, -1, D) for a in np.split(rows, [H * D, (H + Hkv) * D], axis=1))
    pos = (np.concatenate([np.arange(n) + h for h, n in zip(lens, new)] + [[9, 9]]) + far).astype(np.int32)
    dev = torch.from_numpy(rows).to(device=DEV, dtype=p.dt)
    parts = [t.unflatten(1, (-1, D)) for t in dev.split([H * D, Hkv * D, Hkv * D], 1)]
    q_out = torch.full((M + 2, H, D), 7.0, dtype=p.dt, device=DEV)
    say("append8", sh.dtype, H, Hkv, D, "style", sh.rope_style, "page", p.page, p.order, list(zip(lens, new)))
    qb.qcf_page8_append(p.desc, p.cache, len(new), *parts, i64(off), M + 2, i32(lens), i32(pos) if rotated else None, q_out)
    torch.cuda.synchronize()
    want = orc.page8_append(p.codes, p.scales, p.bounds, p.table, lens, off, k[:M], v[:M], pos[:M] if rotated else None, sh.rope_base,
                            sh.rope_style)
    q64 = orc.rope_at(q[:M], pos[:M], sh.rope_base, sh.rope_style) if rotated else np.asarray(q[:M], dtype=np.float64)
    return want, q64, q_out, float(np.nanmax(np.where(np.isfinite(rows), np.abs(rows), 0.0)))


def _check_append(p, want, q64, q_out, largest, rotated):
    (codes, scales, bounds), slack = want, 2.0 ** -21 * 2 * largest if rotated else 0.0
    k, v, s = p.got()
    assert np.array_equal(v, codes[1], equal_nan=True) and np.array_equal(s[:, :, 1], scales[:, :, 1])
    if not rotated:
        assert np.array_equal(k, codes[0], equal_nan=True) and np.array_equal(s, scales)
    # (a scale that differs is off by a factor of two, in few blocks)
    same = s[:, :, 0] == scales[:, :, 0]
    assert np.mean(same) > 0.99 and np.all(same | (s[:, :, 0] == 2 * scales[:, :, 0]) | (2 * s[:, :, 0] == scales[:, :, 0]))
    got, ref = orc.page8_values([k, k], s)[0], orc.page8_values(codes, scales)[0]
    step = np.repeat(np.maximum(s, scales)[:, :, 0], 16, axis=2).transpose(0, 2, 1)[..., None]
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    fine = ~np.isnan(ref)
    # got and ref are both within half a step and slack of the turned element
    assert np.all((np.abs(got - ref) <= np.maximum(2 * 2.0 ** -4 * (np.abs(ref) + slack) * 1.07, 2 * 2.0 ** -10 * step) + slack)[fine])
    assert np.mean((got == ref)[fine]) > 0.999                                  # (an element within slack of the middle of a step)
    assert np.all(np.abs(to_np(q_out)[:len(q64)] - q64) <= (HALF_STEP[p.sh.dtype] if rotated else 0.0) * np.abs(q64) + slack)
    assert np.all(to_np(q_out)[len(q64):] == 7.0)
    if p.bd is not None:
        # bounds: exactly those of what is stored, where codes and scales are the oracle's
        b = to_np(p.bd)
        pages = np.array([np.array_equal(got[i], ref[i], equal_nan=True) for i in range(len(got))])
        assert np.array_equal(b[pages], bounds[pages], equal_nan=True)


@pytest.mark.parametrize("bounds", [True, False])             # (a workgroup to a page, or to a block of it)
@pytest.mark.parametrize("case", APPENDS)
def test_append(case, bounds):
    dtype, H, Hkv, D, style, page, order, requests, rotated = case
    rng = np.random.default_rng(21)
    lens, new = [h for h, _ in requests], [n for _, n in requests]
    p = Paged8(rng, shape(H, Hkv, D, dtype, style), page, [h + n for h, n in requests], order, bounds=bounds)
    _check_append(p, *_append(p, rng, lens, new, rotated), rotated)


@pytest.mark.parametrize("bounds", [True, False])
@pytest.mark.parametrize("size", [2.0 ** -40, 1e-3, 30.0, 1e4])
def test_scales_that_grow_and_scales_that_stay(size, bounds):
    """Rows far smaller or larger than what their block holds: the block's tokens stay as they are, or are rounded again."""
    for dtype, D, page, order in [("bf16", 128, 16, "token"), ("f32", 64, 64, "head"), ("f32", 128, 32, "token"), ("bf16", 64, 128, "head")]:
        rng = np.random.default_rng(22)
        lens, new = [5, 15, 47, 16, 1, 30], [1, 1, 3, 2, 15, 40]
        p = Paged8(rng, shape(4, 2, D, dtype), page, [h + n for h, n in zip(lens, new)], order, bounds=bounds)
        _check_append(p, *_append(p, rng, lens, new, False, size=size), False)


@pytest.mark.parametrize("dtype,H,Hkv,D,style", [("bf16", 8, 8, 128, 0), ("bf16", 8, 8, 64, 1), ("f32", 4, 4, 128, 1), ("f32", 8, 8, 64, 0)])
def test_rotated_keys_get_the_codes_of_the_formula(dtype, H, Hkv, D, style):
    """A key turned in 64 bits is at most 2^-41 of its pair off (positions below 2000, angles to 2^-52 of theirs); of a million elements, with
    middles between codes at least 2^-4 of them apart, 2^-16 may be expected to lie that close to one: all codes are the oracle's."""
    rng = np.random.default_rng(41)
    p = Paged8(rng, shape(H, Hkv, D, dtype, style), 32, [1203, 900, 5], "token", bounds=True)
    (codes, scales, bounds), _, _, _ = _append(p, rng, [3, 0, 0], [1200, 900, 5], True)
    k, v, s = p.got()
    assert np.array_equal(k, codes[0], equal_nan=True) and np.array_equal(v, codes[1], equal_nan=True) and np.array_equal(s, scales)
    assert np.array_equal(to_np(p.bd), bounds, equal_nan=True)


@pytest.mark.parametrize("dtype,far", [("f32", 3000000), ("bf16", 2000000000), ("f32", -100000)])
def test_append_at_far_positions(dtype, far):
    rng = np.random.default_rng(23)
    p = Paged8(rng, shape(4, 2, 128, dtype, 0, 10000.0), 16, [40])
    _check_append(p, *_append(p, rng, [3], [37], True, far), True)


@pytest.mark.parametrize("bounds", [True, False])
def test_steps_of_one_token_fill_a_page(bounds):
    """A page token by token, then again from its middle (drafts that were not accepted): the oracle's bits after every step."""
    rng = np.random.default_rng(24)
    sh = shape(8, 2, 128, "bf16")
    p = Paged8(rng, sh, 16, [0, 0], spare=5, bounds=bounds)
    p.table = np.array([[3], [1]], dtype=np.int32)
    p.scales[:] = np.nan                                                         # (a new page may hold anything)
    p.upload(bounds)
    held = 0
    for step in range(24):
        lens = [held, held]
        want, q64, q_out, largest = _append(p, rng, lens, [1, 1], False, size=float(np.exp(rng.standard_normal() * 3)))
        k, v, s = p.got()
        for b in range(2):
            page = p.table[b, 0]
            assert np.array_equal(k[page, :held + 1], want[0][0][page, :held + 1]) and np.array_equal(v[page, :held + 1], want[0][1][page, :held + 1])
            assert np.array_equal(s[page], want[1][page])
        p.codes, p.scales, p.bounds = [c for c in want[0]], want[1], want[2]
        held = 7 if step == 14 else held + 1


@pytest.mark.parametrize("bounds", [True, False])
def test_append_drops_what_has_no_page_and_takes_special_values(bounds):
    rng = np.random.default_rng(25)
    for dtype, D in [("bf16", 128), ("f32", 64)]:
        sh = shape(4, 2, D, dtype)
        p = Paged8(rng, sh, 16, [64, 64, 20], spare=2)
        p.table[0, 1], p.table[1, 2] = -1, 10 ** 6                               # pages that are not there
        p.upload(bounds)
        lens, new = [10, 30, 60], [30, 40, 9]                                    # the second and the third run beyond the table
        M = sum(new)
        rows = normal(rng, (M + 2, 8 * D), dtype)
        rows[2, 4 * D + 3], rows[2, 4 * D + 5], rows[3, 6 * D] = np.nan, np.inf, -np.inf
        rows[31] = np.float32(2.0 ** 101)                                        # a row beyond what is stored
        rows[5, 4 * D] = np.float32(-2.0 ** 100)                                 # the largest element
        want, q64, q_out, _ = _append(p, rng, lens, new, False, rows=rows)
        _check_append(p, want, np.where(np.isnan(q64), 0, q64)[:0], q_out[:0], 1.0, False)


def test_append_without_queries_or_bounds_and_queries_in_place():
    rng = np.random.default_rng(26)
    sh = shape(8, 2, 128, "bf16")
    p, plain = (Paged8(np.random.default_rng(3), sh, 32, [90], bounds=b) for b in (True, False))
    k, v, q = (torch.from_numpy(normal(rng, (50, n, 128), "bf16")).to(device=DEV, dtype=torch.bfloat16) for n in (2, 2, 8))
    args = i64([0, 50]), 50, i32([40]), i32(np.arange(40, 90))
    out = torch.empty_like(q)
    qb.qcf_page8_append(p.desc, p.cache, 1, q, k, v, *args, out)
    qb.qcf_page8_append(plain.desc, plain.cache, 1, None, k, v, *args, None)
    qb.qcf_page8_append(p.desc, p.cache, 1, q, k, v, *args, q)
    torch.cuda.synchronize()
    assert torch.equal(p.kd.view(torch.uint8), plain.kd.view(torch.uint8)) and torch.equal(p.sd, plain.sd) and torch.equal(q, out)


@pytest.mark.parametrize("bounds", [True, False])
def test_append_of_many_requests(bounds):
    rng = np.random.default_rng(27)
    lens = rng.integers(0, 40, 700).tolist()
    new = [int(n) if n < 5 else 0 for n in rng.integers(0, 7, 700)]
    new[333] = 50
    p = Paged8(rng, shape(2, 1, 64, "f32"), 16, [h + n for h, n in zip(lens, new)], bounds=bounds)
    _check_append(p, *_append(p, rng, lens, new, True), True)


def test_lengths_below_nothing_and_rows_behind_the_last_request():
    """Rows that would be tokens before the first are not stored, their queries are turned; offsets beyond the rows are cut off."""
    rng = np.random.default_rng(28)
    for bounds in (True, False):
        sh = shape(4, 2, 64, "bf16")
        p = Paged8(rng, sh, 32, [64, 64], bounds=bounds)
        k, v, q = (torch.from_numpy(normal(rng, (40, n, 64), "bf16")).to(device=DEV, dtype=p.dt) for n in (2, 2, 4))
        pos, out = i32(np.arange(40) + 100), torch.full_like(q, 7.0)
        qb.qcf_page8_append(p.desc, p.cache, 2, q, k, v, i64([0, 30, 90]), 38, i32([-21, 31]), pos, out)
        torch.cuda.synchronize()
        want = orc.rope_at(to_np(q)[:38], np.arange(38) + 100, sh.rope_base, 0)
        assert np.abs(to_np(out)[:38] - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-5 and (out[38:] == 7.0).all()
        kc, vc, s = p.got()
        turned = orc.rope_at(to_np(k)[:38], np.arange(38) + 100, sh.rope_base, 0)
        # request 0: rows 21 to 29 are tokens 0 to 8; request 1: rows 30 to 37 are tokens 31 to 38
        for b, first, rows in ((0, 0, range(21, 30)), (1, 31, range(30, 38))):
            for i, m in enumerate(rows):
                page, slot = p.table[b, (first + i) // 32], (first + i) % 32
                for g in range(2):
                    sv, sk = s[page, g, 1, slot // 16], s[page, g, 0, slot // 16]
                    assert np.array_equal(vc[page, slot, g], orc.e4m3(to_np(v)[m, g] / sv))
                    assert np.abs(kc[page, slot, g] * sk - turned[m, g]).max() <= 2.0 ** -4 * np.abs(turned[m, g]).max() + 1e-5
        used = {(p.table[b, t // 32], t % 32) for b, ts in ((0, range(9)), (1, range(31, 39))) for t in ts}
        for page in range(len(kc)):
            for slot in range(32):
                if (page, slot) not in used and (page, slot // 16) != (p.table[1, 0], 1):       # (that block's scale may have grown)
                    assert np.array_equal(kc[page, slot], p.codes[0][page, slot]) and np.array_equal(vc[page, slot], p.codes[1][page, slot])


# ------------------------------------------------------------------ attention

def _attend_and_check(p, rng, seen, pages=None, q=None, with_lse=True):
    sh = p.sh
    H, D = sh.n_q_heads, sh.head_dim
    B, n_q = seen.shape
    q = normal(rng, (B, n_q, H, D), sh.dtype, 1.5) if q is None else q
    qd = torch.from_numpy(q).to(device=DEV, dtype=p.dt)
    o = torch.full((B, n_q, H, D), 7.0, dtype=p.dt, device=DEV)
    lse = torch.full((B, n_q, H), 7.0, dtype=torch.float32, device=DEV) if with_lse else None
    n_keep = 0 if pages is None else pages.shape[-1]
    say("attention8", sh.dtype, H, sh.n_kv_heads, D, "page", p.page, p.order, "seen", seen.tolist() if seen.size < 40 else seen.shape, "keep", n_keep)
    qb.qcf_page8_attn(p.desc, p.cache, B, n_q, qd, i32(seen), None if pages is None else i32(pages), n_keep, o, lse)
    torch.cuda.synchronize()
    got, z = to_np(o), to_np(lse) if with_lse else None
    k, v = p.values()
    for b in range(B):
        for i in range(n_q):
            ref, ref_z = orc.page_attn(q[b, i], k, v, p.table[b], seen[b, i], None if pages is None else pages[b, i])
            used = [x for x in p.table[b, :-(-seen[b, i] // p.page)] if 0 <= x < len(k)] if seen[b, i] > 0 else []
            if not used or not np.isfinite(ref_z).any():
                assert not got[b, i].any() and (not with_lse or np.all(z[b, i] == -np.inf)), (b, i)
                continue
            rows = [np.where(np.isfinite(x), x, 0.0) for x in (k[used].reshape(-1, sh.n_kv_heads, D), v[used].reshape(-1, sh.n_kv_heads, D))]
            x = np.asarray(q[b, i], dtype=np.float64)
            terms = max((np.abs(rows[0][:, h // (H // sh.n_kv_heads)]) @ np.abs(x[h])).max() for h in range(H))
            eps, T = (D + 5) * 2.0 ** -24 * terms / math.sqrt(D), len(rows[0])
            out = (2 * eps + 2.0 ** -22 + (T + 1) * 2.0 ** -24 + (2.0 ** -15 if sh.dtype == "bf16" else 0.0)) * np.abs(rows[1]).max()
            assert np.all(np.abs(got[b, i] - ref) <= HALF_STEP[sh.dtype] * np.abs(ref) + out), (b, i, np.abs(got[b, i] - ref).max(), out)
            if with_lse:
                seeing = np.isfinite(ref_z)
                assert np.all(z[b, i][~seeing] == -np.inf)
                off = np.abs(z[b, i][seeing] - ref_z[seeing])
                assert np.all(off <= eps + T * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(ref_z[seeing]))), (b, i)
    return o, lse


ATTENTIONS = [
    # dtype, H, Hkv, D, page, order, seen [B][n_q]
    ("bf16", 32, 8, 128, 16, "token", [[731]]),
    ("bf16", 8, 2, 128, 16, "token", [[1], [2], [15], [16], [17], [0], [31], [32], [33]]),
    ("bf16", 4, 4, 128, 32, "head", [[127], [128], [129], [300], [5]]),
    ("bf16", 64, 8, 128, 64, "token", [[97, 98, 99, 100], [61, 62, 0, 0], [1, 2, 3, 4]]),
    ("bf16", 10, 2, 128, 16, "head", [[50, 3, 0, 77, 20, 16, 48], [0] * 7, [7] * 7]),
    ("bf16", 48, 2, 64, 128, "token", [[200], [129]]),
    ("bf16", 8, 4, 64, 16, "token", [[513, 514], [2000, 1999]]),
    ("bf16", 3, 1, 64, 256, "head", [[255, 256, 257]]),
    ("bf16", 16, 1, 128, 16, "token", [[64 + i for i in range(16)]]),
    ("f32", 4, 2, 64, 32, "token", [[1], [33], [600], [0], [64]]),
    ("f32", 8, 8, 128, 16, "head", [[100, 101], [17, 0]]),
    ("f32", 20, 1, 64, 16, "token", [[40, 41, 42, 43, 44]]),
    ("f32", 6, 2, 128, 256, "token", [[700]]),
    ("f32", 24, 1, 128, 64, "head", [[300, 17], [5, 64]]),
    # rows of one request that see very different parts of it; more contexts than ranges, and more than 64
    ("bf16", 16, 2, 128, 32, "token", [[5000, 2500, 0, 64, 4999], [1, 2, 3, 4, 2000]]),
    ("bf16", 32, 32, 128, 16, "token", [[97 * i % 1300] for i in range(80)]),
    ("f32", 16, 16, 64, 32, "token", [[61 * i % 500, 7 * i] for i in range(70)]),
    ("bf16", 2, 1, 64, 64, "token", [[30001]]),
    # several rows of heads that ranges read side by side, in one tile of rows and in two
    ("bf16", 16, 4, 128, 16, "token", [[700, 701, 640, 0], [1, 2, 3, 4], [33, 32, 31, 2000]]),
    ("f32", 4, 2, 128, 32, "token", [[64, 65, 66, 67, 68], [0, 0, 0, 0, 1000]]),
    ("bf16", 64, 8, 128, 64, "token", [[4000, 100, 4001]]),
]


@pytest.mark.parametrize("wide", [False, True])               # (a wide table: contexts are divided over the GPU and joined)
@pytest.mark.parametrize("case", ATTENTIONS)
def test_attention(case, wide):
    dtype, H, Hkv, D, page, order, seen = case
    rng = np.random.default_rng(31)
    seen = np.array(seen, dtype=np.int32)
    p = Paged8(rng, shape(H, Hkv, D, dtype), page, np.maximum(seen.max(1), 1).tolist(), order, width=131072 // page if wide else None)
    _attend_and_check(p, rng, seen)


@pytest.mark.parametrize("case", ATTENTIONS)
def test_results_do_not_depend_on_what_the_workspace_holds(case):
    dtype, H, Hkv, D, page, order, seen = case
    rng = np.random.default_rng(40)
    seen = np.array(seen, dtype=np.int32)
    B, n_q = seen.shape
    p = Paged8(rng, shape(H, Hkv, D, dtype), page, np.maximum(seen.max(1), 1).tolist(), order, width=131072 // page)
    q = torch.from_numpy(normal(rng, (B, n_q, H, D), dtype)).to(device=DEV, dtype=p.dt)
    n = qb.qcf_page8_attn_workspace_bytes(p.desc, p.cache, B, n_q, 0)
    got = []
    for fill in (0.0, math.nan, 1e19):
        ws = torch.full((n // 4 + 1,), fill, device=DEV).view(torch.uint8)
        o, lse = torch.full_like(q, 7.0), torch.full((B, n_q, H), 7.0, device=DEV)
        qb.qcf_page8_attn(p.desc, p.cache, B, n_q, q, i32(seen), None, 0, o, lse, ws)
        torch.cuda.synchronize()
        got.append((o, lse))
    assert all(torch.equal(o, got[0][0]) and torch.equal(z, got[0][1]) for o, z in got[1:])


@pytest.mark.parametrize("width", [9, 8192])
def test_attention_does_not_read_what_is_not_seen(width):
    """NaN codes behind `seen`, in page 0 (read in the place of absent pages) and in pages of no request; scales there that are NaN or
    infinite, in blocks without a token that is seen."""
    for dtype, D, n_q, page in [("bf16", 128, 1, 16), ("bf16", 64, 3, 16), ("f32", 64, 2, 32), ("bf16", 128, 8, 32), ("f32", 128, 1, 16), ("f32", 128, 6, 16)]:
        rng = np.random.default_rng(32)
        seen = np.array([[75 - n_q + 1 + i for i in range(n_q)], [16] * n_q, [33] * n_q, [0] * n_q], dtype=np.int32)
        p = Paged8(rng, shape(8, 2, D, dtype), page, [75, 16, 33, 40], width=width)
        free = np.setdiff1d(np.arange(len(p.codes[0])), p.table)
        for c in p.codes:
            c[free] = np.nan
        p.scales[free] = np.nan
        for b, n in enumerate([75, 16, 33, 0]):
            for t in range(n, -(-[75, 16, 33, 40][b] // page) * page):
                for c in p.codes:
                    c[p.table[b, t // page], t % page] = np.nan
            for blk in range(-(-n // 16), -(-[75, 16, 33, 40][b] // page) * page // 16):
                p.scales[p.table[b, blk * 16 // page], :, :, blk * 16 % page // 16] = np.inf if blk % 2 else np.nan
        mine = free[free > 0][0]                                            # page 0 of the pool belongs to nobody
        if 0 in p.table:
            for c in p.codes:
                c[mine] = c[0]
            p.scales[mine] = p.scales[0]
            p.table[p.table == 0] = mine
        p.table[0, 1] = -5                                                  # a page in the middle is not there
        for c in p.codes:
            c[0] = np.nan
        p.scales[0] = np.nan
        p.upload(bounds=False)
        _attend_and_check(p, rng, seen)


@pytest.mark.parametrize("width", [4, 16384])                 # (whole, in ranges)
@pytest.mark.parametrize("H", [8, 20])                        # rows in one tile and in two
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_values_that_only_later_drafts_see_do_not_reach_earlier_ones(dtype, D, H, width):
    rng = np.random.default_rng(33)
    p = Paged8(rng, shape(H, 2, D, dtype), 16, [60], width=width)
    p.codes[1][p.table[0, 59 // 16], 59 % 16] = np.nan
    p.upload()
    q = torch.from_numpy(normal(rng, (1, 4, H, D), dtype)).to(device=DEV, dtype=p.dt)
    o, alone = torch.empty_like(q), torch.empty_like(q)
    qb.qcf_page8_attn(p.desc, p.cache, 1, 4, q, i32([[57, 58, 59, 60]]), None, 0, o, None)
    qb.qcf_page8_attn(p.desc, p.cache, 1, 4, q, i32([[57, 58, 59, 57]]), None, 0, alone, None)
    torch.cuda.synchronize()
    assert torch.isfinite(o[:, :3].float()).all() and torch.isnan(o[:, 3].float()).all()
    assert (o[:, :3].float() - alone[:, :3].float()).abs().max() <= 2 * HALF_STEP[dtype] * alone.float().abs().max()


def test_a_key_that_is_nan_makes_its_heads_rows_nan():
    rng = np.random.default_rng(34)
    for dtype, D in [("bf16", 128), ("f32", 64)]:
        p = Paged8(rng, shape(8, 4, D, dtype), 16, [50])
        p.codes[0][p.table[0, 1], 3, 2] = np.nan
        p.upload()
        q = torch.from_numpy(normal(rng, (1, 1, 8, D), dtype)).to(device=DEV, dtype=p.dt)
        o, lse = torch.empty_like(q), torch.empty(1, 1, 8, device=DEV)
        qb.qcf_page8_attn(p.desc, p.cache, 1, 1, q, i32([[50]]), None, 0, o, lse)
        torch.cuda.synchronize()
        bad = torch.isnan(o[0, 0].float()).all(-1).cpu().tolist()
        assert bad == [False] * 4 + [True] * 2 + [False] * 2 and torch.isnan(lse[0, 0]).cpu().tolist() == bad


@pytest.mark.parametrize("dtype,H,Hkv,D,page,keep", [
    ("bf16", 32, 8, 128, 16, 11), ("bf16", 8, 2, 64, 64, 11), ("f32", 4, 2, 64, 32, 11), ("bf16", 32, 8, 128, 16, 3000), ("f32", 4, 2, 64, 32, 900),
    ("bf16", 24, 1, 128, 32, 2000)])
def test_attention_over_listed_pages(dtype, H, Hkv, D, page, keep):
    rng = np.random.default_rng(35)
    lens = [page * 21 + 3, page * 2, 1, page * 9 - 1]
    p = Paged8(rng, shape(H, Hkv, D, dtype), page, lens, width=4096 if keep > 100 else None)
    seen = np.array([[n - 1, n] for n in lens], dtype=np.int32)
    pages = np.full((4, 2, Hkv, keep), -1, dtype=np.int32)
    for b, n in enumerate(lens):
        count = -(-n // page)
        for i in range(2):
            for g in range(Hkv):
                some = rng.permutation(count)[:min(keep, max(1, count - 1))]
                pages[b, i, g, :len(some)] = some
    pages[0, 0, 0, :] = -1                                      # nothing at all
    pages[0, 0, Hkv - 1, 3:6] = [-7, 22, 10 ** 9]               # no pages of this row
    pages[0, 1, 0, :4] = [21, 3, 3, 0]                          # the same page twice
    _attend_and_check(p, rng, seen, pages)


def test_scales_that_are_no_powers_of_two():
    rng = np.random.default_rng(36)
    for dtype, D in [("bf16", 128), ("f32", 128)]:
        p = Paged8(rng, shape(8, 2, D, dtype), 32, [200])
        p.scales = (p.scales * rng.uniform(1, 2, p.scales.shape)).astype(np.float32).astype(np.float64)
        p.upload(bounds=False)
        _attend_and_check(p, rng, np.array([[200]], dtype=np.int32))


def test_selection_reads_the_bounds_that_append_keeps():
    """append -> select -> attention over the pages that it keeps, in 8 bits."""
    rng = np.random.default_rng(37)
    sh = shape(8, 2, 128, "bf16")
    p = Paged8(rng, sh, 16, [300, 90])
    want, _, _, _ = _append(p, rng, [0, 0], [300, 90], False)
    p.codes, p.scales, p.bounds = list(want[0]), want[1], want[2]
    q = normal(rng, (2, 1, 8, 128), "bf16")
    seen, keep = np.array([[300], [90]], dtype=np.int32), 5
    pages = torch.empty(2, 1, 2, keep, dtype=torch.int32, device=DEV)
    qb.qcf_page_select(p.desc, p.cache, 2, 1, torch.from_numpy(q).to(device=DEV, dtype=p.dt), i32(seen), keep, 1, 1, pages)
    torch.cuda.synchronize()
    for b in range(2):
        count = -(-seen[b, 0] // 16)
        score = orc.page_scores(q[b, 0], p.bounds, p.table[b, :count])
        assert np.array_equal(pages[b, 0].cpu().numpy(), orc.page_select(score, keep, 1, 1))
    _attend_and_check(p, rng, seen, pages.cpu().numpy(), q)


def test_pools_beyond_32_bits_of_bytes():
    """Slots more than 2^32 bytes behind the beginning of their pool."""
    sh = shape(2, 1, 64, "bf16")
    rng = np.random.default_rng(38)
    n_pages, page = 17000, 16
    pool = [torch.zeros(n_pages, page, 1, 1 << 14, dtype=torch.uint8, device=DEV)[..., :64] for _ in range(2)]
    scales = torch.ones(n_pages, 1, 2, 1, device=DEV)
    far = [16900, 16999, 3]
    assert far[0] * page * (1 << 14) > 2 ** 32
    table = i32([far])
    cache = qb.page8_cache(pool[0].view(E4M3), pool[1].view(E4M3), scales, None, table, torch.bfloat16)
    desc = qb.make_desc(sh)
    k, v = (torch.from_numpy(normal(rng, (40, 1, 64), "bf16")).to(device=DEV, dtype=torch.bfloat16) for _ in range(2))
    qb.qcf_page8_append(desc, cache, 1, None, k, v, i64([0, 40]), 40, i32([0]), None, None)
    q = torch.from_numpy(normal(rng, (1, 1, 2, 64), "bf16")).to(device=DEV, dtype=torch.bfloat16)
    o = torch.empty_like(q)
    qb.qcf_page8_attn(desc, cache, 1, 1, q, i32([[40]]), None, 0, o, None)
    torch.cuda.synchronize()
    got = pool[1][16999, 0, 0].cpu().view(E4M3).double().numpy() * scales[16999, 0, 1, 0].item()
    assert np.array_equal(got, orc.e4m3(to_np(v)[16, 0] / scales[16999, 0, 1, 0].item()) * scales[16999, 0, 1, 0].item())
    vals = [np.concatenate([pool[i][f, :, 0].cpu().view(E4M3).double().numpy() * scales[f, 0, i, 0].item() for f in far])[:40] for i in range(2)]
    for h in range(2):
        z = vals[0] @ to_np(q)[0, 0, h] / 8.0
        e = np.exp(z - z.max())
        assert np.abs(to_np(o)[0, 0, h] - e @ vals[1] / e.sum()).max() <= 2.0 ** -8 * 4 + 1e-4


def test_steps_replay_from_a_captured_graph_and_on_another_stream():
    rng = np.random.default_rng(39)
    sh = shape(8, 2, 128, "bf16")
    start, room = [40, 7], 8
    p = Paged8(rng, sh, 16, [n + room for n in start], width=1024)
    first = [t.clone() for t in (p.kd.view(torch.uint8), p.vd.view(torch.uint8), p.sd, p.bd)]
    lens, seen = i32(start), i32(start)[:, None] + 1
    qkv = torch.from_numpy(normal(rng, (2, 12 * 128), "bf16")).to(device=DEV, dtype=p.dt)
    parts = [t.unflatten(1, (-1, 128)) for t in qkv.split([8 * 128, 256, 256], 1)]
    q, o, lse, off = torch.empty(2, 8, 128, dtype=p.dt, device=DEV), torch.empty(2, 1, 8, 128, dtype=p.dt, device=DEV), torch.empty(2, 1, 8, device=DEV), i64([0, 1, 2])
    ws = torch.empty(qb.qcf_page8_attn_workspace_bytes(p.desc, p.cache, 2, 1, 0), dtype=torch.uint8, device=DEV)

    def step():
        qb.qcf_page8_append(p.desc, p.cache, 2, *parts, off, 2, lens, lens, q)
        qb.qcf_page8_attn(p.desc, p.cache, 2, 1, q, seen, None, 0, o, lse, ws)
        lens.add_(1), seen.add_(1), qkv.mul_(1.5)

    def reset():
        for t, f in zip((p.kd.view(torch.uint8), p.vd.view(torch.uint8), p.sd, p.bd), first):
            t.copy_(f)
        lens.copy_(i32(start)), seen.copy_(i32(start)[:, None] + 1), qkv.copy_(rows)

    rows, eager = qkv.clone(), []
    for _ in range(6):
        step()
        torch.cuda.synchronize()
        eager.append([t.clone() for t in (o, lse, p.kd.view(torch.uint8), p.sd, p.bd)])
    reset()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for i in range(6):
            step()
            for got, want in zip((o, lse, p.kd.view(torch.uint8), p.sd, p.bd), eager[i]):
                assert torch.equal(got, want), i
        reset()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(6):
        o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((o, lse, p.kd.view(torch.uint8), p.sd, p.bd), eager[i]):
            assert torch.equal(got, want), i
