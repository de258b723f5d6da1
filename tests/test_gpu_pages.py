"""GPU parity of the paged calls (qcf_pages.h) against the float64 oracle on identical inputs.

Tolerances, derived: a stored result is off by at most half a step, 2^-8 (bf16) or 2^-24 (f32) of its value, plus what was computed.
  rotation   (cos, sin) are off by less than 8 * 2^-24, the two products and their sum by 2^-23 more: 2^-20 (|a| + |b|).
  attention  a logit z = q . k / sqrt(d) of d products in 32 bits is off by at most eps = (d + 4) 2^-24 sum |q k| / sqrt(d); all
             weights then by a factor of exp(2 eps), and by 2^-22 for the exponential; sums over T tokens add T 2^-24 in any order;
             weights that enter the product as two bf16 terms 2^-16.  All of these are relative to sum p |v| <= max |v|.
  lse        eps + T 2^-24 + 2^-22 (1 + |lse|).
"""
import math

import numpy as np
import pytest
import torch

from oracle import qcf_oracle as orc
from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd import inputs
import page_rules
from gpu_util import DEV, i32, i64, to_np

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def say(*a):
    print(*a, flush=True)


def shape(H, Hkv, D, dtype, style=0, base=500000.0):
    return inputs.LayerShape(H * D, H, Hkv, D, base, dtype, style)


def normal(rng, size, dtype, std=1.0):
    return inputs.round_to_dtype((rng.standard_normal(size) * std).astype(np.float32), dtype)


class Paged:
    """Pools of random values in shuffled pages, and the same on the GPU; `order` puts heads or tokens next to each other."""

    def __init__(self, rng, sh, page, lens, order="token", spare=3, width=None, std=1.0, bounds=True):
        self.sh, self.page = sh, page
        Hkv, D, dt = sh.n_kv_heads, sh.head_dim, inputs.torch_dtype(sh.dtype)
        counts = [-(-n // page) for n in lens]
        n_pages = sum(counts) + spare
        perm = rng.permutation(n_pages)
        self.table = np.full((len(lens), max(counts + [1]) if width is None else width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(counts):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.k, self.v = normal(rng, (n_pages, page, Hkv, D), sh.dtype, std), normal(rng, (n_pages, page, Hkv, D), sh.dtype)
        self.bounds = np.stack([self.k.min(1), self.k.max(1)], axis=2)
        self.dt, self.order = dt, order
        self.upload(bounds)

    def upload(self, bounds=True):
        def pool(a):
            t = torch.from_numpy(np.ascontiguousarray(a)).to(device=DEV, dtype=self.dt)
            return t.transpose(1, 2).contiguous().transpose(1, 2) if self.order == "head" else t
        self.kd, self.vd = pool(self.k), pool(self.v)
        self.bd = torch.from_numpy(np.ascontiguousarray(self.bounds)).to(device=DEV, dtype=self.dt) if bounds else None
        self.td = i32(self.table)
        self.cache = qb.page_cache(self.kd, self.vd, self.bd, self.td)
        self.desc = qb.make_desc(self.sh)


# ------------------------------------------------------------------ append

APPENDS = [
    # dtype, H, Hkv, D, style, page, order, (held, new) of each request, rotated
    ("bf16", 32, 8, 128, 0, 16, "token", [(0, 1), (15, 1), (16, 1), (777, 1)], True),
    ("bf16", 8, 2, 128, 1, 16, "head", [(5, 40), (0, 0), (31, 2), (16, 16)], True),
    ("bf16", 4, 4, 64, 0, 64, "token", [(45, 131)], True),
    ("bf16", 6, 2, 64, 1, 256, "token", [(0, 300), (250, 7)], True),
    ("bf16", 8, 8, 128, 0, 128, "token", [(0, 257), (3, 1)], False),
    ("f32", 4, 2, 64, 1, 32, "head", [(7, 9), (0, 33), (63, 1)], True),
    ("f32", 16, 1, 128, 0, 16, "token", [(0, 17), (1, 1), (2, 30)], True),
    ("f32", 2, 2, 64, 0, 128, "token", [(100, 100)], False),
]


def _append(p, rng, lens, new, rotated, far=0):
    sh = p.sh
    H, Hkv, D = sh.n_q_heads, sh.n_kv_heads, sh.head_dim
    M = sum(new)
    off = np.concatenate([[0], np.cumsum(new)])
    rows = normal(rng, (M + 2, (H + 2 * Hkv) * D), sh.dtype)                    # two rows behind the last: padding
    q, k, v = (a.reshape(M + 2, -1, D) for a in np.split(rows, [H * D, (H + Hkv) * D], axis=1))
    pos = (np.concatenate([np.arange(n) + h for h, n in zip(lens, new)] + [[9, 9]]) + far).astype(np.int32)
    dev = torch.from_numpy(rows).to(device=DEV, dtype=p.dt)
    parts = [t.unflatten(1, (-1, D)) for t in dev.split([H * D, Hkv * D, Hkv * D], 1)]
    q_out = torch.full((M + 2, H, D), 7.0, dtype=p.dt, device=DEV)
    say("append", sh.dtype, H, Hkv, D, "style", sh.rope_style, "page", p.page, p.order, list(zip(lens, new)))
    qb.qcf_page_append(p.desc, p.cache, len(new), *parts, i64(off), M + 2, i32(lens), i32(pos) if rotated else None, q_out)
    torch.cuda.synchronize()
    pools = orc.page_append((p.k, p.v, p.bounds), p.table, lens, off, k[:M], v[:M], pos[:M] if rotated else None, sh.rope_base,
                            sh.rope_style)
    q64 = orc.rope_at(q[:M], pos[:M], sh.rope_base, sh.rope_style) if rotated else np.asarray(q[:M], dtype=np.float64)
    return pools, q64, q_out, max(np.abs(rows).max(), 1.0)


def _check_append(p, pools, q64, q_out, largest, rotated):
    step = HALF_STEP[p.sh.dtype] if rotated else 0.0
    slack = 2.0 ** -20 * 2 * largest if rotated else 0.0
    got_k, got_v, got_b = to_np(p.kd), to_np(p.vd), to_np(p.bd)
    for got, ref in ((got_k, pools[0]), (to_np(q_out)[:len(q64)], q64)):
        assert np.all(np.abs(got - ref) <= step * np.abs(ref) + slack)
    assert np.array_equal(got_v, pools[1])
    untouched = pools[0] == np.asarray(p.k, dtype=np.float64)                   # (a turned key is never the old one by chance)
    assert np.array_equal(got_k[untouched], pools[0][untouched])
    assert np.all(to_np(q_out)[len(q64):] == 7.0)
    assert np.all(np.abs(got_b - pools[2]) <= step * np.abs(pools[2]) + slack)
    return got_k, got_b


@pytest.mark.parametrize("case", APPENDS)
def test_append(case):
    dtype, H, Hkv, D, style, page, order, requests, rotated = case
    rng = np.random.default_rng(1)
    lens, new = [r[0] for r in requests], [r[1] for r in requests]
    p = Paged(rng, shape(H, Hkv, D, dtype, style), page, [a + b for a, b in requests], order)
    pools, q64, q_out, largest = _append(p, rng, lens, new, rotated)
    got_k, got_b = _check_append(p, pools, q64, q_out, largest, rotated)
    # the bounds are those of the keys as they are stored: exactly, page by page
    for b, (held, n) in enumerate(requests):
        for pg in range(held // page, -(-(held + n) // page)) if n else ():
            t0, t1 = max(held, pg * page), min(held + n, (pg + 1) * page)
            rows = got_k[p.table[b, pg], t0 - pg * page:t1 - pg * page]
            lo, hi = rows.min(0), rows.max(0)
            if t0 % page:
                lo, hi = np.minimum(lo, p.bounds[p.table[b, pg], :, 0]), np.maximum(hi, p.bounds[p.table[b, pg], :, 1])
            assert np.array_equal(got_b[p.table[b, pg], :, 0], lo) and np.array_equal(got_b[p.table[b, pg], :, 1], hi)


@pytest.mark.parametrize("dtype,far", [("f32", 3000000), ("bf16", 2000000000), ("f32", -100000)])
def test_append_at_far_positions(dtype, far):
    """Positions beyond what a float holds, and backwards: the angle's fraction is taken in 64 bits (at 2^31 positions the product
    with a frequency of at most 1 / 2 pi is off by 2^-25 of a turn, which the bound on the factors includes)."""
    rng = np.random.default_rng(2)
    p = Paged(rng, shape(4, 2, 64, dtype), 16, [40])
    out = _append(p, rng, [3], [37], True, far)
    _check_append(p, *out, True)


def test_append_drops_what_has_no_page_and_takes_special_values():
    rng = np.random.default_rng(3)
    sh = shape(4, 2, 64, "bf16")
    p = Paged(rng, sh, 16, [40, 20, 30, 16])
    p.table[0, 1] = -1                                         # rows 13.. of request 0: no page
    p.table[1, 0] = 10 ** 6
    p.k[p.table[2, 0], 0, 0, 3] = np.nan                       # an old key that was not a number is in the old bounds
    p.bounds = np.stack([p.k.min(1), p.k.max(1)], axis=2)
    p.upload()
    lens, new = [3, 0, 2, -4], [33, 20, 5, 9]                  # request 2 continues its page; request 3 begins before token 0
    before = to_np(p.kd)
    pools, q64, q_out, largest = _append(p, rng, lens, new, True)
    got_b = to_np(p.bd)
    assert np.isnan(got_b[p.table[2, 0], 0, :, 3]).all() and np.isfinite(got_b[p.table[3, 0]]).all()
    k = to_np(p.kd)
    written = np.zeros(k.shape[:2], dtype=bool)
    for b, pg, s in [(0, 0, slice(3, 16)), (0, 2, slice(0, 4)), (1, 1, slice(0, 4)), (2, 0, slice(2, 7)), (3, 0, slice(0, 5))]:
        written[p.table[b, pg], s] = True
    assert np.array_equal(k[~written], before[~written], equal_nan=True)
    assert np.all(np.abs(k[written] - pools[0][written]) <= 2.0 ** -8 * np.abs(pools[0][written]) + 2.0 ** -19 * largest)
    assert np.all(np.abs(to_np(q_out)[:67] - q64) <= 2.0 ** -8 * np.abs(q64) + 2.0 ** -19 * largest)
    # rows past the table's last page
    p2 = Paged(rng, sh, 16, [32])
    _, _, q_out, _ = _append(p2, rng, [30], [10], False)
    assert np.array_equal(to_np(p2.kd)[p2.table[0, 0]], np.asarray(p2.k[p2.table[0, 0]], dtype=np.float64))


def test_append_without_queries_or_bounds_and_queries_in_place():
    rng = np.random.default_rng(4)
    p = Paged(rng, shape(4, 2, 64, "f32"), 32, [50], bounds=False)
    k, v, q = (torch.randn(20, n, 64, device=DEV) for n in (2, 2, 4))
    pos = i32(np.arange(20))
    other = torch.empty_like(q)
    qb.qcf_page_append(p.desc, p.cache, 1, q, k, v, i64([0, 20]), 20, i32([30]), pos, other)
    once = p.kd.clone()
    qb.qcf_page_append(p.desc, p.cache, 1, None, k, v, i64([0, 20]), 20, i32([30]), pos, None)
    qb.qcf_page_append(p.desc, p.cache, 1, q, k, v, i64([0, 20]), 20, i32([30]), pos, q)
    torch.cuda.synchronize()
    assert torch.equal(once, p.kd) and torch.equal(q, other)


# ------------------------------------------------------------------ attention

def _bounds_on_error(sh, k_rows, v_rows, q, tokens):
    """(on a logit, on an output element) for queries q [H, d] over rows [T, H_kv, d]."""
    G = sh.group
    D = sh.head_dim
    terms = np.stack([np.abs(k_rows[:, h // G]) @ np.abs(q[h]) for h in range(q.shape[0])]).max()
    eps = (D + 4) * 2.0 ** -24 * terms / math.sqrt(D)
    rel = 2 * eps + 2.0 ** -22 + tokens * 2.0 ** -24 + (2.0 ** -16 if sh.dtype == "bf16" else 0.0)
    return eps, rel * np.abs(v_rows).max()


def _attend_and_check(p, rng, seen, pages=None, q=None, with_lse=True):
    sh = p.sh
    H, D = sh.n_q_heads, sh.head_dim
    B, n_q = seen.shape
    q = normal(rng, (B, n_q, H, D), sh.dtype, 1.5) if q is None else q
    qd = torch.from_numpy(q).to(device=DEV, dtype=p.dt)
    o = torch.full((B, n_q, H, D), 7.0, dtype=p.dt, device=DEV)
    lse = torch.full((B, n_q, H), 7.0, dtype=torch.float32, device=DEV) if with_lse else None
    n_keep = 0 if pages is None else pages.shape[-1]
    say("attention", sh.dtype, H, sh.n_kv_heads, D, "page", p.page, p.order, "seen", seen.tolist() if seen.size < 40 else seen.shape, "keep", n_keep)
    qb.qcf_page_attn(p.desc, p.cache, B, n_q, qd, i32(seen), None if pages is None else i32(pages), n_keep, o, lse)
    torch.cuda.synchronize()
    got, z = to_np(o), to_np(lse) if with_lse else None
    for b in range(B):
        for i in range(n_q):
            ref, ref_z = orc.page_attn(q[b, i], p.k, p.v, p.table[b], seen[b, i], None if pages is None else pages[b, i])
            used = [x for x in p.table[b, :-(-seen[b, i] // p.page)] if 0 <= x < len(p.k)] if seen[b, i] > 0 else []
            if not used or not np.isfinite(ref_z).any():
                assert not got[b, i].any() and (not with_lse or np.all(z[b, i] == -np.inf)), (b, i)
                continue
            rows = p.k[used].reshape(-1, sh.n_kv_heads, D), p.v[used].reshape(-1, sh.n_kv_heads, D)
            rows = [np.where(np.isfinite(r), r, 0.0).astype(np.float64) for r in rows]
            eps, out = _bounds_on_error(sh, *rows, np.asarray(q[b, i], dtype=np.float64), len(rows[0]))
            assert np.all(np.abs(got[b, i] - ref) <= HALF_STEP[sh.dtype] * np.abs(ref) + out), (b, i, np.abs(got[b, i] - ref).max(), out)
            if with_lse:
                seeing = np.isfinite(ref_z)
                assert np.all(z[b, i][~seeing] == -np.inf)
                off = np.abs(z[b, i][seeing] - ref_z[seeing])
                assert np.all(off <= eps + len(rows[0]) * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(ref_z[seeing]))), (b, i)
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
]


@pytest.mark.parametrize("case", ATTENTIONS)
def test_attention_over_all_pages_in_ranges(case):
    """The same contexts in a table that is wide enough for long ones: divided over the GPU and joined."""
    dtype, H, Hkv, D, page, order, seen = case
    rng = np.random.default_rng(15)
    seen = np.array(seen, dtype=np.int32)
    sh = shape(H, Hkv, D, dtype)
    p = Paged(rng, sh, page, seen.max(1).tolist(), order, width=65536 // page)
    assert page_rules.division(p.desc, p.cache, seen.shape[0], seen.shape[1], 0)["whole"] == 0
    _attend_and_check(p, rng, seen)


@pytest.mark.parametrize("case", ATTENTIONS)
def test_attention_over_all_pages(case):
    dtype, H, Hkv, D, page, order, seen = case
    rng = np.random.default_rng(5)
    seen = np.array(seen, dtype=np.int32)
    p = Paged(rng, shape(H, Hkv, D, dtype), page, seen.max(1).tolist(), order)
    _attend_and_check(p, rng, seen)


@pytest.mark.parametrize("dtype,H,Hkv,D,page,seen", [
    # rows of one request that see very different parts of it, in ranges that begin and end among them
    ("bf16", 8, 2, 128, 16, [[3000, 17, 1500, 2999], [40, 900, 0, 33]]),
    ("bf16", 16, 2, 128, 32, [[5000, 2500, 0, 64, 4999], [1, 2, 3, 4, 2000]]),           # 40 rows: three blocks of 16 or two of 32
    ("bf16", 128, 2, 64, 16, [[700], [2100]]),                                           # 64 rows of one token
    ("f32", 24, 2, 128, 64, [[1000, 999, 31], [3, 640, 0]]),
    ("f32", 8, 1, 64, 16, [[4000, 100, 3999, 2048, 2047, 0, 5, 9]]),
    # more contexts than ranges (64 KV heads: 8 ranges), and more than 64
    ("bf16", 64, 64, 64, 16, [[37 * i % 900 + 1] for i in range(30)]),
    ("bf16", 32, 32, 128, 16, [[97 * i % 1300] for i in range(80)]),
    ("f32", 16, 16, 64, 32, [[61 * i % 500, 7 * i] for i in range(70)])])
def test_attention_of_uneven_rows_and_contexts_in_ranges(dtype, H, Hkv, D, page, seen):
    rng = np.random.default_rng(16)
    seen = np.array(seen, dtype=np.int32)
    p = Paged(rng, shape(H, Hkv, D, dtype), page, np.maximum(seen.max(1), 1).tolist(), width=131072 // page)
    assert page_rules.division(p.desc, p.cache, seen.shape[0], seen.shape[1], 0)["whole"] == 0
    _attend_and_check(p, rng, seen)


@pytest.mark.parametrize("dtype,H,Hkv,D,page,lens", [
    ("bf16", 8, 2, 128, 16, [20000, 1, 300, 5000]), ("bf16", 2, 1, 64, 64, [60001]), ("f32", 4, 2, 64, 16, [9000, 40]),
    ("bf16", 4, 4, 128, 32, [100 + 37 * i for i in range(70)])])
def test_attention_divided_over_long_and_many_contexts(dtype, H, Hkv, D, page, lens):
    rng = np.random.default_rng(6)
    p = Paged(rng, shape(H, Hkv, D, dtype), page, lens)
    o, lse = _attend_and_check(p, rng, np.array(lens, dtype=np.int32)[:, None])
    assert torch.isfinite(o.float()).all()


@pytest.mark.parametrize("width", [9, 8192])                  # contexts taken whole, and in ranges
def test_attention_does_not_read_what_is_not_seen(width):
    """NaN and infinities in slots behind `seen`, in absent pages' place (page 0 of the pool) and in pages of no request."""
    rng = np.random.default_rng(7)
    for dtype, D, n_q in [("bf16", 128, 1), ("bf16", 64, 3), ("f32", 64, 2), ("bf16", 128, 8), ("f32", 128, 1), ("f32", 128, 6)]:
        seen = np.array([[75 - n_q + 1 + i for i in range(n_q)], [16] * n_q, [33] * n_q, [0] * n_q], dtype=np.int32)
        p = Paged(rng, shape(8, 2, D, dtype), 16, [75, 16, 33, 40], width=width)
        free = np.setdiff1d(np.arange(len(p.k)), p.table)
        p.k[free], p.v[free] = np.nan, np.inf
        for b, n in enumerate([75, 16, 33, 0]):
            for t in range(n, 80 if b == 0 else 48 if b == 2 else n):
                p.k[p.table[b, t // 16], t % 16], p.v[p.table[b, t // 16], t % 16] = (np.nan, -np.inf) if t % 2 else (np.inf, np.nan)
        mine = free[free > 0][0]                                            # page 0 of the pool belongs to nobody
        if 0 in p.table:
            p.k[mine], p.v[mine] = p.k[0], p.v[0]
            p.table[p.table == 0] = mine
        p.table[0, 2] = -5                                                  # a page in the middle is not there
        p.k[0], p.v[0] = np.nan, np.nan
        p.upload(bounds=False)
        _attend_and_check(p, rng, seen)


@pytest.mark.parametrize("width", [4, 16384])                 # (whole, in ranges)
@pytest.mark.parametrize("H", [8, 20])                        # rows in one tile and in two
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_values_that_only_later_drafts_see_do_not_reach_earlier_ones(dtype, D, H, width):
    rng = np.random.default_rng(8)
    p = Paged(rng, shape(H, 2, D, dtype), 16, [60], width=width)
    p.v[p.table[0, 58 // 16], 58 % 16] = np.inf
    p.v[p.table[0, 59 // 16], 59 % 16] = np.nan
    p.upload()
    q = torch.from_numpy(normal(rng, (1, 4, H, D), dtype)).to(device=DEV, dtype=p.dt)
    o, alone = torch.empty_like(q), torch.empty_like(q)
    qb.qcf_page_attn(p.desc, p.cache, 1, 4, q, i32([[57, 58, 59, 60]]), None, 0, o, None)
    qb.qcf_page_attn(p.desc, p.cache, 1, 4, q, i32([[57, 58, 57, 57]]), None, 0, alone, None)
    torch.cuda.synchronize()
    assert torch.isfinite(o[:, :2].float()).all()
    assert (o[:, :2].float() - alone[:, :2].float()).abs().max() <= 2 * HALF_STEP[dtype] * alone.float().abs().max()
    assert torch.isinf(o[:, 2].float()).all() and torch.isnan(o[:, 3].float()).all()


def test_logits_that_are_not_finite():
    rng = np.random.default_rng(9)
    for dtype, D in [("bf16", 128), ("f32", 64)]:
        p = Paged(rng, shape(4, 4, D, dtype), 16, [50])
        at = lambda t: (p.table[0, t // 16], t % 16)
        p.k[at(7)][0] = -np.inf                    # head 0: one logit -inf or NaN by the query's sign: a query of ones makes it -inf
        p.k[at(8)][1] = np.inf                     # head 1: a logit of +inf: NaN
        for t in range(50):
            p.k[at(t)][2] = -np.inf                # head 2: all logits -inf: NaN
        p.v[at(9)][3] = -np.inf                    # head 3: an infinite value
        p.upload()
        q = torch.ones(1, 1, 4, D, device=DEV, dtype=p.dt)
        o, lse = torch.empty_like(q), torch.empty(1, 1, 4, device=DEV)
        qb.qcf_page_attn(p.desc, p.cache, 1, 1, q, i32([[50]]), None, 0, o, lse)
        p.k[at(7)][0] = -60.0                      # weighs nothing either way
        p.upload()
        same = torch.empty_like(q)
        qb.qcf_page_attn(p.desc, p.cache, 1, 1, q, i32([[50]]), None, 0, same, None)
        torch.cuda.synchronize()
        assert torch.equal(o[0, 0, 0], same[0, 0, 0])
        assert torch.isnan(o[0, 0, 1].float()).all() and torch.isnan(o[0, 0, 2].float()).all()
        assert (o[0, 0, 3].float() == -math.inf).all()
        assert torch.isfinite(lse[0, 0, 0]) and torch.isfinite(lse[0, 0, 3])


@pytest.mark.parametrize("dtype,H,Hkv,D,page,keep", [
    ("bf16", 32, 8, 128, 16, 11), ("bf16", 8, 2, 64, 64, 11), ("f32", 4, 2, 64, 32, 11),
    ("bf16", 32, 8, 128, 16, 3000), ("f32", 4, 2, 64, 32, 900), ("bf16", 24, 1, 128, 32, 2000)])     # (long lists are divided)
def test_attention_over_listed_pages(dtype, H, Hkv, D, page, keep):
    rng = np.random.default_rng(10)
    lens = [page * 21 + 3, page * 2, 1, page * 9 - 1]
    p = Paged(rng, shape(H, Hkv, D, dtype), page, lens, width=4096 if keep > 100 else None)
    n_q = 2
    assert page_rules.division(p.desc, p.cache, 4, n_q, keep)["whole"] == (keep < 100)
    seen = np.array([[n - 1, n] for n in lens], dtype=np.int32)
    pages = np.full((4, n_q, Hkv, keep), -1, dtype=np.int32)
    for b, n in enumerate(lens):
        count = -(-n // page)
        for i in range(n_q):
            for g in range(Hkv):
                some = rng.permutation(count)[:min(keep, max(1, count - 1))]
                pages[b, i, g, :len(some)] = some
    pages[0, 0, 0, :] = -1                                      # nothing at all
    pages[0, 0, Hkv - 1, 3:6] = [-7, 22, 10 ** 9]               # no pages of this row
    pages[0, 1, 0, :4] = [21, 3, 3, 0]                          # the same page twice
    _attend_and_check(p, rng, seen, pages)


@pytest.mark.parametrize("dtype,H,Hkv,D,page,keep,width", [
    ("bf16", 32, 8, 128, 16, 30, None), ("f32", 4, 2, 64, 32, 12, None), ("bf16", 8, 2, 64, 64, 700, 1024), ("bf16", 8, 2, 64, 64, 700, 600),
    ("bf16", 32, 8, 128, 16, 1500, 2048), ("f32", 4, 2, 64, 16, 1100, 2048), ("bf16", 24, 1, 128, 32, 2000, 2048)])
def test_listed_pages_behind_more_entries_than_the_row_has_pages(dtype, H, Hkv, D, page, keep, width):
    """Entries that are no page of the row, before and between those that are, and pages listed again, in lists wider than the row."""
    rng = np.random.default_rng(22)
    lens = [page * 2 - 3, 5, page * 4, page * 7 + 1]
    p = Paged(rng, shape(H, Hkv, D, dtype), page, lens, width=width)
    pages = np.full((4, 2, Hkv, keep), -1, dtype=np.int32)
    for b, n in enumerate(lens):
        count = -(-n // page)
        for i in range(2):
            for g in range(Hkv):
                at = rng.permutation(keep)[:min(10, keep // 2)]
                pages[b, i, g, at] = rng.integers(0, count + 2, len(at))        # (pages of the row, some again, and pages behind it)
                pages[b, i, g, -1] = count - 1
    pages[1, 1, :, :-1], pages[1, 1, :, -1] = 9, 0                      # the last entry alone
    pages[2, 0] = -1                                                    # none
    pages[3, 1, 0, -1] = -1
    _attend_and_check(p, rng, np.array([[n - 1, n] for n in lens], dtype=np.int32), pages)
    _attend_and_check(p, rng, np.array([[0, n] for n in lens], dtype=np.int32), pages)


def test_a_list_of_all_pages_is_no_list():
    rng = np.random.default_rng(11)
    p = Paged(rng, shape(8, 2, 128, "bf16"), 16, [16 * 40 - 5])
    q = normal(rng, (1, 1, 8, 128), "bf16")
    seen = np.array([[16 * 40 - 5]], dtype=np.int32)
    a, _ = _attend_and_check(p, rng, seen, None, q)
    b, _ = _attend_and_check(p, rng, seen, np.tile(np.arange(40, dtype=np.int32)[::-1], (1, 1, 2, 1)), q)
    assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * a.float().abs().max()


def test_parts_without_finite_logits_beside_others():
    """A part of a context, joined with others, whose logits are all -inf weighs nothing; a context of such parts is NaN."""
    rng = np.random.default_rng(17)
    for dtype, D in [("bf16", 128), ("bf16", 64), ("f32", 64)]:
        p = Paged(rng, shape(2, 2, D, dtype), 16, [2000, 300], width=8192)
        keys = p.k[p.table[0, :125]]
        keys[10:60, :, 0] = -np.inf                            # head 0: tokens 160..959
        keys[:, :, 1] = -np.inf
        p.k[p.table[0, :125]] = keys
        p.upload()
        q = torch.ones(2, 1, 2, D, device=DEV, dtype=p.dt)
        o, lse = torch.empty_like(q), torch.empty(2, 1, 2, device=DEV)
        qb.qcf_page_attn(p.desc, p.cache, 2, 1, q, i32([[2000], [300]]), None, 0, o, lse)
        torch.cuda.synchronize()
        got = to_np(o)
        z = np.concatenate([keys[:10, :, 0], keys[60:, :, 0]]).reshape(-1, D).astype(np.float64).sum(-1) / math.sqrt(D)
        v = np.concatenate([p.v[p.table[0, :10], :, 0], p.v[p.table[0, 60:125], :, 0]]).reshape(-1, D).astype(np.float64)
        w = np.exp(z - z.max())
        ref = w @ v / w.sum()
        assert np.all(np.abs(got[0, 0, 0] - ref) <= HALF_STEP[dtype] * np.abs(ref) + 2.0 ** -10 * np.abs(v).max())
        assert np.isnan(got[0, 0, 1]).all() and np.isfinite(got[1]).all() and np.isfinite(to_np(lse)[0, 0, 0])


def test_lengths_beyond_the_table_and_below_nothing():
    rng = np.random.default_rng(18)
    p = Paged(rng, shape(8, 2, 128, "bf16"), 16, [64, 48])
    q = torch.from_numpy(normal(rng, (2, 2, 8, 128), "bf16")).to(device=DEV, dtype=p.dt)
    outs = []
    for seen in ([[2 ** 31 - 1, -5], [1000, 48]], [[64, 0], [48, 48]]):
        o, lse = torch.empty_like(q), torch.empty(2, 2, 8, device=DEV)
        pages = torch.empty(2, 2, 2, 3, dtype=torch.int32, device=DEV)
        qb.qcf_page_attn(p.desc, p.cache, 2, 2, q, i32(seen), None, 0, o, lse)
        qb.qcf_page_select(p.desc, p.cache, 2, 2, q, i32(seen), 3, 1, 1, pages)
        outs.append((o, lse, pages))
    torch.cuda.synchronize()
    for a, b in zip(outs[0][:2], outs[1][:2]):
        assert torch.equal(a, b)
    # (the last pages of the table are not there for the second request: its own last page is the third)
    assert torch.equal(outs[0][2][0], outs[1][2][0]) and not outs[0][0][0, 1].any()


def test_a_pool_beyond_32_bits_of_elements():
    """Pages 16 MB apart: offsets of 6e9 elements, appended to, selected from and attended to."""
    rng = np.random.default_rng(19)
    sh = shape(8, 2, 128, "bf16")
    n_pages, stride = 720, 1 << 23
    pools = [torch.empty(n_pages * stride, dtype=torch.bfloat16, device=DEV).as_strided((n_pages, 16, 2, 128), (stride, 256, 128, 1)) for _ in range(2)]
    bounds = torch.empty(n_pages, 2, 2, 128, dtype=torch.bfloat16, device=DEV)
    table = np.array([[719, 3, 700, 650, 1, 718]], dtype=np.int32)
    cache = qb.page_cache(*pools, bounds, i32(table))
    desc = qb.make_desc(sh)
    k, v, q = (normal(rng, (n, h, 128), "bf16") for n, h in ((90, 2), (90, 2), (1, 8)))
    dev = lambda a: torch.from_numpy(a).to(device=DEV, dtype=torch.bfloat16)
    qb.qcf_page_append(desc, cache, 1, None, dev(k), dev(v), i64([0, 90]), 90, i32([0]), None, None)
    pages = torch.empty(1, 1, 2, 4, dtype=torch.int32, device=DEV)
    o, some = torch.empty(1, 1, 8, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, 1, 8, 128, dtype=torch.bfloat16, device=DEV)
    qb.qcf_page_attn(desc, cache, 1, 1, dev(q), i32([[90]]), None, 0, o, None)
    qb.qcf_page_select(desc, cache, 1, 1, dev(q), i32([[90]]), 4, 0, 1, pages)
    qb.qcf_page_attn(desc, cache, 1, 1, dev(q), i32([[90]]), pages, 4, some, None)
    torch.cuda.synchronize()
    small = np.zeros((6, 16, 2, 128)), np.zeros((6, 16, 2, 128)), np.zeros((6, 2, 2, 128))
    kp, vp, bp = orc.page_append(small, np.arange(6)[None], [0], [0, 90], k, v, None, 1e4)
    want = orc.page_select(orc.page_scores(q[0], bp, np.arange(6)), 4, 0, 1)
    assert np.array_equal(pages.cpu().numpy()[0, 0], want)
    for got, listed in ((o, None), (some, want)):
        ref, _ = orc.page_attn(q[0], kp, vp, np.arange(6), 90, listed)
        assert np.all(np.abs(to_np(got)[0, 0] - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-3)


# ------------------------------------------------------------------ selection

@pytest.mark.parametrize("dtype,H,Hkv,D,page,lens,n_q,keep,first,last", [
    ("bf16", 32, 8, 128, 16, [16 * 70 + 3, 16 * 9, 5], 1, 8, 1, 2),
    ("bf16", 64, 8, 128, 32, [32 * 40], 3, 12, 0, 1),
    ("bf16", 6, 2, 64, 64, [64 * 33 + 1, 64 * 31], 2, 5, 0, 0),
    ("bf16", 40, 2, 64, 16, [16 * 130], 1, 129, 1, 1),
    ("bf16", 7, 1, 128, 16, [16 * 20], 1, 3, 2, 1),
    ("f32", 4, 2, 64, 16, [16 * 100 + 9, 33], 2, 7, 1, 1),
    ("f32", 8, 8, 128, 128, [128 * 17], 1, 1, 0, 0),
    ("bf16", 4, 4, 64, 16, [16 * 1500], 1, 64, 1, 2), ("bf16", 2, 1, 64, 16, [16 * 9000 + 2], 1, 400, 0, 3),
    ("bf16", 1, 1, 64, 16, [16 * 40000], 1, 300, 1, 1)])
def test_selection(dtype, H, Hkv, D, page, lens, n_q, keep, first, last):
    rng = np.random.default_rng(12)
    p = Paged(rng, shape(H, Hkv, D, dtype), page, lens)
    seen = np.array([[max(0, n - n_q + 1 + i) for i in range(n_q)] for n in lens], dtype=np.int32)
    q = normal(rng, (len(lens), n_q, H, D), dtype)
    pages = torch.full((len(lens), n_q, Hkv, keep), 99, dtype=torch.int32, device=DEV)
    say("selection", dtype, H, Hkv, D, "page", page, lens, "keep", keep, first, last)
    qb.qcf_page_select(p.desc, p.cache, len(lens), n_q, torch.from_numpy(q).to(device=DEV, dtype=p.dt), i32(seen), keep, first, last, pages)
    torch.cuda.synchronize()
    got = pages.cpu().numpy()
    for b in range(len(lens)):
        for i in range(n_q):
            count = -(-seen[b, i] // page)
            s = orc.page_scores(q[b, i], p.bounds.astype(np.float64), p.table[b, :count])
            assert np.array_equal(got[b, i], orc.page_select(s, keep, first, last)), (b, i)


@pytest.mark.parametrize("dtype,H,Hkv,D,B,n_q", [
    ("bf16", 64, 8, 128, 20, 16),                                            # a workgroup takes all pages of its row
    ("bf16", 12, 2, 64, 25, 12), ("f32", 6, 3, 64, 40, 6), ("f32", 10, 2, 128, 21, 9)])     # two or four share them
def test_selection_where_workgroups_take_turns(dtype, H, Hkv, D, B, n_q):
    rng = np.random.default_rng(21)
    p = Paged(rng, shape(H, Hkv, D, dtype), 16, [16 * 350])
    p.table = np.stack([rng.permutation(350) for _ in range(B)]).astype(np.int32)        # (pages may be shared by requests)
    p.upload()
    counts = np.array([0, 1, 63, 64, 65, 127, 128, 129, 200, 256, 257, 320, 321, 349, 350])[rng.integers(0, 15, (B, n_q))]
    seen = np.maximum(16 * counts - rng.integers(0, 16, (B, n_q)), 0).astype(np.int32)
    q = normal(rng, (B, n_q, H, D), dtype)
    pages = torch.full((B, n_q, Hkv, 9), 99, dtype=torch.int32, device=DEV)
    say("selection in turns", dtype, H, Hkv, D, B, n_q)
    qb.qcf_page_select(p.desc, p.cache, B, n_q, torch.from_numpy(q).to(device=DEV, dtype=p.dt), i32(seen), 9, 1, 2, pages)
    torch.cuda.synchronize()
    got = pages.cpu().numpy()
    for b in range(B):
        for i in range(n_q):
            s = orc.page_scores(q[b, i], p.bounds.astype(np.float64), p.table[b, :counts[b, i]])
            assert np.array_equal(got[b, i], orc.page_select(s, 9, 1, 2)), (b, i, counts[b, i])


def test_selection_of_ties_absent_pages_and_values_that_are_not_finite():
    rng = np.random.default_rng(13)
    for dtype in ("bf16", "f32"):
        p = Paged(rng, shape(4, 2, 64, dtype), 16, [16 * 12, 16 * 12, 16 * 12, 0])
        p.k[p.table[1, :12]] = p.k[p.table[1, 0]]                            # all alike
        p.k[p.table[0, 5], 3, 0, 7], p.k[p.table[0, 9], 1, 1, 0] = np.nan, -np.inf
        p.bounds = np.stack([p.k.min(1), p.k.max(1)], axis=2)
        p.table[2, 3:9] = -1                                                 # half of the pages are gone
        p.upload()
        seen = np.array([[190], [192], [180], [0]], dtype=np.int32)
        q = normal(rng, (4, 1, 4, 64), dtype)
        pages = torch.full((4, 1, 2, 8), 99, dtype=torch.int32, device=DEV)
        say("selection of special values", dtype)
        qb.qcf_page_select(p.desc, p.cache, 4, 1, torch.from_numpy(q).to(device=DEV, dtype=p.dt), i32(seen), 8, 0, 1, pages)
        torch.cuda.synchronize()
        got = pages.cpu().numpy()[:, 0]
        for b in range(4):
            s = orc.page_scores(q[b, 0], p.bounds.astype(np.float64), p.table[b, :-(-seen[b, 0] // 16)])
            assert np.array_equal(got[b], orc.page_select(s, 8, 0, 1)), b
        assert 5 in got[0, 0] and 9 in got[0, 1] and got[1].tolist() == [[0, 1, 2, 3, 4, 5, 6, 11]] * 2
        assert {0, 1, 2, 9, 10, 11} <= set(got[2, 0]) and (got[3] == -1).all()


# ------------------------------------------------------------------ together

def test_a_step_replays_from_a_captured_graph_and_on_another_stream():
    """append -> select -> attention, captured once and replayed as the request grows (lengths and positions live on the device)."""
    rng = np.random.default_rng(14)
    sh = shape(8, 2, 128, "bf16")
    lens = [300, 31]
    p = Paged(rng, sh, 16, [n + 8 for n in lens])
    q_in, k, v = (torch.randn(2, n, 128, device=DEV).to(p.dt) for n in (8, 2, 2))
    held, pos, seen = i32(lens), i32(lens), i32([[n + 1] for n in lens])
    off = i64([0, 1, 2])
    q = torch.empty(2, 8, 128, dtype=p.dt, device=DEV)
    pages = torch.empty(2, 1, 2, 6, dtype=torch.int32, device=DEV)
    o, lse = torch.empty_like(q), torch.empty(2, 8, device=DEV)
    ws = [torch.empty(max(n, 1), dtype=torch.uint8, device=DEV) for n in (
        qb.qcf_page_select_workspace_bytes(p.desc, p.cache, 2, 1, 6), qb.qcf_page_attn_workspace_bytes(p.desc, p.cache, 2, 1, 6))]

    def step():
        qb.qcf_page_append(p.desc, p.cache, 2, q_in, k, v, off, 2, held, pos, q)
        qb.qcf_page_select(p.desc, p.cache, 2, 1, q, seen, 6, 1, 2, pages, ws[0])
        qb.qcf_page_attn(p.desc, p.cache, 2, 1, q, seen, pages, 6, o, lse, ws[1])

    def grow(n):
        for t in (held, pos, seen):
            t.add_(n)

    start = p.kd.clone(), p.vd.clone(), p.bd.clone()

    def reset():
        p.kd.copy_(start[0]), p.vd.copy_(start[1]), p.bd.copy_(start[2])

    eager = []
    for i in range(6):
        step()
        eager.append((o.clone(), lse.clone(), pages.clone(), p.kd.clone(), p.bd.clone()))
        grow(1)
    grow(-6)
    reset()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for i in range(6):
            step()
            for got, want in zip((o, lse, pages, p.kd, p.bd), eager[i]):
                assert torch.equal(got, want), i
            grow(1)
        grow(-6)
        reset()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(6):
        o.fill_(3.0), pages.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((o, lse, pages, p.kd, p.bd), eager[i]):
            assert torch.equal(got, want), i
        grow(1)


def test_two_graphs_that_share_a_workspace_take_turns():
    """Two captured calls over different requests, divided, replayed in turn with eager calls between them: the same bits each time."""
    rng = np.random.default_rng(20)
    sh = shape(32, 8, 128, "bf16")
    a, b = (Paged(rng, sh, 16, lens, width=4096) for lens in ([3000, 50], [700, 900, 4000]))
    calls = []
    ws = torch.empty(max(qb.qcf_page_attn_workspace_bytes(sh_p.desc, sh_p.cache, n, 1, 0) for sh_p, n in ((a, 2), (b, 3))), dtype=torch.uint8, device=DEV)
    for p, lens in ((a, [3000, 50]), (b, [700, 900, 4000])):
        q = torch.from_numpy(normal(rng, (len(lens), 1, 32, 128), "bf16")).to(device=DEV, dtype=p.dt)
        o, lse = torch.empty_like(q), torch.empty(len(lens), 1, 32, device=DEV)
        calls.append((lambda p=p, q=q, s=i32(lens)[:, None].contiguous(), o=o, lse=lse: qb.qcf_page_attn(p.desc, p.cache, len(q), 1, q, s, None, 0, o, lse, ws), o, lse))
    graphs, want = [], []
    for call, o, lse in calls:
        call()
        torch.cuda.synchronize()
        want.append((o.clone(), lse.clone()))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for turn in range(3):
        for i in (0, 1):
            calls[i][1].fill_(2.0), calls[i][2].fill_(2.0)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(calls[i][1], want[i][0]) and torch.equal(calls[i][2], want[i][1]), (turn, i)
            calls[1 - i][0]()
            torch.cuda.synchronize()
            assert torch.equal(calls[1 - i][1], want[1 - i][0]), (turn, i)


def test_calls_on_two_streams_at_once():
    """Divided attention over two caches, each with a workspace of its own, on two streams: the bits of the calls alone."""
    rng = np.random.default_rng(22)
    sh = shape(32, 8, 128, "bf16")
    jobs = []
    for lens in ([9000, 4000, 77], [15000]):
        p = Paged(rng, sh, 16, lens, width=2048)
        q = torch.from_numpy(normal(rng, (len(lens), 1, 32, 128), "bf16")).to(device=DEV, dtype=p.dt)
        ws = torch.empty(qb.qcf_page_attn_workspace_bytes(p.desc, p.cache, len(lens), 1, 0), dtype=torch.uint8, device=DEV)
        o, lse = torch.empty_like(q), torch.empty(len(lens), 1, 32, device=DEV)
        jobs.append((p, q, i32(lens), o, lse, ws, torch.cuda.Stream()))
    run = lambda j: qb.qcf_page_attn(j[0].desc, j[0].cache, len(j[1]), 1, j[1], j[2], None, 0, j[3], j[4], j[5])
    alone = []
    for j in jobs:
        run(j)
        torch.cuda.synchronize()
        alone.append((j[3].clone(), j[4].clone()))
        j[3].fill_(0.0)
    torch.cuda.synchronize()
    for _ in range(20):
        for j in jobs:
            with torch.cuda.stream(j[6]):
                run(j)
    torch.cuda.synchronize()
    for j, (o, lse) in zip(jobs, alone):
        assert torch.equal(j[3], o) and torch.equal(j[4], lse)


def test_append_of_many_requests():
    """More requests than a wave has lanes, some without rows, lengths all over a page."""
    for dtype, B in [("bf16", 300), ("f32", 65), ("bf16", 64), ("f32", 4097), ("bf16", 4500)]:
        rng = np.random.default_rng(21)
        lens = rng.integers(0, 40, B).tolist()
        new = (rng.integers(0, 5, B) * (rng.random(B) < 0.8)).astype(int).tolist()
        p = Paged(rng, shape(4, 2, 64, dtype), 16, [a + b for a, b in zip(lens, new)], width=4)
        _check_append(p, *_append(p, rng, lens, new, True), True)
