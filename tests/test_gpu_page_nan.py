"""Attention over pages: a key that is not a number, and values beside logits of -inf, wherever a division of the context puts them."""
import numpy as np
import pytest
import torch

from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd import inputs
import page_rules
from gpu_util import DEV, i32

pytestmark = pytest.mark.gpu


class Context:
    """One request of `tokens` tokens in pages of 16, two KV heads, and calls over it."""

    def __init__(self, dtype, D, G, tokens, seen, width, keep):
        rng = np.random.default_rng(51)
        self.tokens, self.keep, self.n_q = tokens, keep, len(seen)
        self.sh = inputs.LayerShape(2 * G * D, 2 * G, 2, D, 10000.0, dtype)
        self.dt, self.desc = inputs.torch_dtype(dtype), qb.make_desc(self.sh)
        n = -(-tokens // 16)
        self.k, self.v = (torch.from_numpy(rng.standard_normal((n, 16, 2, D)).astype(np.float32)).to(DEV, self.dt) for _ in range(2))
        self.q = torch.from_numpy(rng.standard_normal((1, self.n_q, 2 * G, D)).astype(np.float32)).to(DEV, self.dt)
        table = np.full((1, width), -1, dtype=np.int32)
        table[0, :n] = np.arange(n)
        self.table, self.seen = i32(table), i32([seen])
        pages = np.full((1, self.n_q, 2, keep), -1, dtype=np.int32)
        pages[..., :n] = np.arange(n)[:keep]
        self.pages = i32(pages) if keep else None

    def rule(self):
        return page_rules.division(self.desc, qb.page_cache(self.k, self.v, None, self.table), 1, self.n_q, self.keep)

    def run(self, k=None, v=None):
        cache = qb.page_cache(self.k if k is None else k, self.v if v is None else v, None, self.table)
        o, lse = torch.empty_like(self.q), torch.empty(1, self.n_q, self.sh.n_q_heads, device=DEV)
        qb.qcf_page_attn(self.desc, cache, 1, self.n_q, self.q, self.seen, self.pages, self.keep, o, lse)
        torch.cuda.synchronize()
        return o[0], lse[0]

    def changed(self, pool, tokens, value):
        """The pool with `value` in head 0 of some tokens."""
        new = pool.clone()
        t = torch.as_tensor(tokens, device=DEV)
        new[t // 16, t % 16, 0] = value
        return new


CASES = [
    # dtype, D, heads of a group, tokens, seen by the new rows, width of the table, listed pages
    ("bf16", 128, 4, 33, [33], 3, 0), ("bf16", 64, 4, 33, [33], 3, 0), ("f32", 64, 2, 33, [33], 3, 0), ("f32", 128, 2, 17, [17], 2, 0),
    ("bf16", 128, 4, 300, [300, 299, 298], 19, 0), ("bf16", 64, 4, 33, [33], 3, 3),
    ("bf16", 128, 4, 33, [33], 8192, 0), ("bf16", 128, 4, 3000, [3000], 8192, 0), ("f32", 128, 4, 3000, [3000], 8192, 0),
    ("bf16", 64, 4, 3000, [3000, 2999], 8192, 0), ("f32", 64, 2, 3000, [3000, 17, 2998, 0], 8192, 0),
    ("bf16", 128, 10, 3000, [3000, 2999], 65536, 0), ("f32", 64, 20, 3000, [3000], 65536, 0),
    ("bf16", 128, 4, 3000, [3000], 8192, 4000), ("f32", 64, 4, 3000, [3000], 8192, 4000)]


@pytest.mark.parametrize("case", CASES)
def test_a_key_that_is_not_a_number_makes_its_rows_not_numbers(case):
    c = Context(*case)
    seen, G = case[4], case[2]
    assert c.rule()["whole"] == (case[5] < 100)
    base, base_lse = c.run()
    assert torch.isfinite(base.float()).all()
    n = case[3]
    poisoned = [[n - 1], [0], [n // 2], list(range(n // 3, 2 * n // 3)), list(range(16 * (n // 16), n)), list(range(n))]
    for tokens in poisoned:
        print("nan key", case, len(tokens), "from", tokens[0], flush=True)
        o, lse = c.run(k=c.changed(c.k, tokens, float("nan")))
        for i, s in enumerate(seen):
            if s > tokens[0]:
                assert torch.isnan(o[i, :G]).all() and torch.isnan(lse[i, :G]).all(), (tokens[0], len(tokens), i)
            else:
                assert torch.equal(o[i, :G], base[i, :G]) and torch.equal(lse[i, :G], base_lse[i, :G])
        assert torch.equal(o[:, G:], base[:, G:]) and torch.equal(lse[:, G:], base_lse[:, G:])


@pytest.mark.parametrize("case", CASES)
def test_values_that_are_not_finite_beside_logits_of_minus_infinity(case):
    """0 times such a value is not 0: the row is NaN, as it is where other tokens of the same tile have finite logits."""
    c = Context(*case)
    seen, G = case[4], case[2]
    c.q.abs_()                                                 # a key of -inf makes its logit -inf
    n = case[3]
    for tokens in [[n - 1], [n // 2], list(range(n // 3, 2 * n // 3)), list(range(16 * (n // 16), n))]:
        k = c.changed(c.k, tokens, -float("inf"))
        base, base_lse = c.run(k=k)
        assert torch.isfinite(base.float()).all()
        for value in (float("nan"), float("inf")):
            print("values", value, case, len(tokens), "from", tokens[0], flush=True)
            o, lse = c.run(k=k, v=c.changed(c.v, tokens[-1:], value))
            for i, s in enumerate(seen):
                if s > tokens[-1]:
                    assert torch.isnan(o[i, :G]).all(), (tokens[0], len(tokens), i)
                else:
                    assert torch.equal(o[i, :G], base[i, :G])
            assert torch.equal(o[:, G:], base[:, G:]) and torch.equal(lse, base_lse)
