"""Pins of the oracle's paged functions against facts that they do not compute themselves."""
import numpy as np
import pytest
from scipy.special import logsumexp, softmax

from oracle import qcf_oracle as orc

RNG = np.random.default_rng


def _paged(rng, tokens, page, n_kv, d, spare=3):
    """A dense context [tokens, n_kv, d] twice (keys, values) and the same in shuffled pages."""
    k, v = rng.standard_normal((2, tokens, n_kv, d))
    n = -(-tokens // page)
    order = rng.permutation(n + spare)[:n]
    pools = [np.full((n + spare, page, n_kv, d), np.nan) for _ in range(2)] + [np.zeros((n + spare, n_kv, 2, d))]
    pools = orc.page_append(pools, order[None], [0], [0, tokens], k, v, None, 1e4)
    return k, v, pools, order


@pytest.mark.parametrize("tokens,page", [(1, 16), (16, 16), (45, 16), (70, 32)])
def test_attention_over_shuffled_pages_is_attention_over_the_context(tokens, page):
    rng = RNG(tokens)
    k, v, (kp, vp, _), order = _paged(rng, tokens, page, 2, 8)
    q = rng.standard_normal((4, 8))
    o, lse = orc.page_attn(q, kp, vp, order, tokens)
    for h in range(4):
        z = k[:, h // 2] @ q[h] / np.sqrt(8)
        assert np.allclose(o[h], softmax(z) @ v[:, h // 2], atol=1e-12) and np.isclose(lse[h], logsumexp(z))
    every = np.tile(np.arange(len(order)), (2, 1))
    again, _ = orc.page_attn(q, kp, vp, order, tokens, every[:, ::-1])
    assert np.allclose(again, o, atol=1e-12)
    none, z = orc.page_attn(q, kp, vp, order, 0)
    assert not none.any() and np.all(z == -np.inf)


def test_appending_in_parts_is_appending_at_once():
    rng = RNG(3)
    k, v = rng.standard_normal((2, 37, 2, 8))
    pools = [rng.standard_normal((6, 16, 2, 8)) for _ in range(2)] + [rng.standard_normal((6, 2, 2, 8))]
    table = np.array([[4, 0, 5]])
    pos = np.arange(37)
    whole = orc.page_append(pools, table, [0], [0, 37], k, v, pos, 1e4)
    part = pools
    for a, b in [(0, 5), (5, 6), (6, 32), (32, 37)]:
        part = orc.page_append(part, table, [a], [0, b - a], k[a:b], v[a:b], pos[a:b], 1e4)
    for a, b in zip(whole, part):
        assert np.array_equal(a, b)
    assert np.array_equal(whole[0][1:4], pools[0][1:4]) and np.array_equal(whole[0][5, 5:], pools[0][5, 5:])
    turned = orc.rope_at(k, pos, 1e4)
    assert np.array_equal(whole[2][5, :, 0], turned[32:].min(0)) and np.array_equal(whole[2][4, :, 1], turned[:16].max(0))


def test_score_bounds_every_product_and_is_reached():
    rng = RNG(4)
    k, _, (_, _, bounds), order = _paged(rng, 64, 16, 2, 8)
    q = rng.standard_normal((4, 8))
    s = orc.page_scores(q, bounds, order)
    for g in range(2):
        dots = np.einsum("tpe,he->thp", k[:, g].reshape(4, 16, 8), q[2 * g:2 * g + 2]).max((1, 2))
        assert np.all(dots <= s[g] + 1e-12)
    one = np.repeat(bounds[:, :, :1], 2, axis=2)                # a page of one key: the product itself
    assert np.allclose(orc.page_scores(q, one, order)[1], [max(one[p, 1, 0] @ q[2], one[p, 1, 0] @ q[3]) for p in order])
    bounds[order[1], 0, 1, 3] = np.inf
    assert orc.page_scores(q, bounds, [order[1], -1, 99])[0].tolist() == [np.inf, -np.inf, -np.inf]


def test_selection_by_hand():
    s = np.array([[1.0, 5, 3, 5, 2, 0, 4]])
    assert orc.page_select(s, 3, 0, 0).tolist() == [[1, 3, 6]]
    assert orc.page_select(s, 3, 1, 1).tolist() == [[0, 1, 6]]
    assert orc.page_select(s, 2, 1, 1).tolist() == [[0, 6]]
    assert orc.page_select(s, 9, 1, 1).tolist() == [[0, 1, 2, 3, 4, 5, 6, -1, -1]]
    assert orc.page_select(np.zeros((1, 5)), 2, 0, 0).tolist() == [[0, 1]]


def test_scores_that_are_not_finite_or_beyond_32_bits():
    q = np.array([[np.inf, 1.0]])
    bounds = np.zeros((3, 1, 2, 2))
    bounds[0, 0, :, 0] = [-2.0, -1.0]                           # inf * -1: a sum of -inf
    bounds[1, 0, :, 0] = [1.0, 2.0]                             # +inf
    assert orc.page_scores(q, bounds, [0, 1, 2, 9])[0].tolist() == [np.inf, np.inf, np.inf, -np.inf]      # (inf * 0: not a number)
    s = np.array([[-np.inf, -1e300, 1e39, 3.0, 1e300, np.inf, -3e38]])
    order = [orc.page_select(s, n, 0, 0)[0].tolist() for n in range(1, 7)]
    assert order == [[5], [2, 5], [2, 4, 5], [2, 3, 4, 5], [2, 3, 4, 5, 6], [1, 2, 3, 4, 5, 6]]
