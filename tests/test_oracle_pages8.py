"""Pins of the oracle of 8-bit pages, weights and eviction: against torch's own conversion and small cases by hand."""
import math

import numpy as np
import torch

from oracle import qcf_oracle as orc


def test_rounding_is_that_of_the_format():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    finite = np.sort(codes[np.isfinite(codes)])
    assert finite.max() == 448.0 and np.array_equal(orc.e4m3(finite), finite)
    middle = (finite[1:] + finite[:-1]) / 2
    x = np.concatenate([middle, np.nextafter(middle, 1000), np.nextafter(middle, -1000), np.random.default_rng(0).standard_normal(4000) * 30])
    x = x.astype(np.float32)
    assert np.array_equal(orc.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(orc.e4m3(np.nan))


def test_scales():
    for amax, s in [(448.0, 1.0), (np.nextafter(448.0, 1000), 2.0), (1.75, 2.0 ** -8), (1.0, 2.0 ** -8), (1.76, 2.0 ** -7), (0.0, 2.0 ** -100),
                    (2.0 ** 100, 2.0 ** 92), (np.inf, 2.0 ** -100), (np.nan, 2.0 ** -100)]:
        assert orc.page8_scale([0.0, -amax]) == s, amax


def test_a_block_whose_scale_grows_is_rounded_again():
    codes, scales, bounds = np.zeros((2, 1, 16, 1, 2)), np.ones((1, 1, 2, 1)), np.zeros((1, 1, 2, 2))
    codes[0, 0, 0, 0] = [1.0, 2.0 ** -9]                       # 1 and the least value, at a scale of 1
    out, s, b = orc.page8_append(codes, scales, bounds, np.zeros((1, 1), int), [1], [0, 1], np.array([[[896.0, 3.0]]]), np.zeros((1, 1, 2)),
                                 None, 10000.0)
    assert s[0, 0, 0, 0] == 2.0 and s[0, 0, 1, 0] == 1.0       # (the values' does not shrink)
    assert out[0][0, 0, 0].tolist() == [0.5, 0.0]              # 2^-10: half a step, to even
    assert out[0][0, 1, 0].tolist() == [448.0, 1.5]
    assert b[0, 0, 0].tolist() == [0.0, 0.0] and b[0, 0, 1].tolist() == [896.0, 3.0]


def test_weights_sum_to_the_rows_and_forget_fresh_tokens():
    rng = np.random.default_rng(1)
    k, q = rng.standard_normal((3, 16, 2, 64)), rng.standard_normal((2, 4, 64))
    table, seen = np.array([2, 0]), [20, 21]
    lse = np.stack([orc.page_attn(q[i], k, k, table, seen[i])[1] for i in range(2)])
    w = orc.page_weigh(np.full((2, 32), 9.0), q, k, table, seen, lse, 20, 0.5, 1.0)
    assert np.all(w[:, 21:] == 9.0) and np.allclose(w[:, :20].sum(1) + w[:, 20], 20 * 4.5 + 4.0)


def test_tokens_that_stay():
    w = np.array([[5.0, 0.0, 3.0, 3.0, math.nan, 1.0, 0.0]])
    assert orc.page_evict(w, 7, 4, 1, 1).tolist() == [[0, 2, 4, 6]]
    assert orc.page_evict(w, 7, 3, 0, 0).tolist() == [[0, 2, 4]]
    assert orc.page_evict(w, 2, 3, 1, 1).tolist() == [[0, 1, -1]]
    assert orc.page_evict(w, 0, 2, 1, 1).tolist() == [[-1, -1]]
