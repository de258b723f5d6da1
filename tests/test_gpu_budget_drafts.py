"""Decoding with a budget (pipeline.paged_layer, decode_step, advance, evict): whose attention the tokens' weights hold.

Rows that a request accepts, once each: not the drafts that it rejects, not a step that is run again.  Tolerance of a step's weights as for
qcf_page_weigh: exp(z - lse) with z of d products in 32 bits, off by (d + 5) 2^-24 sum |q k| / sqrt(d), z - lse by 2^-23 (1 + |z - lse|) more
and the exponential by 2^-22; a sum of R weights R 2^-24, each step's addition 2^-23.  Queries, keys and lse are the layer's own."""
import math

import numpy as np
import pytest
import torch

from oracle import qcf_oracle as orc
from paper_2604_08585_amd import inputs, pipeline
from gpu_util import DEV, to_np
from test_gpu_decode8 import _held

pytestmark = pytest.mark.gpu

SHAPE = inputs.LayerShape(256, 4, 2, 64, 10000.0, "f32")


def _layer(batch, **kw):
    wl = inputs.make_config(4, orc.PlantOps(), scale=1 / 16, batch=batch, shape=SHAPE)
    L = pipeline.upload(wl, DEV)
    pipeline.fuse_layer(L)
    return L, pipeline.paged_layer(L, **kw)


def _rows(rng, n):
    return torch.from_numpy(rng.standard_normal((n, SHAPE.d_model)).astype(np.float32)).to(DEV)


class Mirror:
    """The weights of accepted rows in 64 bits, and how far the layer's may be off, relative."""

    def __init__(self, P, lens):
        self.w = [np.zeros((2, n)) for n in lens]
        self.rel = 0.0

    def take(self, P, b, rows):
        """Request b accepts the first `rows` rows of the step that was run last."""
        n = self.w[b].shape[1]
        k, _ = _held(P, b, n + P.new)
        q, lse = to_np(P.q)[b], to_np(P.lse)[b]
        w = np.concatenate([self.w[b], np.zeros((2, rows))], axis=1)
        largest = 0.0
        for i in range(rows):
            for h in range(4):
                z = k[h // 2][:n + i + 1] @ q[i, h] / 8.0
                w[h // 2][:n + i + 1] += np.exp(z - lse[i, h])
                largest = max(largest, (np.abs(k[h // 2]) @ np.abs(q[i, h])).max() / 8.0)
        x = 2 * largest + math.log(n + rows)                       # |z - lse| at most
        self.rel = max(self.rel, 69 * 2.0 ** -24 * largest + 2.0 ** -23 * (1 + x) + 2.0 ** -22)
        self.w[b] = w

    def check(self, P, steps):
        got = P.weights.double().cpu().numpy()
        for b, w in enumerate(self.w):
            n = w.shape[1]
            assert P.held[b].item() == n
            off = np.abs(got[b, :, :n] - w)
            assert np.all(off <= (self.rel + 2 * P.new * 2.0 ** -24 + steps * 2.0 ** -23) * w), (b, (off / np.maximum(w, 1e-30)).max())


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("batch,new,accepted", [
    (3, 3, [[3, 0, 1], [2, 3, 1], [0, 1, 3]]), (2, 4, [2, [0, 3], 4, 0, 1]), (2, 1, [1, 0, 1, [0, 1]]), (4, 2, [[2, 1, 0, 2], 1, [2, 2, 2, 2]])])
def test_rejected_drafts_and_repeated_steps_leave_no_weight(batch, new, accepted, eight):
    L, P = _layer(batch, more=new * len(accepted), new=new, eight=eight, budget=40)
    rng = np.random.default_rng(73)
    m = Mirror(P, L.ctx_lens)
    for step, taken in enumerate(accepted):
        for _ in range(1 + step % 2):                              # (every other step is run twice, with other drafts)
            pipeline.decode_step(P, _rows(rng, batch * new), L.w_qkv)
        torch.cuda.synchronize()
        for b in range(batch):
            m.take(P, b, taken if isinstance(taken, int) else taken[b])
        pipeline.advance(P, taken)
        print("step", step, "of", new, "rows, taken", taken, "8 bits" if eight else "", flush=True)
        m.check(P, step + 1)
    # what stays is chosen by the weights of accepted rows
    was, held = P.weights.cpu().numpy(), P.held.tolist()
    pipeline.evict(P, 1, 4)
    torch.cuda.synchronize()
    for b in range(batch):
        want = orc.page_evict(was[b], held[b], 40, 1, 4)
        assert np.array_equal(P.kept[b].cpu().numpy(), want)
        m.w[b] = np.take_along_axis(m.w[b], want[:, :min(held[b], 40)], axis=1)
    m.check(P, len(accepted))
    # and goes on behind the eviction
    pipeline.decode_step(P, _rows(rng, batch * new), L.w_qkv)
    torch.cuda.synchronize()
    for b in range(batch):
        m.take(P, b, new)
    pipeline.advance(P, new)
    m.check(P, len(accepted) + 1)


def test_a_step_that_is_not_taken_yet_shows_in_the_weights_and_leaves_them():
    """Between a step and `advance` the weights hold all of its rows; what `advance` does not take is gone, bit for bit."""
    L, P = _layer(2, more=9, new=3, budget=40)
    rng = np.random.default_rng(74)
    pipeline.decode_step(P, _rows(rng, 6), L.w_qkv)
    pipeline.advance(P, 3)
    before = P.weights
    held = P.held[0].item()
    pipeline.decode_step(P, _rows(rng, 6), L.w_qkv)
    inside = P.weights
    assert (inside[0, :, :held].double().sum() - before[0, :, :held].double().sum()).item() > 0.5
    assert (inside[0, :, :held + 3].double().sum(1) - 12.0).abs().max().item() < 1e-3          # (6 rows so far, two heads each)
    pipeline.advance(P, 0)
    assert torch.equal(P.weights, before)
    pipeline.advance(P, 0)
    assert torch.equal(P.weights, before)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,inside", [(1, True), (3, True), (3, False)])
def test_captured_steps_weigh_what_is_taken(new, inside, eight):
    """A step and its `advance` in one graph, or the step alone and what is taken told between replays: the bits of eager steps."""
    rng = np.random.default_rng(75)
    rows = [_rows(rng, 2 * new) for _ in range(5)]
    taken = [new, new, new, new, new] if inside else [2, [3, 0], 0, [1, 2], 3]

    def after(P):
        n = P.held.tolist()
        return [P.weights[b, :, :n[b]] for b in range(2)]

    L, P = _layer(2, more=5 * new, new=new, eight=eight, budget=40)
    want = []
    for x, t in zip(rows, taken):
        pipeline.decode_step(P, x, L.w_qkv)
        pipeline.advance(P, t)
        want.append(after(P))
    L, P = _layer(2, more=5 * new + new, new=new, eight=eight, budget=40)
    x = rows[0].clone()
    pipeline.decode_step(P, x, L.w_qkv)                            # (a first step outside, which is not taken)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pipeline.decode_step(P, x, L.w_qkv)
        if inside:
            pipeline.advance(P, new)
    for i, t in enumerate(taken):
        x.copy_(rows[i])
        graph.replay()
        if not inside:
            pipeline.advance(P, t)
        torch.cuda.synchronize()
        got = after(P)
        for b in range(2):
            assert torch.equal(got[b], want[i][b]), (i, b)
