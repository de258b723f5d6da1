"""Host side of a layer's decoding steps (pipeline.paged_layer, decode_step, advance): what they count and what they refuse."""
import types

import pytest
import torch

from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd import pipeline
from paper_2604_08585_amd.inputs import LayerShape

DESC = qb.make_desc(LayerShape(d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, rope_base=10000.0, dtype="f32"))


def _layer(B, new, room, held=None):
    """The host's side of a PagedLayer, on the CPU."""
    held = torch.tensor(held or [10 * (b + 1) for b in range(B)], dtype=torch.int32)
    step = torch.arange(new, dtype=torch.int32)
    return types.SimpleNamespace(desc=DESC, B=B, new=new, room=[room] * B, held=held, seen=held[:, None] + 1 + step,
                                 pos=(held[:, None] + step).flatten(), qkv=torch.zeros(B * new, 512))


def _state(P):
    return P.held.tolist(), P.seen.tolist(), P.pos.tolist()


def test_a_step_beyond_the_room_is_refused():
    P = _layer(2, 3, 7)
    x, w = torch.zeros(6, 256), torch.zeros(512, 256)
    for taken in (3, 2):
        with pytest.raises((qb.QcfError, AttributeError)):       # (room for it: goes on to the projection, which wants a GPU)
            pipeline.decode_step(P, x, w)
        pipeline.advance(P, taken)
    assert P.room == [2, 2]
    with pytest.raises(ValueError, match="room for 2"):
        pipeline.decode_step(P, x, w)


@pytest.mark.parametrize("tokens", [-1, 4, 3])
def test_advance_refuses_what_no_step_appended_and_what_has_no_room(tokens):
    P = _layer(2, 3, 3 if tokens == 4 else 2)
    before = _state(P)
    with pytest.raises(ValueError, match="in a step"):
        pipeline.advance(P, tokens)
    assert _state(P) == before and P.room == [3 if tokens == 4 else 2] * 2


def test_advance_moves_lengths_and_positions():
    P = _layer(2, 3, 9)
    pipeline.advance(P, 2)
    pipeline.advance(P, 0)
    assert P.room == [7, 7] and _state(P) == _state(_layer(2, 3, 9, held=[12, 22]))


@pytest.mark.parametrize("kind", [list, tuple, lambda t: torch.tensor(t), lambda t: torch.tensor(t, dtype=torch.int32).numpy()])
def test_requests_accept_different_numbers(kind):
    for B, new, taken in [(3, 3, [3, 0, 2]), (2, 3, [1, 3]), (1, 4, [2])]:        # (as many requests as rows, and not)
        P = _layer(B, new, 9)
        pipeline.advance(P, kind(taken))
        assert P.room == [9 - t for t in taken]
        assert _state(P) == _state(_layer(B, new, 9, held=[10 * (b + 1) + t for b, t in enumerate(taken)]))


@pytest.mark.parametrize("taken,word", [([1, 2], "2 numbers"), ([1, 2, 3, 0], "4 numbers"), ([1, 4, 0], "4 tokens more"), ([1, -1, 0], "-1 tokens more"),
                                        ([0, 3, 2], "room for 2")])
def test_numbers_that_do_not_fit_change_nothing(taken, word):
    P = _layer(3, 3, 2)
    before = _state(P)
    with pytest.raises(ValueError, match=word):
        pipeline.advance(P, taken)
    with pytest.raises(TypeError):
        pipeline.advance(P, [0.5, 1, 1])
    assert _state(P) == before and P.room == [2, 2, 2]


def test_the_request_with_the_least_room_stops_a_step():
    P = _layer(2, 2, 4)
    pipeline.advance(P, [1, 2])
    pipeline.advance(P, [0, 1])
    assert P.room == [3, 1]
    with pytest.raises(ValueError, match="room for 1 more behind request 1"):
        pipeline.decode_step(P, torch.zeros(4, 256), torch.zeros(512, 256))


@pytest.mark.parametrize("kw", [dict(more=-1), dict(more=4, new=17), dict(more=4, new=-1), dict(more=4, keep=1), dict(more=4, keep=-3),
                                dict(more=4, keep=8, first=-1), dict(more=4, keep=8, first=4, last=5)])
def test_layers_whose_steps_would_fail_are_refused_before_anything_is_appended(kw):
    with pytest.raises(ValueError, match="room for|pages kept"):
        pipeline.paged_layer(None, **kw)
