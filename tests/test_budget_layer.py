"""Host side of a layer with a budget (pipeline.paged_layer, evict): what it refuses."""
import types

import pytest
import torch

from paper_2604_08585_amd import pipeline


@pytest.mark.parametrize("kw", [dict(budget=-1), dict(budget=8, keep=4)])
def test_budgets_that_no_layer_takes(kw):
    with pytest.raises(ValueError, match="budget"):
        pipeline.paged_layer(None, more=4, **kw)


@pytest.mark.parametrize("budget,first,last,word", [(0, 1, 1, "budget="), (8, -1, 0, "8 in all"), (8, 5, 4, "8 in all")])
def test_evictions_that_no_layer_takes(budget, first, last, word):
    P = types.SimpleNamespace(budget=budget, held=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match=word):
        pipeline.evict(P, first, last)
