"""The bounds of pages that a verified batch of trees writes."""

import numpy as np
import pytest
import torch

from paper_2606_09061_amd import cache
from test_gpu_cache_model import CFG, _check_bounds, _model, _prompts, _start

pytestmark = pytest.mark.gpu


def test_verify_takes_the_bounds_of_a_layer_once(monkeypatch):
    """Behind the moves: the attention to the trees reads none."""
    rng = np.random.default_rng(5)
    prompts = _prompts(rng, [75, 30])
    m = _model(2, page_bounds=True)
    _start(m, prompts)
    calls, real = [], cache.page_bounds
    monkeypatch.setattr(cache, "page_bounds", lambda *a: calls.append(a[1]) or real(*a))
    rows = [(0, 75, 9, 84), (1, 30, 20, 50)]
    tokens = torch.from_numpy(rng.integers(0, CFG.vocab, 29).astype(np.int32)).to(m.dev)
    parents = torch.tensor([-1, 0, 0, 1, 2, 2, 5, 5, 7, -1, *range(19)], dtype=torch.int32,
                           device=m.dev)
    m.verify(rows, tokens, parents)
    assert [k.data_ptr() for k in calls] == [k.data_ptr() for k in m.kc]
    _check_bounds(m, rows)
    m.forward([(0, 77, 1, 78)], budget=4)
    assert len(calls) == 2 * CFG.layers
    _check_bounds(m, [(0, 0, 0, 78)])
