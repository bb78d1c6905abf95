"""Chunks over the cache whose two tiles of query rows list very different numbers of pages, many short items to a CTA."""
import numpy as np
import pytest
import torch

from cache_util import PAGE, filled, ints
from paper_2505_21036_b200 import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("most", [(1, 1), (0, 1), (1, 3)])
def test_streams_with_no_tile_or_one(D, most):
    """450 items, three a CTA: one stream's first scores are another item's before the other stream has looked at its own."""
    heads, M = 450, 2 * PAGE
    p, rng = filled(1, heads, D, [300], seed=D)
    sched = api.CacheSchedule.empty(p.dev, heads, M, 3)
    sched.pages.fill_(-5)
    lists = [[[sorted(rng.choice(3, int(rng.integers(0, m + 1)), replace=False).tolist()) for m in most] for _ in range(heads)]]
    for h in range(heads):
        for t, x in enumerate(lists[0][h]):
            sched.count[0, h, t] = len(x)
            sched.pages[0, h, t, :len(x)] = ints(x)
    p.attend(rng.standard_normal((1, heads, M, D)), sched=sched, lists=lists)


@pytest.mark.parametrize("D", [64, 96, 128])
def test_streams_that_see_nothing(D):
    """Causal chunks longer than what the cache holds: the first tile of every item sees no key, the second a few."""
    p, rng = filled(3, 160, D, [90, 0, 5], seed=D)
    p.attend(rng.standard_normal((3, 160, 2 * PAGE, D)), [2 * PAGE, 2 * PAGE, PAGE + 3], 1)
