"""V's pages in a chunk's units: what a row does not attend to must not take bits from what it does."""
import numpy as np
import pytest

from cache_util import PAGE, Pair, ints
from paper_2505_21036_b200 import api

pytestmark = pytest.mark.gpu


def pages_of(exponents, D, seed, heads=1):
    """A sequence whose page i holds values of V of about 2^exponents[i]."""
    p = Pair(1, heads, D, len(exponents) + 2, len(exponents) + 1)
    rng = np.random.default_rng(seed)
    for e in exponents:
        p.append(rng.standard_normal((1, heads, PAGE, D)), rng.standard_normal((1, heads, PAGE, D)) * 2.0 ** e, [PAGE])
    return p, rng


def schedule(p, M, lists):
    sched = api.CacheSchedule.empty(p.dev, 1, M, max(len(x) for x in lists))
    for t, x in enumerate(lists):
        sched.count[0, 0, t] = len(x)
        sched.pages[0, 0, t, :len(x)] = ints(x)
    return sched, [[lists]]


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("gap", [16, 20, 26, 40, 90, 180])
@pytest.mark.parametrize("order", [0, 1])
def test_neighbouring_tiles_with_pages_of_their_own(D, gap, order):
    """Two tiles of query rows that list no page in common, one of them pages 2^gap smaller: each to the bits of its own."""
    e = [gap // 2 if (i + order) % 2 else -(gap - gap // 2) for i in range(6)]
    p, rng = pages_of(e, D, gap)
    sched, lists = schedule(p, 2 * PAGE, [[0, 2, 4], [1, 3, 5]])
    p.attend(rng.standard_normal((1, 1, 2 * PAGE, D)), sched=sched, lists=lists)


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("e", [(30, 0, 1, 0), (50, 25, 0, 0), (0, 70, 0, 70), (-90, 90, 90, 90), (45, -15, -15, -15), (40, -10, 40, -10)])
@pytest.mark.parametrize("causal", [0, PAGE])
def test_small_pages_that_hold_all_of_the_weight(D, e, causal):
    """Queries that find their keys in the small pages alone: the large ones' weights are zero to 2^-120 and less."""
    rng, small = np.random.default_rng(abs(sum(e)) + D), min(e)
    q = rng.standard_normal((1, 1, 4 * PAGE, D)) * 0.01
    mine = [i for i, x in enumerate(e) if x == small]
    # column 0 of K: 1 in the small pages' tokens, -1 in the others'
    p = Pair(1, 1, D, len(e) + 2, len(e) + 1)
    for i, x in enumerate(e):
        k = rng.standard_normal((1, 1, PAGE, D)) * 0.1
        k[..., 0] = 1.0 if i in mine else -1.0
        p.append(k, rng.standard_normal((1, 1, PAGE, D)) * 2.0 ** x, [PAGE])
    q[..., 0] = 200.0
    if causal:      # rows that see no small page attend to large ones, which is fine as well
        q = q[:, :, -2 * PAGE:]
    p.attend(q, causal=causal, scale=1.0)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_end_before_a_large_page(D):
    """Frame by frame: the first rows see small pages alone, the large ones lie behind."""
    p, rng = pages_of([-80, -80, 95, 95], D, 7)
    p.attend(rng.standard_normal((1, 1, 4 * PAGE, D)), causal=PAGE)
    for e, heads in (([-20] * 40 + [60] * 2, 20), ([-80, -80, 95, 95], 90)):       # in many pieces, which are joined; some items a CTA
        p, rng = pages_of(e, D, 8, heads)
        p.attend(rng.standard_normal((1, heads, 4 * PAGE, D)), causal=PAGE)
