"""More items than a CTA has threads, tables wider than eight tiles' scores, padding that is no number."""
import numpy as np
import pytest
import torch

from cache_util import Pair, bf16, filled, ints
from paper_2505_21036_b200 import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("M,G", [(1, 1), (3, 3), (20, 1), (129, 1)])
@pytest.mark.parametrize("causal", [0, 3])
def test_more_items_than_threads(D, M, G, causal):
    """1500 K/V heads of sequences, some of them empty: three and more items to a thread that adds up the line."""
    lens = [0, 5, 0, 130, 1]
    p, rng = filled(5, 300, D, lens, seed=D)
    p.attend(rng.standard_normal((5, 300 * G, M, D)), [M, min(M, 2), 0, M, M], causal)


def test_a_thousand_sequences():
    lens = [(i * 37) % 140 for i in range(1024)]
    p, rng = filled(1024, 1, 64, lens, seed=1)
    p.attend(rng.standard_normal((1024, 2, 1, 64)), [i % 2 for i in range(1024)], 1)
    p.attend(rng.standard_normal((1024, 1, 18, 64)), [i % 19 for i in range(1024)], 7)


@pytest.mark.parametrize("M,G", [(300, 1), (70, 5), (1, 1)])
@pytest.mark.parametrize("max_pages", [2048, 2049, 9000, 16384])
def test_selection_in_wide_tables(M, G, max_pages):
    """One tile a CTA where the scores of eight do not fit."""
    rng = np.random.default_rng(M)
    p = Pair(2, 1, 64, 40, max_pages)
    p.append(rng.standard_normal((2, 1, 2500, 64)), rng.standard_normal((2, 1, 2500, 64)), [2500, 700])
    q = bf16(rng.standard_normal((2, G, M, 64)) + rng.standard_normal((2, G, 1, 64)))
    for causal, keep in ((0, (1, 1, 4)), (100, (0, 2, 7)), (1, (0, 0, 1))):
        sched = api.CacheSchedule.empty(p.dev, G, M, sum(keep))
        sched.pages.fill_(-9)
        api.rf_cache_select(p.dev, q.cuda(), sched, ints([M, M]), causal, *keep, p.status)
        lists = p.model.select(q.double().numpy(), [M, M], causal, *keep)
        for b in range(2):
            for t, x in enumerate(lists[b][0]):
                assert sched.pages[b, 0, t].tolist() == x + [-9] * (sum(keep) - len(x)) and int(sched.count[b, 0, t]) == len(x)
        p.attend(q.float().numpy(), [M, M], causal, sched=sched, lists=lists)


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("M,G", [(4, 2), (100, 1), (90, 3), (300, 1)])
def test_padding_that_is_no_number(D, M, G):
    """What rows behind q_len hold does not matter, to the lists and to the other rows, bit for bit."""
    p, rng = filled(2, 2, D, [900, 260], seed=M)
    q_len = [M - 3, M // 2]
    q = bf16(rng.standard_normal((2, 2 * G, M, D)))
    got = []
    for value in (0.0, float("nan"), float("inf"), -3.3e38):
        x = q.clone()
        for b in range(2):
            x[b, :, q_len[b]:] = value
        sched = api.CacheSchedule.empty(p.dev, 2 * G, M, 4)
        api.rf_cache_select(p.dev, x.cuda(), sched, ints(q_len), 50, 1, 1, 2, p.status)
        o, lse = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), torch.full(q.shape[:3], 7.0, device="cuda")
        api.rf_cache_attn_fwd(p.dev, x.cuda(), o, lse, sched, ints(q_len), 50, dev_status=p.status)
        o2 = torch.full_like(o, 7.0)
        api.rf_cache_attn_fwd(p.dev, x.cuda(), o2, None, None, ints(q_len), 50, dev_status=p.status)
        got.append((sched.count, sched.pages, o, lse, o2))
    assert int(p.status.item()) == 0 and all(torch.equal(a, b) for g in got[1:] for a, b in zip(got[0], g))
    for b in range(2):
        assert (got[0][2][b, :, q_len[b]:] == 7.0).all() and not torch.isnan(got[0][2][b, :, :q_len[b]].float()).any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("M", [3, 140])
def test_a_page_that_one_row_names_often(D, M):
    """The same page in several columns of one row: the same keys several times."""
    p, rng = filled(1, 1, D, [640], seed=D)
    row = [p.model.rows[0][i] for i in (0, 1, 0, 0, 4)]
    p.model.rows[0] = row
    p.dev.page_table[0, :5] = ints(row)
    p.attend(rng.standard_normal((1, 2, M, D)))
    p.attend(rng.standard_normal((1, 2, M, D)), causal=70)
