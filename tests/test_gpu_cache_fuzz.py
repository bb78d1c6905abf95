"""Seeded random caches, queries, masks and lists: selection equal to the model's, attention within the bound that it claims."""
import numpy as np
import pytest
import torch

from cache_bounds import HALF_FP32, tight
from cache_util import PAGE, Pair, bf16, ints
from paper_2505_21036_b200 import api

pytestmark = pytest.mark.gpu


def case(rng):
    while True:
        D, B, H, G = (int(rng.choice(x)) for x in ((64, 96, 128), (1, 1, 2, 3, 5), (1, 1, 2, 3, 7), (1, 1, 2, 5)))
        M = int(rng.choice([1, 1, 2, 5, 17, 60, 128, 129, 200, 257, 300, 513]))
        lens = [int(rng.choice([0, 1, 5, 127, 128, 129, 300, 500, 900, 1300])) for _ in range(B)]
        if B * H * G * M * max(lens) <= 3e6:
            return D, B, H, G, M, lens


def some_lists(p, lens, H, n_q, rng):
    sched = api.CacheSchedule.empty(p.dev, H, PAGE * n_q, p.dev.max_pages)
    sched.pages.fill_(-5)
    lists = [[[sorted(rng.choice(max(-(-L // PAGE), 1), int(rng.integers(0, -(-L // PAGE) + 1)), replace=False).tolist()) for _ in range(n_q)]
              for _ in range(H)] for L in lens]
    for b, heads in enumerate(lists):
        for h, tiles in enumerate(heads):
            for t, x in enumerate(tiles):
                sched.count[b, h, t] = len(x)
                sched.pages[b, h, t, :len(x)] = ints(x)
    return sched, lists


@pytest.mark.parametrize("seed", range(60))
def test_random_case(seed):
    rng = np.random.default_rng(9000 + seed)
    D, B, H, G, M, lens = case(rng)
    p = Pair(B, H, D, sum(-(-n // PAGE) for n in lens) + 8, max(1, max(-(-n // PAGE) for n in lens)))
    left, spread_of_v = list(lens), int(rng.choice([0, 8, 28]))
    while any(left):                                        # V's pages up to 2^56 apart
        n = [min(x, int(rng.choice([128, 128, 256, 77]))) for x in left]
        x = [rng.standard_normal((B, H, max(n), D)) for _ in range(2)]
        p.append(x[0] * 2.0 ** int(rng.integers(-3, 2)), x[1] * 2.0 ** int(rng.integers(-spread_of_v, spread_of_v + 1)), n)
        left = [a - b for a, b in zip(left, n)]
    q = bf16(rng.standard_normal((B, H * G, M, D)) * rng.choice([0.1, 1, 6, 40]))
    q_len = [int(rng.choice([M, M, 0, rng.integers(0, M + 1)])) for _ in range(B)]
    causal, origin = int(rng.choice([0, 0, 1, 50, 128, 513])), [int(rng.choice([0, rng.integers(-600, 1400)])) for _ in range(B)]
    p.model.origin, n_q, sched, lists = list(origin), -(-G * M // PAGE), None, None
    how = rng.choice(["all", "own", "selected"])
    if how == "own":
        sched, lists = some_lists(p, lens, H, n_q, rng)
    elif how == "selected":
        keep = [int(x) for x in rng.integers(0, 3, 3)]
        sched = api.CacheSchedule.empty(p.dev, H * G, M, max(1, min(p.dev.max_pages, sum(keep))))
        api.rf_cache_select(p.dev, q.cuda(), sched, ints(q_len), causal, *keep, p.status, ints(origin))
        lists = p.model.select(q.double().numpy(), q_len, causal, *keep)
        for b in range(B):
            for h in range(H):
                for t in range(n_q):
                    assert sched.pages[b, h, t].tolist()[:int(sched.count[b, h, t])] == lists[b][h][t]
    o, lse = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full(q.shape[:3], 12345.0, device="cuda")
    api.rf_cache_attn_fwd(p.dev, q.cuda(), o, lse, sched, ints(q_len), causal, None, None, p.status, ints(origin))
    got, got_lse = o.float().cpu().double().numpy(), lse.cpu().double().numpy()
    ref, ref_lse, spread, reach, wide = p.model.attend(q.double().numpy(), q_len, causal, None, lists)
    assert int(p.status.item()) == 0
    p.mem.check()
    for b in range(B):
        n = lens[b]
        assert np.isnan(got[b, :, q_len[b]:]).all() and (got_lse[b, :, q_len[b]:] == 12345.0).all()
        for h in range(H * G):
            at = (b, h, slice(0, q_len[b]))
            largest = np.abs(p.model.tokens("v", b, h // G)).max(initial=0.0)
            assert (np.abs(got[at] - ref[at]) <= tight(ref[at], spread[at], reach[at], wide[at], n, D, largest) + 1e-37).all(), (b, h)
            empty = np.isneginf(ref_lse[at])
            finite = np.where(empty, 0.0, ref_lse[at])
            assert np.array_equal(np.isneginf(got_lse[at]), empty)
            e_s = (D + 8) * HALF_FP32 * reach[at] + 2.0 ** -21 * wide[at] + 2.0 ** -21      # as in cache_util.check_attention
            assert (np.abs(np.where(empty, 0.0, got_lse[at]) - finite) <= e_s + (n + 16) * HALF_FP32 + 4 * HALF_FP32 * np.abs(finite)).all(), (b, h)
