"""The paged 8-bit K/V cache on the GPU against its CPU model: exact for what is stored, within derived bounds for the attention."""
import numpy as np
import pytest
import torch

from cache_util import PAGE, Pair, bf16, filled, ints
from oracle import cache_oracle as co
from paper_2505_21036_b200 import api

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ append and page operations
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("H", [1, 3])
def test_append_in_pieces(D, H):
    rng = np.random.default_rng(D + H)
    p = Pair(4, H, D, 24, 6)
    for i, n in enumerate([[1, 0, 127, 128], [1, 1, 1, 1], [0, 255, 129, 0], [300, 0, 0, 2], [0, 0, 0, 0], [5, 384, 7, 9]]):
        M = max(max(n), 1)
        amp = 10.0 ** rng.uniform(-4, 3)          # scales grow and stay
        p.append(rng.standard_normal((4, H, M, D)) * amp, rng.standard_normal((4, H, M, D)) / amp, n)
        p.check(f"append {i}")
    p.append(rng.standard_normal((4, H, 3, D)), rng.standard_normal((4, H, 3, D)), [3] * 4, whole=True)
    p.check("every sequence")


@pytest.mark.parametrize("seed", range(8))
def test_random_histories(seed):
    """Appends, forks, drops and compactions in any order: the whole state after every call."""
    rng = np.random.default_rng(100 + seed)
    B, H, D = int(rng.integers(1, 6)), int(rng.choice([1, 2, 5])), int(rng.choice([64, 96, 128]))
    p = Pair(B, H, D, 80, 9)
    for step in range(14):
        what = rng.choice(["append", "append", "append", "fork", "drop", "cut", "compact"])
        if what == "append":
            n = [int(min(rng.choice([0, 1, 2, 100, 128, 200, 257]), 9 * PAGE - p.model.len[b])) for b in range(B)]
            M = max(max(n), 1) + int(rng.integers(0, 3))
            if sum(-(-(p.model.len[b] + n[b]) // PAGE) + 1 for b in range(B)) > 80:
                continue
            amp = 10.0 ** rng.uniform(-3, 3)
            p.append(rng.standard_normal((B, H, M, D)) * amp, rng.standard_normal((B, H, M, D)) * amp, n)
        elif what == "fork":
            p.fork([int(x) for x in rng.integers(-1, B, B)])
        elif what == "drop":
            p.drop([int(x) for x in rng.integers(0, 5, B)], [int(x) for x in rng.integers(0, 4, B)],
                   [int(x) for x in rng.integers(0, 1200, B)] if rng.random() < 0.5 else None)
        elif what == "cut":
            p.drop(max_len=[int(x) for x in rng.integers(0, 1200, B)])
        else:
            p.compact()
        p.check(f"step {step}: {what}")


def test_a_rewritten_chunk_takes_the_same_pages():
    """The chunk of a denoising step is cut off and written again: nothing else moves."""
    p, rng = filled(2, 2, 64, [300, 77], M=200)
    lens = list(p.model.len)
    for step in range(3):
        p.drop(max_len=lens)
        p.append(rng.standard_normal((2, 2, 200, 64)), rng.standard_normal((2, 2, 200, 64)), [200, 131])
        p.check(f"step {step}")
        rows = [list(r) for r in p.model.rows]
        assert step == 0 or rows == before
        before = rows


@pytest.mark.parametrize("case", ["pool", "row"])
def test_no_room_leaves_the_cache_as_it_was(case):
    p, rng = Pair(2, 1, 64, *((5, 9) if case == "pool" else (9, 4))), np.random.default_rng(4)
    p.append(rng.standard_normal((2, 1, 200, 64)), rng.standard_normal((2, 1, 200, 64)), [100, 200])
    k = bf16(rng.standard_normal((2, 1, 400, 64))).cuda()
    api.rf_cache_append(p.dev, k, k, ints([1, 400]), p.status)
    p.check(case, status=8)
    p.status.zero_()
    p.append(rng.standard_normal((2, 1, 9, 64)), rng.standard_normal((2, 1, 9, 64)), [9, 0])
    p.check("what fits still goes in")


@pytest.mark.parametrize("D", [64, 128])
def test_values_that_are_not_finite(D):
    rng = np.random.default_rng(3)
    p = Pair(1, 2, D, 4, 2)
    k, v = rng.standard_normal((1, 2, 130, D)), rng.standard_normal((1, 2, 130, D))
    k[0, 0, 5, 3], k[0, 0, 6, 4], k[0, 1, 128, 0] = np.nan, np.inf, -np.inf
    v[0, 1, 129, :] = np.inf                       # and a page whose only other token is finite
    p.append(k, v, [130])
    p.check("not finite", status=9)


def test_extreme_magnitudes():
    """Zeros, subnormal bf16 numbers, the largest ones: the exponent stays within its bounds."""
    p = Pair(1, 1, 64, 8, 8)
    for x in (0.0, 1e-40, 3.3e38, 2.0 ** -100, 2.0 ** 109, 448.0, 450.0):
        k = np.full((1, 1, 128, 64), x)
        k[..., ::2] *= -1
        if p.model.len[0] < 7 * 128:
            p.append(k, k / 3, [128])
            p.check(str(x))


def test_broken_arguments_are_reported_and_change_nothing():
    p, rng = filled(3, 1, 64, [130, 5, 260], M=100)
    k = bf16(rng.standard_normal((3, 1, 50, 64))).cuda()
    for call in (lambda: api.rf_cache_append(p.dev, k, k, ints([1, 51, 1]), p.status), lambda: api.rf_cache_append(p.dev, k, k, ints([1, -1, 1]), p.status),
                 lambda: api.rf_cache_fork(p.dev, ints([0, 3, 1]), p.status), lambda: api.rf_cache_fork(p.dev, ints([0, -2, 1]), p.status),
                 lambda: api.rf_cache_drop(p.dev, ints([0, -1, 0]), ints([0, 0, 0]), None, p.status),
                 lambda: api.rf_cache_drop(p.dev, ints([0, 1, 0]), ints([0, 0, -5]), None, p.status),
                 lambda: api.rf_cache_drop(p.dev, None, None, ints([5, 5, -5]), p.status)):
        call()
        p.check("refused", status=1)
        p.status.zero_()
    # a table that names a page which does not exist
    good = p.dev.page_table.clone()
    live = ints([5])
    for bad in (-1, p.dev.n_pages, 1 << 30):
        p.dev.page_table[0, 1] = bad
        api.rf_cache_append(p.dev, k, k, ints([1, 1, 1]), p.status)
        torch.cuda.synchronize()
        assert int(p.status.item()) == 1
        p.status.zero_()
        api.rf_cache_compact(p.dev, live, p.status)
        torch.cuda.synchronize()
        assert int(p.status.item()) == 1 and int(live.item()) == -1
        p.status.zero_()
        p.dev.page_table.copy_(good)
        p.check("as before")


@pytest.mark.parametrize("bad", [-1, 3 * 128 + 1])
def test_a_broken_length_is_reported_and_changes_nothing(bad):
    p, rng = filled(3, 1, 64, [130, 5, 260], M=100)
    k, live = bf16(rng.standard_normal((3, 1, 50, 64))).cuda(), ints([0])
    p.dev.seq_len[1] = bad
    table = p.dev.page_table.clone()
    for call in (lambda: api.rf_cache_append(p.dev, k, k, None, p.status), lambda: api.rf_cache_fork(p.dev, ints([2, 0, 1]), p.status),
                 lambda: api.rf_cache_drop(p.dev, ints([0] * 3), ints([1] * 3), ints([9] * 3), p.status),
                 lambda: api.rf_cache_compact(p.dev, live, p.status)):
        call()
        torch.cuda.synchronize()
        assert int(p.status.item()) == 1 and torch.equal(p.dev.page_table, table) and p.dev.seq_len.tolist() == [130, bad, 260]
        p.status.zero_()
    assert int(live.item()) == -1
    p.dev.seq_len[1] = 5
    p.check("as before")


def test_many_sequences_and_a_large_pool():
    rng = np.random.default_rng(5)
    p = Pair(700, 1, 64, 40000, 3)
    p.append(rng.standard_normal((700, 1, 3, 64)), rng.standard_normal((700, 1, 3, 64)), [int(x) for x in rng.integers(0, 4, 700)])
    p.fork([int(x) for x in rng.integers(-1, 700, 700)])
    p.append(rng.standard_normal((700, 1, 130, 64)), rng.standard_normal((700, 1, 130, 64)), [int(x) for x in rng.integers(0, 131, 700)])
    p.drop([int(x) for x in rng.integers(0, 2, 700)], [int(x) for x in rng.integers(0, 2, 700)])
    p.compact()
    p.check("700 sequences")


# ------------------------------------------------------------------------------------------------ attention
LENS = [0, 1, 127, 128, 129, 257, 640]


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("M,G", [(1, 1), (1, 6), (1, 16), (1, 17), (2, 3), (5, 5)])
@pytest.mark.parametrize("causal", [0, 1, 50])
def test_few_rows(D, M, G, causal):
    p, rng = filled(7, 2, D, LENS, seed=D + M)
    q = rng.standard_normal((7, 2 * G, M, D))
    p.attend(q, None if M == 1 else [M, 1, 0, M, M - 1, M, M], causal, lse=G != 3)


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("M,G", [(128, 1), (100, 2), (255, 1), (43, 3), (257, 1), (300, 2)])
@pytest.mark.parametrize("causal", [0, 1, 100])
def test_chunks(D, M, G, causal):
    lens = [0, 1, 128, 300, 1000]
    p, rng = filled(5, 2, D, lens, seed=D + M)
    q = rng.standard_normal((5, 2 * G, M, D))
    p.attend(q, [M, M // 2, 0, min(M, 300), M], causal, lse=G != 2)


@pytest.mark.parametrize("M", [1, 200])
def test_scores_of_every_size(M):
    """Maxima that jump late by many orders, weights that vanish beside them, a scale of the caller's."""
    p = Pair(1, 1, 128, 12, 12)
    rng = np.random.default_rng(7)
    for page in range(10):
        k = rng.standard_normal((1, 1, 128, 128))
        k[0, 0, 17] *= 3.0 + 2 * (page % 5)
        p.append(k, rng.standard_normal((1, 1, 128, 128)), [128])
    q = rng.standard_normal((1, 1, M, 128)) * 3
    p.attend(q, scale=0.3)
    p.attend(q, scale=1e-3)
    p.attend(q * 0, scale=1.0)


@pytest.mark.parametrize("M", [1, 256])
def test_scales_past_the_exponent_that_one_product_reaches(M):
    """Pages of very large and very small values (2^e with e above and below 7, the two-step widening)."""
    p = Pair(1, 2, 64, 6, 6)
    rng = np.random.default_rng(8)
    for e in (40, -60, 0, 8, 7):
        p.append(rng.standard_normal((1, 2, 128, 64)) * 2.0 ** -10, rng.standard_normal((1, 2, 128, 64)) * 2.0 ** e, [128])
    p.attend(rng.standard_normal((1, 2, M, 64)))
    p2 = Pair(1, 2, 64, 6, 6)
    for e in (20, 12, 10):
        p2.append(rng.standard_normal((1, 2, 128, 64)) * 2.0 ** e, rng.standard_normal((1, 2, 128, 64)), [128])
    p2.attend(rng.standard_normal((1, 2, M, 64)) * 2.0 ** -14)


@pytest.mark.parametrize("M", [1, 9, 200])
@pytest.mark.parametrize("large", [30.0, 3000.0])
def test_queries_with_one_large_element(M, large):
    """Where the keys have nothing, so that the scores come from the small ones."""
    p = Pair(1, 1, 128, 5, 5)
    rng = np.random.default_rng(12)
    k = rng.standard_normal((1, 1, 500, 128))
    k[..., 7] = 0.0
    p.append(k, rng.standard_normal((1, 1, 500, 128)), [500])
    q = rng.standard_normal((1, 1, M, 128))
    q[..., 7] = large
    p.attend(q)


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("M,causal", [(1, 0), (640, 128), (640, 1), (300, 0)])
def test_values_whose_scale_varies_from_page_to_page(D, M, causal):
    """V's pages 2^-14 to 2^16 apart: units that change under rows that see some of them only.  (Within 2^15 below the largest, where V is
    exact in any unit.)"""
    p = Pair(1, 2, D, 10, 10)
    rng = np.random.default_rng(D + M)
    for e in (0, 9, -5, 12, 1):
        p.append(rng.standard_normal((1, 2, 128, D)), rng.standard_normal((1, 2, 128, D)) * 2.0 ** e, [128])
    p.attend(rng.standard_normal((1, 4, M, D)) * 3, causal=causal)


@pytest.mark.parametrize("M", [1, 130])
def test_a_query_that_is_no_number_spoils_its_own_row_only(M):
    p, rng = filled(1, 1, 64, [300])
    q = bf16(rng.standard_normal((1, 2, M, 64)))
    good = torch.empty_like(q, device="cuda")
    api.rf_cache_attn_fwd(p.dev, q.cuda(), good)
    q[0, 1, M // 2, 5] = float("nan")
    bad = torch.empty_like(good)
    api.rf_cache_attn_fwd(p.dev, q.cuda(), bad)
    assert torch.isnan(bad[0, 1, M // 2]).all()
    bad[0, 1, M // 2] = good[0, 1, M // 2]
    assert torch.equal(bad, good)


@pytest.mark.parametrize("D,M,G", [(64, 1, 3), (128, 1, 1), (96, 130, 1), (128, 256, 2), (64, 300, 1)])
def test_schedules_of_the_callers_own(D, M, G):
    p, rng = filled(3, 2, D, [900, 1, 500])
    q = rng.standard_normal((3, 2 * G, M, D))
    n_q = -(-G * M // PAGE)
    lists = [[[sorted(rng.choice(-(-L // PAGE), int(rng.integers(0, -(-L // PAGE) + 1)), replace=False).tolist()) for _ in range(n_q)]
              for _ in range(2)] for L in (900, 1, 500)]
    lists[0][0][0] = []                                       # a tile without any page
    sched = api.CacheSchedule.empty(p.dev, 2 * G, M, 9)
    sched.pages.fill_(-5)                                     # entries behind the count are not looked at
    for b in range(3):
        for g in range(2):
            for t in range(n_q):
                x = lists[b][g][t]
                sched.count[b, g, t] = len(x)
                sched.pages[b, g, t, :len(x)] = ints(x)
    p.attend(q, None, 0, sched=sched, lists=lists)
    p.attend(q, [M, 1, M], 1, sched=sched, lists=lists)


@pytest.mark.parametrize("M", [1, 140])
def test_schedules_that_name_no_page_of_the_sequence(M):
    p, rng = filled(1, 1, 64, [300])
    q = bf16(rng.standard_normal((1, 1, M, 64))).cuda()
    n_q = -(-M // PAGE)
    for bad in (-1, 3, 1 << 30):
        sched = api.CacheSchedule.empty(p.dev, 1, M, 2)
        sched.count.fill_(2)
        sched.pages[..., 1] = bad
        o = torch.empty_like(q)
        api.rf_cache_attn_fwd(p.dev, q, o, sched=sched, dev_status=p.status)
        torch.cuda.synchronize()
        assert int(p.status.item()) == 1
        p.status.zero_()
        lists = [[[[0]] * n_q]]
        ref = p.model.attend(q.cpu().double().numpy(), [M], lists=lists)[0]
        assert np.abs(o.cpu().double().numpy() - ref).max() < 0.05           # the other page was attended to
    sched.count.fill_(99)                                                    # counts past the row are cut
    sched.pages[..., 1] = 1
    p.attend(q.cpu().float().numpy(), sched=sched, lists=[[[[0, 1]] * n_q]])


# ------------------------------------------------------------------------------------------------ selection
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("M,G,causal", [(1, 1, 0), (1, 4, 1), (150, 1, 100), (70, 3, 0), (300, 1, 1)])
@pytest.mark.parametrize("keep", [(0, 0, 3), (1, 2, 1), (2, 0, 0), (0, 1, 100)])
def test_selection(D, M, G, causal, keep):
    first, last, top = keep
    lens = [0, 100, 129, 1900]
    p, rng = filled(4, 2, D, lens, seed=D)
    q = bf16(rng.standard_normal((4, 2 * G, M, D)) + rng.standard_normal((4, 2 * G, 1, D)))
    q_len = [M, min(M, 100), M // 2, M]
    cap = min(p.dev.max_pages, first + last + top)
    sched = api.CacheSchedule.empty(p.dev, 2 * G, M, cap)
    sched.pages.fill_(-9)
    api.rf_cache_select(p.dev, q.cuda(), sched, ints(q_len), causal, first, last, top, p.status)
    lists = p.model.select(q.double().numpy(), q_len, causal, first, last, top)
    for b in range(4):
        for g in range(2):
            for t, x in enumerate(lists[b][g]):
                n = int(sched.count[b, g, t])
                assert sched.pages[b, g, t].tolist() == x + [-9] * (cap - len(x)) and n == len(x), (b, g, t, x)
    p.attend(q.float().numpy(), q_len, causal, sched=sched, lists=lists)
    p.check("selection leaves the cache alone")


def test_selection_after_a_cut():
    """Two sequences share pages, one of them is cut inside one: its score is that of the tokens it keeps."""
    p, rng = filled(2, 2, 64, [500, 0])
    p.fork([0, 0])
    p.drop(max_len=[500, 290])
    for lens in ([500, 290], [500, 257]):
        p.drop(max_len=lens)
        for seed in range(6):
            q = bf16(np.random.default_rng(seed).standard_normal((2, 2, 1, 64)))
            sched = api.CacheSchedule.empty(p.dev, 2, 1, 1)
            api.rf_cache_select(p.dev, q.cuda(), sched, top_k=1, dev_status=p.status)
            lists = p.model.select(q.double().numpy(), [1, 1], 0, 0, 0, 1)
            assert [[sched.pages[b, g, 0].tolist() for g in range(2)] for b in range(2)] == [[x[0] for x in y] for y in lists], seed


def test_selection_of_pages_that_score_alike():
    """Copies of one page: the lowest of them.  Queries of zero: the lowest pages.  Queries that are no numbers: the lowest pages."""
    rng = np.random.default_rng(9)
    p = Pair(1, 1, 64, 700, 700)
    k = np.tile(rng.standard_normal((1, 1, 128, 64)), (1, 1, 600, 1))
    p.append(k, k, [600 * 128])
    sched = api.CacheSchedule.empty(p.dev, 1, 1, 20)
    for q in (rng.standard_normal((1, 1, 1, 64)), np.zeros((1, 1, 1, 64)), np.full((1, 1, 1, 64), np.nan)):
        api.rf_cache_select(p.dev, bf16(q).cuda(), sched, keep_first=3, keep_last=2, top_k=15)
        assert sched.pages[0, 0, 0].tolist() == list(range(18)) + [598, 599]


def test_selection_over_a_long_sequence():
    """16384 pages, the most there may be; random sums, so that every score is distinct."""
    p = Pair(1, 1, 64, 16384, 16384)
    g = torch.Generator("cuda").manual_seed(1)
    p.dev.page_table.copy_(torch.randperm(16384, generator=g, device="cuda", dtype=torch.int32).view(1, -1))
    p.dev.seq_len.fill_(16384 * 128)
    p.dev.k_sum.copy_(torch.randn(p.dev.k_sum.shape, generator=g, device="cuda"))
    q = torch.randn((1, 1, 1, 64), generator=g, device="cuda").to(torch.bfloat16)
    for first, last, top in ((1, 4, 500), (0, 0, 1), (5000, 3000, 8000)):
        sched = api.CacheSchedule.empty(p.dev, 1, 1, first + last + top)
        api.rf_cache_select(p.dev, q, sched, keep_first=first, keep_last=last, top_k=top, dev_status=p.status)
        score = (p.dev.k_sum[p.dev.page_table[0].long(), 0].double() @ q[0, 0, 0].double()) / 128
        rest = torch.arange(first, 16384 - last, device="cuda")
        best = rest[score[rest].argsort(descending=True, stable=True)[:top]]
        want = torch.cat([torch.arange(first, device="cuda"), best.sort().values, torch.arange(16384 - last, 16384, device="cuda")])
        assert int(sched.count.item()) == first + last + top
        assert torch.equal(sched.pages[0, 0, 0].long(), want)
    assert int(p.status.item()) == 0


# ------------------------------------------------------------------------------------------------ as it is used
@pytest.mark.parametrize("M", [1, 160])
def test_offsets_past_32_bits(M):
    """A pool of more than 2^32 bytes, the sequence's pages at its end."""
    H, D, n_pages = 24, 128, 11200
    c = api.KVCache.empty(2, H, D, n_pages, n_pages, "cuda")
    assert c.k.numel() > 2 ** 32
    # the first sequence takes every page but the last ones; it is never read
    c.page_table[0] = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    c.seq_len[0] = (n_pages - 5) * 128
    g = torch.Generator("cuda").manual_seed(2)
    k, v = (torch.randn((2, H, 600, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.rf_cache_append(c, k, v, ints([0, 600]), status)
    q = torch.randn((2, H, M, D), generator=g, device="cuda").to(torch.bfloat16)
    o = torch.empty_like(q)
    api.rf_cache_attn_fwd(c, q, o, q_len=ints([0, M]), dev_status=status)
    assert int(status.item()) == 0 and c.page_table[1, :5].tolist() == list(range(n_pages - 5, n_pages))
    m = co.Cache(1, 2, D, 5, 5)
    m.append(k[1:, :2].double().cpu().numpy(), v[1:, :2].double().cpu().numpy(), [600])
    ref = m.attend(q[1:, :2].double().cpu().numpy(), [M])[0]
    assert np.abs(o[1:, :2].double().cpu().numpy() - ref).max() < 2e-2


def test_long_row_keeps_small_weights():
    """One key of weight 1 beside 40 000 of 2^-15: the sums are held in more bits than the weights."""
    n = 40000
    c = api.KVCache.empty(1, 1, 64, 400, 400, "cuda")
    k = torch.zeros((1, 1, n, 64), dtype=torch.bfloat16, device="cuda")
    k[..., 0] = -15 * 0.693147 * 8
    k[0, 0, 77, 0] = 0
    v = torch.zeros_like(k)
    v[..., 1] = 1.0
    v[0, 0, 77] = 0
    v[0, 0, 77, 2] = 1.0
    api.rf_cache_append(c, k, v)
    for M in (1, 256):
        q = torch.zeros((1, 1, M, 64), dtype=torch.bfloat16, device="cuda")
        q[..., 0] = 1.0
        o, lse = torch.empty_like(q), torch.empty((1, 1, M), device="cuda")
        api.rf_cache_attn_fwd(c, q, o, lse)
        s = float(c.k[0, 0, 0, 0].float() * c.k_scale[0, 0]) / 8         # the stored score of the small ones
        w = (n - 1) * np.exp(s) / (1 + (n - 1) * np.exp(s))
        assert abs(float(lse[0, 0, -1]) - np.log1p((n - 1) * np.exp(s))) < 2e-5
        assert abs(float(o[0, 0, -1, 1]) - w) <= 2 ** -8 * w * 2.1 and abs(float(o[0, 0, 0, 2]) - (1 - w)) <= 2 ** -8 * (1 - w) * 2.1


@pytest.mark.parametrize("M", [1, 200])
def test_same_bits_every_time_and_with_any_workspace(M):
    p, rng = filled(2, 3, 128, [3000, 777])
    q = bf16(rng.standard_normal((2, 6, M, 128))).cuda()
    first, l1 = torch.empty_like(q), torch.empty((2, 6, M), device="cuda")
    api.rf_cache_attn_fwd(p.dev, q, first, l1)
    for fill in (0, 255):
        o, l = torch.empty_like(q), torch.empty_like(l1)
        ws = api.alloc_cache_attn_workspace(p.dev, 6, M).fill_(fill)
        api.rf_cache_attn_fwd(p.dev, q, o, l, ws=ws)
        assert torch.equal(o, first) and torch.equal(l, l1)
    # without lse: the same outputs
    o = torch.empty_like(q)
    api.rf_cache_attn_fwd(p.dev, q, o)
    assert torch.equal(o, first)


@pytest.mark.parametrize("M", [1, 200])
def test_two_streams_at_once(M):
    pairs = [filled(1, 4, 64, [5000 + 300 * i], seed=i)[0] for i in range(2)]
    g = torch.Generator("cuda").manual_seed(3)
    q = torch.randn((1, 4, M, 64), generator=g, device="cuda").to(torch.bfloat16)
    want = [torch.empty_like(q) for _ in range(2)]
    for p, o in zip(pairs, want):
        api.rf_cache_attn_fwd(p.dev, q, o)
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[torch.empty_like(q) for _ in range(20)] for _ in range(2)]
    ws = [api.alloc_cache_attn_workspace(p.dev, 4, M) for p in pairs]
    torch.cuda.synchronize()
    for i in range(20):
        for s, p, o, w in zip(streams, pairs, got, ws):
            with torch.cuda.stream(s):
                api.rf_cache_attn_fwd(p.dev, q, o[i], ws=w)
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        assert all(torch.equal(x, w) for x in o)


@pytest.mark.parametrize("M", [1, 150])
def test_a_captured_step_replayed(M):
    """Cut, append, select, attend as one graph: the lengths and pages on the device decide, at every replay anew."""
    p, rng = filled(2, 2, 64, [1000, 300], M=8 * M, spare=20)
    k, v = (torch.zeros((2, 2, M, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((2, 2, M, 64), dtype=torch.bfloat16, device="cuda")
    o, new = torch.zeros_like(q), ints([M, M])
    sched = api.CacheSchedule.empty(p.dev, 2, M, 6)
    ws = api.alloc_cache_attn_workspace(p.dev, 2, M)

    def step():
        api.rf_cache_append(p.dev, k, v, new, p.status)
        api.rf_cache_select(p.dev, q, sched, new, 1, 1, 1, 4, p.status)
        api.rf_cache_attn_fwd(p.dev, q, o, None, sched, new, 1, None, ws, p.status)
    lens = list(p.model.len)
    step()                                             # attributes are set on first use, outside any capture
    p.drop(max_len=lens)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        kk, vv, qq = (bf16(rng.standard_normal((2, 2, M, 64))) for _ in range(3))
        n = [M, max(M - i, 1)]
        k.copy_(kk); v.copy_(vv); q.copy_(qq); new.copy_(ints(n))
        o.fill_(float("nan"))
        g.replay()
        p.model.append(kk.double().numpy(), vv.double().numpy(), n)
        p.check(f"replay {i}")
        lists = p.model.select(qq.double().numpy(), n, 1, 1, 1, 4)
        from cache_util import check_attention
        check_attention(o, None, *p.model.attend(qq.double().numpy(), n, 1, None, lists), p.model, n, f"replay {i}")


def test_a_clip_in_chunks():
    """Four frames at a time: every denoising step rewrites the chunk and attends; then branch, choose, slide, compact."""
    B, H, D, S = 3, 2, 96, 70
    p = Pair(B, H, D, 60, 12)
    rng = np.random.default_rng(11)
    for chunk in range(3):
        base = list(p.model.len)
        for step in range(2):
            p.drop(max_len=base)
            p.append(rng.standard_normal((B, H, 4 * S, D)), rng.standard_normal((B, H, 4 * S, D)), [4 * S, 3 * S, 4 * S - 1])
            p.attend(rng.standard_normal((B, H, 4 * S, D)), [4 * S, 3 * S, 4 * S - 1], S, what=f"chunk {chunk} step {step}")
        p.fork([0, 0, 2])
        p.check(f"chunk {chunk}")
    p.drop([1, 0, 0], [2, 1, 0])
    p.attend(rng.standard_normal((B, H, 5, D)), causal=1)
    p.compact()
    p.check("end")
    p.attend(rng.standard_normal((B, H, 200, D)), causal=S)


def test_the_binding_refuses():
    c = api.KVCache.empty(2, 2, 64, 4, 2, "cuda")
    q = torch.zeros((2, 2, 3, 64), dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    for bad in (q.float(), q.transpose(1, 2).contiguous().transpose(1, 2), q[:1], q.cpu(), q[..., :32].contiguous()):
        with pytest.raises(api.RainFusionError):
            api.rf_cache_append(c, bad, bad)
        with pytest.raises(api.RainFusionError):
            api.rf_cache_attn_fwd(c, bad, o)
    with pytest.raises(api.RainFusionError):
        api.rf_cache_attn_fwd(c, q, o[:, :, :2].contiguous())
    with pytest.raises(api.RainFusionError):
        api.rf_cache_attn_fwd(c, q, o, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(api.RainFusionError):
        api.rf_cache_append(c, q, q, new_len=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(api.RainFusionError):
        api.rf_cache_select(c, q, api.CacheSchedule.empty(c, 2, 3, 1), top_k=2)       # no room for the list
    with pytest.raises(api.RainFusionError):
        api.rf_cache_attn_fwd(c, torch.zeros((2, 3, 3, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 3, 3, 64), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(api.RainFusionError):
        api.rf_cache_drop(c, first=ints([0, 0]))


def test_the_most_sequences_and_pages():
    """1024 sequences, 524288 pages: every free page is handed out, then there are none, then half of them come back."""
    B, P, C = 1024, 1 << 19, 512
    c = api.KVCache.empty(B, 1, 64, P, C, "cuda")
    g = torch.Generator("cuda").manual_seed(4)
    perm = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    c.page_table[:, :511] = perm[:B * 511].view(B, 511)
    c.seq_len.fill_(511 * 128)
    c.k_sum.copy_(torch.arange(P, device="cuda")[:, None, None].expand(P, 1, 64).float())      # a page's mark
    status, live = ints([0]), ints([0])
    x = torch.ones((B, 1, 1, 64), dtype=torch.bfloat16, device="cuda")
    api.rf_cache_append(c, x, x, None, status)
    assert int(status.item()) == 0
    assert torch.equal(c.page_table[:, 511], perm[B * 511:].sort().values) and bool((c.seq_len == 511 * 128 + 1).all())
    before = c.page_table.clone()
    y = torch.ones((B, 1, 128, 64), dtype=torch.bfloat16, device="cuda")
    api.rf_cache_append(c, y, y, None, status)
    assert int(status.item()) == 8 and torch.equal(c.page_table, before) and bool((c.seq_len == 511 * 128 + 1).all())
    status.zero_()
    first, count = ints([0] * B), ints([256] * B)
    api.rf_cache_drop(c, first, count, None, status)
    assert torch.equal(c.page_table[:, :256], before[:, 256:])
    marks = c.k_sum[c.page_table[:, :256].long(), 0, 0].clone()
    api.rf_cache_compact(c, live, status)
    now = c.page_table[:, :256].long()
    assert int(live.item()) == B * 256 and int(status.item()) == 0 and torch.equal(now.flatten().sort().values, torch.arange(B * 256, device="cuda"))
    assert torch.equal(c.k_sum[now, 0, 0], marks)
    stays = before[:, 256:].long() < B * 256
    assert torch.equal(now[stays], before[:, 256:].long()[stays])


@pytest.mark.parametrize("M", [1, 130])
def test_two_calls_on_one_cache_at_once(M):
    """Readers of one cache on two streams, a workspace each, one of them with a schedule."""
    p, rng = filled(2, 2, 96, [2000, 900])
    q = [bf16(rng.standard_normal((2, 4, M, 96))).cuda() for _ in range(2)]
    sched = api.CacheSchedule.empty(p.dev, 4, M, 6)
    api.rf_cache_select(p.dev, q[1], sched, keep_last=2, top_k=4)
    want = [torch.empty_like(x) for x in q]
    for x, o, s in zip(q, want, (None, sched)):
        api.rf_cache_attn_fwd(p.dev, x, o, sched=s)
    ws, streams = [api.alloc_cache_attn_workspace(p.dev, 4, M) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    got = [[torch.empty_like(x) for _ in range(12)] for x in q]
    torch.cuda.synchronize()
    for i in range(12):
        for j in range(2):
            with torch.cuda.stream(streams[j]):
                api.rf_cache_attn_fwd(p.dev, q[j], got[j][i], sched=(None, sched)[j], ws=ws[j])
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for o, w in zip(got, want) for x in o)


@pytest.mark.parametrize("H,heads", [(1, 1), (48, 48), (40, 5), (64, 1)])
def test_head_layouts(H, heads):
    for M in (1, 3, 129):
        p, rng = filled(1, heads, 64, [400], seed=H + M)
        p.attend(rng.standard_normal((1, H, M, 64)), causal=1)
