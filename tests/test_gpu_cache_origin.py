"""Causal blocks that begin where the caller says: prompts in front of the frames, borders that a slide has moved."""
import pytest
import torch

from cache_util import bf16, check_attention, filled, ints
from paper_2505_21036_b200 import api

pytestmark = pytest.mark.gpu
LENS = [0, 1, 300, 640, 1000, 513]
ORIGINS = [[0] * 6, [5, 1, 77, 639, 1000, -13], [-1, 0, 300, 641, -2 ** 31, 2 ** 31 - 1], [-50, 100, 301, -7777, 128, 500]]


def attend(p, q, q_len, causal, origin, sched=None, lists=None):
    p.model.origin = list(origin)
    qb = bf16(q)
    o, l = torch.full(qb.shape, float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full(qb.shape[:3], 12345.0, device="cuda")
    api.rf_cache_attn_fwd(p.dev, qb.cuda(), o, l, sched, ints(q_len), causal, None, None, p.status, ints(origin))
    assert int(p.status.item()) == 0
    check_attention(o, l, *p.model.attend(qb.double().numpy(), q_len, causal, None, lists), p.model, q_len, str(origin))


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("M,G", [(1, 1), (3, 2), (1, 12), (5, 3), (17, 1), (200, 1), (150, 2), (300, 1)])
@pytest.mark.parametrize("causal", [1, 50, 513])
def test_attention(D, M, G, causal):
    p, rng = filled(6, 2, D, LENS, seed=D + M)
    for origin in ORIGINS:
        attend(p, rng.standard_normal((6, 2 * G, M, D)), [M, 1, M, M // 2, M, M], causal, origin)


@pytest.mark.parametrize("M,G", [(1, 1), (150, 1), (70, 3), (300, 1)])
def test_selection(M, G):
    p, rng = filled(6, 2, 64, LENS, seed=M)
    for causal in (1, 100):
        for origin in ORIGINS:
            q, q_len = bf16(rng.standard_normal((6, 2 * G, M, 64))), [M, 1, M, M // 2, M, M]
            sched = api.CacheSchedule.empty(p.dev, 2 * G, M, 5)
            api.rf_cache_select(p.dev, q.cuda(), sched, ints(q_len), causal, 1, 1, 3, p.status, ints(origin))
            p.model.origin = list(origin)
            lists = p.model.select(q.double().numpy(), q_len, causal, 1, 1, 3)
            for b in range(6):
                for g in range(2):
                    for t, x in enumerate(lists[b][g]):
                        assert sched.pages[b, g, t].tolist()[:int(sched.count[b, g, t])] == x, (causal, origin, b, g, t)
            attend(p, q.float().numpy(), q_len, causal, origin, sched, lists)


def test_frames_behind_a_prompt():
    """7 frames of 513 tokens behind a prompt of 77: every row of the last two sees its own frame to its end and nothing of the next."""
    prompt, S, frames = 77, 513, 7
    L = prompt + frames * S
    c = api.KVCache.empty(1, 1, 64, 40, 40, "cuda")
    k = torch.zeros((1, 1, L, 64), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    frame = (torch.arange(L, device="cuda") - prompt).div(S, rounding_mode="floor") + 1        # 0: the prompt
    v[0, 0, torch.arange(L, device="cuda"), frame] = 1.0                                       # V says which frame a token is of
    api.rf_cache_append(c, k, v)
    M = 2 * S
    q = torch.zeros((1, 1, M, 64), dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    api.rf_cache_attn_fwd(c, q, o, causal_block=S, block_origin=ints([prompt]))
    mine = frame[L - M:]
    seen = torch.bincount(frame, minlength=64).float() * (torch.arange(64, device="cuda")[None] <= mine[:, None])
    want = seen / seen.sum(1, keepdim=True)
    assert (o[0, 0].float() - want).abs().max() < 2.0 ** -8      # alike weights: o is rounded to bf16, and the frames' counts are exact
    # an unaligned or foreign origin is refused
    with pytest.raises(api.RainFusionError):
        api.rf_cache_attn_fwd(c, q, o, causal_block=S, block_origin=torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(api.RainFusionError):
        api.rf_cache_select(c, q, api.CacheSchedule.empty(c, 1, M, 1), top_k=1, block_origin=ints([0, 0]))
