"""layer.StreamingAttention: a clip in chunks as a sampler drives it, against the cache's CPU model."""
import numpy as np
import pytest
import torch

from cache_util import PAGE, bf16, check_attention, ints
from oracle import cache_oracle as co
from paper_2505_21036_b200 import api, layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top_k,graph", [(None, False), (2, False), (2, True)])
def test_chunks_branches_and_a_sliding_window(top_k, graph):
    B, H, G, D, S, frames = 2, 2, 2, 64, 50, 3
    M, steps = frames * S, 4
    cache = api.KVCache.empty(B, H, D, 24, 10, "cuda")
    model = co.Cache(B, H, D, 24, 10)
    net = layer.StreamingAttention(cache, H * G, M, causal_block=S, top_k=top_k, keep_first=1, keep_last=2, dense_fraction=0.25)
    assert [net.is_dense_step(i, steps) for i in range(steps)] == ([True] * 4 if top_k is None else [True, False, False, False])
    rng = np.random.default_rng(5)
    q, k, v = (torch.zeros((B, n, M, D), dtype=torch.bfloat16, device="cuda") for n in (H * G, H, H))
    o, lse, new = torch.zeros_like(q), torch.zeros((B, H * G, M), device="cuda"), ints([M, M])
    replay = None
    for chunk in range(4):
        net.begin_chunk()
        base = list(model.len)
        n = [M, M - 7 * chunk]
        new.copy_(ints(n))
        for step in range(steps):
            qb, kb, vb = (bf16(rng.standard_normal(t.shape)) for t in (q, k, v))
            q.copy_(qb); k.copy_(kb); v.copy_(vb)
            o.fill_(float("nan")); lse.fill_(12345.0)
            if graph and not net.is_dense_step(step, steps):
                if replay is None:
                    net(q, k, v, o, lse, new, step, steps)      # attributes are set on first use, outside any capture
                    torch.cuda.synchronize()
                    replay = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(replay):
                        net(q, k, v, o, lse, new, step, steps)
                o.fill_(float("nan")); lse.fill_(12345.0)
                replay.replay()
            else:
                net(q, k, v, o, lse, new, step, steps)
            net.check()
            model.drop(max_len=base)
            model.append(kb.double().numpy(), vb.double().numpy(), n)
            lists = None if net.is_dense_step(step, steps) else model.select(qb.double().numpy(), n, S, 1, 2, top_k)
            check_attention(o, lse, *model.attend(qb.double().numpy(), n, S, None, lists), model, n, f"chunk {chunk} step {step}")
        if chunk == 1:
            net.fork(ints([1, 1]))
            model.fork([1, 1])
        if chunk == 2:
            net.drop(ints([1, 0]), ints([2, 1]))
            model.drop([1, 0], [2, 1])
            assert int(net.compact().item()) == model.compact()
    assert cache.seq_len.tolist() == model.len
    assert [cache.page_table[b, :len(r)].tolist() for b, r in enumerate(model.rows)] == model.rows


def test_errors_are_raised():
    cache = api.KVCache.empty(1, 1, 64, 2, 4, "cuda")
    net = layer.StreamingAttention(cache, 1, 300)
    x = torch.zeros((1, 1, 300, 64), dtype=torch.bfloat16, device="cuda")
    net.begin_chunk()
    net(x, x, x, torch.empty_like(x))
    with pytest.raises(api.RainFusionError, match="room"):
        net.check()
    net.check()
    with pytest.raises(ValueError):
        layer.StreamingAttention(cache, 1, 300, dense_fraction=1.5)
