"""What the cache's binding refuses before it calls the library, on host tensors."""
import pytest
import torch

from paper_2505_21036_b200 import api


def test_numbers_that_do_not_fit_32_bits():
    """Cut to 32 bits, 2**32 would be no mask at all and 2**32 + 5 pages five."""
    c = api.KVCache.empty(1, 1, 64, 4, 4, "cpu")
    q = torch.zeros((1, 1, 3, 64), dtype=torch.bfloat16)
    o, sched = torch.empty_like(q), api.CacheSchedule.empty(c, 1, 3, 4)
    for bad in (2 ** 32, 2 ** 32 + 5, 2 ** 31, -2 ** 31 - 1):
        with pytest.raises(api.RainFusionError, match="causal_block"):
            api.rf_cache_attn_fwd(c, q, o, causal_block=bad)
        with pytest.raises(api.RainFusionError, match="causal_block"):
            api.rf_cache_select(c, q, sched, causal_block=bad, top_k=1)
        for name in ("keep_first", "keep_last", "top_k"):
            with pytest.raises(api.RainFusionError, match=name):
                api.rf_cache_select(c, q, sched, **{name: bad})
        with pytest.raises(api.RainFusionError, match="M = "):
            api.alloc_cache_attn_workspace(c, 1, bad)
    assert c.query(q, 2 ** 31 - 1, None)


def test_a_scale_that_changes_in_place():
    """The query's sizes are kept from call to call by their values, not by the object that held them."""
    c = api.KVCache.empty(1, 1, 64, 4, 4, "cpu")
    q = torch.zeros((1, 1, 3, 64), dtype=torch.bfloat16)
    scale, block = torch.tensor(0.25), torch.tensor(7)
    first = c.query(q, block, scale)[1]._obj
    assert (first.scale, first.causal_block) == (0.25, 7)
    scale.fill_(0.5)
    block.fill_(9)
    now = c.query(q, block, scale)[1]._obj
    assert (now.scale, now.causal_block) == (0.5, 9)
    assert c.query(q, 9, 0.5)[1]._obj is now and c.query(q, 9, None)[1]._obj.scale == 0.0
    for bad in (7.5, "7"):
        with pytest.raises(TypeError):
            c.query(q, bad, None)


def test_a_workspace_with_gaps():
    """Its bytes would be counted without the gaps and written with them."""
    c = api.KVCache.empty(1, 1, 64, 4, 4, "cpu")
    q = torch.zeros((1, 1, 3, 64), dtype=torch.bfloat16)
    whole = api.alloc_cache_attn_workspace(c, 1, 3)
    with pytest.raises(api.RainFusionError, match="contiguous"):
        api.rf_cache_attn_fwd(c, q, torch.empty_like(q), ws=torch.empty(2 * whole.numel(), dtype=torch.uint8)[::2])
