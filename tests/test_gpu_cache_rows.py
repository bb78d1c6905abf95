"""Rows of a chunk that see no key, or none of a tile's."""
import numpy as np
import pytest
import torch

from cache_util import PAGE, bf16, check_attention
from paper_2505_21036_b200 import api
from test_gpu_cache_units import pages_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("M", [1, 16, 128, 300])
def test_rows_without_keys_whose_query_is_no_number(D, M):
    """Zeros and -inf, whatever the query holds: rows before the first key, and rows whose listed pages lie behind what they see."""
    for value in (float("nan"), float("inf")):
        p, rng = pages_of([0, 0], D, M)
        p.drop(max_len=[130])
        q = bf16(rng.standard_normal((1, 2, M, D)))
        rows = []
        n_q = -(-2 * M // PAGE)
        for causal, sched in ((1, None), (1, "last")):
            q_len = [M]
            lists = None
            if sched:
                sched = api.CacheSchedule.empty(p.dev, 2, M, 1)
                sched.count.fill_(1)
                sched.pages.fill_(1)
                lists = [[[[1]] * n_q]]
            clean = q.double().numpy()
            ref, ref_lse, spread, reach, wide = p.model.attend(clean, q_len, causal, None, lists)
            empty = np.isneginf(ref_lse)
            bad = q.clone()
            bad[torch.from_numpy(empty)] = value
            o, lse = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full(q.shape[:3], 12345.0, device="cuda")
            api.rf_cache_attn_fwd(p.dev, bad.cuda(), o, lse, sched, None, causal, None, None, p.status)
            check_attention(o, lse, ref, ref_lse, spread, reach, wide, p.model, q_len, f"{value} {causal}")
            rows.append(int(empty.sum()))
        assert M == 1 or sum(rows) > 0
