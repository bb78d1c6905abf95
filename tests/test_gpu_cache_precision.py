"""The attention kernels within the bound that they claim: weights to 11 bits, V exact."""
import numpy as np
import pytest
import torch

from cache_bounds import tight
from cache_util import PAGE, Pair, bf16
from paper_2505_21036_b200 import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("M,G", [(1, 1), (8, 1), (3, 5), (17, 1), (100, 2), (256, 1)])
@pytest.mark.parametrize("keys", [2, 3, 6, 40, 129, 300])
def test_o(D, M, G, keys):
    """Values of both signs and of all of e4m3's bits, so that weights that were rounded further would show where o is small beside them."""
    rng = np.random.default_rng(D + M + keys)
    p = Pair(2, 2, D, 12, 4)
    for lo in range(0, keys, PAGE):                            # a page at a time, V's scales 2^14 apart at most
        n = min(PAGE, keys - lo)
        v = np.sign(rng.standard_normal((2, 2, n, D))) * rng.choice([1.0, 1.125, 1.25, 1.375, 1.5, 1.625, 1.75, 1.875], (2, 2, n, D))
        p.append(rng.standard_normal((2, 2, n, D)), v * 2.0 ** (0, 7, -7)[lo // PAGE], [n, n])
    qb = bf16(rng.standard_normal((2, 2 * G, M, D)) * 1.5)
    o = torch.full(qb.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    api.rf_cache_attn_fwd(p.dev, qb.cuda(), o, dev_status=p.status)
    got = o.float().cpu().double().numpy()
    ref, _, spread, reach, wide = p.model.attend(qb.double().numpy(), [M, M])
    largest = max(np.abs(p.model.tokens("v", b, h)).max() for b in range(2) for h in range(2))
    ratio = np.abs(got - ref) / tight(ref, spread, reach, wide, keys, D, largest)
    assert int(p.status.item()) == 0 and ratio.max() <= 1.0, float(ratio.max())
