"""The tight bound tells weights of fp16 from weights of bf16: mistakes are planted in a model, not in a kernel."""
import numpy as np
import pytest
import torch

from cache_bounds import tight
from oracle import cache_oracle as co


@pytest.mark.parametrize("keys", [2, 3, 6])
@pytest.mark.parametrize("kind,fits", [("fp16", True), ("bf16", False), ("v", False)])
def test_what_fits(keys, kind, fits):
    rng = np.random.default_rng(keys)
    D, M = 64, 200
    c = co.Cache(1, 1, D, 1, 1)
    c.append(rng.standard_normal((1, 1, keys, D)), np.sign(rng.standard_normal((1, 1, keys, D))) * rng.choice([1.0, 1.125, 1.875], (1, 1, keys, D)), [keys])
    q = torch.from_numpy(rng.standard_normal((1, 1, M, D))).to(torch.bfloat16).double().numpy()
    ref, _, spread, reach, wide = c.attend(q, [M])
    k, v = c.tokens("k", 0, 0), c.tokens("v", 0, 0)
    s = q[0, 0] @ k.T / 8.0
    w = torch.from_numpy(np.exp(s - s.max(1, keepdims=True)) * 2.0 ** 7)
    w = w.to(torch.bfloat16 if kind == "bf16" else torch.float16).double().numpy()
    if kind == "v":                                  # one bit less of V
        v = np.where(np.abs(v) == 1.125, np.sign(v), v)
    o = torch.from_numpy((w @ v) / w.sum(1, keepdims=True)).to(torch.bfloat16).double().numpy()
    bound = tight(ref, spread, reach, wide, keys, D, np.abs(v).max())[0, 0]
    assert bool((np.abs(o - ref[0, 0]) <= bound).all()) == fits
