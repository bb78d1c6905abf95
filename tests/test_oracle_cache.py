"""The cache model that the GPU tests compare with, pinned on its own: rounding, scales, page bookkeeping, attention."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co


def test_rounding_is_that_of_every_e4m3_value_and_its_ties():
    codes = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(co.round_e4m3(codes), codes)
    mid = (codes[1:] + codes[:-1]) / 2
    even = np.where(np.arange(126) % 2 == 0, codes[:-1], codes[1:])
    assert np.array_equal(co.round_e4m3(mid), even)
    assert np.array_equal(co.round_e4m3(-np.nextafter(mid, 1e9)), -codes[1:])
    assert np.array_equal(co.round_e4m3([464.0, 1e9, -1e9, 0.0]), [448.0, 448.0, -448.0, 0.0])


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.5, 1), (1.75, -8), (1.76, -7), (0.0, -100), (1e38, 100), (3.5, -7), (1e-38, -100)])
def test_scale_exponent(amax, e):
    assert co.scale_exponent(amax) == e


def test_pages_are_shared_copied_dropped_and_moved():
    rng = np.random.default_rng(0)
    c = co.Cache(3, 1, 4, 8, 4)
    k, v = rng.standard_normal((3, 1, 200, 4)), rng.standard_normal((3, 1, 200, 4))
    c.append(k, v, [200, 0, 5])
    assert c.rows == [[0, 1], [], [2]] and c.len == [200, 0, 5]
    c.fork([0, 0, -1])
    assert c.rows == [[0, 1], [0, 1], []]
    before = c.tokens("k", 0, 0).copy()
    c.append(k, v, [0, 3, 0])                    # page 1 is shared and partly filled: a copy
    assert c.rows == [[0, 1], [0, 2], []] and c.len == [200, 203, 0]
    assert np.array_equal(c.tokens("k", 0, 0), before)
    c.drop([0, 0, 0], [1, 0, 0], [1 << 30, 203, 0])
    assert c.rows == [[1], [0, 2], []] and c.len == [72, 203, 0]
    c.fork([-1, 1, -1])
    assert c.compact() == 2 and c.rows == [[], [0, 1], []]
    with pytest.raises(co.CacheFull):
        c.append(np.zeros((3, 1, 1000, 4)), np.zeros((3, 1, 1000, 4)), [1000, 0, 0])


def test_attention_equals_torch_on_the_stored_tokens():
    rng = np.random.default_rng(1)
    c = co.Cache(2, 2, 8, 8, 4)
    k, v = rng.standard_normal((2, 2, 150, 8)), rng.standard_normal((2, 2, 150, 8))
    c.append(k, v, [150, 40])
    q = rng.standard_normal((2, 4, 10, 8))
    for causal in (0, 1, 7):
        o, lse, *_ = c.attend(q, [10, 10], causal)
        for b in range(2):
            L = c.len[b]
            p = torch.arange(10) + L - 10
            keep = torch.arange(L)[None, :] < (torch.full((10, 1), L) if causal == 0 else ((p // causal + 1) * causal)[:, None])
            for h in range(4):
                kk, vv = (torch.from_numpy(c.tokens(w, b, h // 2)) for w in "kv")
                s = (torch.from_numpy(q[b, h]) @ kk.T / 8 ** 0.5).masked_fill(~keep, -float("inf"))
                assert np.allclose(o[b, h], (s.softmax(1) @ vv).numpy(), atol=1e-12)
                assert np.allclose(lse[b, h], s.logsumexp(1).numpy(), atol=1e-12)


def test_selecting_every_page_is_attending_to_all_and_rows_can_be_empty():
    rng = np.random.default_rng(2)
    c = co.Cache(1, 1, 8, 8, 4)
    c.append(rng.standard_normal((1, 1, 300, 8)), rng.standard_normal((1, 1, 300, 8)), [300])
    q = rng.standard_normal((1, 1, 140, 8))
    lists = c.select(q, [140], 0, 0, 0, 3)
    assert lists == [[[[0, 1, 2], [0, 1, 2]]]]
    assert np.array_equal(c.attend(q, [140])[0], c.attend(q, [140], lists=lists)[0])
    o, lse, *_ = c.attend(q, [140], lists=[[[[], [1]]]])
    assert np.all(o[0, 0, :128] == 0) and np.all(np.isneginf(lse[0, 0, :128])) and np.all(np.isfinite(lse[0, 0, 128:]))
    # identical pages: the lower one
    c.append(np.zeros((1, 1, 84, 8)), np.zeros((1, 1, 84, 8)), [84])
    for w in (c.val["k"], c.exp["k"]):
        w[c.rows[0][1]] = w[c.rows[0][2]] = w[c.rows[0][0]]
    assert c.select(q[:, :, :1], [1], 0, 0, 0, 1) == [[[[0]]]] and c.select(-q[:, :, :1], [1], 0, 0, 0, 2) == [[[[0, 1]]]]
