"""layer.StreamingAttention: where its chunk begins, over a cache that is not empty and with page operations between steps."""
import numpy as np
import pytest
import torch

from cache_util import PAGE, bf16, check_attention, ints
from oracle import cache_oracle as co
from paper_2505_21036_b200 import api, layer

pytestmark = pytest.mark.gpu


class Clip:
    """The layer and the cache's model in step; base: tokens of finished chunks, counted one by one."""

    def __init__(self, lens, M, begin):
        B = len(lens)
        self.cache, self.model = api.KVCache.empty(B, 1, 64, 40, 12, "cuda"), co.Cache(B, 1, 64, 40, 12)
        self.rng, self.M, self.B = np.random.default_rng(3), M, B
        k, v = (bf16(self.rng.standard_normal((B, 1, max(lens), 64))) for _ in range(2))
        api.rf_cache_append(self.cache, k.cuda(), v.cuda(), ints(lens))
        self.model.append(k.double().numpy(), v.double().numpy(), lens)
        self.net = layer.StreamingAttention(self.cache, 1, M)
        if begin:
            self.net.begin_chunk()
        self.base = list(lens)

    def step(self, new):
        q, k, v = (bf16(self.rng.standard_normal((self.B, 1, self.M, 64))) for _ in range(3))
        o = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        self.net(q.cuda(), k.cuda(), v.cuda(), o, new_len=ints(new))
        self.net.check()
        self.model.drop(max_len=self.base)
        self.model.append(k.double().numpy(), v.double().numpy(), new)
        self.same()
        check_attention(o, None, *self.model.attend(q.double().numpy(), new), self.model, new)

    def same(self):
        assert self.cache.seq_len.tolist() == self.model.len and self.net.base.tolist() == self.base
        assert [self.cache.page_table[b, :len(r)].tolist() for b, r in enumerate(self.model.rows)] == self.model.rows

    def fork(self, parent):
        self.net.fork(ints(parent))
        self.model.fork(parent)
        self.base = [self.base[p] if p >= 0 else 0 for p in parent]
        self.same()

    def drop(self, first, count):
        self.net.drop(ints(first), ints(count))
        self.base = [sum(not f <= t // PAGE < f + n for t in range(base)) for f, n, base in zip(first, count, self.base)]
        self.model.drop(first, count)
        self.same()


@pytest.mark.parametrize("begin", [False, True])
def test_what_the_cache_held_before_stays(begin):
    clip = Clip([300, 0, 128], 150, begin)
    clip.step([150, 20, 1])
    clip.step([100, 150, 150])


def test_forks_between_steps():
    clip = Clip([300, 10, 128], 150, True)
    clip.step([150, 20, 1])
    clip.fork([1, 0, 0])                  # a child of a longer parent, of a shorter one
    clip.step([9, 150, 130])
    clip.fork([0, -1, 1])
    clip.step([150, 150, 0])
    clip.net.begin_chunk()
    clip.base = list(clip.model.len)
    clip.step([1, 2, 3])


def test_pages_dropped_between_steps():
    clip = Clip([700, 300, 128], 200, True)
    clip.step([200, 200, 200])
    clip.drop([1, 2, 0], [2, 1, 1])       # finished pages; the page that the chunk begins in; all that was finished
    clip.step([200, 200, 100])
    clip.drop([4, 0, 9], [9, 9, 9])       # from the chunk on; everything; nothing
    clip.step([200, 1, 200])


def test_what_the_library_refuses_changes_nothing():
    clip = Clip([300, 10, 128], 150, True)
    clip.step([150, 20, 1])
    for call in (lambda: clip.net.fork(ints([0, 3, 1])), lambda: clip.net.fork(ints([0, -2, 1])), lambda: clip.net.drop(ints([0, -1, 0]), ints([1, 1, 1]))):
        call()
        with pytest.raises(api.RainFusionError):
            clip.net.check()
        clip.same()
    clip.step([10, 20, 30])
