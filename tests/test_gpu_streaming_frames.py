"""layer.StreamingAttention frame by frame: what a row may see is told by the frame that each token was made for, not by its place in the cache."""
import warnings

import numpy as np
import pytest
import torch

from cache_util import PAGE, bf16, check_attention, ints
from oracle import cache_oracle as co
from paper_2505_21036_b200 import api, layer

pytestmark = pytest.mark.gpu


class Clip(co.Cache):
    """The cache's model with the frame of every token (-1: the prompt).  at[b]: the clip's token, counted from the prompt's end, that the
    chunk begins with; made[b]: tokens of the chunk."""

    def __init__(self, prompts, S, *sizes):
        super().__init__(len(prompts), *sizes)
        self.S, self.prompts = S, prompts
        self.frame = [[] for _ in prompts]
        self.at, self.made, self.base = [-p for p in prompts], [0] * self.B, [0] * self.B

    def sees(self, b, q_len, causal):
        f = self.frame[b]
        assert len(f) == self.len[b] and f == sorted(f)
        return [sum(x <= mine for x in f) for mine in f[len(f) - q_len:]]

    def begin(self, new_frame):
        for b in range(self.B):
            self.at[b] += self.made[b]
            if new_frame:
                self.at[b] = max(0, -(-self.at[b] // self.S) * self.S)
        self.made, self.base = [0] * self.B, list(self.len)

    def step(self, k, v, n):
        self.drop(max_len=self.base)
        self.append(k, v, n)
        for b in range(self.B):
            self.frame[b] = self.frame[b][:self.base[b]] + [max(-1, (self.at[b] + i) // self.S) for i in range(n[b])]
        self.made = list(n)

    def slide(self, first, count):
        kept = [[not f <= t // PAGE < f + n for t in range(L)] for f, n, L in zip(first, count, self.len)]
        self.frame = [[x for x, keep in zip(f, k) if keep] for f, k in zip(self.frame, kept)]
        self.base = [sum(k[:n]) for k, n in zip(kept, self.base)]
        self.drop(first, count)

    def branch(self, parent):
        self.fork(parent)
        pick = lambda x, empty: [x[p] if p >= 0 else empty(b) for b, p in enumerate(parent)]      # noqa: E731
        self.frame = [list(f) for f in pick(self.frame, lambda b: [])]
        self.at, self.made, self.base = pick(self.at, lambda b: -self.prompts[b]), pick(self.made, lambda b: 0), pick(self.base, lambda b: 0)


def run(seed, D, heads, top_k, graph, S=50, M=150, prompts=(77, 0, 30), chunks=6):
    rng, B = np.random.default_rng(seed), len(prompts)
    cache, clip = api.KVCache.empty(B, 1, D, 60, 14, "cuda"), Clip(list(prompts), S, 1, D, 60, 14)
    net = layer.StreamingAttention(cache, heads, M, causal_block=S, top_k=top_k, keep_first=1, keep_last=2, dense_fraction=0.5,
                                   prompt_tokens=prompts[0] if len(set(prompts)) == 1 else ints(prompts))
    q, k, v = (torch.zeros((B, h, M, D), dtype=torch.bfloat16, device="cuda") for h in (heads, 1, 1))
    o, new, replay, seen = torch.zeros_like(q), ints([M] * B), None, set()

    def operation():
        what = rng.choice(["fork", "slide", "compact", "nothing"])
        if what == "fork":
            parent = [int(x) for x in rng.integers(-1 if rng.random() < 0.3 else 0, B, B)]
            net.fork(ints(parent))
            clip.branch(parent)
        elif what == "slide":
            first, count = ([int(x) for x in rng.integers(0, 4, B)] for _ in range(2))
            net.drop(ints(first), ints(count))
            clip.slide(first, count)
        elif what == "compact":
            assert int(net.compact().item()) == clip.compact()
        net.check()
        assert cache.seq_len.tolist() == clip.len and net.base.tolist() == clip.base, what

    for chunk in range(chunks):
        fresh = bool(chunk and rng.random() < 0.4)
        net.begin_chunk(fresh)
        clip.begin(fresh)
        n = [min(M, int(rng.choice([M, M, S, S + 3, rng.integers(0, M + 1)]))) if L + M <= 14 * PAGE else 0 for L in clip.len]
        new.copy_(ints(n))
        for step in range(2):
            qb, kb, vb = (bf16(rng.standard_normal(t.shape)) for t in (q, k, v))
            q.copy_(qb); k.copy_(kb); v.copy_(vb)
            o.fill_(float("nan"))
            if graph and step == 1:
                if replay is None:
                    net(q, k, v, o, None, new, 1, 2)
                    torch.cuda.synchronize()
                    replay = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(replay):
                        net(q, k, v, o, None, new, 1, 2)
                o.fill_(float("nan"))
                replay.replay()
            else:
                net(q, k, v, o, None, new, step, 2)
            net.check()
            clip.step(kb.double().numpy(), vb.double().numpy(), n)
            lists = None if net.is_dense_step(step, 2) else clip.select(qb.double().numpy(), n, S, 1, 2, top_k)
            check_attention(o, None, *clip.attend(qb.double().numpy(), n, S, None, lists), clip, n, f"chunk {chunk} step {step}")
            # what the test is there for: rows whose frame ends at no multiple of S
            seen |= {x % S for b in range(B) for x in clip.sees(b, n[b], S) if x < clip.len[b]}
            if rng.random() < 0.4:
                operation()
        operation()
    return seen


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("top_k,graph", [(None, False), (2, False), (2, True)])
def test_histories(seed, top_k, graph):
    seen = run(seed, 64, 2, top_k, graph)
    assert seen - {0}


@pytest.mark.parametrize("seed", range(3))
def test_tokens(seed):
    """Three tokens a chunk, the few-rows kernel."""
    run(100 + seed, 128, 2, None, False, S=5, M=3, prompts=(4, 4), chunks=14)


def test_arguments():
    cache = api.KVCache.empty(2, 1, 64, 8, 4, "cuda")
    with pytest.raises(ValueError):
        layer.StreamingAttention(cache, 1, 50, prompt_tokens=3)                       # no blocks to begin anywhere
    with pytest.raises(ValueError):
        layer.StreamingAttention(cache, 1, 50, causal_block=50).begin_chunk(True)
    with pytest.raises(RuntimeError):
        layer.StreamingAttention(cache, 1, 50, causal_block=50, prompt_tokens=[1, 2, 3])
    none = ints([0, 0])
    with pytest.warns(UserWarning, match="prompt_tokens"):
        layer.StreamingAttention(cache, 1, 50, causal_block=50).drop(none, none)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        layer.StreamingAttention(cache, 1, 50, causal_block=64).drop(none, none)      # pages are whole blocks
        layer.StreamingAttention(cache, 1, 50).drop(none, none)
        layer.StreamingAttention(cache, 1, 50, causal_block=50, prompt_tokens=0).drop(none, none)
