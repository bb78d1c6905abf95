"""One attention layer's call sequence, as the sampler of a video DiT would drive it.

Policy only: which entry points of the C ABI run at which denoising step, with which buffers.  Every
arithmetic step is a kernel of the library.

  * the first `dense_fraction` of the sampling steps run dense attention (Sec. 4.2 keeps the first tenth of
    the timesteps dense);
  * every later step runs ARM -> tile schedule -> pattern-masked attention (Fig. 2a: the head categories are
    determined online, per call);
  * with `graph=True` the three calls of a sparse step are captured once into a CUDA graph per set of
    tensor addresses and replayed: the kernels take no host decision between them (head_class stays on
    the device), so a replay is the same work with one launch from the host.
"""
from __future__ import annotations

import math
import warnings

from . import api


class RainFusionAttention:
    def __init__(self, shape: api.rf_shape, params: api.rf_params, device, dense_fraction: float = 0.1,
                 graph: bool = False, bandwidths=None):
        import torch
        if not (0.0 <= dense_fraction <= 1.0):
            raise ValueError("dense_fraction must be in [0, 1]")
        self.shape, self.params, self.device = shape, params, device
        self.dense_fraction = dense_fraction
        self.use_graph = graph
        self.bandwidths = list(bandwidths) if bandwidths else None      # RainFusion+ (Sec. 4.3) when given
        self.ws = api.alloc_workspace(shape, params, device)
        self.sched = api.Schedule(shape, params, device)
        self.head_class = torch.zeros((shape.B, shape.H), dtype=torch.int32, device=device)
        self.head_window = (torch.zeros((shape.B, shape.H), dtype=torch.int32, device=device)
                            if self.bandwidths else None)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self._graphs = {}

    # ------------------------------------------------------------------ policy
    def dense_steps(self, num_steps: int) -> int:
        """Number of leading sampling steps that stay dense."""
        return int(math.ceil(self.dense_fraction * num_steps - 1e-9))

    def is_dense_step(self, step: int, num_steps: int) -> bool:
        return step < self.dense_steps(num_steps)

    # ------------------------------------------------------------------ calls
    def _sparse(self, q, k, v, o, lse):
        api.rf_sparse_call(self.shape, self.params, self.bandwidths, q, k, v, self.head_class, self.head_window, self.sched, o,
                           lse, self.ws, self.status)

    def _sparse_graphed(self, q, k, v, o, lse):
        import torch
        key = (q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), None if lse is None else lse.data_ptr())
        g = self._graphs.get(key)
        if g is None:
            # one eager call first: per-device kernel attributes are set on first use, outside any capture
            self._sparse(q, k, v, o, lse)
            torch.cuda.current_stream().synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                self._sparse(q, k, v, o, lse)
            self._graphs[key] = g
        g.replay()

    def __call__(self, q, k, v, o, lse=None, step: int = 0, num_steps: int = 1):
        """Attention of one layer at sampling step `step` of `num_steps`; writes o (and lse)."""
        if self.is_dense_step(step, num_steps):
            api.rf_dense_attn_fwd(self.shape, q, k, v, o, lse, self.status)
        elif self.use_graph:
            self._sparse_graphed(q, k, v, o, lse)
        else:
            self._sparse(q, k, v, o, lse)

    def check(self):
        """Raises if a kernel reported an error since the last check (reads the device status word)."""
        code = int(self.status.item())
        if code != 0:
            self.status.zero_()
            raise api.RainFusionError(f"device status {code}: {api.load().rf_status_string(code).decode()}")

    def expected_attention_speedup(self, num_steps: int, density: float) -> float:
        """Whole-run attention speed-up if a sparse step costs `density` of a dense one (Sec. 4.2's arithmetic)."""
        d = self.dense_steps(num_steps)
        return num_steps / (d + (num_steps - d) * density)


class StreamingAttention:
    """One attention layer of a clip that is generated chunk by chunk: K and V of the finished chunks stay in a paged 8-bit cache, and at
    every denoising step the chunk's queries attend to them and to the chunk itself.  Policy only, as above.

      layer.begin_chunk()
      for step in range(num_steps):
          layer(q, k, v, o, step=step, num_steps=num_steps)    # the step's K and V replace the last step's in the cache
      # the last step's stay; further operations, between chunks or between steps: fork, drop, compact

    What the cache holds when the layer is made belongs to finished chunks.

    The first `dense_fraction` of the steps attend to every page; with `top_k` set, the others attend to the pages that are selected
    for every 128 query rows (the first `keep_first` and last `keep_last` always: prompt and first frame, the chunk itself and its
    neighbours).  Everything that varies between steps is on the device, so a step can be captured into a graph.

    With `causal_block` a row attends to its own block of that many tokens and to what lies before it.  Frames want `prompt_tokens` too: how many
    tokens stand in front of a sequence's first frame (a number, or int32 [n_seqs]; 0 where there is no prompt).  The blocks are then the
    clip's frames, counted from the end of the prompt: fork and drop carry their borders along, and begin_chunk can set a new one.  Without it
    they are blocks of positions in the cache as it is now, counted from its first token, whatever has been dropped before it."""

    def __init__(self, cache: api.KVCache, heads: int, chunk_tokens: int, causal_block: int = 0, top_k=None, keep_first: int = 0,
                 keep_last: int = 0, dense_fraction: float = 0.1, prompt_tokens=None):
        import torch
        if not (0.0 <= dense_fraction <= 1.0):
            raise ValueError("dense_fraction must be in [0, 1]")
        self.cache, self.heads, self.chunk_tokens, self.causal_block = cache, heads, chunk_tokens, causal_block
        self.top_k, self.keep_first, self.keep_last, self.dense_fraction = top_k, keep_first, keep_last, dense_fraction
        self.base = cache.seq_len.clone()              # tokens of finished chunks: where the chunk begins
        # where the frames begin for the chunk that begins at base, and where they do in a sequence that starts anew (fork's -1)
        self.origin = self.first_origin = None
        if prompt_tokens is not None:
            if causal_block <= 0:
                raise ValueError("prompt_tokens says where causal blocks begin: causal_block is wanted too")
            self.first_origin = torch.as_tensor(prompt_tokens, dtype=torch.int32, device=cache.device).expand(cache.n_seqs).contiguous()
            self.origin = self.first_origin.clone()
            self.gone = torch.zeros_like(self.origin)  # tokens from base on that drop took out since the last step
        self.status = torch.zeros(1, dtype=torch.int32, device=cache.device)
        self.live = torch.zeros(1, dtype=torch.int32, device=cache.device)
        self.ws = api.alloc_cache_attn_workspace(cache, heads, chunk_tokens)
        self.sched = (None if top_k is None else
                      api.CacheSchedule.empty(cache, heads, chunk_tokens, max(1, min(cache.max_pages, keep_first + keep_last + top_k))))

    def is_dense_step(self, step: int, num_steps: int) -> bool:
        return self.top_k is None or step < int(math.ceil(self.dense_fraction * num_steps - 1e-9))

    def begin_chunk(self, new_frame: bool = False):
        """What the cache holds now belongs to finished chunks.  new_frame: the chunk begins a frame, also where the last one ended short."""
        if new_frame and self.origin is None:
            raise ValueError("frames are counted where prompt_tokens is given")
        self.base.copy_(self.cache.seq_len)
        if new_frame:
            self.origin.copy_(self.base)
        elif self.origin is not None:
            self._move_origin(self.gone)
        if self.origin is not None:
            self.gone.zero_()

    def _move_origin(self, n):
        """Borders move n[b] positions down, with the tokens behind them.  One that is no longer there stands for those whole frames behind it."""
        moved = self.origin - n
        self.origin.copy_(moved.where(moved >= 0, moved.remainder(self.causal_block)))

    def __call__(self, q, k, v, o, lse=None, new_len=None, step: int = 0, num_steps: int = 1):
        """q, o [n_seqs, heads, chunk_tokens, D], k, v [n_seqs, cache.heads, chunk_tokens, D]; new_len: int32 [n_seqs] on the device, tokens
        that each sequence's chunk really has (None: chunk_tokens)."""
        api.rf_cache_drop(self.cache, max_len=self.base, dev_status=self.status)
        api.rf_cache_append(self.cache, k, v, new_len, self.status)
        if self.origin is not None:
            self.gone.zero_()                          # the chunk is whole again
        sched = None
        if not self.is_dense_step(step, num_steps):
            sched = self.sched
            api.rf_cache_select(self.cache, q, sched, new_len, self.causal_block, self.keep_first, self.keep_last, self.top_k, self.status,
                                self.origin)
        api.rf_cache_attn_fwd(self.cache, q, o, lse, sched, new_len, self.causal_block, None, self.ws, self.status, self.origin)

    def fork(self, parent):
        """Every sequence b continues sequence parent[b] (int32 on the device; -1: it ends), its unfinished chunk included."""
        before = self.cache.seq_len.clone()
        api.rf_cache_fork(self.cache, parent, self.status)
        # a call that the library refuses changes nothing here either
        valid = ((parent >= -1) & (parent < self.cache.n_seqs) & (before >= 0) & (before <= self.cache.max_pages * api.CACHE_PAGE)).all()
        source = parent.clamp(0, self.cache.n_seqs - 1).long()
        for x, empty in ((self.base, 0),) if self.origin is None else ((self.base, 0), (self.gone, 0), (self.origin, self.first_origin)):
            x.copy_(x.where(~valid, x[source].where(parent >= 0, empty)))

    def drop(self, first, count):
        """Sequence b lets go of its pages [first[b], first[b] + count[b]): a window that slides."""
        if self.causal_block > 0 and self.origin is None and api.CACHE_PAGE % self.causal_block != 0:
            warnings.warn("StreamingAttention: causal blocks of cache positions are no frames behind dropped pages; give prompt_tokens (0 without a prompt)",
                          stacklevel=2)
        before = self.cache.seq_len.long()
        api.rf_cache_drop(self.cache, first, count, None, self.status)
        gone = before - self.cache.seq_len                         # tokens [start, start + gone); none if the library refused
        start = first.long() * api.CACHE_PAGE
        finished = ((start + gone).minimum(self.base) - start).clamp(min=0).int()
        self.base -= finished
        if self.origin is not None:
            self._move_origin(finished)
            self.gone += gone.int() - finished                     # the chunk's own: back with the next step, or finished with begin_chunk

    def compact(self):
        """Pages in use move to the front of the pool; returns how many there are (on the device)."""
        api.rf_cache_compact(self.cache, self.live, self.status)
        return self.live

    def check(self):
        """Raises if a kernel reported an error since the last check (reads the device status word)."""
        code = int(self.status.item())
        if code != 0:
            self.status.zero_()
            raise api.RainFusionError(f"device status {code}: {api.load().rf_status_string(code).decode()}")


class HostStagedAttention:
    """The whole path for callers whose Q, K, V and O live in (pinned) host memory: a thin wrapper over the
    library's rf_host_pipeline_* calls, which pipeline groups of heads over a copy-in stream, two alternating compute
    streams and a copy-out stream (heads are independent at every stage: Algorithm 1 classifies per head; masks and attention are per
    head).  Per call every byte of Q, K, V still crosses to the device and every byte of O comes back; only the
    waiting is overlapped, inside a call and between calls made back to back."""

    def __init__(self, shape: api.rf_shape, params: api.rf_params, device, groups: int = 4):
        heads = shape.B * shape.H
        if groups < 1 or heads % groups != 0:
            raise ValueError("groups must divide B*H")
        self.shape, self.params, self.device, self.groups = shape, params, device, groups
        self.N = shape.T * shape.frame_h * shape.frame_w + shape.L_text
        self.pipe = api.HostPipeline(shape, params, device, groups)
        self.h2d_bytes = 3 * heads * self.N * shape.D * 2
        self.d2h_bytes = heads * self.N * shape.D * 2

    def __call__(self, qh, kh, vh, oh):
        """qh, kh, vh, oh: pinned host bf16 tensors of [B, H, N, D]; the inputs must be complete in host memory
        when the call is made.  Returns when the work is enqueued; the current stream waits for the output copy."""
        for t in (qh, kh, vh, oh):
            if t.is_cuda or not t.is_contiguous():
                raise ValueError("host-staged call takes contiguous host tensors")
        self.pipe.run(qh, kh, vh, oh)

    @property
    def status(self):
        """Object with .item(): the pipeline's device status word."""
        pipe = self.pipe

        class _S:
            def item(self_inner):
                return pipe.status()
        return _S()
