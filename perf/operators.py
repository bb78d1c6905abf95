"""The operators of the paged 8-bit K/V cache whose speed this repository keeps track of.

A clip that is generated chunk by chunk keeps K and V of its finished frames in pages of 128 tokens, in e4m3 with a
power-of-two scale for each page and head.  One case is one pass through an operator, as a sampler's layer makes it:

  append   the chunk's K and V go into the cache (again at every denoising step: the last step's tokens are dropped first)
  branch   the sequences are forked, and every branch appends its own chunk (partly filled pages are copied on write)
  compact  the live pages move to the lowest places of the pool
  attend   the chunk's queries (or single tokens) attend to the whole cache
  select   pages are chosen for every 128 query rows by a pooled score, and the queries attend to those alone

With `own` false the operators are computed in plain torch operations; with `own` true by the framework.  `exact` has
them in 64 bits.  The page tables are random permutations of the pool, as after some time of service.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 128
MOST_SCORES = 1.7e9     # query rows x keys x heads of the largest listed dense case
MOST_TOKENS = 3.0e6     # tokens x heads of the largest listed cache


def _case(name, kind, H, Hkv, D, lens, M, new=None, causal=0, lse=False, keep=(0, 0), top=0, live=0.5, amp=1.0):
    """lens: tokens in the cache before the pass (attend, select: with the chunk's own), by sequence.  M: tokens a chunk's
    tensors have room for; new: tokens the chunk really has, by sequence.  Both lists as texts, to be plain values."""
    c = dict(kind=kind, H=H, Hkv=Hkv, D=D, lens=" ".join(map(str, lens)), M=M, new=" ".join(map(str, new or [M] * len(lens))),
             causal=causal, lse=lse, first=keep[0], last=keep[1], top=top, live=live, amp=amp)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token for each of eight sequences: a token-wise sampler's step, all latency
        _case("append_token", "append", 24, 24, 128, [8448, 1, 0, 127, 128, 4000, 2146, 777], 1),
        # a frame of the HunyuanVideo-720p-shaped layer behind eight frames
        _case("append_frame", "append", 24, 24, 128, [8 * 3600 + 256], 3600),
        # four branches of one CogVideoX-shaped clip, each with a chunk of its own length
        _case("branch_d64", "branch", 48, 48, 64, [4 * 1350 + 226, 3 * 1350 + 77, 1350, 0], 1350, [1350, 1001, 1, 350]),
        # upkeep of a small pool, and of one that holds a 720p-shaped clip
        _case("compact_d96", "compact", 24, 24, 96, [3600, 1777, 513], 1, live=0.4),
        _case("compact_d128", "compact", 24, 24, 128, [16 * 2040 + 256, 8448], 1, live=0.6),
        # a token against the clip of 33 frames; a ragged batch of tokens whose heads share K and V, one without any keys
        _case("token_33x3600", "attend", 24, 24, 128, [33 * 3600 + 256], 1),
        _case("token_batch_gqa", "attend", 24, 4, 128, [8448, 5337, 129, 1, 0, 2146, 128, 8000, 7777, 31, 4096, 640, 8448, 300, 65, 6001], 1, lse=True),
        # a unit-test-sized chunk; chunks of odd length that see their own frames and the earlier ones; a frame against 16
        _case("chunk_tiny_d64", "attend", 3, 3, 64, [4 * 64 + 16], 64),
        _case("chunk_ragged_d96", "attend", 24, 12, 96, [7 * 513 + 77, 3 * 513, 700], 1026, [1026, 513, 701], causal=513, lse=True),
        _case("chunk_16x2040", "attend", 24, 24, 128, [16 * 2040 + 256], 2040),
        # selected pages: tokens against long clips, a frame against 33
        _case("select_token", "select", 24, 8, 128, [33 * 3600 + 256, 16 * 2040, 8448, 50], 1, keep=(2, 4), top=58),
        _case("select_33x3600", "select", 24, 24, 128, [33 * 3600 + 256], 3600, keep=(2, 30), top=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(("append", "branch", "compact", "attend", "attend", "select"))
        D, Hkv, B = rng.choice((64, 96, 128)), rng.choice((1, 3, 4, 8, 12, 24)), rng.choice((1, 1, 2, 3, 5, 8))
        G = rng.choice((1, 1, 2, 3, 6)) if kind in ("attend", "select") else 1
        lens = [_log_int(rng, 1, 120000) - rng.choice((0, 0, 1)) for _ in range(B)]
        M = rng.choice((1, 1, 2, 7, _log_int(rng, 16, 4000), _log_int(rng, 16, 4000)))
        new = [rng.choice((M, M, rng.randint(0, M))) for _ in range(B)]
        if kind in ("attend", "select"):
            lens = [max(l, n) for l, n in zip(lens, new)]      # the chunk's own tokens are in the cache
        causal = rng.choice((0, 0, 1, _log_int(rng, 30, 4000))) if kind in ("attend", "select") else 0
        keep, top = ((rng.randint(0, 4), rng.randint(1, 8)), rng.randint(0, 64)) if kind == "select" else ((0, 0), 0)
        c = _case(None, kind, Hkv * G, Hkv, D, lens, M, new, causal, rng.random() < 0.5, keep, top, rng.uniform(0.2, 0.9))
        rows, span = Hkv * G * M * B, max(lens) if kind != "select" else min(max(lens), PAGE * (sum(keep) + top))
        if (sum(lens) + B * M) * Hkv <= MOST_TOKENS and (kind not in ("attend", "select") or rows * max(span, PAGE) <= MOST_SCORES):
            return c


# ------------------------------------------------------------------------------------------------ the cache, in plain form
def _ints(text):
    return [int(x) for x in text.split()]


def _scale(amax):
    """2^e, e the least exponent with amax <= 448 * 2^e, within [-100, 100]."""
    m, e = torch.frexp(amax)                         # amax = m * 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(amax > 0, e, torch.full_like(e, -100)).clamp(-100, 100)
    return torch.ldexp(torch.ones_like(amax), e)


def _encode(x, scale):
    """The e4m3 values of x / scale (finite x), saturating."""
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _paged(x, pages):
    """[H, n, D] as pages [pages, H, 128, D], zeros behind the last token."""
    H, n, D = x.shape
    return torch.nn.functional.pad(x, (0, 0, 0, pages * PAGE - n)).view(H, pages, PAGE, D).transpose(0, 1)


def _cache(c, gen, spare):
    """A cache of random content whose pages lie all over the pool; `spare` pages are free."""
    H, D, lens = c["Hkv"], c["D"], _ints(c["lens"])
    used = [-(-n // PAGE) for n in lens]
    room = [-(-(n + c["M"]) // PAGE) for n in lens]
    total = sum(used) + spare
    place = torch.randperm(total, generator=gen, device="cuda")
    k = torch.zeros((total, H, PAGE, D), dtype=torch.float8_e4m3fn, device="cuda")
    v = torch.zeros_like(k)
    k_scale, v_scale = (torch.ones((total, H), device="cuda") for _ in range(2))
    k_sum = torch.zeros((total, H, D), device="cuda")
    table = torch.zeros((len(lens), max(max(room), 1)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(lens):
        p = place[at:at + used[b]]
        at += used[b]
        table[b, :used[b]] = p.to(torch.int32)
        if n == 0:
            continue
        for data, scales, keys in ((k, k_scale, True), (v, v_scale, False)):
            x = torch.randn((H, n, D), generator=gen, device="cuda")
            if keys:   # tokens of one stretch of frames have something in common: what the selection is there to find
                x += c["amp"] * torch.randn((H, -(-n // 512), 1, D), generator=gen, device="cuda").expand(-1, -1, 512, -1).reshape(H, -1, D)[:, :n]
            x = _paged(x.to(torch.bfloat16).float(), used[b])
            s = _scale(x.abs().amax((2, 3)))
            codes = _encode(x, s[..., None, None])
            data.view(torch.uint8)[p] = codes.view(torch.uint8)
            scales[p] = s
            if keys:
                k_sum[p] = (codes.double().sum(2) * s[..., None].double()).float()
    return dict(k=k, v=v, k_scale=k_scale, v_scale=v_scale, k_sum=k_sum, table=table,
                lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    c = case
    gen = torch.Generator("cuda").manual_seed(seed)
    lens, new, M, B = _ints(c["lens"]), _ints(c["new"]), c["M"], len(_ints(c["lens"]))
    grow = sum(-(-(n + M) // PAGE) for n in lens)
    used = sum(-(-n // PAGE) for n in lens)
    spare = int(used / c["live"]) - used + 1 if c["kind"] == "compact" else grow - used + B if c["kind"] == "append" else grow + B
    s = dict(case=c, cache=_cache(c, gen, spare))
    s["start_table"], s["start_lens"] = s["cache"]["table"].clone(), s["cache"]["lens"].clone()
    s["new"] = torch.tensor(new, dtype=torch.int32, device="cuda")
    if c["kind"] in ("append", "branch"):
        s["k_new"], s["v_new"] = (torch.randn((B, c["Hkv"], M, c["D"]), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        # every branch but the last continues the first sequence
        s["parent"] = torch.tensor([0] * (B - 1) + [B - 1], dtype=torch.int32, device="cuda")
    elif c["kind"] == "compact":
        s["live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    else:
        q = torch.randn((B, c["H"], M, c["D"]), generator=gen, device="cuda")
        q += c["amp"] * torch.randn((B, c["H"], 1, c["D"]), generator=gen, device="cuda")
        s["q"] = q.to(torch.bfloat16)
        s["o"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros((B, c["H"], M), device="cuda")
        n_q = -(-(c["H"] // c["Hkv"]) * M // PAGE)
        if c["kind"] == "select":
            cap = max(1, min(s["cache"]["table"].shape[1], c["first"] + c["last"] + c["top"]))
            s["count"] = torch.zeros((B, c["Hkv"], n_q), dtype=torch.int32, device="cuda")
            s["pages"] = torch.zeros((B, c["Hkv"], n_q, cap), dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _columns(table):
    return torch.arange(table.shape[1], device=table.device)


def _append(s, lens, table):
    """The chunk's tokens behind `lens`: the cache's new tensors."""
    a, M, D = s["cache"], s["k_new"].shape[2], s["k_new"].shape[3]
    B, H = s["k_new"].shape[:2]
    new, col = s["new"], _columns(table)
    total = a["k"].shape[0]
    old_pages, all_pages = (lens + PAGE - 1) // PAGE, (lens + new + PAGE - 1) // PAGE
    named = torch.zeros(total, dtype=torch.int64, device=table.device)
    in_use = col[None, :] < old_pages[:, None]
    named.index_add_(0, table.long().clamp(0, total - 1).flatten(), in_use.long().flatten())
    # pages that are written: from the one that holds position lens on; fresh where there was none or others name it too
    written = (col[None, :] >= (lens // PAGE)[:, None]) & (col[None, :] < all_pages[:, None]) & (new > 0)[:, None]
    fresh = written & (~in_use | (named[table.long().clamp(0, total - 1)] > 1))
    free = torch.nonzero(named == 0).flatten()
    rank = fresh.flatten().long().cumsum(0) - 1
    table2 = torch.where(fresh, free[rank.clamp(0, max(free.numel() - 1, 0))].view(table.shape).to(torch.int32), table)
    b, c = torch.nonzero(written, as_tuple=True)
    src, dst = table[b, c].long(), table2[b, c].long()
    pos = c[:, None] * PAGE + torch.arange(PAGE, device=table.device)                  # [w, 128] positions in the sequence
    from_old = pos < lens[b][:, None]
    there = pos < (lens + new)[b][:, None]
    at = (pos - lens[b][:, None]).clamp(0, M - 1)
    out = {}
    for name, x in (("k", s["k_new"]), ("v", s["v_new"])):
        chunk = x[b[:, None], :, at].float().transpose(1, 2)                           # [w, H, 128, D]
        chunk = torch.where((there & ~from_old)[:, None, :, None], chunk, 0.0)
        kept_scale = torch.where(from_old.any(1)[:, None], a[name + "_scale"][src], 0.0)
        kept = torch.where(from_old[:, None, :, None], a[name].view(torch.uint8)[src].view(torch.float8_e4m3fn).float(), 0.0)
        scale = torch.maximum(kept_scale, _scale(chunk.abs().amax((2, 3))))
        whole = torch.where(from_old[:, None, :, None], kept * kept_scale[..., None, None], chunk)
        codes = _encode(whole, scale[..., None, None])
        stay = ~there[:, None, :, None]                                                # behind the last token: as it was
        dst_codes = torch.where(stay, a[name].view(torch.uint8)[dst], codes.view(torch.uint8))
        out[name], out[name + "_scale"] = a[name].view(torch.uint8).clone(), a[name + "_scale"].clone()
        out[name][dst] = dst_codes
        out[name] = out[name].view(torch.float8_e4m3fn)
        out[name + "_scale"][dst] = scale
        if name == "k":
            out["k_sum"] = a["k_sum"].clone()
            out["k_sum"][dst] = (torch.where(stay, 0.0, codes.double()).sum(2) * scale[..., None].double()).float()
    return dict(out, table=table2, lens=lens + new)


def _compact(s):
    a, table, lens = s["cache"], s["start_table"], s["start_lens"]
    total = a["k"].shape[0]
    in_use = _columns(table)[None, :] < ((lens + PAGE - 1) // PAGE)[:, None]
    live = torch.zeros(total, dtype=torch.bool, device=table.device)
    live[table[in_use].long()] = True
    n = live.sum()
    place = torch.arange(total, device=table.device)
    holes, movers = torch.nonzero(~live & (place < n)).flatten(), torch.nonzero(live & (place >= n)).flatten()
    to = place.clone()
    to[movers] = holes
    out = {}
    for name in ("k", "v", "k_scale", "v_scale", "k_sum"):
        x = a[name].view(torch.uint8).clone() if a[name].dtype == torch.float8_e4m3fn else a[name].clone()
        x[holes] = x[movers]
        out[name] = x.view(a[name].dtype)
    return dict(out, table=torch.where(in_use, to[table.long()].to(torch.int32), table), lens=lens, live=n.view(1).to(torch.int32))


def _visible(c, lens, new, rows):
    """Keys that each of the rows [G * M] of a K/V head sees, by sequence: [B, rows]; -1 for a row that is not there."""
    i = torch.arange(rows, device=lens.device) % c["M"]
    p = (lens - new)[:, None] + i[None, :]
    sees = lens[:, None].expand_as(p)
    if c["causal"] > 0:
        sees = torch.where(p < 0, 0, torch.minimum(sees, (torch.div(p, c["causal"], rounding_mode="floor") + 1) * c["causal"]))
    return torch.where(i[None, :] < new[:, None], sees, -1)


def _select(s, dtype):
    """(count, pages): the pages of every 128 rows of a K/V head, ascending."""
    c, a = s["case"], s["cache"]
    lens, table = a["lens"], a["table"].long()
    B, H, M, D = s["q"].shape
    Hkv, rows = c["Hkv"], H // c["Hkv"] * M
    n_q, cap = s["pages"].shape[2:]
    sees = _visible(c, lens, s["new"], rows)
    pad = n_q * PAGE - rows
    sees = torch.nn.functional.pad(sees, (0, pad), value=-1).view(B, 1, n_q, PAGE)
    q = torch.nn.functional.pad(s["q"].view(B, Hkv, rows, D), (0, 0, 0, pad)).view(B, Hkv, n_q, PAGE, D)
    pooled = torch.where((sees >= 0)[..., None], q, 0).to(dtype).sum(3)
    col = _columns(table)
    tokens = (lens[:, None] - col * PAGE).clamp(1, PAGE)                                # of each page
    sums = a["k_sum"][table].to(dtype)                                                  # [B, pages, Hkv, D]
    score = torch.einsum("bhtd,bchd->bhtc", pooled, sums) / tokens[:, None, None, :]
    n = (sees.amax(3).clamp(min=0) + PAGE - 1) // PAGE                                  # candidate pages [B, 1, n_q]
    there = col < n[..., None]
    always = there & ((col < c["first"]) | (col >= n[..., None] - c["last"]))
    rest = (there & ~always).expand_as(score)
    order = torch.where(rest, score, -math.inf).sort(dim=-1, descending=True, stable=True).indices
    best = torch.zeros_like(rest).scatter_(-1, order[..., :c["top"]], True) & rest
    chosen = best | always
    count = chosen.sum(-1)
    first = torch.where(chosen, col, table.shape[1]).sort(dim=-1).values[..., :cap]
    return count.to(torch.int32), torch.where(first < table.shape[1], first, 0).to(torch.int32)


def _gathered(a, which, pages):
    """The tokens of these physical pages [B, Hkv, ..., n] as values, [B, Hkv, ..., n * 128, D]."""
    heads = torch.arange(pages.shape[1], device=pages.device).view([1, -1] + [1] * (pages.dim() - 2))
    x = a[which].view(torch.uint8)[pages, heads].view(torch.float8_e4m3fn)
    x = x.to(a["dtype"]) * a[which + "_scale"][pages, heads].to(a["dtype"])[..., None, None]
    return x.flatten(-3, -2)


def _attend(s, dtype, selection=None):
    """(o, lse) in `dtype`, before any rounding; rows without keys are zeros and -inf.  All rows, those that are not there too."""
    c, a = s["case"], dict(s["cache"], dtype=dtype)
    B, H, M, D = s["q"].shape
    Hkv, rows = c["Hkv"], H // c["Hkv"] * M
    sees = _visible(c, a["lens"], s["new"], rows)
    q = s["q"].view(B, Hkv, rows, D).to(dtype)
    table = a["table"].long()
    if selection is None:
        pages = table[:, None, :].expand(-1, Hkv, -1)
        pos = torch.arange(table.shape[1] * PAGE, device=q.device)
        seen = pos < sees[:, None, :, None]                                             # [B, 1, rows, keys]
    else:
        count, logical = selection
        n_q, cap = logical.shape[2:]
        pad = n_q * PAGE - rows
        q = torch.nn.functional.pad(q, (0, 0, 0, pad)).view(B, Hkv, n_q, PAGE, D)
        sees = torch.nn.functional.pad(sees, (0, pad), value=-1).view(B, 1, n_q, PAGE)
        pages = table[torch.arange(B, device=q.device).view(B, 1, 1, 1), logical.long()]
        pos = (logical.long()[..., None] * PAGE + torch.arange(PAGE, device=q.device)).flatten(-2)
        listed_ = (torch.arange(cap, device=q.device) < count[..., None]).repeat_interleave(PAGE, -1)
        seen = (pos[..., None, :] < sees[..., None]) & listed_[..., None, :]
    score = q @ _gathered(a, "k", pages).transpose(-1, -2)
    score = torch.where(seen, score * (D ** -0.5), -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    score = torch.exp_(score.sub_(top))
    total = score.sum(-1)
    o = (score @ _gathered(a, "v", pages)) / torch.where(total > 0, total, 1.0)[..., None]
    lse = torch.log(total) + top[..., 0]
    if selection is not None:
        o, lse = o.flatten(2, 3)[:, :, :rows], lse.flatten(2, 3)[:, :, :rows]
    return o.reshape(B, H, M, D), lse.reshape(B, H, M)


def _present(s):
    """Which rows [B, 1, M] are there."""
    return torch.arange(s["case"]["M"], device="cuda")[None, None, :] < s["new"][:, None, None]


# ------------------------------------------------------------------------------------------------ one pass
def _handle(s):
    """The framework's view of the cache: what a program builds once, with its tensors."""
    if "handle" not in s:
        from paper_2505_21036_b200 import api
        a, c = s["cache"], s["case"]
        s["handle"] = api.KVCache(a["k"], a["v"], a["k_scale"], a["v_scale"], a["k_sum"], a["table"], a["lens"])
        if c["kind"] == "select":
            s["sched"] = api.CacheSchedule(s["count"], s["pages"])
        if c["kind"] in ("attend", "select"):
            s["ws"] = api.alloc_cache_attn_workspace(s["handle"], c["H"], c["M"])
    return s["handle"]


def _state(a, live=None):
    """The updated cache."""
    out = dict(k=a["k"], v=a["v"], k_scale=a["k_scale"], v_scale=a["v_scale"], k_sum=a["k_sum"], table=a["table"], lens=a["lens"])
    return out if live is None else dict(out, live=live)


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if own:
        from paper_2505_21036_b200 import api
        cache, a = _handle(s), s["cache"]
        if kind == "append":
            api.rf_cache_drop(cache, max_len=s["start_lens"])
            api.rf_cache_append(cache, s["k_new"], s["v_new"], s["new"])
            return _state(a)
        if kind in ("branch", "compact"):   # the pass begins from the same page table every time
            a["table"].copy_(s["start_table"])
            a["lens"].copy_(s["start_lens"])
            if kind == "branch":
                api.rf_cache_fork(cache, s["parent"])
                api.rf_cache_append(cache, s["k_new"], s["v_new"], s["new"])
                return _state(a)
            api.rf_cache_compact(cache, s["live"])
            return _state(a, s["live"])
        if kind == "select":
            api.rf_cache_select(cache, s["q"], s["sched"], q_len=s["new"], causal_block=c["causal"], keep_first=c["first"],
                                keep_last=c["last"], top_k=c["top"])
        api.rf_cache_attn_fwd(cache, s["q"], s["o"], s["lse"] if c["lse"] else None, s["sched"] if kind == "select" else None,
                              q_len=s["new"], causal_block=c["causal"], ws=s["ws"])
        out = dict(o=s["o"], lse=s["lse"]) if c["lse"] else dict(o=s["o"])
        return dict(out, count=s["count"], pages=s["pages"]) if kind == "select" else out
    if kind == "append":
        return _state(_append(s, torch.minimum(s["cache"]["lens"], s["start_lens"]), s["cache"]["table"]))
    if kind == "branch":
        parent = s["parent"].long()
        return _state(_append(s, s["start_lens"][parent], s["start_table"][parent]))
    if kind == "compact":
        new = _compact(s)
        return _state(new, new["live"])
    selection = _select(s, torch.float64) if kind == "select" else None
    o, lse = _attend(s, torch.float32, selection)
    there = _present(s)
    s["o"].copy_(torch.where(there[..., None], o, 0.0))
    s["lse"].copy_(torch.where(there, lse, 0.0))
    out = dict(o=s["o"], lse=s["lse"]) if c["lse"] else dict(o=s["o"])
    return dict(out, count=selection[0], pages=selection[1]) if kind == "select" else out


def work(case):
    """Bytes: what goes into and comes out of the operator, each once; flops: two products a pair of query row and key."""
    c, D, Hkv, G = case, case["D"], case["Hkv"], case["H"] // case["Hkv"]
    lens, new = _ints(c["lens"]), _ints(c["new"])
    side = 2 * 4 * Hkv + 4 * Hkv * D                                       # scales and key sums of a page
    if c["kind"] in ("append", "branch"):
        if c["kind"] == "branch":
            lens = [lens[0]] * (len(lens) - 1) + lens[-1:]
        old = sum(l % PAGE for l, n in zip(lens, new) if n)                # tokens of the pages that are written further
        pages = sum(-(-(l + n) // PAGE) - l // PAGE for l, n in zip(lens, new) if n)
        return {"bytes": (4 + 2) * sum(new) * Hkv * D + 2 * old * Hkv * D + pages * side, "flops": 0}
    if c["kind"] == "compact":
        used = sum(-(-n // PAGE) for n in lens)
        moved = used * (1 - c["live"])                                     # those that lie behind the live pages' number
        return {"bytes": int(2 * moved * (2 * Hkv * PAGE * D + side)), "flops": 0}
    pairs = keys = 0
    for l, n in zip(lens, new):
        span = min(l, PAGE * (c["first"] + c["last"] + c["top"])) if c["kind"] == "select" else l
        part = 1.0 if c["causal"] == 0 else max(0.5, 1 - n / (2 * max(l, 1)))   # of them a causal row sees
        pairs += n * span * part
        tiles = -(-G * n // PAGE)
        keys += min(l, tiles * span) if n else 0
    chosen = sum(-(-l // PAGE) * 4 * Hkv * D for l in lens) if c["kind"] == "select" else 0
    return {"bytes": int(2 * keys * Hkv * D + 2 * 2 * sum(new) * c["H"] * D + chosen), "flops": int(4 * pairs * c["H"] * D)}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _round_e4m3(x):
    """The nearest value of three mantissa bits, ties to even, least step 2^-9, largest 448."""
    e = torch.frexp(x)[1].to(torch.float64) - 1                             # |x| in [2^e, 2^(e+1))
    step = torch.exp2(e.clamp(min=-6) - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_append(s, lens, table):
    """Token by token of every written page, from the definition."""
    a, new = s["cache"], s["new"].tolist()
    total, M = a["k"].shape[0], s["case"]["M"]
    lens, table = lens.tolist(), table.tolist()
    names = [0] * total
    for b, n in enumerate(lens):
        for col in range(-(-n // PAGE)):
            names[table[b][col]] += 1
    free = [p for p in range(total) if names[p] == 0]
    out = {w: a[w].double() for w in ("k", "v", "k_scale", "v_scale", "k_sum")}
    begin = {w: out[w].clone() for w in ("k", "v", "k_scale", "v_scale")}
    for b, n in enumerate(lens):
        if new[b] == 0:
            continue
        for col in range(n // PAGE, -(-(n + new[b]) // PAGE)):
            held = max(0, min(PAGE, n - col * PAGE))                       # tokens that were there
            end = min(PAGE, n + new[b] - col * PAGE)
            src = table[b][col]
            dst = src if held and names[src] == 1 else free.pop(0)
            table[b][col] = dst
            lo = col * PAGE + held - n
            for w, x in (("k", s["k_new"]), ("v", s["v_new"])):
                fresh = x[b, :, lo:lo + end - held].double()
                amax = fresh.abs().amax((1, 2))
                e = torch.ceil(torch.log2(amax / 448.0)).clamp(-100, 100)
                scale = torch.exp2(e)
                old = begin[w][src, :, :held] * begin[w + "_scale"][src][:, None, None]
                if held:
                    scale = torch.maximum(scale, begin[w + "_scale"][src])
                codes = _round_e4m3(torch.cat((old, fresh), 1) / scale[:, None, None])
                out[w][dst, :, :end] = codes
                out[w + "_scale"][dst] = scale
                if w == "k":
                    out["k_sum"][dst] = codes.sum(1) * scale[:, None]
    return dict(out, table=torch.tensor(table, dtype=torch.int32).cuda(), lens=torch.tensor([n + m for n, m in zip(lens, new)], dtype=torch.int32).cuda())


def _exact_attend(s, selection):
    """Sequence by sequence and K/V head by K/V head, over the keys that a tile of rows really has."""
    c, a = s["case"], s["cache"]
    B, H, M, D = s["q"].shape
    G = H // c["Hkv"]
    o = torch.zeros((B, H, M, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, H, M), dtype=torch.float64, device="cuda")
    for b, (n, m) in enumerate(zip(_ints(c["lens"]), _ints(c["new"]))):
        if m == 0:
            continue
        position = torch.arange(m, device="cuda") + n - m
        limit = torch.full_like(position, n)
        if c["causal"]:
            limit = ((position // c["causal"] + 1) * c["causal"]).clamp(max=n)
        phys = a["table"][b, :-(-n // PAGE)].long()
        for g in range(c["Hkv"]):
            k, v = (((a[w].view(torch.uint8)[phys, g].view(torch.float8_e4m3fn).double()) * a[w + "_scale"][phys, g].double()[:, None, None]).reshape(-1, D)[:n]
                    for w in ("k", "v"))
            key = torch.arange(n, device="cuda")
            for h in range(G):
                score = s["q"][b, g * G + h, :m].double() @ k.T / math.sqrt(D)
                hide = key[None, :] >= limit[:, None]
                if selection is not None:
                    on = torch.zeros((selection[0].shape[2], phys.numel() + 1), dtype=torch.bool, device="cuda")
                    spot = torch.arange(selection[1].shape[3], device="cuda") < selection[0][b, g][:, None]
                    on.scatter_(1, torch.where(spot, selection[1][b, g].long(), phys.numel()), True)
                    tile = (h * M + torch.arange(m, device="cuda")) // PAGE
                    hide = hide | ~on[tile][:, key // PAGE]
                score = score.masked_fill_(hide, -math.inf)
                total = torch.logsumexp(score, 1) if n else torch.full((m,), -math.inf, dtype=torch.float64, device="cuda")
                lse[b, g * G + h, :m] = total
                weight = torch.exp_(score.sub_(torch.where(torch.isfinite(total), total, 0.0)[:, None]))
                o[b, g * G + h, :m] = weight @ v
    return o, lse


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "append":
        return _exact_append(s, s["start_lens"], s["start_table"])
    if c["kind"] == "branch":
        parent = s["parent"].long()
        return _exact_append(s, s["start_lens"][parent], s["start_table"][parent])
    if c["kind"] == "compact":   # pages move as they are
        new = _compact(s)
        return {w: x.double() if x.is_floating_point() else x for w, x in _state(new, new["live"]).items()}
    if c["kind"] == "select" and sum(_ints(c["lens"])) * c["H"] * c["M"] > 2e10:
        return None
    selection = _select(s, torch.float64) if c["kind"] == "select" else None
    o, lse = _exact_attend(s, selection)
    out = dict(o=o, lse=lse) if c["lse"] else dict(o=o)
    return dict(out, count=selection[0], pages=selection[1]) if selection is not None else out
