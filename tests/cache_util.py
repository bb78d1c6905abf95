"""A cache on the GPU beside its CPU model, with guarded buffers, and the error bounds of the attention."""
import numpy as np
import torch

from gpu_util import Guarded
from oracle import cache_oracle as co
from paper_2505_21036_b200 import api

PAGE = co.PAGE
BF16, FP32 = 2.0 ** -8, 2.0 ** -24       # half a step, relative to the value


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


class Pair:
    """KVCache and its model.  Whatever no operator may read starts as NaN codes, NaN scales and page numbers out of range."""

    def __init__(self, B, H, D, n_pages, max_pages):
        self.model = co.Cache(B, H, D, n_pages, max_pages)
        self.mem = Guarded()
        a = self.mem.alloc
        self.dev = api.KVCache(a((n_pages, H, PAGE, D), torch.uint8, 255, "k"), a((n_pages, H, PAGE, D), torch.uint8, 127, "v"),
                               a((n_pages, H), torch.float32, float("nan"), "k_scale"), a((n_pages, H), torch.float32, float("nan"), "v_scale"),
                               a((n_pages, H, D), torch.float32, float("nan"), "k_sum"), a((B, max_pages), torch.int32, 1 << 30, "table"),
                               a((B,), torch.int32, 0, "seq_len"))
        self.dev.ws = a((self.dev.ws.numel(),), torch.uint8, 0xEE, "ws")
        self.status = a((1,), torch.int32, 0, "status")

    def append(self, k, v, new_len, whole=False):
        kb, vb = bf16(k), bf16(v)
        api.rf_cache_append(self.dev, kb.cuda(), vb.cuda(), None if whole else ints(new_len), self.status)
        self.model.append(kb.double().numpy(), vb.double().numpy(), new_len)

    def fork(self, parent):
        api.rf_cache_fork(self.dev, ints(parent), self.status)
        self.model.fork(parent)

    def drop(self, first=None, count=None, max_len=None):
        api.rf_cache_drop(self.dev, *(None if x is None else ints(x) for x in (first, count, max_len)), self.status)
        self.model.drop(first, count, max_len)

    def compact(self):
        live = self.mem.alloc((1,), torch.int32, -7, "live")
        api.rf_cache_compact(self.dev, live, self.status)
        assert int(live.item()) == self.model.compact()

    def check(self, what="", status=0):
        """Every entry, token, scale and sum that the cache holds equals the model's."""
        torch.cuda.synchronize()
        d, m = self.dev, self.model
        assert int(self.status.item()) == status, (what, int(self.status.item()))
        assert d.seq_len.cpu().tolist() == m.len, what
        table = d.page_table.cpu().tolist()
        values = {w: getattr(d, w).view(torch.float8_e4m3fn).cpu().double().numpy() for w in "kv"}
        scales = {w: getattr(d, w + "_scale").cpu().double().numpy() for w in "kv"}
        sums = d.k_sum.cpu().double().numpy()
        for b, row in enumerate(m.rows):
            assert table[b][:len(row)] == row, (what, b, table[b][:len(row)], row)
            for c, p in enumerate(row):
                end = min(PAGE, m.len[b] - c * PAGE)
                for w in "kv":
                    assert np.array_equal(scales[w][p], 2.0 ** m.exp[w][p].astype(np.float64)), (what, b, c, w)
                    assert np.array_equal(values[w][p, :, :end], m.val[w][p, :, :end]), (what, b, c, w)
                # an integer sum, rounded once to fp32 (of what the page held when it was last written)
                assert np.array_equal(sums[p], m.k_sum[p].astype(np.float32).astype(np.float64)), (what, b, c)
        self.mem.check(what)

    def attend(self, q, q_len=None, causal=0, scale=None, lse=True, sched=None, lists=None, what=""):
        """Runs the kernel and compares with the model; rows that are padding must stay as they were."""
        m, qb = self.model, bf16(q)
        B, H, M, D = qb.shape
        o = self.mem.alloc((B, H, M, D), torch.bfloat16, float("nan"), "o")
        l = self.mem.alloc((B, H, M), torch.float32, 12345.0, "lse") if lse else None
        n = api.alloc_cache_attn_workspace(self.dev, H, M).numel()
        ws = self.mem.alloc((n,), torch.uint8, 0xEE, "attn ws")
        api.rf_cache_attn_fwd(self.dev, qb.cuda(), o, l, sched, None if q_len is None else ints(q_len), causal, scale, ws, self.status)
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0, (what, int(self.status.item()))
        self.mem.check(what)
        lens = [M] * B if q_len is None else q_len
        check_attention(o, l, *m.attend(qb.double().numpy(), lens, causal, scale, lists), m, lens, what)
        return o, l


def check_attention(o, lse, ref, ref_lse, spread, reach, wide, model, q_len, what=""):
    """o (bf16) and lse (fp32) against fp64.  With s a score in nats, its error is at most the fp32 sums' of D exact products of
    bf16 numbers, the scaling's and the maximum's subtraction: (D + 8) * 2^-24 * sum |q k| scale =: e_s, and an exponential adds
    2^-21; chunks take a query row as two 8-bit numbers that miss an element by 2^-21.8 of the row's largest at most, which adds 2^-21 *
    max |q| * scale * sum |k| (`wide`).  Each weight is rounded to bf16 (2^-8 of itself) and O is the mean of V under the rounded weights, so the error of
    an element is at most (2^-8 + e_s + 2^-21) * (sum w |v| + |o|), times 1 / (1 - 2^-8), plus the fp32 sums of n terms, n * 2^-24 of sum
    w |v|, plus the rounding of o itself.  The log-sum-exp has e_s, the exponentials and the fp32 sum of n positive terms, and
    its own rounding."""
    B, H, M, D = ref.shape
    got = o.float().cpu().double().numpy()
    for b in range(B):
        n = model.len[b]
        at = (b, slice(None), slice(0, q_len[b]))
        e_s = ((D + 8) * FP32 * reach[at] + 2.0 ** -21 * wide[at] + 2.0 ** -21)
        mass = spread[at] + np.abs(ref[at])
        bound = (BF16 + e_s[..., None]) * mass * (1 + 2 * BF16) + n * FP32 * spread[at] + BF16 * np.abs(ref[at]) + 1e-37
        err = np.abs(got[at] - ref[at])
        assert (err <= bound).all(), (what, b, float((err / bound).max()), np.unravel_index(np.argmax(err / bound), err.shape))
        assert np.isnan(got[b, :, q_len[b]:]).all(), (what, b, "padding rows were written")
        if lse is not None:
            l = lse.cpu().double().numpy()
            inf = np.isneginf(ref_lse[at])
            assert np.array_equal(np.isneginf(l[at]), inf), (what, b)
            tol = e_s + (n + 16) * FP32 + 4 * FP32 * np.abs(np.where(inf, 0.0, ref_lse[at]))
            d = np.abs(np.where(inf, 0.0, l[at]) - np.where(inf, 0.0, ref_lse[at]))
            assert (d <= tol).all(), (what, b, float((d / tol).max()))
            assert (l[b, :, q_len[b]:] == 12345.0).all(), (what, b)


def filled(B, H, D, lens, seed=0, spare=4, M=0, amp=1.0, shuffle=True):
    """A cache with `lens` tokens, its pages scattered over the pool."""
    rng = np.random.default_rng(seed)
    pages = sum(-(-(n + M) // PAGE) for n in lens) + spare
    p = Pair(B, H, D, max(pages, 1), max(1, max(-(-(n + M) // PAGE) for n in lens)))
    if shuffle:      # sequence by sequence in pieces of odd length, so that their pages interleave
        left = list(lens)
        while any(left):
            n = [min(x, int(rng.integers(1, 400))) for x in left]
            cap = max(n)
            p.append(rng.standard_normal((B, H, cap, D)) * amp, rng.standard_normal((B, H, cap, D)), n)
            left = [x - y for x, y in zip(left, n)]
    return p, rng
