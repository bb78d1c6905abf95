"""CPU model of the paged 8-bit K/V cache (numpy, fp64): the operators' definitions, step by step, without the library's code.

Values are kept as numbers, not as codes: an entry of the pool is what the code stands for before the page's scale."""
from __future__ import annotations

import math

import numpy as np

PAGE = 128


class CacheFull(Exception):
    pass


def round_e4m3(x: np.ndarray) -> np.ndarray:
    """The nearest e4m3 value: three mantissa bits, least step 2^-9, ties to even, saturating at 448."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    with np.errstate(divide="ignore"):
        e = np.where(a > 0, np.floor(np.log2(np.where(a > 0, a, 1.0))), -6.0)
    step = np.exp2(np.maximum(e, -6.0) - 3.0)
    return np.sign(x) * np.minimum(np.round(a / step) * step, 448.0)      # np.round: ties to even


def scale_exponent(amax: float) -> int:
    """Least e in -100..100 with amax <= 448 * 2^e."""
    e = -100
    while e < 100 and amax > 448.0 * 2.0 ** e:
        e += 1
    return e


class Cache:
    def __init__(self, n_seqs, heads, D, n_pages, max_pages):
        self.B, self.H, self.D, self.P, self.C = n_seqs, heads, D, n_pages, max_pages
        self.val = {w: np.zeros((n_pages, heads, PAGE, D)) for w in "kv"}
        self.exp = {w: np.full((n_pages, heads), -100) for w in "kv"}
        self.k_sum = np.zeros((n_pages, heads, D))
        self.rows = [[] for _ in range(n_seqs)]
        self.len = [0] * n_seqs
        self.origin = [0] * n_seqs      # where a sequence's causal blocks begin: the caller's to keep

    def named(self):
        n = [0] * self.P
        for row in self.rows:
            for p in row:
                n[p] += 1
        return n

    def append(self, k, v, new_len):
        """k, v: [B, H, M, D] numbers.  CacheFull: nothing has changed."""
        named = self.named()
        free = [p for p in range(self.P) if named[p] == 0]
        plan, used = [], 0
        for b, n in enumerate(new_len):
            pages = -(-(self.len[b] + n) // PAGE)
            shared = n > 0 and self.len[b] % PAGE != 0 and named[self.rows[b][-1]] > 1
            need = pages - len(self.rows[b]) + int(shared) if n > 0 else 0
            if pages > self.C:
                raise CacheFull
            plan.append((shared, free[used:used + need]))
            used += need
        if used > len(free):
            raise CacheFull
        old = {w: (self.val[w].copy(), self.exp[w].copy()) for w in "kv"}
        for b, n in enumerate(new_len):
            if n == 0:
                continue
            shared, fresh = plan[b]
            row = list(self.rows[b])
            held_in = row[-1] if self.len[b] % PAGE else None
            if shared:
                row[-1], fresh = fresh[0], fresh[1:]
            row += fresh
            L = self.len[b]
            for c in range(L // PAGE, len(row)):
                held = max(0, min(PAGE, L - c * PAGE))
                end = min(PAGE, L + n - c * PAGE)
                lo = c * PAGE + held - L
                for w, x in (("k", k), ("v", v)):
                    for h in range(self.H):
                        chunk = np.asarray(x[b, h, lo:lo + end - held], dtype=np.float64)
                        fin = np.isfinite(chunk)
                        e = scale_exponent(float(np.abs(chunk[fin]).max()) if fin.any() else 0.0)
                        before = np.zeros((0, self.D))
                        if held:
                            e = max(e, int(old[w][1][held_in, h]))
                            before = old[w][0][held_in, h, :held] * 2.0 ** float(old[w][1][held_in, h])
                        chunk = np.where(np.isnan(chunk), 0.0, np.clip(chunk, -1e300, 1e300))
                        p = row[c]
                        self.val[w][p, h, :end] = round_e4m3(np.concatenate([before, chunk]) / 2.0 ** e)
                        self.exp[w][p, h] = e
                        if w == "k":
                            self.k_sum[p, h] = self.val[w][p, h, :end].sum(0) * 2.0 ** e
            self.rows[b] = row
            self.len[b] = L + n

    def fork(self, parent):
        rows, lens = [list(r) for r in self.rows], list(self.len)
        for b, p in enumerate(parent):
            self.rows[b], self.len[b] = (list(rows[p]), lens[p]) if p >= 0 else ([], 0)

    def drop(self, first=None, count=None, max_len=None):
        for b in range(self.B):
            if max_len is not None:
                self.len[b] = min(self.len[b], max_len[b])
            self.rows[b] = self.rows[b][:-(-self.len[b] // PAGE)]
            if first is not None:
                gone = [t // PAGE for t in range(self.len[b])]
                kept = [t for t in gone if not first[b] <= t < first[b] + count[b]]
                self.rows[b] = [p for c, p in enumerate(self.rows[b]) if not first[b] <= c < first[b] + count[b]]
                self.len[b] = len(kept)

    def compact(self):
        live = sorted({p for row in self.rows for p in row})
        n = len(live)
        holes = [p for p in range(n) if p not in set(live)]
        to = dict(zip([p for p in live if p >= n], holes))
        for src, dst in to.items():
            for w in "kv":
                self.val[w][dst], self.exp[w][dst] = self.val[w][src], self.exp[w][src]
            self.k_sum[dst] = self.k_sum[src]
        self.rows = [[to.get(p, p) for p in row] for row in self.rows]
        return n

    def tokens(self, which, b, h):
        """[len, D]: what the cache holds for a sequence."""
        x = [self.val[which][p, h] * 2.0 ** float(self.exp[which][p, h]) for p in self.rows[b]]
        return np.concatenate(x)[:self.len[b]] if x else np.zeros((0, self.D))

    def sees(self, b, q_len, causal):
        """Keys that each of the q_len rows sees: those up to the end of its block, where blocks end at the origin and every `causal` positions on."""
        L, o = self.len[b], self.origin[b]
        p = [L - q_len + i for i in range(q_len)]
        if causal == 0:
            return [L] * q_len
        return [0 if x < 0 else min(L, o if x < o else o + ((x - o) // causal + 1) * causal) for x in p]

    def select(self, q, q_len, causal, keep_first, keep_last, top_k):
        """q [B, H, M, D]; lists [b][g][tile]."""
        B, H, M, _ = q.shape
        G = H // self.H
        out = []
        for b in range(B):
            sees = self.sees(b, q_len[b], causal)
            heads = []
            for g in range(self.H):
                rows = [(h, i) for h in range(G) for i in range(M)]
                tiles = []
                for t0 in range(0, len(rows), PAGE):
                    tile = [(h, i) for h, i in rows[t0:t0 + PAGE] if i < q_len[b]]
                    n = -(-max([sees[i] for _, i in tile], default=0) // PAGE)
                    kept = [c for c in range(n) if c < keep_first or c >= n - keep_last]
                    rest = [c for c in range(n) if c not in set(kept)]
                    if rest and 0 < top_k < len(rest):
                        pooled = np.array([q[b, g * G + h, i] for h, i in tile], dtype=np.float64).sum(0)
                        score = []
                        for c in rest:
                            n_tok, page = min(PAGE, self.len[b] - c * PAGE), self.rows[b][c]
                            sums = self.val["k"][page, g, :n_tok].sum(0) * 2.0 ** float(self.exp["k"][page, g])
                            s = float(pooled @ sums.astype(np.float32).astype(np.float64)) / n_tok
                            score.append(-math.inf if math.isnan(s) else s)
                        rest = [rest[i] for i in sorted(range(len(rest)), key=lambda i: (-score[i], i))[:top_k]]
                    elif top_k == 0:
                        rest = []
                    tiles.append(sorted(kept + rest))
                heads.append(tiles)
            out.append(heads)
        return out

    def attend(self, q, q_len, causal=0, scale=None, lists=None):
        """(o, lse, spread, reach, wide) for q [B, H, M, D], each [B, H, M(, D)]; padding rows are NaN.  spread = sum of weights *
        |v|, reach = the largest scale * sum |q| |k| of a row, wide = scale * max |q| * the largest sum |k|: what the error bounds are made of."""
        B, H, M, D = q.shape
        G, scale = H // self.H, D ** -0.5 if scale is None else scale
        o, spread = np.full((B, H, M, D), np.nan), np.full((B, H, M, D), np.nan)
        lse, reach, wide = (np.full((B, H, M), np.nan) for _ in range(3))
        for b in range(B):
            m = q_len[b]
            if m == 0:
                continue
            sees = np.array(self.sees(b, m, causal))
            key = np.arange(self.len[b])
            for h in range(H):
                g = h // G
                k, v = self.tokens("k", b, g), self.tokens("v", b, g)
                x = q[b, h, :m].astype(np.float64)
                s = scale * (x @ k.T)
                keep = key[None, :] < sees[:, None]
                if lists is not None:
                    tile = ((h % G) * M + np.arange(m)) // PAGE
                    for t in np.unique(tile):
                        on = np.zeros(len(self.rows[b]) + 1, dtype=bool)
                        on[lists[b][g][t]] = True
                        keep[tile == t] &= on[key // PAGE][None, :]
                s = np.where(keep, s, -np.inf)
                top = s.max(1, initial=-np.inf, keepdims=True)
                w = np.exp(s - np.where(np.isfinite(top), top, 0.0))
                total = w.sum(1)
                w = w / np.where(total > 0, total, 1.0)[:, None]
                with np.errstate(divide="ignore"):
                    lse[b, h, :m] = np.log(total) + np.where(np.isfinite(top), top, 0.0)[:, 0]
                o[b, h, :m], spread[b, h, :m] = w @ v, w @ np.abs(v)
                wide[b, h, :m] = (np.where(keep, abs(scale) * np.abs(k).sum(1)[None, :], 0.0)).max(1, initial=0.0) * np.abs(x).max(1)
                reach[b, h, :m] = (np.where(keep, abs(scale) * (np.abs(x) @ np.abs(k).T), 0.0)).max(1, initial=0.0)
        return o, lse, spread, reach, wide
