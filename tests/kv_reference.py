"""Plain implementations in 64 bits of the paged cache's operators, on the CPU,
and the bounds that a kernel with 32-bit sums and weights rounded to the
inputs' type can be held to."""
import math

import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def attention(q, k, v, length_before, causal=True, window=0, softcap=0.0, scale=None, begin=0):
    """One sequence: q [n, heads, dim], k and v [tokens, kv heads, dim] as
    float64 numpy arrays, the queries being those of tokens length_before ...
    (which may be negative). Returns out, lse, and (for the bounds) the
    weighted sum of |v|, the largest sum of |q k|, and the sum of |v| over the
    unnormalised weights' sum."""
    n, heads, dim = q.shape
    tokens, kv_heads, _ = k.shape
    scale = 1 / math.sqrt(dim) if scale is None else scale
    out, mass = np.zeros((n, heads, dim)), np.zeros((n, heads, dim))
    lse, spread, small = np.full((n, heads), -np.inf), np.zeros((n, heads)), np.zeros((n, heads, dim))
    for j in range(n):
        p = length_before + j
        t = np.arange(tokens)
        seen = t >= begin
        if causal:
            seen &= t <= p
        if window:
            seen &= t > p - window
        if not seen.any():
            continue
        for h in range(heads):
            kk, vv = k[seen, h // (heads // kv_heads)], v[seen, h // (heads // kv_heads)]
            with np.errstate(all="ignore"):
                s = scale * (kk @ q[j, h])
                if softcap:
                    s = softcap * np.tanh(s / softcap)
                top = s.max()
                if top == -np.inf:
                    continue
                w = np.exp(s - top)
                out[j, h] = (w[:, None] * vv).sum(0) / w.sum()
                lse[j, h] = top + np.log(w.sum())
                mass[j, h] = (w[:, None] * np.abs(vv)).sum(0) / w.sum()
                spread[j, h] = (np.abs(kk) @ np.abs(q[j, h])).max() * abs(scale)
                small[j, h] = np.abs(vv).sum(0) / w.sum()
    return out, lse, mass, spread, small


def attention_bounds(out, lse, mass, spread, small, tokens, dim, dtype, out_dtype):
    """(|out error|, |lse error|): weights rounded to dtype (relative error
    one unit; in float16 also an absolute one of half its smallest number,
    2^-25, where the largest weight is at least 2^-9 of the sum's scale), the
    result to out_dtype, and 32-bit sums of dim products and of `tokens`
    weights."""
    e32 = 2.0 ** -24 * (2 * (dim + 8) * spread + tokens + 64)
    rel = UNIT[dtype] + e32[..., None]
    bound = rel * mass + (UNIT[out_dtype] + 2.0 ** -22) * np.abs(out) + 1e-30
    if dtype == torch.float16:
        bound = bound + 2.0 ** -24 * small
    if out_dtype == torch.float16:
        bound = bound + 2.0 ** -25
    return bound, e32 + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0)) + 2.0 ** -22


def close(got, want, bound, what):
    """Equal infinities and NaN places; the rest within the bound."""
    got, want, bound = np.asarray(got, dtype=np.float64), np.asarray(want), np.broadcast_to(bound, np.shape(want))
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), f"{what}: infinities differ"
    fine = np.isfinite(want)
    assert np.isfinite(got[fine]).all(), f"{what}: not finite"
    off = np.abs(got[fine] - want[fine]) - bound[fine]
    assert not off.size or off.max() <= 0, f"{what}: {off.max():.3g} over a bound of {bound[fine][off.argmax()]:.3g}"


class Pages:
    """The page calls' definition on lists: numbers only."""

    def __init__(self, n_pages, page, max_seqs):
        self.page, self.ref, self.rows, self.length = page, [0] * n_pages, [[] for _ in range(max_seqs)], [0] * max_seqs
        self.copies = []                     # (from, to, tokens) of partial pages and moved pages, in order

    def need(self, tokens):
        return -(-tokens // self.page)

    def free_ids(self):
        return [p for p, r in enumerate(self.ref) if r == 0]

    def _take(self, count):
        ids = self.free_ids()[:count]
        assert len(ids) == count
        for p in ids:
            self.ref[p] = 1
        return ids

    def fork(self, src, dst, keep, new_len):
        rows, copies = {}, []
        for s, d, k, n in zip(src, dst, keep, new_len):
            rows[d] = self.rows[s][:k // self.page] if s >= 0 else []
        for d in rows.values():
            for p in d:
                self.ref[p] += 1
        for s, d, k, n in zip(src, dst, keep, new_len):
            full = k // self.page
            old = self.rows[s][full] if k % self.page else None
            fresh = self._take(self.need(n) - full)
            if old is not None:
                copies.append((old, fresh[0], k % self.page))
            rows[d] = rows[d] + fresh
        for s, d, k, n in zip(src, dst, keep, new_len):
            self.rows[d], self.length[d] = rows[d], n
        self.copies = copies

    def extend(self, seqs, new_len):
        copies, shared = [], []
        for s, n in zip(seqs, new_len):
            now = self.length[s]
            shared.append(n > now and now % self.page and self.ref[self.rows[s][now // self.page]] > 1)
        drops = []
        for s, n, cow in zip(seqs, new_len, shared):
            have = self.need(self.length[s])
            if cow:
                have -= 1
                old = self.rows[s][have]
            fresh = self._take(self.need(n) - have)
            if cow:
                copies.append((old, fresh[0], self.length[s] % self.page))
                drops.append(old)
            self.rows[s] = self.rows[s][:have] + fresh
            self.length[s] = n
        for p in drops:
            self.ref[p] -= 1
        self.copies = copies

    def free(self, seqs, keep=None):
        for i, s in enumerate(seqs):
            k = 0 if keep is None else keep[i]
            for p in self.rows[s][self.need(k):]:
                self.ref[p] -= 1
            self.rows[s], self.length[s] = self.rows[s][:self.need(k)], k

    def compact(self):
        used = [p for p, r in enumerate(self.ref) if r]
        holes = [p for p in range(len(used)) if self.ref[p] == 0]
        movers = [p for p in used if p >= len(used)]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.ref[b], self.ref[a] = self.ref[a], 0
        self.rows = [[to.get(p, p) for p in row] for row in self.rows]
        self.copies = [(a, b, self.page) for a, b in to.items()]
        return len(used)
