"""Performance cases of the paged K/V cache: what a server calls that holds the
prompts of a layout in a cache and answers on them.

Six kinds of work, each through the public calls of
`paper_2609_13692_amd.kv`:

* ``attend``   attention of each sequence's newest tokens (one, or a chunk)
               over all of its tokens in the pages;
* ``append``   a chunk's keys and values written into the pages;
* ``admit``    requests forked off cached prefixes, grown, and freed again;
* ``turnover`` the older half of a cache freed, the pages compacted, the newer
               half renamed, and new requests admitted;
* ``copy``     a list of pages copied inside the cache;
* ``merge``    attention over parts of a context joined by their statistics.

`run` with `own` false is the plain form: elementary torch operations in 32
bits over padded batches. `exact` computes the same from the definitions in 64
bits, sequence by sequence.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# --- cases --------------------------------------------------------------------

def _attend(n, q, l, heads, kv_heads, dim, page, **more):
    """n sequences with q[0] .. q[1] new tokens after l[0] .. l[1] cached ones."""
    c = {"kind": "attend", "n": n, "q_lo": q[0], "q_hi": q[1], "l_lo": l[0], "l_hi": l[1], "heads": heads,
         "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": "bf16", "causal": True, "window": 0,
         "softcap": 0.0, "heads_first": False}
    c.update(more)
    return c


def _append(n, q, l, kv_heads, dim, page, **more):
    c = {"kind": "append", "n": n, "q_lo": q[0], "q_hi": q[1], "l_lo": l[0], "l_hi": l[1], "kv_heads": kv_heads,
         "dim": dim, "page": page, "dtype": "bf16", "heads_first": False}
    c.update(more)
    return c


def _pages(kind, n, l, layers, kv_heads, dim, page, **more):
    c = {"kind": kind, "n": n, "l_lo": l[0], "l_hi": l[1], "layers": layers, "kv_heads": kv_heads, "dim": dim,
         "page": page, "dtype": "bf16", "heads_first": False}
    c.update(more)
    return c


def _merge(rows, heads, dim, parts, **more):
    c = {"kind": "merge", "rows": rows, "heads": heads, "dim": dim, "parts": parts, "dtype": "bf16"}
    c.update(more)
    return c


def listed():
    return [
        # one request of the middle retrieval workload (10 passages of about
        # 180 tokens) producing its next token: nothing but latency
        _attend(1, (1, 1), (1800, 1800), 32, 8, 128, 16, name="decode_1"),
        # a batch of the largest workload's requests (50 passages each), one
        # token each, at all stages of being cached
        _attend(64, (1, 1), (700, 9000), 32, 8, 128, 16, name="decode_64"),
        # small heads, seven query heads to a key head, single-token pages (a
        # radix cache's own granularity), an odd number of short contexts
        _attend(37, (1, 1), (1, 5003), 14, 2, 64, 1, dtype="f16", name="decode_37_f16"),
        # the largest workload's 25 requests, each computing the tokens that
        # no other request has cached: chunks of one to three passages
        _attend(25, (60, 600), (1000, 8400), 32, 8, 128, 16, name="chunk_25"),
        # wide heads, capped scores and a window, pages with the heads outside
        _attend(9, (33, 411), (17, 4099), 8, 4, 256, 64, dtype="f16", window=1024, softcap=30.0, heads_first=True,
                name="chunk_9_window"),
        # the long end: chunks of 1024 tokens, 16k of context
        _attend(4, (1024, 1024), (15000, 15360), 32, 8, 128, 16, name="chunk_4_long"),
        # the decode batch's new keys and values, then a prefill batch's
        _append(64, (1, 1), (700, 9000), 8, 128, 16, name="append_64"),
        _append(25, (60, 1201), (0, 8400), 8, 128, 16, name="append_25_chunks"),
        # nine requests of the smallest batch forked off cached prefixes
        _pages("admit", 9, (90, 731), 4, 8, 128, 16, name="admit_9"),
        # half of a cache replaced
        _pages("turnover", 48, (1000, 9000), 4, 8, 128, 16, name="turnover_48"),
        # a decode batch's shared prefix and own suffix; a prefill's four
        # levels of the trie
        _merge(64, 32, 128, 2, name="merge_64"),
        _merge(8191, 32, 128, 4, name="merge_8191"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attend",) * 6 + ("append", "append", "admit", "admit", "turnover", "copy", "merge", "merge"))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    first = rng.random() < 0.3
    page = rng.choice((1, 4, 16, 16, 32, 64, 128))
    dim = rng.choice((64, 128, 128, 128, 256, 80, 96))
    kv_heads = rng.choice((1, 2, 4, 8, 8))
    if kind == "attend":
        heads = kv_heads * rng.choice((1, 2, 4, 4, 7, 8))
        while True:
            n = _log(rng, 1, 128)
            q_hi = rng.choice((1, 1, rng.randint(2, 16), _log(rng, 17, 1500)))
            l_hi = _log(rng, 16, 16000)
            # the plain form's scores, and its copies of keys and values
            if n * heads * q_hi * (q_hi + l_hi) * max(dim, 128) <= 1 << 38 and n * kv_heads * dim * (q_hi + l_hi) <= 560 << 20:
                break
        return _attend(n, (max(1, int(q_hi * rng.uniform(0.1, 1.0))), q_hi), (int(l_hi * rng.uniform(0, 1)), l_hi),
                       heads, kv_heads, dim, page, dtype=dtype, causal=rng.random() < 0.85,
                       window=rng.choice((0, 0, 0, _log(rng, 16, 4096))), softcap=rng.choice((0.0, 0.0, 0.0, 30.0)),
                       heads_first=first)
    if kind == "append":
        while True:
            n = _log(rng, 1, 128)
            q_hi = rng.choice((1, _log(rng, 2, 16384)))
            l_hi = _log(rng, 16, 9000)
            if n * q_hi * kv_heads * dim <= 15 << 20 and n * (q_hi + l_hi) * kv_heads * dim <= 400 << 20:
                break
        return _append(n, (max(1, q_hi // rng.randint(1, 9)), q_hi), (int(l_hi * rng.uniform(0, 1)), l_hi), kv_heads,
                       dim, page, dtype=dtype, heads_first=first)
    if kind == "merge":
        rows = _log(rng, 1, 8191)
        heads = rng.choice((1, 7, 8, 14, 32))
        return _merge(rows, heads, dim if dim <= 128 else 64, rng.randint(2, 4), dtype=dtype)
    page = rng.choice((16, 16, 32, 64))
    l_hi = _log(rng, 40, 9000)
    while True:
        n, layers = _log(rng, 1, 48), rng.randint(1, 4)
        if n * l_hi * layers * kv_heads * dim <= 24 * 9000 * 4 * 8 * 128:
            break
    return _pages(kind, n, (int(l_hi * rng.uniform(0.1, 1)) + 1, l_hi), layers, kv_heads, dim, page,
                  dtype=dtype, heads_first=first)


# --- inputs -------------------------------------------------------------------

def _spread(lo, hi, n):
    """n whole numbers from lo to hi (the same for every seed)."""
    return np.rint(np.linspace(lo, hi, n) if n > 1 else np.array([hi])).astype(np.int64)


def _sizes(case, order=None):
    """New and total tokens of the sequences of an attend or append case."""
    n = case["n"]
    q, l = _spread(case["q_lo"], case["q_hi"], n), np.roll(_spread(case["l_lo"], case["l_hi"], n), n // 3)
    if order is not None:
        q, l = q[order], l[order]
    return q, q + l


def _pool(case, layers, n_pages, gen):
    """Keys and values [layer, page, slot, head, dim], the heads outside the
    slots in memory where `heads_first`; and the tables of an empty cache."""
    p, h, d = case["page"], case["kv_heads"], case["dim"]
    shape = (layers, n_pages, h, p, d) if case["heads_first"] else (layers, n_pages, p, h, d)
    kv = []
    for _ in range(2):
        x = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=gen)
        kv.append(x.transpose(2, 3) if case["heads_first"] else x)
    return kv


def _bits(ref):
    """One bit per page, set where nothing refers to it, in words of 64."""
    free = torch.zeros((ref.numel() + 63) // 64 * 64, dtype=torch.int64, device=ref.device)
    free[:ref.numel()] = ref == 0
    return (free.view(-1, 64) << torch.arange(64, device=ref.device)).sum(1)


def _tables(lengths, max_seqs, max_len, page, n_pages, rng):
    """Sequences of the given lengths in slots 0, 1, ... on pages drawn from
    all over the pool; the rest of the slots are empty."""
    pages = -(-lengths // page)
    table = torch.full((max_seqs, max(1, -(-max_len // page))), -1, dtype=torch.int32)
    ids = torch.from_numpy(rng.permutation(n_pages)[:int(pages.sum())].astype(np.int32))
    at = np.arange(int(pages.sum())) - np.repeat(np.cumsum(pages) - pages, pages)
    table[torch.from_numpy(np.repeat(np.arange(len(pages)), pages)), torch.from_numpy(at)] = ids
    length = torch.zeros(max_seqs, dtype=torch.int32)
    length[:len(lengths)] = torch.from_numpy(lengths.astype(np.int32))
    ref = torch.zeros(n_pages, dtype=torch.int32)
    ref[ids.long()] = 1
    ref = ref.cuda()
    return {"table": table.cuda(), "length": length.cuda(), "ref": ref, "free_bits": _bits(ref),
            "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def prepare(case, seed):
    rng = np.random.default_rng([int(seed), 1 + case.get("n", case.get("rows", 0)), case["dim"]])
    gen = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 40)))
    rand = lambda *shape: torch.empty(shape, device="cuda").normal_(generator=gen)  # noqa: E731
    dtype = DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if case["kind"] == "merge":
        shape = (case["rows"], case["heads"])
        s["o"] = [rand(*shape, case["dim"]) for _ in range(case["parts"])]
        # later parts are shorter; some rows see nothing of a part but the first
        s["lse"] = [rand(*shape) + 8.0 - p for p in range(case["parts"])]
        for p in range(1, case["parts"]):
            s["lse"][p][torch.rand(shape, device="cuda", generator=gen) < 0.05] = -math.inf
        return s
    n, page = case["n"], case["page"]
    if case["kind"] in ("attend", "append"):
        q, length = _sizes(case, rng.permutation(n))
        n_pages = int((-(-length // page)).sum()) + 7
        max_len = int(length.max())
        s["k"], s["v"] = _pool(case, 1, n_pages, gen)
        s |= _tables(length, n, max_len, page, n_pages, rng)
        s |= {"seqs": _ints(np.arange(n)), "q_off": _ints(np.concatenate([[0], np.cumsum(q)])), "max_q": int(q.max()),
              "max_len": max_len}
        tokens = int(q.sum())
        if case["kind"] == "attend":
            s["q"] = (rand(tokens, case["heads"], case["dim"]) * 1.5).to(dtype)
        else:
            s["k_new"], s["v_new"] = (rand(tokens, case["kv_heads"], case["dim"]).to(dtype) for _ in range(2))
        return s
    length = _spread(case["l_lo"], case["l_hi"], n)[rng.permutation(n)]
    top = case["l_hi"]
    if case["kind"] == "copy":
        pages = int((-(-length // page)).sum())
        s["k"], s["v"] = _pool(case, case["layers"], 2 * pages, gen)
        ids = rng.permutation(2 * pages)
        s |= _tables(length, n, top, page, 2 * pages, rng)
        s |= {"src": _ints(ids[:pages]), "dst": _ints(ids[pages:])}
    elif case["kind"] == "admit":
        # slots 0 .. n-1 are cached; each new request shares a part of one
        keep = np.minimum((rng.permutation(n) + 1) * length // n, length)
        new = keep + _spread(1, max(1, top // 4), n)[rng.permutation(n)]
        grown = new + rng.integers(0, 2 * page, n)
        n_pages = int((-(-length // page)).sum()) + n * (-(-(top + top // 4) // page) + 3)
        s["k"], s["v"] = _pool(case, case["layers"], n_pages, gen)
        s |= _tables(length, 2 * n, int(max(top, grown.max())), page, n_pages, rng)
        s |= {"src": _ints(rng.permutation(n)), "dst": _ints(n + np.arange(n)), "new_len": _ints(new), "grown": _ints(grown)}
        keep = np.minimum(keep, length[s["src"].cpu().numpy()])
        s["keep"] = _ints(keep)
    else:
        # slots 0 .. n-1 hold the older half, n .. 2n-1 the newer
        length = np.concatenate([length, length[::-1]])
        n_pages = int((-(-length // page)).sum()) + 2 * n + 7
        s["k"], s["v"] = _pool(case, case["layers"], n_pages, gen)
        s |= _tables(length, 2 * n, top, page, n_pages, rng)
        s |= {"old": _ints(np.arange(n)), "new": _ints(n + np.arange(n)), "none": _ints(np.full(n, -1)),
              "zero": _ints(np.zeros(n)), "new_len": _ints(length[n:]), "old_len": _ints(length[:n]), "turn": 0}
    return s


# --- one pass -----------------------------------------------------------------

def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "merge":
        if own:
            from paper_2609_13692_amd import kv
            return kv.merge(s["o"], s["lse"], out_dtype=DTYPES[case["dtype"]])
        lse = torch.stack(s["lse"])
        top = lse.amax(0)
        w = torch.exp(lse - top)
        total = w.sum(0)
        out = (torch.stack(s["o"]) * w[..., None]).sum(0) / total[..., None]
        return out.to(DTYPES[case["dtype"]]), top + torch.log(total)
    if own:
        if "cache" not in s:          # the handle that a program keeps
            from paper_2609_13692_amd import kv
            s["cache"] = kv.KvCache(s["k"], s["v"], s["table"], s["length"], s["ref"], s["free_bits"], s["status"])
        ops = s["cache"]
    else:
        ops = _Plain(s)
    if kind == "attend":
        return ops.attend(0, s["q"], s["q_off"], s["seqs"], causal=case["causal"], window=case["window"],
                          softcap=case["softcap"])
    if kind == "append":
        ops.append(0, s["k_new"], s["v_new"], s["q_off"], s["seqs"])
        return s["k"], s["v"]
    if kind == "copy":
        ops.copy(s["src"], s["dst"])
        return s["k"], s["v"]
    if kind == "admit":
        ops.fork(s["src"], s["dst"], s["keep"], s["new_len"])
        ops.extend(s["dst"], s["grown"])
        ops.free(s["dst"])
        return s["k"], s["v"], s["table"], s["length"], s["ref"]
    # what the new slots hold this turn was admitted in the last one
    held, coming = (s["new_len"], s["old_len"]) if s["turn"] % 2 == 0 else (s["old_len"], s["new_len"])
    s["turn"] += 1
    ops.free(s["old"])
    ops.compact()
    ops.fork(s["new"], s["old"], held, held)
    ops.free(s["new"])
    ops.fork(s["none"], s["new"], s["zero"], coming)
    return s["k"], s["v"], s["table"], s["length"], s["ref"]


class _Plain:
    """The operators in elementary torch operations on the state's tensors."""

    def __init__(self, s):
        self.s = s
        self.k, self.v, self.table, self.length, self.ref = s["k"], s["v"], s["table"], s["length"], s["ref"]
        self.page = s["k"].shape[2]

    def attend(self, layer, q, q_off, seqs, causal, window, softcap):
        s, page = self.s, self.page
        n, heads, dim = seqs.numel(), q.shape[1], q.shape[2]
        kv_heads = self.k.shape[3]
        group = heads // kv_heads
        counts = (q_off[1:] - q_off[:-1]).long()
        length = self.length[seqs.long()].long()
        t = torch.arange(s["max_len"], device=q.device)
        j = torch.arange(s["max_q"], device=q.device)
        pages = self.table[seqs.long()][:, t // page].long().clamp(min=0)
        k = self.k[layer][pages, t % page].float().permute(0, 2, 3, 1).contiguous()     # [n, kv head, dim, t]
        v = self.v[layer][pages, t % page].float().permute(0, 2, 1, 3).contiguous()     # [n, kv head, t, dim]
        rows = (q_off[:-1, None].long() + j).clamp(max=q.shape[0] - 1)
        x = q[rows].float().view(n, s["max_q"], kv_heads, group, dim).permute(0, 2, 3, 1, 4)
        x = x.reshape(n, kv_heads, group * s["max_q"], dim).contiguous()
        scores = torch.matmul(x, k) * (1.0 / math.sqrt(dim))
        if softcap:
            scores = softcap * torch.tanh(scores / softcap)
        at = (length - counts)[:, None] + j                                              # [n, max_q]
        seen = (t < length[:, None, None]).expand(n, s["max_q"], s["max_len"])
        if causal:
            seen = seen & (t <= at[:, :, None])
        if window:
            seen = seen & (t > at[:, :, None] - window)
        scores = scores.view(n, kv_heads, group, s["max_q"], s["max_len"])
        scores.masked_fill_(~seen[:, None, None], -math.inf)
        top = scores.amax(-1, keepdim=True)
        p = torch.exp_(scores.sub_(top))
        total = p.sum(-1, keepdim=True)
        out = torch.matmul(p.view(n, kv_heads, group * s["max_q"], s["max_len"]), v)
        out = out.view(n, kv_heads, group, s["max_q"], dim) / total
        lse = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2).reshape(n, s["max_q"], heads)
        out = out.permute(0, 3, 1, 2, 4).reshape(n, s["max_q"], heads, dim)
        there = j < counts[:, None]
        return out[there].to(q.dtype), lse[there]

    def append(self, layer, k_new, v_new, q_off, seqs):
        token = torch.arange(k_new.shape[0], device=k_new.device)
        entry = torch.searchsorted(q_off[1:].contiguous(), token.int(), right=True)
        slot = seqs.long()[entry]
        at = self.length[slot].long() - q_off[1:][entry].long() + token
        pages = self.table[slot, at // self.page].long()
        self.k[layer][pages, at % self.page] = k_new
        self.v[layer][pages, at % self.page] = v_new

    def copy(self, src, dst):
        self.k[:, dst.long()] = self.k[:, src.long()]
        self.v[:, dst.long()] = self.v[:, src.long()]

    def _need(self, length):
        return (length.long() + self.page - 1) // self.page

    def _give(self, slots, have, want):
        """Fresh pages for entries have .. want-1 of the slots' rows, the
        lowest-numbered free ones in order."""
        need = want - have
        first = need.cumsum(0) - need
        free = (self.ref == 0).nonzero()[:, 0]
        j = torch.arange(self.table.shape[1], device=slots.device)
        fresh = (j >= have[:, None]) & (j < want[:, None])
        ids = free[(first[:, None] + j - have[:, None]).clamp(0, max(0, free.numel() - 1))]
        self.table[slots] = torch.where(fresh, ids.int(), self.table[slots])
        self.ref[ids[fresh]] = 1

    def fork(self, src, dst, keep, new_len):
        src, dst, keep = src.long().clamp(min=0), dst.long(), keep.long()
        full, part = keep // self.page, keep % self.page
        j = torch.arange(self.table.shape[1], device=src.device)
        shared = j < full[:, None]
        rows = self.table[src]
        self.table[dst] = torch.where(shared, rows, self.table[dst])
        self.ref.index_add_(0, rows[shared].long(), torch.ones_like(rows[shared]))
        self._give(dst, full, self._need(new_len))
        cut = (part > 0).nonzero()[:, 0]
        a, b = self.table[src[cut], full[cut]].long(), self.table[dst[cut], full[cut]].long()
        moved = (torch.arange(self.page, device=src.device) < part[cut, None])[None, :, :, None, None]
        for x in (self.k, self.v):
            x[:, b] = torch.where(moved, x[:, a], x[:, b])
        self.length[dst] = new_len

    def extend(self, seqs, new_len):
        seqs = seqs.long()
        self._give(seqs, self._need(self.length[seqs]), self._need(new_len))
        self.length[seqs] = new_len

    def free(self, seqs):
        seqs = seqs.long()
        j = torch.arange(self.table.shape[1], device=seqs.device)
        ids = self.table[seqs][j < self._need(self.length[seqs])[:, None]].long()
        self.ref.index_add_(0, ids, torch.full_like(ids, -1, dtype=torch.int32))
        self.length[seqs] = 0

    def compact(self):
        used = self.ref > 0
        live = used.sum()
        ids = torch.arange(self.ref.numel(), device=used.device)
        src, dst = ids[used & (ids >= live)], ids[~used & (ids < live)]
        self.copy(src, dst)
        to = ids.clone()
        to[src] = dst
        j = torch.arange(self.table.shape[1], device=used.device)
        held = j < self._need(self.length)[:, None]
        self.table.copy_(torch.where(held, to[self.table.long().clamp(min=0)].int(), self.table))
        self.ref[dst] = self.ref[src]
        self.ref[src] = 0


# --- what a pass cannot do without --------------------------------------------

def _visible(case):
    """(keys some query sees, pairs of a query and a key it sees) of the
    sequences of an attend case, summed."""
    keys = pairs = 0
    for q, length in zip(*_sizes(case)):
        at = np.arange(length - q, length)
        hi = np.minimum(at + 1, length) if case["causal"] else np.full(q, length)
        lo = np.maximum(0, at + 1 - case["window"]) if case["window"] else np.zeros(q, dtype=np.int64)
        keys += int(hi.max() - lo.min())
        pairs += int(np.maximum(0, hi - lo).sum())
    return keys, pairs


def work(case):
    size = 4 if case["kind"] == "merge" else DTYPES[case["dtype"]].itemsize
    if case["kind"] == "merge":
        rows = case["rows"] * case["heads"]
        return {"bytes": rows * (case["parts"] * (4 * case["dim"] + 4) + DTYPES[case["dtype"]].itemsize * case["dim"] + 4),
                "flops": 2 * rows * case["parts"] * case["dim"]}
    row = case["kv_heads"] * case["dim"] * size                      # one token's keys, or its values
    if case["kind"] == "attend":
        keys, pairs = _visible(case)
        tokens = int(_sizes(case)[0].sum())
        return {"bytes": 2 * keys * row + tokens * case["heads"] * (2 * case["dim"] * size + 4),
                "flops": 4 * pairs * case["heads"] * case["dim"]}
    if case["kind"] == "append":
        return {"bytes": 4 * int(_sizes(case)[0].sum()) * row, "flops": 0}
    length = _spread(case["l_lo"], case["l_hi"], case["n"])
    pages = int((-(-length // case["page"])).sum())
    if case["kind"] == "admit":                                      # half a page each, and the rows of the table
        return {"bytes": 4 * case["n"] * case["page"] // 2 * row * case["layers"] + 16 * pages, "flops": 0}
    return {"bytes": 4 * pages * case["page"] * row * case["layers"], "flops": 0}


# --- the definitions in 64 bits -----------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "merge":
        lse = torch.stack([x.double() for x in s["lse"]])
        total = torch.logsumexp(lse, 0)
        out = torch.zeros(s["o"][0].shape, dtype=torch.float64, device="cuda")
        for o, x in zip(s["o"], lse):
            out += o.double() * torch.exp(x - total)[..., None]
        return out, total
    table, length = s["table"].cpu().numpy(), s["length"].cpu().numpy()
    if case["kind"] == "attend":
        return _exact_attend(case, s, table, length)
    page = case["page"]
    if case["kind"] == "append":
        off = s["q_off"].cpu().numpy()
        k, v = s["k"].double(), s["v"].double()
        for i, slot in enumerate(s["seqs"].tolist()):
            at = np.arange(length[slot] - (off[i + 1] - off[i]), length[slot])
            p, o = (torch.from_numpy(x).cuda() for x in (table[slot, at // page].astype(np.int64), at % page))
            k[0, p, o] = s["k_new"][off[i]:off[i + 1]].double()
            v[0, p, o] = s["v_new"][off[i]:off[i + 1]].double()
        return k, v
    if case["kind"] == "copy":
        k, v = s["k"].double(), s["v"].double()
        a, b = s["src"].cpu().numpy().astype(np.int64), s["dst"].cpu().numpy().astype(np.int64)
        for lo in range(0, len(a), 64):
            i, j = torch.from_numpy(a[lo:lo + 64]).cuda(), torch.from_numpy(b[lo:lo + 64]).cuda()
            k[:, j], v[:, j] = s["k"][:, i].double(), s["v"][:, i].double()
        return k, v
    model = _Pages(s, table, length)
    if case["kind"] == "admit":
        model.fork(s["src"].tolist(), s["dst"].tolist(), s["keep"].tolist(), s["new_len"].tolist())
        model.extend(s["dst"].tolist(), s["grown"].tolist())
        model.free(s["dst"].tolist())
    else:
        old, new = s["old"].tolist(), s["new"].tolist()
        model.free(old)
        model.compact()
        model.fork(new, old, s["new_len"].tolist(), s["new_len"].tolist())
        model.free(new)
        model.fork(s["none"].tolist(), new, s["zero"].tolist(), s["old_len"].tolist())
    return s["k"].double(), s["v"].double(), *(torch.from_numpy(np.asarray(x, dtype=np.int32))
                                               for x in (model.table, model.length, model.ref))


def _exact_attend(case, s, table, length):
    page, dim, group = case["page"], case["dim"], case["heads"] // case["kv_heads"]
    off = s["q_off"].cpu().numpy()
    outs, lses = [], []
    for i, slot in enumerate(s["seqs"].tolist()):
        n_new, total = int(off[i + 1] - off[i]), int(length[slot])
        t = np.arange(total)
        pages, slots = (torch.from_numpy(x).cuda() for x in (table[slot, t // page].astype(np.int64), t % page))
        at = torch.arange(total - n_new, total, device="cuda")[:, None]
        t = torch.arange(total, device="cuda")[None]
        hidden = torch.zeros((n_new, total), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= t > at
        if case["window"]:
            hidden |= t <= at - case["window"]
        out = torch.empty((n_new, case["heads"], dim), dtype=torch.float64, device="cuda")
        lse = torch.empty((n_new, case["heads"]), dtype=torch.float64, device="cuda")
        for h in range(case["heads"]):
            kh = s["k"][0][pages, slots, h // group].double()
            vh = s["v"][0][pages, slots, h // group].double()
            x = torch.mm(s["q"][off[i]:off[i + 1], h].double(), kh.t().contiguous()) / math.sqrt(dim)
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            x[hidden] = -math.inf
            lse[:, h] = torch.logsumexp(x, 1)
            out[:, h] = torch.mm(torch.exp(x - lse[:, h, None]), vh)
        outs.append(out)
        lses.append(lse)
    return torch.cat(outs), torch.cat(lses)


class _Pages:
    """Pages one by one: sets of numbers and lists, and the contents moved
    with them (in place, in the given state's keys and values)."""

    def __init__(self, s, table, length):
        self.k, self.v, self.page = s["k"], s["v"], s["k"].shape[2]
        self.table, self.length = table.tolist(), length.tolist()
        self.ref = s["ref"].tolist()

    def _move(self, pairs):
        for x in (self.k, self.v):
            taken = [x[:, a, :n].clone() for a, _, n in pairs]
            for (_, b, n), y in zip(pairs, taken):
                x[:, b, :n] = y

    def _take(self, count):
        ids = [p for p, r in enumerate(self.ref) if r == 0][:count]
        for p in ids:
            self.ref[p] = 1
        return ids

    def fork(self, src, dst, keep, new_len):
        moves = []
        for a, b, k, n in zip(src, dst, keep, new_len):
            for j in range(k // self.page):
                self.table[b][j] = self.table[a][j]
                self.ref[self.table[a][j]] += 1
        for a, b, k, n in zip(src, dst, keep, new_len):
            full, total = k // self.page, -(-n // self.page)
            self.table[b][full:total] = self._take(total - full)
            if k % self.page:
                moves.append((self.table[a][full], self.table[b][full], k % self.page))
            self.length[b] = n
        self._move(moves)

    def extend(self, seqs, new_len):
        for a, n in zip(seqs, new_len):
            have, total = -(-self.length[a] // self.page), -(-n // self.page)
            self.table[a][have:total] = self._take(total - have)
            self.length[a] = n

    def free(self, seqs):
        for a in seqs:
            for p in self.table[a][:-(-self.length[a] // self.page)]:
                self.ref[p] -= 1
            self.length[a] = 0

    def compact(self):
        used = [p for p, r in enumerate(self.ref) if r]
        holes = [p for p in range(len(used)) if not self.ref[p]]
        movers = [p for p in used if p >= len(used)]
        self._move([(a, b, self.page) for a, b in zip(movers, holes)])
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.ref[b], self.ref[a] = self.ref[a], 0
        for row, n in zip(self.table, self.length):
            for j in range(-(-n // self.page)):
                row[j] = to.get(row[j], row[j])
