"""Performance cases of rotated appends and of the cache in 4 bits: what a server
calls that holds the prompts of a layout as a model with rotated positions
computes them, in 16 bits or in 4.

Four kinds of work, each through the public calls of
`paper_2609_13692_amd.kv`:

* ``rotate``  new keys rotated to their positions and written into the pages of
              a 16-bit cache with their values, their queries rotated beside them;
* ``store``   the same into a cache of 4 bits, and the new tokens read back as
              the 16-bit values that they have there;
* ``read``    cached prefixes of a 4-bit cache read out in 16 bits;
* ``attend``  attention of each sequence's newest tokens (one, or a chunk) over
              all of its tokens in a 4-bit cache.

4 bits: 32 consecutive elements of a row share a byte E and have a code each, a
sign and one of eight magnitudes; an element is its code's value times
2^(E - 127). E - 127 is the smallest exponent (of those whose values the 16-bit
type holds) at which the largest magnitude is at most 7, codes are the nearest
ones, of two the even one.

`run` with `own` false is the plain form: elementary torch operations in 32
bits (64 for angles, and for what is rounded to 4 bits) over padded batches.
`exact` computes the same from the definitions in 64 bits, sequence by sequence.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EXPONENTS = {"bf16": (-125, 125), "f16": (-23, 13)}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# --- cases --------------------------------------------------------------------

def _new(kind, n, q, l, heads, kv_heads, dim, page, **more):
    """n sequences with q[0] .. q[1] new tokens after l[0] .. l[1] cached ones."""
    c = {"kind": kind, "n": n, "q_lo": q[0], "q_hi": q[1], "l_lo": l[0], "l_hi": l[1], "heads": heads,
         "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": "bf16", "heads_first": kind != "rotate"}
    c |= {"causal": True, "window": 0, "softcap": 0.0} if kind == "attend" else \
        {"rot": dim, "interleaved": False, "base": 10000.0}
    c.update(more)
    return c


def _read(n, l, kv_heads, dim, page, **more):
    c = {"kind": "read", "n": n, "l_lo": l[0], "l_hi": l[1], "kv_heads": kv_heads, "dim": dim, "page": page,
         "dtype": "bf16", "heads_first": True}
    c.update(more)
    return c


def listed():
    return [
        # a decode batch of an odd size with small heads, half of each rotated
        # in neighbouring pairs, single-token pages (a radix cache's own
        # granularity)
        _new("rotate", 37, (1, 1), (1, 5003), 14, 2, 64, 1, dtype="f16", rot=32, interleaved=True, name="rotate_37_f16"),
        # the largest workload's 25 requests, each computing the tokens that
        # no other request has cached: chunks of one to three passages
        _new("rotate", 25, (60, 600), (1000, 8400), 32, 8, 128, 16, name="rotate_25_chunks"),
        # a decode batch of that workload into the cache in 4 bits, and a
        # prefill's chunks, from none cached on
        _new("store", 64, (1, 1), (700, 9000), 32, 8, 128, 16, name="store_64"),
        _new("store", 25, (60, 1201), (0, 8400), 32, 8, 128, 16, name="store_25_chunks"),
        # cached prefixes of the smallest batch, and half of a cache, taken
        # out of it
        _read(9, (90, 731), 2, 64, 32, dtype="f16", heads_first=False, name="read_9_f16"),
        _read(48, (1000, 9000), 8, 128, 16, name="read_48"),
        # one request of the middle retrieval workload (10 passages of about
        # 180 tokens) producing its next token: nothing but latency
        _new("attend", 1, (1, 1), (1800, 1800), 32, 8, 128, 16, name="decode_1"),
        # the decode batch, at all stages of being cached
        _new("attend", 64, (1, 1), (700, 9000), 32, 8, 128, 16, name="decode_64"),
        # seven query heads to a key head, an odd number of short contexts
        _new("attend", 37, (1, 1), (1, 5003), 14, 2, 64, 1, dtype="f16", heads_first=False, name="decode_37_f16"),
        # the prefill's chunks
        _new("attend", 25, (60, 600), (1000, 8400), 32, 8, 128, 16, name="chunk_25"),
        # wide heads, capped scores and a window
        _new("attend", 9, (33, 411), (17, 4099), 8, 4, 256, 64, dtype="f16", window=1024, softcap=30.0,
             name="chunk_9_window"),
        # the long end: chunks of 1024 tokens, 16k of context
        _new("attend", 4, (1024, 1024), (15000, 15360), 32, 8, 128, 16, name="chunk_4_long"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attend",) * 6 + ("rotate", "rotate", "store", "store", "read"))
    how = {"dtype": rng.choice(("bf16", "bf16", "f16")), "heads_first": rng.random() < (0.3 if kind == "rotate" else 0.7)}
    page = rng.choice((1, 4, 16, 16, 32, 64, 128))
    dim = rng.choice((64, 128, 128, 128, 256, 96))
    kv_heads = rng.choice((1, 2, 4, 8, 8))
    heads = kv_heads * rng.choice((1, 2, 4, 4, 7, 8))
    if kind == "attend":
        while True:
            n = _log(rng, 1, 128)
            q_hi = rng.choice((1, 1, rng.randint(2, 16), _log(rng, 17, 1500)))
            l_hi = _log(rng, 16, 16000)
            # the plain form's scores, and its copies of keys and values
            if n * heads * q_hi * (q_hi + l_hi) * max(dim, 128) <= 1 << 38 and n * kv_heads * dim * (q_hi + l_hi) <= 560 << 20:
                break
        return _new("attend", n, (max(1, int(q_hi * rng.uniform(0.1, 1.0))), q_hi), (int(l_hi * rng.uniform(0, 1)), l_hi),
                    heads, kv_heads, dim, page, causal=rng.random() < 0.85, window=rng.choice((0, 0, 0, _log(rng, 16, 4096))),
                    softcap=rng.choice((0.0, 0.0, 0.0, 30.0)), **how)
    if kind == "read":
        while True:
            n, l_hi = _log(rng, 1, 64), _log(rng, 40, 9000)
            if n * l_hi * kv_heads * dim <= 48 * 5000 * 8 * 128:
                break
        return _read(n, (int(l_hi * rng.uniform(0.1, 1)) + 1, l_hi), kv_heads, dim, page, **how)
    while True:
        n = _log(rng, 1, 128)
        q_hi = rng.choice((1, _log(rng, 2, 8192)))
        l_hi = _log(rng, 16, 30000)
        if n * q_hi * (kv_heads + heads) * dim <= 60 << 20 and n * (q_hi + l_hi) * kv_heads * dim <= 400 << 20:
            break
    return _new(kind, n, (max(1, q_hi // rng.randint(1, 9)), q_hi), (int(l_hi * rng.uniform(0, 1)), l_hi), heads, kv_heads,
                dim, page, rot=rng.choice((dim, dim, 32, 64)), interleaved=rng.random() < 0.3,
                base=rng.choice((10000.0, 500000.0)), **how)


# --- inputs -------------------------------------------------------------------

def _spread(lo, hi, n):
    """n whole numbers from lo to hi (the same for every seed)."""
    return np.rint(np.linspace(lo, hi, n) if n > 1 else np.array([hi])).astype(np.int64)


def _sizes(case, order=None):
    """New and total tokens of the sequences of a case."""
    n = case["n"]
    l = np.roll(_spread(case["l_lo"], case["l_hi"], n), n // 3)
    q = _spread(case["q_lo"], case["q_hi"], n) if "q_lo" in case else np.zeros(n, dtype=np.int64)
    if order is not None:
        q, l = q[order], l[order]
    return q, q + l


def _gains(dim, gen):
    """Keys have some dimensions that are larger than the others everywhere."""
    return torch.exp(0.5 * torch.empty(dim, device="cuda").normal_(generator=gen))


def _pool(case, n_pages, gen, four):
    """Keys and values [1, page, slot, head, dim], the heads outside the slots
    in memory where `heads_first`; in 4 bits the codes, two to a byte, and the
    bytes E as well."""
    p, h, d = case["page"], case["kv_heads"], case["dim"]
    shape = (1, n_pages, h, p) if case["heads_first"] else (1, n_pages, p, h)
    turn = (lambda x: x.transpose(2, 3)) if case["heads_first"] else (lambda x: x)
    pools = []
    for gain in (_gains(d, gen), 1.0):
        if not four:
            pools.append(turn(torch.empty((*shape, d), dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=gen)))
            continue
        codes = torch.empty((*shape, d // 2), dtype=torch.uint8, device="cuda")
        scale = torch.empty((*shape, d // 32), dtype=torch.uint8, device="cuda")
        step = max(1, (64 << 20) // (p * h * d))
        for a in range(0, n_pages, step):        # in pieces: a pool is as large as a cache
            x = torch.empty((min(step, n_pages - a), *shape[2:], d), device="cuda").normal_(generator=gen) * gain
            codes[0, a:a + step], scale[0, a:a + step] = _codes(x, *EXPONENTS[case["dtype"]])
        pools.append((turn(codes), turn(scale)))
    return pools


def _codes(x, lo, hi):
    """Codes (two to a byte) and bytes E of x [..., dim]."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    part, power = torch.frexp(top)               # top = part 2^power, 1/2 <= part < 1
    e = torch.where(part <= 0.875, power - 3, power - 2)
    e = torch.where(top == 0, lo, e).clamp(lo, hi)
    size = x.abs() * torch.exp2(-e.to(x.dtype))[..., None]
    code = (size > 0.25).to(torch.uint8)
    code += size >= 0.75
    code += size > 1.25
    code += size >= 1.75
    code += size > 2.5
    code += size >= 3.5
    code += size > 5.0
    code = (code + 8 * (x < 0)).to(torch.uint8).flatten(-2)
    return code[..., ::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def _bits(ref):
    """One bit per page, set where nothing refers to it, in words of 64."""
    free = torch.zeros((ref.numel() + 63) // 64 * 64, dtype=torch.int64, device=ref.device)
    free[:ref.numel()] = ref == 0
    return (free.view(-1, 64) << torch.arange(64, device=ref.device)).sum(1)


def _tables(lengths, page, n_pages, rng):
    """Sequences of the given lengths in slots 0, 1, ... on pages drawn from
    all over the pool."""
    pages = -(-lengths // page)
    table = torch.full((len(lengths), max(1, int(pages.max()))), -1, dtype=torch.int32)
    ids = torch.from_numpy(rng.permutation(n_pages)[:int(pages.sum())].astype(np.int32))
    at = np.arange(int(pages.sum())) - np.repeat(np.cumsum(pages) - pages, pages)
    table[torch.from_numpy(np.repeat(np.arange(len(pages)), pages)), torch.from_numpy(at)] = ids
    ref = torch.zeros(n_pages, dtype=torch.int32)
    ref[ids.long()] = 1
    ref = ref.cuda()
    return {"table": table.cuda(), "length": _ints(lengths), "ref": ref, "free_bits": _bits(ref),
            "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def prepare(case, seed):
    rng = np.random.default_rng([int(seed), 1 + case["n"], case["dim"]])
    gen = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 40)))
    rand = lambda *shape: torch.empty(shape, device="cuda").normal_(generator=gen)  # noqa: E731
    dtype, kind, n, page = DTYPES[case["dtype"]], case["kind"], case["n"], case["page"]
    q, length = _sizes(case, rng.permutation(n))
    n_pages = int((-(-length // page)).sum()) + 7
    s = {"case": dict(case), "seqs": _ints(np.arange(n)), "max_q": int(q.max()), "max_len": int(length.max())}
    s |= _tables(length, page, n_pages, rng)
    if kind == "rotate":
        s["k"], s["v"] = _pool(case, n_pages, gen, False)
    else:
        (s["k"], s["k_scale"]), (s["v"], s["v_scale"]) = _pool(case, n_pages, gen, True)
    if kind == "read":
        s |= {"off": _ints(np.concatenate([[0], np.cumsum(length)])), "tokens": int(length.sum())}
        return s
    tokens = int(q.sum())
    s |= {"q_off": _ints(np.concatenate([[0], np.cumsum(q)])), "tokens": tokens,
          "q": (rand(tokens, case["heads"], case["dim"]) * 1.5).to(dtype)}
    if kind != "attend":
        s["k_new"] = (rand(tokens, case["kv_heads"], case["dim"]) * _gains(case["dim"], gen)).to(dtype)
        s["v_new"] = rand(tokens, case["kv_heads"], case["dim"]).to(dtype)
        i = torch.arange(case["rot"] // 2, device="cuda", dtype=torch.float64)
        s["freq"] = torch.pow(case["base"], -2 * i / case["rot"]).float()      # radians a position
    return s


# --- one pass -----------------------------------------------------------------

def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2609_13692_amd import kv
        if "cache" not in s:          # the handle that a program keeps
            four = {} if kind == "rotate" else {"k_scale": s["k_scale"], "v_scale": s["v_scale"], "dtype": DTYPES[case["dtype"]]}
            s["cache"] = kv.KvCache(s["k"], s["v"], s["table"], s["length"], s["ref"], s["free_bits"], s["status"], **four)
        cache = s["cache"]
        if kind == "attend":
            return cache.attend(0, s["q"], s["q_off"], s["seqs"], causal=case["causal"], window=case["window"],
                                softcap=case["softcap"])
        if kind == "read":
            return cache.read(0, s["off"], s["seqs"], s["tokens"])
        q = cache.append_rotated(0, s["k_new"], s["v_new"], s["q_off"], s["seqs"], s["freq"], q=s["q"],
                                 interleaved=case["interleaved"])
        if kind == "rotate":
            return s["k"], s["v"], q
        return *cache.read(0, s["q_off"], s["seqs"], s["tokens"]), q
    if kind == "attend":
        return _attend(s, s["q"], case["causal"], case["window"], case["softcap"])
    if kind == "read":
        at = _places(s, s["off"])
        return _values(s, "k", at).to(DTYPES[case["dtype"]]), _values(s, "v", at).to(DTYPES[case["dtype"]])
    at = _places(s, s["q_off"])
    wide = torch.float32 if kind == "rotate" else torch.float64
    angle = at[2].double()[:, None, None] * s["freq"].double()
    turn = torch.cos(angle).to(wide), torch.sin(angle).to(wide)
    k = _rotated(s["k_new"].to(wide), *turn, case["interleaved"])
    q = _rotated(s["q"].float(), turn[0].float(), turn[1].float(), case["interleaved"]).to(s["q"].dtype)
    if kind == "rotate":
        s["k"][0][at[:2]] = k.to(s["k"].dtype)
        s["v"][0][at[:2]] = s["v_new"]
        return s["k"], s["v"], q
    for name, x in (("k", k), ("v", s["v_new"].float())):
        s[name][0][at[:2]], s[name + "_scale"][0][at[:2]] = _codes(x, *EXPONENTS[case["dtype"]])
    return _values(s, "k", at).to(q.dtype), _values(s, "v", at).to(q.dtype), q


def _places(s, off):
    """Page, slot and position of the newest tokens of the sequences, cut by off."""
    token = torch.arange(s["tokens"], device=off.device)
    entry = torch.searchsorted(off[1:].contiguous(), token.int(), right=True)
    slot = s["seqs"].long()[entry]
    at = s["length"][slot].long() - off[1:][entry].long() + token
    page = s["k"].shape[2]
    return s["table"][slot, at // page].long(), at % page, at


def _rotated(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _values(s, name, at):
    """What the codes of tokens stand for, [..., heads, dim] in 32 bits."""
    codes, scale = s[name][0][at[:2]], s[name + "_scale"][0][at[:2]]
    one = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    pair = torch.stack((one.repeat(16), one.repeat_interleave(16)), 1)           # of each byte
    x = pair[codes.int()].flatten(-2).unflatten(-1, (-1, 32))
    return (x * torch.exp2(scale.float() - 127)[..., None]).flatten(-2)


def _attend(s, q, causal, window, softcap):
    page, q_off, seqs = s["k"].shape[2], s["q_off"], s["seqs"].long()
    n, heads, dim, kv_heads = seqs.numel(), q.shape[1], q.shape[2], s["k"].shape[3]
    group = heads // kv_heads
    counts = (q_off[1:] - q_off[:-1]).long()
    length = s["length"][seqs].long()
    t = torch.arange(s["max_len"], device=q.device)
    j = torch.arange(s["max_q"], device=q.device)
    at = s["table"][seqs][:, t // page].long().clamp(min=0), t % page
    k = _values(s, "k", at).permute(0, 2, 3, 1).contiguous()                     # [n, kv head, dim, t]
    v = _values(s, "v", at).permute(0, 2, 1, 3).contiguous()                     # [n, kv head, t, dim]
    rows = (q_off[:-1, None].long() + j).clamp(max=q.shape[0] - 1)
    x = q[rows].float().view(n, s["max_q"], kv_heads, group, dim).permute(0, 2, 3, 1, 4)
    x = x.reshape(n, kv_heads, group * s["max_q"], dim).contiguous()
    scores = torch.matmul(x, k) * (1.0 / math.sqrt(dim))
    if softcap:
        scores = softcap * torch.tanh(scores / softcap)
    stands = (length - counts)[:, None] + j                                      # [n, max_q]
    seen = (t < length[:, None, None]).expand(n, s["max_q"], s["max_len"])
    if causal:
        seen = seen & (t <= stands[:, :, None])
    if window:
        seen = seen & (t > stands[:, :, None] - window)
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
    kind, dim = case["kind"], case["dim"]
    four = 2 * case["kv_heads"] * (dim // 2 + dim // 32)             # a token's keys and values in 4 bits,
    two = 2 * case["kv_heads"] * 2 * dim                             # and in 16
    q, length = _sizes(case)
    tokens = int(q.sum())
    if kind == "read":
        return {"bytes": int(length.sum()) * (four + two), "flops": 0}
    if kind == "attend":
        keys, pairs = _visible(case)
        return {"bytes": keys * four + tokens * case["heads"] * (4 * dim + 4), "flops": 4 * pairs * case["heads"] * dim}
    turn = 4 * case["heads"] * dim                                   # its queries, read and written
    # read back at once, what was stored need not be read from memory
    return {"bytes": tokens * (two + turn + (two if kind == "rotate" else four + two)),
            "flops": 3 * tokens * (case["heads"] + case["kv_heads"]) * case["rot"]}


# --- the definitions in 64 bits -----------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    table, length = s["table"].cpu().numpy(), s["length"].cpu().numpy()
    if case["kind"] == "attend":
        return _exact_attend(case, s, table, length)
    if case["kind"] == "read":
        whole = [_token_rows(case, table[i], np.arange(n)) for i, n in enumerate(length)]
        return tuple(torch.cat([_exact_values(s, name, *at) for at in whole]) for name in ("k", "v"))
    off = s["q_off"].cpu().numpy()
    freq, rot = s["freq"].double(), case["rot"]
    pools = {name: s[name].double() for name in ("k", "v")} if case["kind"] == "rotate" else {}
    outs = {"k": [], "v": [], "q": []}
    for i in range(case["n"]):
        a, b = int(off[i]), int(off[i + 1])
        p = np.arange(length[i] - (b - a), length[i])
        # a rotation is a product with a complex number of size one
        theta = torch.from_numpy(p).cuda().double()[:, None] * freq
        unit = torch.polar(torch.ones_like(theta), theta)[:, None]
        new = {}
        for name, x in (("k", s["k_new"]), ("q", s["q"])):
            x = x[a:b].double()
            z = x[..., :rot]
            z = z.unflatten(-1, (rot // 2, 2)) if case["interleaved"] else z.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.complex(z[..., 0].contiguous(), z[..., 1].contiguous()) * unit)
            z = z if case["interleaved"] else z.transpose(-1, -2)
            new[name] = torch.cat([z.flatten(-2), x[..., rot:]], -1)
        new["v"] = s["v_new"][a:b].double()
        outs["q"].append(new["q"])
        pages, slots = _token_rows(case, table[i], p)
        for name in ("k", "v"):
            if pools:
                pools[name][0, pages, slots] = new[name]
            else:
                outs[name].append(_nearest(new[name], *EXPONENTS[case["dtype"]]))
    k, v = (pools[name] if pools else torch.cat(outs[name]) for name in ("k", "v"))
    return k, v, torch.cat(outs["q"])


def _token_rows(case, row, t):
    return torch.from_numpy(row[t // case["page"]].astype(np.int64)).cuda(), torch.from_numpy(t % case["page"]).cuda()


def _nearest(x, lo, hi):
    """The values in 4 bits that are nearest to x: the magnitudes one by one,
    those with even codes first."""
    blocks = x.reshape(-1, 32)
    top = blocks.abs().max(1, keepdim=True).values
    e = torch.full_like(top, float(lo))
    for k in range(lo + 1, hi + 1):
        e[top > 7 * 2.0 ** (k - 1)] = k
    unit = 2.0 ** e
    best = torch.zeros_like(blocks)
    off = blocks.abs().clone()
    for code in (2, 4, 6, 1, 3, 5, 7):
        value = MAGNITUDES[code] * unit
        near = (blocks.abs() - value).abs()
        best = torch.where(near < off, value.expand_as(best), best)
        off = torch.minimum(near, off)
    return (best * torch.sign(blocks)).reshape(x.shape)


def _exact_values(s, name, pages, slots):
    codes, scale = s[name][0, pages, slots], s[name + "_scale"][0, pages, slots]
    both = torch.empty((*codes.shape, 2), dtype=torch.float64, device="cuda")
    for k, nibble in enumerate((codes % 16, codes // 16)):
        z = torch.zeros(codes.shape, dtype=torch.float64, device="cuda")
        for code, m in enumerate(MAGNITUDES):
            z[nibble % 8 == code] = m
        both[..., k] = torch.where(nibble >= 8, -z, z)
    power = torch.pow(2.0, scale.double() - 127)
    return both.flatten(-2) * power.repeat_interleave(32, -1)


def _exact_attend(case, s, table, length):
    dim, group = case["dim"], case["heads"] // case["kv_heads"]
    off = s["q_off"].cpu().numpy()
    outs, lses = [], []
    for i in range(case["n"]):
        n_new, total = int(off[i + 1] - off[i]), int(length[i])
        at = _token_rows(case, table[i], np.arange(total))
        k, v = _exact_values(s, "k", *at), _exact_values(s, "v", *at)
        stands = torch.arange(total - n_new, total, device="cuda")[:, None]
        t = torch.arange(total, device="cuda")[None]
        hidden = torch.zeros((n_new, total), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= t > stands
        if case["window"]:
            hidden |= t <= stands - case["window"]
        out = torch.empty((n_new, case["heads"], dim), dtype=torch.float64, device="cuda")
        lse = torch.empty((n_new, case["heads"]), dtype=torch.float64, device="cuda")
        for h in range(case["heads"]):
            kh, vh = k[:, h // group].t().contiguous(), v[:, h // group].contiguous()
            x = torch.mm(s["q"][off[i]:off[i + 1], h].double(), kh) / math.sqrt(dim)
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            x[hidden] = -math.inf
            lse[:, h] = torch.logsumexp(x, 1)
            out[:, h] = torch.mm(torch.exp(x - lse[:, h, None]), vh)
        outs.append(out)
        lses.append(lse)
    return torch.cat(outs), torch.cat(lses)
