"""Page calls of the cache (fork, extend, free, compact, copy), appends and
merged parts, against plain implementations on lists and in 64 bits."""
import math
import random

import numpy as np
import pytest
import torch

from kv_reference import UNIT, Pages, close
from paper_2609_13692_amd import kv

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def cache(n_pages, page, max_seqs=12, max_len=400, layers=2, heads=2, dim=16, dtype=torch.bfloat16, heads_first=False):
    c = kv.KvCache.create(layers, n_pages, page, heads, dim, max_seqs, max_len, dtype, heads_first=heads_first)
    c.k.normal_()
    c.v.normal_()
    return c


def same(c, model):
    """Tables, lengths, references and the bits of free pages."""
    length, table, ref = c.length.tolist(), c.table.tolist(), c.ref.tolist()
    assert length == model.length
    assert ref == model.ref
    for row, want in zip(table, model.rows):
        assert row[:len(want)] == want
    bits = [(w >> b) & 1 for w in (x & (2 ** 64 - 1) for x in c.free_bits.tolist()) for b in range(64)]
    assert bits == [int(r == 0) for r in model.ref] + [0] * (len(bits) - len(model.ref))


@pytest.mark.parametrize("page,n_pages,heads_first", [(1, 700, False), (4, 257, True), (16, 64, False), (64, 63, False)])
def test_random_calls(page, n_pages, heads_first):
    """Hundreds of calls on both; every page's contents after each."""
    rng = random.Random(page)
    c, model = cache(n_pages, page, heads_first=heads_first), Pages(n_pages, page, 12)
    k, v = c.k.clone(), c.v.clone()
    for step in range(250):
        used, empty = [s for s in range(12) if model.length[s]], [s for s in range(12) if not model.length[s]]
        kind = rng.choice(["fork", "fork", "extend", "free", "cut", "compact"])
        room = len(model.free_ids())
        model.copies = []
        if kind == "fork" and empty:
            dst = rng.sample(empty, rng.randint(1, min(4, len(empty))))
            src = [rng.choice(used) if used and rng.random() < 0.8 else -1 for _ in dst]
            keep = [rng.randint(0, model.length[s]) if s >= 0 else 0 for s in src]
            new = [k_ + rng.randint(0, 400 - k_) // rng.choice((1, 8)) for k_ in keep]
            if sum(model.need(b) - a // page for a, b in zip(keep, new)) > room:
                with pytest.raises(kv.MptError) as e:
                    c.fork(ints(src), ints(dst), ints(keep), ints(new), check=True)
                assert e.value.name == "MPT_E_PAGES" and c.take_status() == ["no pages"]
            else:
                model.fork(src, dst, keep, new)
                assert c.fork(ints(src), ints(dst), ints(keep), ints(new), check=True) == len(model.free_ids())
        elif kind == "extend" and used:
            seqs = rng.sample(used, rng.randint(1, len(used)))
            new = [min(400, model.length[s] + rng.randint(0, 3 * page)) for s in seqs]
            if sum(model.need(n) - model.need(model.length[s]) + 1 for s, n in zip(seqs, new)) <= room:
                model.extend(seqs, new)
                assert c.extend(ints(seqs), ints(new), check=True) == len(model.free_ids())
        elif kind == "free" and used:
            seqs = rng.sample(range(12), rng.randint(1, 4))
            model.free(seqs)
            assert c.free(ints(seqs), check=True) == len(model.free_ids())
        elif kind == "cut" and used:
            seqs = rng.sample(used, rng.randint(1, len(used)))
            keep = [rng.randint(0, model.length[s]) for s in seqs]
            model.free(seqs, keep)
            c.free(ints(seqs), ints(keep))
        elif kind == "compact":
            live = model.compact()
            assert c.compact(check=True) == live
        same(c, model)
        for x in (k, v):
            taken = [x[:, a, :t].clone() for a, _, t in model.copies]
            for (_, b, t), y in zip(model.copies, taken):
                x[:, b, :t] = y
        assert torch.equal(c.k, k) and torch.equal(c.v, v), (step, kind)
    assert c.take_status() == []


def test_many_entries_and_pages():
    """More list entries and words than one step of the plan takes; fragmented
    pages; a compaction that moves thousands."""
    n, page, n_pages = 1500, 2, 70001
    c = kv.KvCache.create(1, n_pages, page, 1, 8, 2 * n, 64, torch.float16)
    c.k.normal_()
    c.v.normal_()
    model = Pages(n_pages, page, 2 * n)
    rng = random.Random(3)
    lens = [rng.randint(0, 64) for _ in range(n)]
    slots = rng.sample(range(2 * n), n)
    model.fork([-1] * n, slots, [0] * n, lens)
    c.fork(ints([-1] * n), ints(slots), ints([0] * n), ints(lens))
    same(c, model)
    gone = rng.sample(slots, 1100)
    model.free(gone)
    c.free(ints(gone))
    same(c, model)
    empty = [s for s in range(2 * n) if not model.length[s]][:1200]
    src = [rng.choice([s for s in slots if s not in set(gone)]) for _ in empty]
    keep = [rng.randint(0, model.length[s]) for s in src]
    new = [k + rng.randint(0, 64 - k) for k in keep]
    model.fork(src, empty, keep, new)
    c.fork(ints(src), ints(empty), ints(keep), ints(new))
    same(c, model)
    k = c.k.clone()
    gone = rng.sample(range(2 * n), 1500)
    model.free(gone)
    c.free(ints(gone))
    for a, b, t in model.copies:
        k[:, b, :t] = k[:, a, :t]
    live = model.compact()
    k = c.k.clone()
    assert c.compact(check=True) == live
    same(c, model)
    a, b = (torch.tensor(x, device="cuda") for x in zip(*[(a, b) for a, b, _ in model.copies]))
    k[:, b] = k[:, a]
    assert torch.equal(c.k, k)


def test_copy_and_its_refusals():
    c = cache(40, 8, heads_first=True)
    k, v = c.k.clone(), c.v.clone()
    assert c.copy(ints([3, 3, 39, 0]), ints([7, 8, 1, 20]), check=True) == 4
    for x in (k, v):
        x[:, [7, 8, 1, 20]] = x[:, [3, 3, 39, 0]]
    assert torch.equal(c.k, k) and torch.equal(c.v, v)
    for src, dst, name in (([1, 2], [5, 5], "MPT_E_DUP"), ([1, 2], [2, 5], "MPT_E_DUP"), ([40], [1], "MPT_E_RANGE"),
                           ([1], [-1], "MPT_E_RANGE")):
        with pytest.raises(kv.MptError) as e:
            c.copy(ints(src), ints(dst), check=True)
        assert e.value.name == name
    assert c.copy(ints([]), ints([]), check=True) == 0
    assert torch.equal(c.k, k) and torch.equal(c.v, v)
    assert set(c.take_status()) == {"duplicate", "page"}


def test_refused_lists_change_nothing():
    c = cache(20, 4, max_seqs=5, max_len=40)
    c.fork(ints([-1, -1]), ints([0, 1]), ints([0, 0]), ints([10, 7]), check=True)
    before = [x.clone() for x in (c.table, c.length, c.ref, c.free_bits)]
    forks = [([0], [5], [4], [4], "MPT_E_RANGE"), ([5], [2], [4], [4], "MPT_E_RANGE"), ([0], [2], [11], [12], "MPT_E_RANGE"),
             ([0], [2], [5], [4], "MPT_E_RANGE"), ([-1], [2], [1], [4], "MPT_E_RANGE"), ([-1], [2], [0], [41], "MPT_E_RANGE"),
             ([0, 0], [2, 2], [4, 4], [4, 4], "MPT_E_DUP"), ([0], [1], [4], [4], "MPT_E_STATE"), ([0], [2], [-1], [4], "MPT_E_RANGE"),
             ([-1, -1], [2, 3], [0, 0], [40, 40], "MPT_E_PAGES"), ([2], [3], [1], [4], "MPT_E_RANGE"),
             ([-1, 2], [2, 3], [0, 4], [8, 8], "MPT_E_RANGE")]
    for src, dst, keep, new, name in forks:
        with pytest.raises(kv.MptError) as e:
            c.fork(ints(src), ints(dst), ints(keep), ints(new), check=True)
        assert e.value.name == name, (src, dst, keep, new)
        c.fork(ints(src), ints(dst), ints(keep), ints(new))            # unasked: the same, and no exception
    for call, name in (((c.extend, [0], [9]), "MPT_E_RANGE"), ((c.extend, [0, 0], [12, 12]), "MPT_E_DUP"),
                       ((c.extend, [-1], [12]), "MPT_E_RANGE"), ((c.extend, [0, 1, 2], [40, 40, 40]), "MPT_E_PAGES"),
                       ((c.extend, [0], [41]), "MPT_E_RANGE"), ((c.free, [0], [11]), "MPT_E_RANGE"),
                       ((c.free, [0], [-1]), "MPT_E_RANGE"), ((c.free, [1, 1], [0, 0]), "MPT_E_DUP"),
                       ((c.free, [9], [0]), "MPT_E_RANGE")):
        with pytest.raises(kv.MptError) as e:
            call[0](ints(call[1]), ints(call[2]), check=True)
        assert e.value.name == name, call
    for x, y in zip(before, (c.table, c.length, c.ref, c.free_bits)):
        assert torch.equal(x, y)
    assert set(c.take_status()) == {"slot", "length", "duplicate", "not empty", "no pages"} and c.take_status() == []
    with pytest.raises(kv.MptError):
        c.free(ints(range(6)))                                         # more entries than slots
    with pytest.raises(TypeError):
        c.free(torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        c.fork(ints([-1, -1]), ints([2]), ints([0]), ints([1]))


def test_a_cut_inside_a_shared_page_is_copied_before_it_grows():
    c, model = cache(30, 8), Pages(30, 8, 12)
    for call, args in (("fork", ([-1], [0], [0], [30])), ("fork", ([0, 0], [1, 2], [24, 16], [24, 20])),
                       ("free", ([1, 2], [13, 9])), ("extend", ([1, 2], [20, 9])), ("extend", ([2], [10])),
                       ("free", ([0],)), ("compact", ())):
        getattr(model, call)(*args)
        getattr(c, call)(*[ints(a) for a in args], check=True)
        same(c, model)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page,heads,dim,heads_first", [(1, 1, 8, False), (16, 8, 128, False), (64, 3, 80, True)])
def test_append(page, heads, dim, heads_first, dtype):
    lengths, counts = [1, 200, 33, 70, 64], [1, 5, 33, 0, 64]
    c = kv.KvCache.create(2, 400 // page + 10, page, heads, dim, 7, 256, dtype, heads_first=heads_first)
    slots = ints([6, 2, 0, 5, 3])
    c.fork(ints([-1] * 5), slots, ints([0] * 5), ints(lengths), check=True)
    k, v = c.k.clone(), c.v.clone()
    fused = torch.randn((sum(counts), 2 * heads + 1, dim), device="cuda").to(dtype)
    kn, vn = fused[:, :heads], fused[:, heads + 1:]                     # strided rows
    off = np.concatenate([[0], np.cumsum(counts)])
    c.append(1, kn, vn, ints(off), slots)
    for i, s in enumerate(slots.tolist()):
        for j in range(counts[i]):
            t = lengths[i] - counts[i] + j
            p = int(c.table[s, t // page])
            k[1, p, t % page], v[1, p, t % page] = kn[off[i] + j], vn[off[i] + j]
    assert torch.equal(c.k, k) and torch.equal(c.v, v) and c.take_status() == []


def test_append_leaves_shared_pages_and_bad_slots_alone():
    c = cache(20, 4, max_seqs=4, max_len=40)
    c.fork(ints([-1]), ints([0]), ints([0]), ints([10]), check=True)
    c.fork(ints([0]), ints([1]), ints([8]), ints([9]), check=True)
    k = c.k.clone()
    new = torch.randn((3, 2, 16), device="cuda").bfloat16()
    c.append(0, new, new, ints([0, 3]), ints([1]))                      # 6, 7 lie in a page that 0 refers to
    assert c.take_status() == ["shared page"]
    k[0, int(c.table[1, 2]), 0] = new[2]
    assert torch.equal(c.k, k)
    c.append(0, new, new, ints([0, 3]), ints([4]))
    assert c.take_status() == ["slot"]
    c.append(0, new, new, ints([0, 3]), ints([3]))                      # an empty slot
    assert c.take_status() == ["length"]
    assert torch.equal(c.k, k)
    for bad in (dict(layer=2), dict(k_new=new.float()), dict(v_new=new[:2]), dict(q_off=ints([0]))):
        with pytest.raises((ValueError, TypeError, kv.MptError)):
            c.append(**{**dict(layer=0, k_new=new, v_new=new, q_off=ints([0, 3]), seqs=ints([1])), **bad})


def test_append_of_many_entries():
    """More entries than one step of the search takes, some of them empty."""
    n = 5000
    c = kv.KvCache.create(1, n + 10, 4, 1, 8, n, 4, torch.float16)
    c.fork(ints([-1] * n), ints(range(n)), ints([0] * n), ints([3] * n), check=True)
    counts = [i % 4 if i % 4 < 3 else 0 for i in range(n)]
    off = np.concatenate([[0], np.cumsum(counts)])
    new = torch.randn((sum(counts), 1, 8), device="cuda").half()
    c.append(0, new, new, ints(off), ints(range(n)))
    assert c.take_status() == []
    entry = np.repeat(np.arange(n), counts)
    at = 3 - np.array(counts)[entry] + (np.arange(len(entry)) - off[entry])
    page = c.table[torch.from_numpy(entry).cuda(), 0].long()
    assert torch.equal(c.k[0, page, torch.from_numpy(at).cuda()], new)


@pytest.mark.parametrize("dtype,out_dtype", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16),
                                             (torch.float16, torch.float32), (torch.float32, torch.float16)])
@pytest.mark.parametrize("rows,heads,dim,parts", [(1, 1, 8, 1), (5, 7, 80, 3), (333, 4, 128, 2), (64, 3, 256, 16)])
def test_merge(rows, heads, dim, parts, dtype, out_dtype):
    g = torch.Generator().manual_seed(rows)
    o = [torch.randn((rows, heads, dim), generator=g).to(dtype) for _ in range(parts)]
    lse = [torch.randn((rows, heads), generator=g) * 4 for _ in range(parts)]
    for i, l in enumerate(lse):                                         # parts that a row sees nothing of
        l[torch.rand((rows, heads), generator=g) < 0.3] = -math.inf
        o[i][l == -math.inf] = math.nan
    got, total = kv.merge([x.cuda() for x in o], [x.cuda() for x in lse], out_dtype=out_dtype)
    w = np.stack([x.double().numpy() for x in lse])
    x = np.nan_to_num(np.stack([x.double().numpy() for x in o]))
    with np.errstate(all="ignore"):
        top = w.max(0)
        p = np.where(top == -np.inf, 0, np.exp(w - top))
        want_lse = np.where(top == -np.inf, -np.inf, top + np.log(p.sum(0)))
        want = np.where((top == -np.inf)[..., None], 0, (p[..., None] * x).sum(0) / p.sum(0)[..., None])
        mass = np.where((top == -np.inf)[..., None], 0, (p[..., None] * np.abs(x)).sum(0) / p.sum(0)[..., None])
    # differences up to some tens in the exponent, parts + 4 roundings in 32 bits
    e = 2.0 ** -24 * (parts + 64)
    bound = (e * mass + (UNIT[out_dtype] + 2.0 ** -24) * np.abs(want) + (2.0 ** -25 if out_dtype == torch.float16 else 0)
             + 1e-30)
    close(got.double().cpu().numpy(), want, bound, "out")
    close(total.double().cpu().numpy(), want_lse, e + 2.0 ** -23 * np.abs(np.where(np.isfinite(want_lse), want_lse, 0)), "lse")


def test_merge_in_place_and_its_refusals():
    o = [torch.randn((50, 3, 80), device="cuda") for _ in range(2)]
    lse = [torch.randn((50, 3), device="cuda") for _ in range(2)]
    want, want_lse = kv.merge(o, lse)
    out, total = kv.merge(o, lse, out=o[0], lse=lse[1])
    assert out is o[0] and total is lse[1] and torch.equal(out, want) and torch.equal(total, want_lse)
    for parts, lses in (([], []), (o, lse[:1]), ([o[0], o[1].half()], lse), ([o[0], o[1][:49]], lse),
                        ([o[0].cpu(), o[1].cpu()], lse), (o, [lse[0], lse[1].double()]), (o * 9, lse * 9),
                        ([o[0].transpose(0, 1)] * 2, [lse[0].t()] * 2)):
        with pytest.raises((ValueError, TypeError)):
            kv.merge(parts, lses)
    with pytest.raises(kv.MptError):
        kv.merge([torch.zeros((4, 12), device="cuda")], [torch.zeros(4, device="cuda")])
    out, total = kv.merge([torch.zeros((0, 8), device="cuda")], [torch.zeros(0, device="cuda")])
    assert out.shape == (0, 8)


def test_shared_prefix_in_two_parts_is_the_whole():
    """Queries of three forks: the shared prefix in one slot with all of them,
    each one's own part from kv_begin, merged; against one attention."""
    page, prefix, heads, dim = 16, 100, 8, 64
    c = kv.KvCache.create(1, 60, page, 2, dim, 5, 400)
    c.fork(ints([-1]), ints([0]), ints([0]), ints([prefix]), check=True)
    x = torch.randn((prefix, 2, dim), device="cuda").bfloat16()
    c.append(0, x, -x, ints([0, prefix]), ints([0]))
    own, slots = [1, 40, 131], ints([1, 3, 4])
    c.fork(ints([0, 0, 0]), slots, ints([prefix] * 3), ints([prefix + n for n in own]), check=True)
    off = ints(np.concatenate([[0], np.cumsum(own)]))
    kn, vn = (torch.randn((sum(own), 2, dim), device="cuda").bfloat16() for _ in range(2))
    c.append(0, kn, vn, off, slots)
    q = torch.randn((sum(own), heads, dim), device="cuda").bfloat16()
    whole, whole_lse = c.attend(0, q, off, slots, out_dtype=torch.float32)
    parts = [c.attend(0, q, ints([0, sum(own)]), ints([0]), causal=False, out_dtype=torch.float32),
             c.attend(0, q, off, slots, kv_begin=ints([prefix] * 3), out_dtype=torch.float32)]
    out, lse = kv.merge([p[0] for p in parts], [p[1] for p in parts])
    assert c.take_status() == []
    # both sides round weights to bfloat16 (2^-8) of values up to the largest |v|
    assert (out - whole).abs().max() <= 2 * 2.0 ** -8 * max(float(vn.abs().max()), float(x.abs().max()))
    assert (lse - whole_lse).abs().max() <= 1e-4
