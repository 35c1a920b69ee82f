"""Attention over a cache in 4 bits against the definition in 64 bits over the
values that the cache holds: types, head layouts, page sizes, lengths from none
to thousands, masks that leave rows empty, and NaN in what a row sees and does
not see."""
import math

import numpy as np
import pytest
import torch

from kv_reference import attention, attention_bounds, close
from paper_2609_13692_amd import kv
from test_gpu_kv_attention import DT, check, ints

pytestmark = pytest.mark.gpu


def filled(lengths, page, kv_heads, dim, dtype, seed, heads_first=True, extra_pages=5, poison=255):
    """A cache of two layers whose bytes start out as 0xff (NaN), sequences in
    slots in a mixed order, written into layer 1; and their values in 64 bits."""
    g = torch.Generator().manual_seed(seed)
    n = len(lengths)
    pages = sum(-(-l // page) for l in lengths) + extra_pages
    c = kv.KvCache.create(2, pages, page, kv_heads, dim, n + 2, max(max(lengths), 1) + 2 * page, dtype, heads_first=heads_first, bits=4)
    for x in (c.k, c.v, c.k_scale, c.v_scale):
        x.fill_(poison)
    slots = torch.randperm(n + 2, generator=g)[:n].int().cuda()
    c.fork(ints([-1] * n), slots, ints([0] * n), ints(lengths), check=True)
    total = sum(lengths)
    off = np.concatenate([[0], np.cumsum(lengths)])
    k, v = (torch.randn((total, kv_heads, dim), generator=g).to(dtype).cuda() for _ in range(2))
    c.append(1, k, v, ints(off), slots)
    assert c.take_status() == []
    k, v = (x.double().cpu().numpy() for x in c.read(1, ints(off), slots, total))
    return c, slots, [k[a:b] for a, b in zip(off, off[1:])], [v[a:b] for a, b in zip(off, off[1:])]


SHAPES = [
    # lengths, new tokens, heads, kv heads, dim, page
    ([1], [1], 1, 1, 32, 1),
    ([1, 2, 17, 64, 65], [1, 1, 1, 1, 1], 4, 1, 64, 16),
    ([300, 1, 129, 33], [1, 1, 1, 1], 32, 8, 128, 16),
    ([515, 70], [1, 1], 14, 2, 64, 1),
    ([700, 31], [2, 3], 8, 1, 128, 32),                    # 16 and 24 rows of a key head
    ([260, 40, 5], [9, 40, 5], 7, 1, 96, 4),
    ([333, 129], [65, 129], 4, 4, 128, 64),
    ([200, 1000], [100, 70], 8, 2, 256, 128),
    ([600, 31], [1, 2], 8, 1, 256, 8),
    ([96, 97], [96, 33], 6, 2, 96, 8),
    ([300], [300], 16, 2, 128, 16),                        # several tiles of rows
    ([64, 0, 3, 0], [5, 0, 3, 0], 2, 2, 32, 2),            # empty sequences
    ([130], [7], 71, 1, 64, 16),
    ([40, 1025], [17, 260], 4, 2, 192, 256),
    ([400, 90], [1, 3], 5, 5, 160, 16),
    ([400], [64], 2, 1, 224, 16),
    ([700], [200], 8, 1, 64, 32),
    ([700, 900], [300, 20], 8, 2, 64, 32),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"L{max(s[0])}q{max(s[1])}h{s[2]}k{s[3]}d{s[4]}p{s[5]}")
def test_shapes(shape, dtype):
    lengths, counts, heads, kv_heads, dim, page = shape
    c, slots, ks, vs = filled(lengths, page, kv_heads, dim, DT[dtype], 1, heads_first=page != 32)
    check(c, slots, ks, vs, counts, heads, 2, DT[dtype])


@pytest.mark.parametrize("counts", [[1, 1, 1], [3, 9, 1], [70, 129, 90]], ids=["one", "few", "many"])
@pytest.mark.parametrize("how", [dict(causal=False), dict(window=1), dict(window=50), dict(softcap=5.0),
                                 dict(causal=False, window=40), dict(window=64, softcap=20.0), dict(scale=0.3), dict(scale=-0.2),
                                 dict(scale=0.0)], ids=lambda h: "-".join(f"{k}{v}" for k, v in h.items()))
def test_masks_and_scores(counts, how):
    c, slots, ks, vs = filled([140, 129, 500], 16, 2, 64, torch.bfloat16, 3)
    check(c, slots, ks, vs, counts, 8, 4, torch.bfloat16, **how)


@pytest.mark.parametrize("counts", [[1, 1, 1, 1], [40, 33, 7, 80]], ids=["one", "many"])
def test_first_visible_token(counts):
    c, slots, ks, vs = filled([100, 64, 33, 300], 8, 1, 128, torch.float16, 5)
    check(c, slots, ks, vs, counts, 4, 6, torch.float16, begin=[10, 64, 1000, 191])
    check(c, slots, ks, vs, counts, 4, 7, torch.float16, begin=[99, 0, 32, 299], causal=False)


def test_rows_before_the_sequence_see_nothing():
    c, slots, ks, vs = filled([3, 1, 0, 70], 4, 1, 64, torch.bfloat16, 8)
    check(c, slots, ks, vs, [5, 20, 3, 100], 2, 9, torch.bfloat16)
    check(c, slots, ks, vs, [5, 20, 3, 100], 2, 9, torch.bfloat16, causal=False)


@pytest.mark.parametrize("counts", [[1, 1], [90, 64]], ids=["one", "many"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_long_contexts_and_output_type(dim, counts):
    """Several workers a tile, and outputs in 32 bits."""
    c, slots, ks, vs = filled([5000, 2777], 16, 1, dim, torch.bfloat16, 10)
    check(c, slots, ks, vs, counts, 2, 11, torch.bfloat16, out_dtype=torch.float32)


def test_many_entries_and_a_slot_listed_twice():
    lengths = [1 + 37 * i % 90 for i in range(300)]
    c, slots, ks, vs = filled(lengths, 8, 1, 64, torch.float16, 12)
    pick = list(range(300)) + [5, 5, 17]
    listed = slots[torch.tensor(pick, device="cuda")].contiguous()
    check(c, listed, [ks[i] for i in pick], [vs[i] for i in pick], [1] * 303, 2, 13, torch.float16)


def test_strided_rows():
    c, slots, ks, vs = filled([77, 200], 16, 2, 64, torch.bfloat16, 10)
    fused = torch.randn((50, 20, 64), device="cuda").bfloat16()
    wide = torch.full((50, 10, 64), 5.0, device="cuda", dtype=torch.bfloat16)
    want, want_lse = c.attend(1, fused[:, 3:11].contiguous(), ints([0, 20, 50]), slots)
    got, lse = c.attend(1, fused[:, 3:11], ints([0, 20, 50]), slots, out=wide[:, 1:9])
    assert torch.equal(got, want) and torch.equal(lse, want_lse) and (wide[:, 0] == 5).all() and (wide[:, 9] == 5).all()


def set_byte(c, name, slot, t, head, block, byte):
    page = c.table[slot, t // c.page_size].item()
    getattr(c, name)[1, page, t % c.page_size, head, block] = byte


@pytest.mark.parametrize("length", [150, 6000])
@pytest.mark.parametrize("count", [1, 3, 100])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_nan(dim, count, length):
    """A NaN among the keys makes rows NaN that see it, one among the values their
    32 dimensions; no other row, head or dimension changes."""
    c, slots, ks, vs = filled([length, 60], 16, 2, dim, torch.bfloat16, 14)
    q = (torch.randn((count + 1, 4, dim), device="cuda") * 1.5).bfloat16()
    off = ints([0, count, count + 1])
    for window in (0, 40):
        clean, clean_lse = c.attend(1, q, off, slots, window=window)
        slot = slots[0].item()
        last = length - 1
        cases = [("v", last, 0, 0), ("v", length - 1 - count // 2, 1, dim // 32 - 1), ("v", length - 30, 0, dim // 64),
                 ("k", length - 1 - count // 3, 1, 1), ("v", 3, 1, 0), ("k", 0, 0, dim // 32 - 1)]
        for name, t, head, block in cases:
            old = getattr(c, name + "_scale").clone()
            set_byte(c, name + "_scale", slot, t, head, block, 255)
            out, lse = c.attend(1, q, off, slots, window=window)
            want, want_lse = clean.clone(), clean_lse.clone()
            for j in range(count):
                p = length - count + j
                if t > p or (window and t <= p - window):
                    continue
                if name == "v":
                    want[j, 2 * head:2 * head + 2, 32 * block:32 * block + 32] = math.nan
                else:
                    want[j, 2 * head:2 * head + 2] = math.nan
                    want_lse[j, 2 * head:2 * head + 2] = math.nan
            where = (name, t, head, block, window)
            assert torch.equal(out.isnan(), want.isnan()), where
            assert torch.equal(lse.isnan(), want_lse.isnan()), where
            # the rest: a block of zeros in the place of one that has a weight of its
            # row's sum would show in the rows that see it alone, whose NaN are apart
            keep = ~want.isnan()
            if name == "v":
                assert torch.equal(out[keep], clean[keep]) and torch.equal(lse, clean_lse), where
            else:
                assert torch.equal(out[keep], clean[keep]) and torch.equal(lse[~want_lse.isnan()], clean_lse[~want_lse.isnan()]), where
            getattr(c, name + "_scale").copy_(old)
    assert c.take_status() == []


@pytest.mark.parametrize("count", [1, 70])
def test_bad_pages_and_slots(count):
    """Pages outside the pool count as tokens of zeros or of the pool, and are
    reported; slots outside the table as empty."""
    c, slots, ks, vs = filled([200, 100], 16, 1, 128, torch.float16, 15, poison=100)
    q = torch.randn((2 * count, 4, 128), device="cuda").half()
    clean, _ = c.attend(1, q, ints([0, count, 2 * count]), slots)
    for page in (-1, 10 ** 9, c.k.shape[1], -2 ** 31):
        row = c.table[slots[0].item()].clone()
        c.table[slots[0].item(), 3] = page
        out, lse = c.attend(1, q, ints([0, count, 2 * count]), slots)
        assert c.take_status() == ["page"] and torch.isfinite(out).all()
        assert torch.equal(out[count:], clean[count:])
        c.table[slots[0].item()] = row
    out, lse = c.attend(1, q, ints([0, count, 2 * count]), torch.cat([slots[:1], ints([50])]))
    # less work is cut in other places: the same sums in another order
    ref = attention(q[:count].double().cpu().numpy(), ks[0], vs[0], 200 - count)
    bo, bl = attention_bounds(*ref, 200, 128, torch.float16, torch.float16)
    close(out[:count].double().cpu().numpy(), ref[0], bo, "out")
    close(lse[:count].double().cpu().numpy(), ref[1], bl, "lse")
    assert c.take_status() == ["slot"]
    assert (out[count:] == 0).all() and (lse[count:] == -math.inf).all()


def test_a_cache_past_four_gigabytes():
    """Codes whose offsets pass 32 bits, and scales whose do."""
    page, heads, dim = 1024, 8, 256
    pages = 4500                                                    # 4.7 GB of codes, 0.3 of scales, each
    c = kv.KvCache.create(1, pages, page, heads, dim, 2, 3 * page, torch.bfloat16, bits=4)
    c.length[:2] = ints([2500, 30])
    c.table[0, :3] = ints([pages - 1, 0, pages - 3])
    c.table[1, :1] = ints([pages - 2])
    c.ref[[pages - 1, 0, pages - 3, pages - 2]] = 1
    k, v = (torch.randn((2530, heads, dim), device="cuda").bfloat16() for _ in range(2))
    slots, off = ints([0, 1]), ints([0, 2500, 2530])
    c.append(0, k, v, off, slots)
    ks, vs = (x.double().cpu().numpy() for x in c.read(0, off, slots, 2530))
    for counts in ([1, 1], [40, 30]):
        q = torch.randn((sum(counts), heads, dim), device="cuda").bfloat16()
        out, lse = c.attend(0, q, ints([0, counts[0], sum(counts)]), slots)
        for i, (a, b, n) in enumerate(((0, 2500, counts[0]), (2500, 2530, counts[1]))):
            first = sum(counts[:i])
            ref = attention(q[first:first + n].double().cpu().numpy(), ks[a:b], vs[a:b], b - a - n)
            bo, bl = attention_bounds(*ref, b - a, dim, torch.bfloat16, torch.bfloat16)
            close(out[first:first + n].double().cpu().numpy(), ref[0], bo, "out")
            close(lse[first:first + n].double().cpu().numpy(), ref[1], bl, "lse")
    assert c.take_status() == []


def test_parts_of_a_context_are_the_whole():
    """A shared prefix and the rest, merged, are attention over all."""
    c, slots, ks, vs = filled([300], 16, 2, 128, torch.bfloat16, 16)
    q = torch.randn((1, 8, 128), device="cuda").bfloat16()
    whole, lse = c.attend(1, q, ints([0, 1]), slots, out_dtype=torch.float32)
    c.fork(slots, ints([next(s for s in range(3) if s != slots.item())]), ints([128]), ints([128]), check=True)
    other = ints([s for s in range(3) if c.length[s] == 128])
    a = c.attend(1, q, ints([0, 1]), other, causal=False, out_dtype=torch.float32)
    b = c.attend(1, q, ints([0, 1]), slots, causal=False, kv_begin=ints([128]), out_dtype=torch.float32)
    got, got_lse = kv.merge([a[0], b[0]], [a[1], b[1]])
    # three sums of weights rounded to 2^-9, each of terms of at most the largest |value|
    assert (got - whole).abs().max() <= 2.0 ** -8 * np.abs(vs[0]).max() + 1e-5
    assert (got_lse - lse).abs().max() <= 1e-5


def test_a_captured_decode_step_of_the_whole_path():
    """Growth, rotated append and attention over 4 bits in one graph, replayed with
    the cache's own work between the replays; each replay against eager calls on
    a cache that went the same way."""
    def build():
        g = torch.Generator(device="cuda").manual_seed(3)
        c = kv.KvCache.create(1, 64, 16, 2, 128, 4, 200, torch.bfloat16, bits=4)
        slots = ints([2, 0])
        c.fork(ints([-1, -1]), slots, ints([0, 0]), ints([70, 33]), check=True)
        x = torch.empty((103, 2, 128), device="cuda").normal_(generator=g).bfloat16()
        freq = torch.pow(10000.0, -torch.arange(64, device="cuda") / 64)
        c.append_rotated(0, x, -x, ints([0, 70, 103]), slots, freq)
        return c, slots, freq, torch.tensor([70, 33], dtype=torch.int32, device="cuda")
    k, v, q = (torch.empty((2, h, 128), device="cuda", dtype=torch.bfloat16).normal_() for h in (2, 2, 8))
    off = ints([0, 1, 2])
    sides = [build(), build()]
    out = torch.empty_like(q)

    def step(c, slots, freq, length, out):
        length.add_(1)
        c.extend(slots, length)
        turned = c.append_rotated(0, k, v, off, slots, freq, q=q)
        return c.attend(0, turned, off, slots, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*sides[0], out)
        step(*sides[1], torch.empty_like(q))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step(*sides[0], out)
    for _ in range(5):
        for x in (k, v, q):
            x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in kept]
        want = step(*sides[1], torch.empty_like(q))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(sides[0][0].k_scale, sides[1][0].k_scale)
    assert sides[0][0].length.tolist() == sides[1][0].length.tolist() == [39, 0, 76, 0]
    assert sides[0][0].take_status() == sides[1][0].take_status() == []


def test_refusals():
    c, slots, _, _ = filled([20], 16, 1, 64, torch.bfloat16, 17)
    q = torch.zeros((1, 2, 64), device="cuda", dtype=torch.bfloat16)
    with pytest.raises(kv.MptError):
        c.attend(1, q, ints([0, 1]), slots, out=torch.zeros((1, 2, 64), device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        c.attend(1, q.half(), ints([0, 1]), slots)
    with pytest.raises(ValueError):
        c.attend(1, torch.zeros((1, 2, 32), device="cuda", dtype=torch.bfloat16), ints([0, 1]), slots)
    assert c.take_status() == []
