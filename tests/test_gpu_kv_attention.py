"""Attention of new tokens over the paged cache against the definition in 64
bits: types, head layouts, page sizes, lengths from none to thousands, masks
that leave rows empty, and what must not reach a row that does not see it."""
import math

import numpy as np
import pytest
import torch

from kv_reference import attention, attention_bounds, close
from paper_2609_13692_amd import kv

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def filled(lengths, page, kv_heads, dim, dtype, seed, heads_first=False, poison=float("nan"), extra_pages=5):
    """A cache of two layers whose pages start out as `poison`, with sequences
    of random keys and values in slots in a mixed order, written by append
    into layer 1; and the float64 copies."""
    g = torch.Generator().manual_seed(seed)
    n = len(lengths)
    pages = sum(-(-l // page) for l in lengths) + extra_pages
    c = kv.KvCache.create(2, pages, page, kv_heads, dim, n + 2, max(max(lengths), 1) + 2 * page, dtype,
                          heads_first=heads_first)
    c.k.fill_(poison)
    c.v.fill_(poison)
    slots = torch.randperm(n + 2, generator=g)[:n].int().cuda()
    c.fork(ints([-1] * n), slots, ints([0] * n), ints(lengths), check=True)
    total = sum(lengths)
    k = torch.randn((total, kv_heads, dim), generator=g).to(dtype)
    v = torch.randn((total, kv_heads, dim), generator=g).to(dtype)
    off = np.concatenate([[0], np.cumsum(lengths)])
    c.append(1, k.cuda(), v.cuda(), ints(off), slots)
    assert c.take_status() == []
    kd, vd = k.double().numpy(), v.double().numpy()
    return c, slots, [kd[a:b] for a, b in zip(off, off[1:])], [vd[a:b] for a, b in zip(off, off[1:])]


def check(c, slots, ks, vs, counts, heads, seed, dtype, out_dtype=None, q=None, begin=None, **how):
    g = torch.Generator().manual_seed(seed)
    total = sum(counts)
    if q is None:
        q = (torch.randn((total, heads, c.head_dim), generator=g) * 1.5).to(dtype)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(int)
    out, lse = c.attend(1, q.cuda(), ints(off), slots, kv_begin=None if begin is None else ints(begin),
                        out_dtype=out_dtype, **how)
    out, lse = out.cpu(), lse.cpu()
    assert c.take_status() == []
    for i in range(len(counts)):
        a, b = off[i], off[i + 1]
        if a == b:
            continue
        ref = attention(q[a:b].double().numpy(), ks[i], vs[i], len(ks[i]) - counts[i],
                        begin=0 if begin is None else begin[i], **how)
        bo, bl = attention_bounds(*ref, len(ks[i]), c.head_dim, dtype, out_dtype or dtype)
        close(out[a:b].double().numpy(), ref[0], bo, f"out of entry {i}")
        close(lse[a:b].double().numpy(), ref[1], bl, f"lse of entry {i}")


DT = {"bf16": torch.bfloat16, "f16": torch.float16}

SHAPES = [
    # lengths, new tokens, heads, kv heads, dim, page
    ([1], [1], 1, 1, 8, 1),
    ([1, 2, 17, 64, 65], [1, 1, 1, 1, 1], 4, 1, 64, 16),
    ([300, 1, 129, 33], [1, 1, 1, 1], 32, 8, 128, 16),
    ([515, 70], [1, 1], 14, 2, 64, 1),
    ([700, 31], [2, 3], 8, 1, 128, 32),                    # 16 and 24 rows of a key head
    ([260, 40, 5], [9, 40, 5], 7, 1, 80, 4),
    ([333, 129], [65, 129], 4, 4, 128, 64),
    ([200, 1000], [100, 70], 8, 2, 256, 128),
    ([96, 97], [96, 33], 6, 2, 96, 8),
    ([300], [300], 16, 2, 128, 16),                        # several tiles of rows
    ([64, 0, 3, 0], [5, 0, 3, 0], 2, 2, 72, 2),            # empty sequences
    ([130], [7], 71, 1, 64, 16),
    ([40, 1025], [17, 260], 4, 2, 192, 256),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"L{max(s[0])}q{max(s[1])}h{s[2]}k{s[3]}d{s[4]}p{s[5]}")
def test_shapes(shape, dtype):
    lengths, counts, heads, kv_heads, dim, page = shape
    c, slots, ks, vs = filled(lengths, page, kv_heads, dim, DT[dtype], 1, heads_first=page == 32)
    check(c, slots, ks, vs, counts, heads, 2, DT[dtype])


@pytest.mark.parametrize("counts", [[1, 1, 1], [3, 9, 1], [70, 129, 90]], ids=["one", "few", "many"])
@pytest.mark.parametrize("how", [dict(causal=False), dict(window=1), dict(window=50), dict(softcap=5.0),
                                 dict(causal=False, window=40), dict(window=64, softcap=20.0), dict(scale=0.3)],
                         ids=lambda h: "-".join(f"{k}{v}" for k, v in h.items()))
def test_masks_and_scores(counts, how):
    c, slots, ks, vs = filled([140, 129, 500], 16, 2, 64, torch.bfloat16, 3)
    check(c, slots, ks, vs, counts, 8, 4, torch.bfloat16, **how)


@pytest.mark.parametrize("counts", [[1, 1, 1, 1], [40, 33, 7, 80]], ids=["one", "many"])
def test_first_visible_token(counts):
    """kv_begin inside, at the end and past the end of a sequence."""
    c, slots, ks, vs = filled([100, 64, 33, 300], 8, 1, 128, torch.float16, 5)
    check(c, slots, ks, vs, counts, 4, 6, torch.float16, begin=[10, 64, 1000, 191])
    check(c, slots, ks, vs, counts, 4, 7, torch.float16, begin=[99, 0, 32, 299], causal=False)


def test_rows_before_the_sequence_see_nothing():
    """More queries than tokens: the first stand before position 0."""
    c, slots, ks, vs = filled([3, 1, 0, 70], 4, 1, 64, torch.bfloat16, 8)
    check(c, slots, ks, vs, [5, 20, 3, 100], 2, 9, torch.bfloat16)
    check(c, slots, ks, vs, [5, 20, 3, 100], 2, 9, torch.bfloat16, causal=False)


@pytest.mark.parametrize("out_dtype", [torch.float32, None], ids=["f32", "own"])
def test_strided_rows_and_output_type(out_dtype):
    """Queries inside a fused projection, outputs into a wider buffer."""
    c, slots, ks, vs = filled([77, 200], 16, 2, 64, torch.bfloat16, 10)
    g = torch.Generator().manual_seed(11)
    fused = torch.randn((60, 12, 64), generator=g).to(torch.bfloat16).cuda()
    q = fused[:, :8]
    wide = torch.zeros((60, 11, 128), dtype=out_dtype or torch.bfloat16, device="cuda")
    out = wide[:, 1:9, 64:]
    got, lse = c.attend(1, q, ints([0, 20, 60]), slots, out=out)
    assert got.data_ptr() == out.data_ptr()
    plain, plain_lse = c.attend(1, q.contiguous(), ints([0, 20, 60]), slots, out_dtype=out_dtype)
    assert torch.equal(out, plain) and torch.equal(lse, plain_lse)
    assert not wide[:, 0].any() and not wide[:, 9:].any() and not wide[:, :, :64].any()
    check(c, slots, ks, vs, [20, 40], 8, 12, torch.bfloat16, out_dtype=out_dtype, q=q.cpu().contiguous())


@pytest.mark.parametrize("counts", [[1, 1], [64, 150]], ids=["one", "many"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_unseen_values_do_not_matter(counts, bad):
    """NaN and infinities in the values and keys of tokens that a row does not
    see: later tokens, tokens before kv_begin, stale pages (the pages start
    out as NaN everywhere)."""
    lengths = [150, 333]
    c, slots, ks, vs = filled(lengths, 16, 1, 128, torch.bfloat16, 13)
    at = [[149 - (counts[0] > 1) * 20, 5], [300, 40]]          # one late, one early token of each
    for i in range(2):
        for t in at[i]:
            page = int(c.table[int(slots[i]), t // 16])
            c.k[1, page, t % 16] = bad
            c.v[1, page, t % 16, :, ::3] = bad
            ks[i][t] = bad
            vs[i][t, :, ::3] = bad
    # the definition leaves out what is not seen: NaN only where it is seen
    check(c, slots, ks, vs, counts, 4, 14, torch.bfloat16, begin=[6, 41])
    check(c, slots, ks, vs, counts, 4, 14, torch.bfloat16, window=30)


def test_infinite_and_nan_values_that_are_seen():
    c, slots, ks, vs = filled([200], 16, 1, 64, torch.bfloat16, 15)
    for t, d, x in ((20, 3, math.inf), (120, 5, -math.inf), (150, 7, math.nan), (160, 3, -math.inf)):
        page = int(c.table[int(slots[0]), t // 16])
        c.v[1, page, t % 16, 0, d] = x
        vs[0][t, 0, d] = x
    check(c, slots, ks, vs, [200], 2, 16, torch.bfloat16)


def test_scores_far_apart_and_large():
    """Scores up to thousands, growing along the sequence and falling, so that
    the running maximum moves at every step or only once."""
    for sign in (1.0, -1.0):
        c, slots, ks, vs = filled([600], 16, 1, 64, torch.bfloat16, 17)
        q = torch.zeros((150, 1, 64), dtype=torch.bfloat16)
        q[:, :, 0] = 16.0
        ramp = (torch.arange(600) * sign).to(torch.bfloat16)
        for t in range(600):
            page = int(c.table[int(slots[0]), t // 16])
            c.k[1, page, t % 16, 0, 0] = ramp[t]
        ks[0][:, 0, 0] = ramp.double().numpy()
        check(c, slots, ks, vs, [150], 1, 18, torch.bfloat16, q=q)
        check(c, slots, ks, vs, [1], 1, 18, torch.bfloat16, q=q[:1])


@pytest.mark.parametrize("counts", [[1], [130]], ids=["one", "many"])
def test_offsets_past_32_bits(counts):
    """Pages more than 2^32 bytes apart, the last beyond 2^32 elements."""
    n_pages, page, heads, dim = 5, 64, 2, 128
    stride = (1 << 30) + 8192                                   # elements between pages
    store = torch.empty(stride * (n_pages - 1) + page * heads * dim, dtype=torch.bfloat16, device="cuda")
    view = lambda: store.as_strided((1, n_pages, page, heads, dim), (0, stride, heads * dim, dim, 1))  # noqa: E731
    i32 = dict(dtype=torch.int32, device="cuda")
    c = kv.KvCache(view(), view(), torch.full((1, 4), -1, **i32), torch.zeros(1, **i32), torch.zeros(n_pages, **i32),
                   torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, **i32))
    c.reset()
    c.fork(ints([-1]), ints([0]), ints([0]), ints([64]), check=True)
    c.free(ints([0]), check=True)
    # pages 1 .. 4: page 0 is held back by hand
    c.ref[0] = 1
    c.free_bits[0] = 0b11110
    c.fork(ints([-1]), ints([0]), ints([0]), ints([250]), check=True)
    assert c.table[0].tolist() == [1, 2, 3, 4]
    g = torch.Generator().manual_seed(19)
    x = torch.randn((250, heads, dim), generator=g).to(torch.bfloat16)
    c.append(0, x.cuda(), x.cuda(), ints([0, 250]), ints([0]))
    q = torch.randn((counts[0], 4, dim), generator=g).to(torch.bfloat16)
    out, lse = c.attend(0, q.cuda(), ints([0, counts[0]]), ints([0]))
    assert c.take_status() == []
    ref = attention(q.double().numpy(), x.double().numpy(), x.double().numpy(), 250 - counts[0])
    bo, bl = attention_bounds(*ref, 250, dim, torch.bfloat16, torch.bfloat16)
    close(out.double().cpu().numpy(), ref[0], bo, "out")
    close(lse.double().cpu().numpy(), ref[1], bl, "lse")


def test_long_context_and_same_result_every_time():
    """One query and a chunk over a context long enough to be split over many
    workgroups, twice, bit for bit; and against the definition."""
    c, slots, ks, vs = filled([20001, 3], 16, 1, 64, torch.float16, 20)
    for counts in ([1, 1], [33, 2]):
        check(c, slots, ks, vs, counts, 4, 21, torch.float16)
        q = torch.randn((sum(counts), 4, 64), device="cuda", dtype=torch.float16)
        off = ints(np.concatenate([[0], np.cumsum(counts)]))
        first = c.attend(1, q, off, slots)
        for _ in range(3):
            again = c.attend(1, q, off, slots)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


LONG = [
    # lengths, new tokens, heads, kv heads, dim, page: tiles of 256 rows, and of 128
    ([1500, 900], [70, 64], 8, 2, 128, 16),
    ([1700, 1300], [33, 50], 8, 1, 64, 256),
    ([1100, 1031], [40, 20], 6, 2, 128, 1),
    ([1000], [16], 4, 1, 64, 4),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", LONG, ids=lambda s: f"h{s[2]}k{s[3]}d{s[4]}p{s[5]}")
def test_many_tokens_that_every_row_sees(shape, dtype):
    """Chunks over contexts of many tiles of keys, which the kernel takes in
    groups where nothing is masked: with the groups starting and ending at all
    places, by lengths, windows and first visible tokens."""
    lengths, counts, heads, kv_heads, dim, page = shape
    c, slots, ks, vs = filled(lengths, page, kv_heads, dim, DT[dtype], 36, heads_first=page == 256)
    check(c, slots, ks, vs, counts, heads, 37, DT[dtype])
    check(c, slots, ks, vs, counts, heads, 38, DT[dtype], window=700, softcap=10.0)
    check(c, slots, ks, vs, counts, heads, 39, DT[dtype], begin=[65 + 3 * i for i in range(len(counts))], causal=False)


def test_bad_pages_inside_a_long_context():
    """Ids outside the pool among many good ones are reported and not
    followed, and do not matter to another sequence."""
    c, slots, ks, vs = filled([1500, 1500], 16, 1, 128, torch.bfloat16, 40)
    q = torch.randn((140, 4, 128), device="cuda").bfloat16()
    off = ints([0, 70, 140])
    want, _ = c.attend(1, q, off, slots)
    for page, bad in ((40, 1 << 30), (41, -1), (93, c.ref.numel())):
        c.table[int(slots[0]), page] = bad
    got, _ = c.attend(1, q, off, slots)
    assert c.take_status() == ["page"]
    assert torch.equal(got[70:], want[70:])


def test_many_short_sequences():
    lengths = [1 + (7 * i) % 90 for i in range(300)]
    c, slots, ks, vs = filled(lengths, 16, 1, 64, torch.bfloat16, 22)
    check(c, slots, ks, vs, [1] * 300, 2, 23, torch.bfloat16)
    check(c, slots, ks, vs, [1 + i % l for i, l in enumerate(lengths)], 2, 24, torch.bfloat16)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_many_entries_of_a_few_rows_each(dtype):
    """More tiles of 128 rows than the card has CUs, on either side of that
    (heads of 128 go by another kernel there), over contexts of all lengths."""
    for n in (128, 131):
        lengths = [10 + (97 * i) % 641 for i in range(n)]
        c, slots, ks, vs = filled(lengths, 16, 2, 128, DT[dtype], 41)
        check(c, slots, ks, vs, [8 + i % 3 for i in range(n)], 8, 42, DT[dtype])
        check(c, slots, ks, vs, [9] * n, 8, 43, DT[dtype], window=300, softcap=15.0)


def test_decodes_and_a_chunk_in_one_batch():
    lengths = [500, 60, 200, 90, 31]
    c, slots, ks, vs = filled(lengths, 16, 2, 128, torch.bfloat16, 25)
    check(c, slots, ks, vs, [1, 1, 150, 1, 1], 8, 26, torch.bfloat16)
    check(c, slots, ks, vs, [1, 40, 1, 0, 1], 8, 27, torch.bfloat16)


def test_a_slot_listed_twice():
    """Two entries that read one sequence."""
    c, slots, ks, vs = filled([90], 16, 1, 64, torch.bfloat16, 28)
    both = torch.cat([slots, slots])
    check(c, both, ks * 2, vs * 2, [3, 40], 4, 29, torch.bfloat16, causal=False)


def test_replays_of_a_captured_call():
    """Capture a decode step (append, attend), replay it on new queries and a
    longer sequence with eager work between, each replay against eager."""
    c, slots, ks, vs = filled([500, 70], 16, 2, 64, torch.bfloat16, 30)
    for heads, counts in ((8, [1, 1]), (8, [30, 17])):
        off = ints(np.concatenate([[0], np.cumsum(counts)]))
        q = torch.randn((sum(counts), heads, 64), device="cuda").bfloat16()
        kn, vn = (torch.randn((sum(counts), 2, 64), device="cuda").bfloat16() for _ in range(2))
        out, lse = c.attend(1, q, off, slots)              # the workspace exists before the capture
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.append(1, kn, vn, off, slots)
            c.attend(1, q, off, slots, out=out, lse=lse)
        for step in range(4):
            q.normal_()
            kn.normal_()
            vn.normal_()
            out.fill_(7)
            if step == 2:
                c.extend(slots, (c.length[slots.long()] + ints(counts)).int(), check=True)
            graph.replay()
            torch.cuda.synchronize()
            c.append(1, kn, vn, off, slots)
            want, want_lse = c.attend(1, q, off, slots)
            assert torch.equal(out, want) and torch.equal(lse, want_lse), step
        assert c.take_status() == []


def test_replays_after_calls_of_other_sizes():
    """A graph captured with the workspace of a decode step, replayed after
    eager calls that need other workspaces, on other streams, and after their
    memory could have been handed out again."""
    c, slots, ks, vs = filled([500, 70], 16, 2, 64, torch.bfloat16, 34)
    q = torch.randn((2, 8, 64), device="cuda").bfloat16()
    off = ints([0, 1, 2])
    out, lse = c.attend(1, q, off, slots)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(1, q, off, slots, out=out, lse=lse)
    side = torch.cuda.Stream()
    for counts in ([30, 17], [300, 70], [1, 1]):
        many = torch.randn((sum(counts), 8, 64), device="cuda").bfloat16()
        side.wait_stream(torch.cuda.current_stream())
        big, _ = c.attend(1, many, ints(np.concatenate([[0], np.cumsum(counts)])), slots, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        filler = [torch.full((1 << 22,), 3.0, device="cuda") for _ in range(24)]
        q.normal_()
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all((x == 3.0).all() for x in filler)
        want, want_lse = c.attend(1, q, off, slots)
        assert torch.equal(out, want) and torch.equal(lse, want_lse), counts
        check(c, slots, ks, vs, counts, 8, 35, torch.bfloat16)
        del filler, big, many
    assert c.take_status() == []


def test_another_stream():
    c, slots, ks, vs = filled([300, 40], 16, 2, 64, torch.bfloat16, 31)
    q = torch.randn((2, 8, 64), device="cuda").bfloat16()
    want, _ = c.attend(1, q, ints([0, 1, 2]), slots)
    off = ints([0, 1, 2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = c.attend(1, q, off, slots, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_bad_device_data_is_flagged_and_not_followed():
    c, slots, ks, vs = filled([100, 60], 16, 1, 64, torch.bfloat16, 32)
    q = torch.randn((2, 4, 64), device="cuda").bfloat16()
    want, _ = c.attend(1, q, ints([0, 1, 2]), slots)
    bad = slots.clone()
    bad[0] = 1 << 20
    got, lse = c.attend(1, q, ints([0, 1, 2]), bad)
    assert c.take_status() == ["slot"]
    assert torch.equal(got[1], want[1]) and not got[0].any() and (lse[0] == -math.inf).all()
    c.table[int(slots[0]), 2] = 1 << 30
    got, _ = c.attend(1, q, ints([0, 1, 2]), slots)
    assert "page" in c.take_status()
    assert torch.equal(got[1], want[1])


def test_refusals():
    c, slots, ks, vs = filled([100], 16, 2, 64, torch.bfloat16, 33)
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    off = ints([0, 1])
    for args in (dict(q=q.half()), dict(q=q.cpu()), dict(q=q[..., :32]), dict(q_off=off.long()), dict(q_off=ints([0])),
                 dict(seqs=slots.cpu()), dict(out=torch.zeros_like(q).half()), dict(lse=torch.zeros(4, device="cuda"))):
        with pytest.raises((ValueError, TypeError, kv.MptError)):
            c.attend(**{**dict(layer=1, q=q, q_off=off, seqs=slots), **args})
    for args in (dict(layer=2), dict(layer=-1), dict(window=-1), dict(softcap=-1.0), dict(softcap=math.nan),
                 dict(scale=math.inf), dict(q=torch.zeros((1, 3, 64), dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(kv.MptError) as e:
            c.attend(**{**dict(layer=1, q=q, q_off=off, seqs=slots), **args})
        assert e.value.name == "MPT_E_INVALID"
    shifted = torch.zeros(4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(1, 4, 64)
    with pytest.raises(kv.MptError):
        c.attend(1, shifted, off, slots)
    out, lse = c.attend(1, q[:0], ints([0]), slots[:0])
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
