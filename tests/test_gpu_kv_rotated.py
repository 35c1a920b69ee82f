"""Appends that rotate keys and queries to their positions, in a cache of 16
bits, against the definition in 64."""
import numpy as np
import pytest
import torch

from kv_reference import UNIT, close
from mx4_reference import partners, rotated
from paper_2609_13692_amd import kv

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def frequencies(rot, base=10000.0):
    return (base ** (-np.arange(rot // 2) / (rot / 2))).astype(np.float32)


def bound(x, y, freq, dtype, interleaved, factor=1.0):
    """One rounding to the type (half its step, and half its smallest number in
    float16), and in 32 bits: cosine and sine rounded, two products, a sum."""
    return (UNIT[dtype] * np.abs(y) + 4 * 2.0 ** -24 * abs(factor) * partners(x, freq, interleaved) * (1 + UNIT[dtype])
            + (2.0 ** -25 if dtype == torch.float16 else 1e-40))


def filled(lengths, page, heads, dim, dtype, max_len=None, heads_first=False, **how):
    pages = sum(-(-l // page) for l in lengths) + 4
    c = kv.KvCache.create(2, pages, page, heads, dim, len(lengths) + 2, max_len or max(max(lengths), 1), dtype,
                          heads_first=heads_first, **how)
    slots = ints(range(len(lengths), 0, -1))
    c.fork(ints([-1] * len(lengths)), slots, ints([0] * len(lengths)), ints(lengths), check=True)
    return c, slots


CASES = [
    # lengths, new tokens, query heads, heads, dim, page, rotated, neighbours, heads first
    ([1], [1], 1, 1, 16, 1, 16, False, False),
    ([1, 200, 33, 70, 64], [1, 5, 33, 0, 64], 4, 2, 64, 16, 64, False, False),
    ([1, 200, 33, 70, 64], [1, 5, 33, 0, 64], 4, 2, 64, 16, 32, True, True),
    ([130, 7], [40, 7], 14, 2, 64, 1, 32, False, False),
    ([90, 300], [90, 2], 32, 8, 128, 16, 128, False, True),
    ([90, 300], [90, 2], 32, 8, 128, 16, 128, True, False),
    ([65, 40], [3, 40], 3, 3, 80, 4, 80, False, False),
    ([65, 40], [3, 40], 3, 1, 72, 4, 48, False, False),
    ([20, 40], [3, 40], 7, 1, 96, 64, 96, False, True),
    ([33], [33], 2, 1, 256, 32, 256, False, False),
    ([33], [33], 2, 1, 248, 32, 16, True, False),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"q{c[2]}h{c[3]}d{c[4]}p{c[5]}r{c[6]}{'n' if c[7] else ''}")
def test_shapes(case, dtype):
    lengths, counts, q_heads, heads, dim, page, rot, neighbours, first = case
    dtype = DT[dtype]
    c, slots = filled(lengths, page, heads, dim, dtype, heads_first=first)
    before = [x.clone() for x in (c.k, c.v)]
    tokens = sum(counts)
    fused = torch.randn((tokens, q_heads + 2 * heads, dim), device="cuda").to(dtype)      # strided rows
    q, k, v = fused[:, :q_heads], fused[:, q_heads:q_heads + heads], fused[:, q_heads + heads:]
    off = np.concatenate([[0], np.cumsum(counts)])
    freq = frequencies(rot)
    out = c.append_rotated(1, k, v, ints(off), slots, torch.tensor(freq, device="cuda"), q=q, interleaved=neighbours)
    assert c.take_status() == [] and out.shape == q.shape and out.dtype is dtype
    pos = np.concatenate([np.arange(l - n, l) for l, n in zip(lengths, counts)])
    x = q.double().cpu().numpy()
    y = rotated(x, pos, freq, neighbours)
    close(out.double().cpu().numpy(), y, bound(x, y, freq, dtype, neighbours), "queries")
    x = k.double().cpu().numpy()
    y = rotated(x, pos, freq, neighbours)
    table = c.table.cpu().numpy()
    slot = np.repeat(slots.cpu().numpy(), counts)
    pages, at = torch.tensor(table[slot, pos // page]).long().cuda(), torch.tensor(pos % page).cuda()
    close(c.k[1, pages, at].double().cpu().numpy(), y, bound(x, y, freq, dtype, neighbours), "keys")
    assert torch.equal(c.v[1, pages, at], v)
    for x, old in zip((c.k, c.v), before):                       # and nothing else has changed
        x = x.clone()
        x[1, pages, at] = old[1, pages, at]
        assert torch.equal(x, old)


@pytest.mark.parametrize("factor", [1.0, 1.25, -0.5])
def test_far_positions_and_a_factor(factor):
    """Angles of a million radians and more are formed in 64 bits."""
    pos = np.array([0, 1, -1, 65535, 1000003, 2 ** 24 + 1, 2 ** 30 - 1, 2 ** 31 - 1, -2 ** 31])
    freq = frequencies(128, 1.0001)                              # all about one radian a position
    c, _ = filled([1], 1, 1, 128, torch.float16)
    q = torch.randn((len(pos), 5, 128), device="cuda").half()
    got = c.append_rotated(0, None, None, None, None, torch.tensor(freq, device="cuda"), q=q, positions=ints(pos), factor=factor)
    x = q.double().cpu().numpy()
    y = rotated(x, pos, freq, factor=factor)
    close(got.double().cpu().numpy(), y, bound(x, y, freq, torch.float16, False, factor), "queries")
    assert c.take_status() == []


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("rot,dim,heads", [(80, 80, 7), (48, 72, 5), (128, 128, 32)])
def test_queries_in_place(rot, dim, heads, neighbours):
    c, slots = filled([50, 9], 4, 1, dim, torch.bfloat16)
    q = torch.randn((30, heads, dim), device="cuda").bfloat16()
    freq = torch.tensor(frequencies(rot), device="cuda")
    off = ints([0, 21, 30])
    want = c.append_rotated(0, None, None, off, slots, freq, q=q, interleaved=neighbours)
    k = torch.randn((30, 1, dim), device="cuda").bfloat16()
    assert c.append_rotated(0, k, k, off, slots, freq, q=q, q_out=q, interleaved=neighbours) is q
    assert torch.equal(q, want)


def test_positions_that_are_given():
    """Keys and queries at given positions, the tokens in the pages that their
    place in the sequence says."""
    c, slots = filled([40], 8, 2, 64, torch.bfloat16)
    k, v, q = (torch.randn((7, 2, 64), device="cuda").bfloat16() for _ in range(3))
    freq = torch.tensor(frequencies(64), device="cuda")
    pos = ints([5, 4, 3, 100, 0, 9, 9])
    got = c.append_rotated(1, k, v, ints([0, 7]), slots, freq, q=q, positions=pos)
    alone = c.append_rotated(1, None, None, None, None, freq, q=torch.cat([k, q], 1), positions=pos)
    assert torch.equal(got, alone[:, 2:])
    kk, vv = c.read(1, ints([0, 7]), slots, 7)
    assert torch.equal(kk, alone[:, :2]) and torch.equal(vv, v)


def test_tokens_that_are_not_written():
    """Shared pages, bad pages, lengths and slots: reported, nothing written, and
    queries rotated where the token has a place."""
    c, slots = filled([20, 20, 3, 20], 8, 1, 64, torch.bfloat16)
    c.fork(slots[:1], ints([5]), ints([16]), ints([16]), check=True)
    c.table[slots[1].item(), 2] = 10 ** 6                        # no page of the pool
    before = [x.clone() for x in (c.k, c.v)]
    listed = torch.cat([slots[:3], ints([77, -1])])
    counts = [6, 2, 5, 2, 1]                                     # 14 .. 19 (two of them shared), 18, 19, -2 .. 2
    k = torch.randn((17, 1, 64), device="cuda").bfloat16()
    q = torch.randn((17, 2, 64), device="cuda").bfloat16()
    q_out = torch.full_like(q, 7.0)
    freq = frequencies(64)
    c.append_rotated(0, k, k, ints([0, 6, 8, 13, 15, 16]), listed, torch.tensor(freq, device="cuda"), q=q, q_out=q_out)
    assert set(c.take_status()) == {"slot", "length", "page", "shared page"}
    pos = np.array([14, 15, 16, 17, 18, 19, 18, 19, -2, -1, 0, 1, 2])
    x = q[:13].double().cpu().numpy()
    y = rotated(x, pos, freq)
    close(q_out[:13].double().cpu().numpy(), y, bound(x, y, freq, torch.bfloat16, False), "queries")
    assert (q_out[13:] == 7).all() and sum(counts) == 16
    row = c.table.cpu().numpy()
    wrote = [(row[slots[0].item(), p // 8], p % 8) for p in (16, 17, 18, 19)] + [(row[slots[2].item(), 0], p) for p in (0, 1, 2)]
    for x, old in zip((c.k, c.v), before):
        changed = (x != old).any(-1).any(-1)
        assert sorted(map(tuple, changed[0].nonzero().tolist())) == sorted(wrote) and not changed[1].any()


def test_captured_and_replayed():
    """A graph of the call reads lengths, positions and rows as they are when it
    is replayed."""
    c, slots = filled([30, 50], 8, 2, 128, torch.bfloat16, max_len=64)
    k, v = (torch.randn((2, 2, 128), device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((2, 8, 128), device="cuda").bfloat16()
    freq, off = torch.tensor(frequencies(128), device="cuda"), ints([0, 1, 2])
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.append_rotated(0, k, v, off, slots, freq, q=q, q_out=out)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.append_rotated(0, k, v, off, slots, freq, q=q, q_out=out)
    for step in range(4):
        c.extend(slots, c.length[slots.long()] + 1, check=True)
        for x in (k, v, q):
            x.normal_()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = c.append_rotated(1, k, v, off, slots, freq, q=q)
        assert torch.equal(got, want)
        for x in (c.k, c.v):
            assert torch.equal(x[0][x[1] != 0], x[1][x[1] != 0])
    assert c.take_status() == []


@pytest.mark.parametrize("first", [None, [0, 5, 90]])
def test_read(first):
    c, slots = filled([40, 17, 100], 8, 3, 72, torch.float16)
    c.k.normal_()
    c.v.normal_()
    counts = [40, 3, 10]
    off = np.concatenate([[0], np.cumsum(counts)])
    wide = torch.full((53, 8, 72), 3.0, device="cuda", dtype=torch.float16)
    k, v = c.read(1, ints(off), slots, 53, first=None if first is None else ints(first), k_out=wide[:, 1:4])
    table, lengths = c.table.cpu(), [40, 17, 100]
    for i, s in enumerate(slots.tolist()):
        a = lengths[i] - counts[i] if first is None else first[i]
        t = torch.arange(a, a + counts[i])
        p, o = table[s][t // 8].long().cuda(), (t % 8).cuda()
        assert torch.equal(k[off[i]:off[i + 1]], c.k[1, p, o]) and torch.equal(v[off[i]:off[i + 1]], c.v[1, p, o])
    assert k.data_ptr() == wide[:, 1:4].data_ptr() and (wide[:, 0] == 3).all() and (wide[:, 4:] == 3).all()
    assert c.take_status() == []


def test_read_of_tokens_that_are_not_there():
    c, slots = filled([10, 20, 20], 8, 1, 64, torch.bfloat16)
    c.k.fill_(1)
    c.v.fill_(1)
    c.table[slots[1].item(), 1] = -5
    k, v = c.read(0, ints([0, 12, 22, 23, 25]), torch.cat([slots[:2], ints([99]), slots[2:]]), 26, first=ints([-1, 2, 0, 18]),
                  k_out=torch.full((26, 1, 64), 9.0, device="cuda", dtype=torch.bfloat16),
                  v_out=torch.full((26, 1, 64), 9.0, device="cuda", dtype=torch.bfloat16))
    want = [0] + [1] * 10 + [0] + [1] * 6 + [0] * 4 + [0] + [1] * 2 + [9]
    for x in (k, v):
        assert x[:, 0, 0].tolist() == want and x.amin(-1).flatten().tolist() == want
    assert set(c.take_status()) == {"slot", "length", "page"}


def test_refusals():
    c, slots = filled([10], 8, 2, 64, torch.bfloat16)
    k = torch.zeros((3, 2, 64), device="cuda", dtype=torch.bfloat16)
    freq, off = torch.ones(32, device="cuda"), ints([0, 3])
    for kw in (dict(freq=torch.ones(33, device="cuda")), dict(freq=torch.ones(4, device="cuda")), dict(layer=2),
               dict(freq=torch.ones(40, device="cuda")), dict(factor=float("nan"))):
        a = {**dict(layer=0, freq=freq, factor=1.0), **kw}
        with pytest.raises(kv.MptError) as e:
            c.append_rotated(a["layer"], k, k, off, slots, a["freq"], factor=a["factor"])
        assert e.value.name == "MPT_E_INVALID"
    for call in (lambda: c.append_rotated(0, k, None, off, slots, freq), lambda: c.append_rotated(0, None, None, off, slots, freq),
                 lambda: c.append_rotated(0, k, k, off, slots, freq.double()),
                 lambda: c.append_rotated(0, k, k, off, slots, freq, q=k[:2]),
                 lambda: c.append_rotated(0, k, k, off, slots, freq, q_out=k),
                 lambda: c.append_rotated(0, k, k, None, None, freq, positions=ints([1, 2, 3])),
                 lambda: c.append_rotated(0, None, None, None, None, freq, q=k),
                 lambda: c.append_rotated(0, k, k, off, slots, freq, positions=ints([1, 2])),
                 lambda: c.append_rotated(0, k.float(), k, off, slots, freq),
                 lambda: c.read(0, off, slots, 3, k_out=k[:2]), lambda: c.read(0, off, slots, 3, v_out=k.float())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(kv.MptError):
        c.read(-1, off, slots, 3)
    wide = torch.zeros((3, 4, 64), device="cuda", dtype=torch.bfloat16)
    with pytest.raises(kv.MptError):                             # in place with other strides
        c.append_rotated(0, None, None, off, slots, freq, q=wide[:, :2], q_out=wide.view(6, 2, 64)[:3])
    assert c.take_status() == []
