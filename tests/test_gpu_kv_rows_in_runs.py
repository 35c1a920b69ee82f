"""Rotated appends and reads whose waves take several tokens each, or lanes the
pieces of several tokens: the bytes of calls over few tokens, which other tests hold
against the definition, and of plain indexing."""
import pytest
import torch

from paper_2609_13692_amd import kv

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("tokens", [40000, 270001])
@pytest.mark.parametrize("heads,q_heads,dim,rot,neighbours,bits", [
    (1, 2, 32, 16, False, 16), (2, 3, 32, 32, True, 16), (1, 1, 64, 48, False, 16), (1, 2, 160, 160, False, 16),
    (1, 2, 32, 16, True, 4), (2, 1, 64, 48, False, 4), (1, 1, 160, 160, True, 4)])
def test_one_call_is_many(tokens, heads, q_heads, dim, rot, neighbours, bits):
    """Three sequences' tokens in one call, and in calls of 5000 at most."""
    g = torch.Generator("cuda").manual_seed(tokens + dim)
    k, v = (torch.empty((tokens, heads, dim), device="cuda").normal_(generator=g).bfloat16() for _ in range(2))
    q = torch.empty((tokens, q_heads, dim), device="cuda").normal_(generator=g).bfloat16()
    freq = 1000.0 ** (torch.arange(rot // 2, device="cuda") / (-rot // 2))
    cuts = [0, 7, tokens // 3, tokens]
    counts = [b - a for a, b in zip(cuts, cuts[1:])]
    def cache():
        return kv.KvCache.create(1, sum(-(-n // 16) for n in counts), 16, heads, dim, 3, max(counts), bits=bits)
    one, many = cache(), cache()
    slots = ints([1, 2, 0])
    one.fork(ints([-1] * 3), slots, ints([0] * 3), ints(counts), check=True)
    got = one.append_rotated(0, k, v, ints(cuts), slots, freq, q=q, interleaved=neighbours)
    want = torch.empty_like(q)
    for slot, a, n in zip([1, 2, 0], cuts, counts):
        for first in range(0, n, 5000):
            last = min(first + 5000, n)
            many.extend(ints([slot]), ints([last]))
            part = slice(a + first, a + last)
            many.append_rotated(0, k[part], v[part], ints([0, last - first]), ints([slot]), freq, q=q[part], q_out=want[part],
                                interleaved=neighbours)
    assert torch.equal(got, want)
    whole = one.read(0, ints(cuts), slots, tokens)
    for slot, a, n in zip([1, 2, 0], cuts, counts):
        for first in range(0, n, 5000):
            last = min(first + 5000, n)
            part = many.read(0, ints([0, last - first]), ints([slot]), last - first, first=ints([first]))
            for x, y in zip(whole, part):
                assert torch.equal(x[a + first:a + last], y)
    if bits == 16:
        assert torch.equal(whole[1], v)
    assert one.take_status() == [] and many.take_status() == []


@pytest.mark.parametrize("tokens", [1, 63, 300, 60000])
@pytest.mark.parametrize("heads,dim", [(1, 8), (3, 8), (1, 24), (1, 64), (4, 64), (5, 56), (1, 256), (2, 136), (8, 128)])
@pytest.mark.parametrize("heads_first", [False, True])
def test_read_is_indexing(heads, dim, tokens, heads_first):
    """Pieces of a token: 1 to 128. Rows before the first offset and past the last stay,
    tokens that are not there are zeros; outputs lie in wider rows."""
    g = torch.Generator("cuda").manual_seed(heads * dim + tokens)
    lengths = [tokens, 40, tokens // 2 + 1]
    pages = [-(-n // 8) for n in lengths]
    c = kv.KvCache.create(2, sum(pages), 8, heads, dim, 3, max(lengths) + 8, heads_first=heads_first)
    c.fork(ints([-1] * 3), ints([0, 1, 2]), ints([0] * 3), ints(lengths), check=True)
    for x in (c.k, c.v):
        x.normal_(generator=g)
    off, first = [2, 2 + tokens, 2 + tokens + 50], [0, 20]
    total = off[-1] + 3
    wide = torch.full((2, total, heads + 1, dim + 8), 7.0, device="cuda", dtype=torch.bfloat16)
    out = [w[:, 1:, :dim] for w in wide]
    c.read(1, ints(off), ints([0, 1]), total, first=ints(first), k_out=out[0], v_out=out[1])
    assert c.take_status() == ["slot", "length"]
    for x, y in zip((c.k, c.v), out):
        want = torch.full((total, heads, dim), 7.0, device="cuda", dtype=torch.bfloat16)
        for slot, a, b, f in zip([0, 1], off, off[1:], first):
            t = torch.arange(f, f + b - a, device="cuda")
            there = t < lengths[slot]
            page = c.table[slot, t.clamp(max=lengths[slot] - 1) // 8].long()
            want[a:b] = torch.where(there[:, None, None], x[1, page, t % 8], torch.zeros_like(want[a:b]))
        assert torch.equal(y, want)
    assert (wide[:, :, 0] == 7).all() and (wide[:, :, :, dim:] == 7).all()
