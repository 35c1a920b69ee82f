"""Caches in 4 bits whose callers lay them out, fill them or order their calls in
other ways: bytes E that appends never write, pools with layers inside pages and
gaps between rows, work on another stream, graphs that share a cache, and the
place of a token in the middle of a cut."""
import numpy as np
import pytest
import torch

from kv_reference import close
from mx4_reference import from_codes, rotated
from paper_2609_13692_amd import kv
from test_gpu_kv_attention import DT, check, ints
from test_gpu_kv_mx4_attention import filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_exponent_byte(dtype):
    """Of a key's, a value's and a read row's 32 elements: every E. Bytes above
    the range of the 16-bit type's values are NaN, bytes below it are values that
    the type rounds (to zero, or to its smallest numbers)."""
    dtype = DT[dtype]
    c, slots, _, _ = filled([256], 16, 1, 32, dtype, 3)
    slot = int(slots[0])
    g = torch.Generator().manual_seed(4)
    codes = torch.randint(0, 256, (256, 16), generator=g, dtype=torch.uint8)
    pages = c.table[slot, :16].tolist()
    for t in range(256):
        for x, e in ((c.k, c.k_scale), (c.v, c.v_scale)):
            x[1, pages[t // 16], t % 16, 0] = codes[t].cuda()
            e[1, pages[t // 16], t % 16, 0] = t
    k, v = (x[:, 0].double().cpu().numpy() for x in c.read(1, ints([0, 256]), slots, 256))
    want = from_codes(codes.numpy(), np.arange(256)[:, None])
    top = 252 if dtype == torch.bfloat16 else 140
    # What a value below the written range may be off by. float16's numbers below
    # 2^-14 are 2^-24 apart: the nearest is off by at most 2^-25, and by nothing
    # from E - 127 = -23 on, where halves of 2^-23 are multiples of 2^-24.
    # bfloat16: numbers below its smallest normal one, 2^-126, may be zeros.
    e = np.arange(top + 1)[:, None]
    if dtype == torch.float16:
        limit = np.where(e >= 104, 0.0, 2.0 ** -25) + 0.0 * want[:top + 1]
    else:
        limit = np.where(np.abs(want[:top + 1]) < 2.0 ** -126, 2.0 ** -126, 0.0)
    for got in (k, v):
        assert np.isnan(got[top + 1:]).all() and not np.isnan(got[:top + 1]).any()
        close(got[:top + 1], want[:top + 1], limit, "values")
    # attention over one token at a time sees what reads see
    q = torch.randn((1, 1, 32), generator=g).to(dtype).cuda()
    for t in (0, 1, top - 1, top, top + 1, 254, 255):
        out, _ = c.attend(1, q, ints([0, 1]), slots, causal=False, kv_begin=ints([t]))
        if t > top:
            assert torch.isnan(out).all()
    c.k_scale[1].fill_(120)                                # keys that can be weighted
    for t in (255, top + 1, top, 127, 104):
        c.free(slots, ints([t + 1]))
        out, _ = c.attend(1, q, ints([0, 1]), slots, kv_begin=ints([t]), out_dtype=torch.float32)
        got = out[0, 0].double().cpu().numpy()
        if t > top:
            assert np.isnan(got).all()
        else:
            close(got, want[t], 2.0 ** -22 * np.abs(want[t]), "the only token's value")


def layers_inside(n_layers, n_pages, page, heads, dim, gap):
    """Pools [pages, slots, layers, heads + gap, row] seen as [layers, pages, slots, heads, row]."""
    def pool(row):
        x = torch.full((n_pages, page, n_layers, heads + gap, row), 0x5a, dtype=torch.uint8, device="cuda")
        return x, x.permute(2, 0, 1, 3, 4)[:, :, :, :heads]
    return [pool(r) for r in (dim // 2, dim // 2, dim // 32, dim // 32)]


@pytest.mark.parametrize("dim,page", [(32, 4), (96, 16), (128, 1)])
def test_layers_inside_pages_and_gaps(dim, page):
    """Strides in another order, rows of other owners between: those stay."""
    heads, lengths, n_pages = 2, [70, 5, 33], 140
    pools = layers_inside(2, n_pages, page, heads, dim, 1)
    k, v, ke, ve = (view for _, view in pools)
    i32 = dict(dtype=torch.int32, device="cuda")
    c = kv.KvCache(k, v, torch.full((4, -(-100 // page)), -1, **i32), torch.zeros(4, **i32), torch.zeros(n_pages, **i32),
                   torch.zeros(-(-n_pages // 64), dtype=torch.int64, device="cuda"), torch.zeros(1, **i32), ke, ve, torch.bfloat16)
    c.reset()
    slots = ints([2, 0, 3])
    c.fork(ints([-1] * 3), slots, ints([0] * 3), ints(lengths), check=True)
    g = torch.Generator().manual_seed(5)
    off = np.concatenate([[0], np.cumsum(lengths)])
    new = [[torch.randn((108, heads, dim), generator=g).bfloat16().cuda() for _ in range(2)] for _ in range(2)]
    for layer in range(2):
        c.append(layer, *new[layer], ints(off), slots)
    c.free(ints([0]))
    c.compact(check=True)
    c.fork(ints([2]), ints([1]), ints([31]), ints([40]), check=True)             # copies a page's part where it is cut
    for layer in range(2):
        x = [t[:9] for t in new[layer]]
        c.append(layer, *x, ints([0, 9]), ints([1]))
    assert c.take_status() == []
    for raw, _ in pools:
        assert (raw[:, :, :, heads:] == 0x5a).all()
    def back(layer, x, which):                             # through a cache in order, whose codes are tested by themselves
        other = kv.KvCache.create(1, 200, 16, heads, dim, 1, 200, bits=4)
        other.fork(ints([-1]), ints([0]), ints([0]), ints([len(x)]), check=True)
        other.append(0, x, x, ints([0, len(x)]), ints([0]))
        return other.read(0, ints([0, len(x)]), ints([0]), len(x))[0]
    for layer in range(2):
        got = c.read(layer, ints([0, 70, 110, 143]), ints([2, 1, 3]), 143)
        ks, vs = [], []
        for which in range(2):
            x = new[layer][which]
            parts = [x[:70], torch.cat([x[:31], x[:9]]), x[75:108]]
            want = [back(layer, p, which) for p in parts]
            assert torch.equal(got[which], torch.cat(want))
            (vs if which else ks).extend(w.double().cpu().numpy() for w in want)
        if layer == 1:
            check(c, ints([2, 1, 3]), ks, vs, [1, 1, 1], 4, 6, torch.bfloat16)
            check(c, ints([2, 1, 3]), ks, vs, [60, 40, 33], 14, 7, torch.bfloat16)


def test_another_stream():
    """A step on a stream of its own, behind work on the current one."""
    c, slots, ks, vs = filled([200, 77], 16, 2, 64, torch.bfloat16, 11)
    side = torch.cuda.Stream()
    g = torch.Generator().manual_seed(12)
    q = torch.randn((2, 8, 64), generator=g).bfloat16().cuda()
    k, v = (torch.randn((2, 2, 64), generator=g).bfloat16().cuda() for _ in range(2))
    freq = 100.0 ** (torch.arange(32, device="cuda") / -32)
    lists = ints([0, 1, 2]), ints([201, 78]), ints([0, 201, 279])
    def step(**how):
        c.extend(slots, lists[1], **how)
        turned = c.append_rotated(1, k, v, lists[0], slots, freq, q=q, **how)
        out, lse = c.attend(1, turned, lists[0], slots, **how)
        return [turned, out, lse, *c.read(1, lists[2], slots, 279, **how)]
    want = [x.clone() for x in step()]
    c.free(slots, ints([200, 77]))
    big = torch.randn((4096, 4096), device="cuda")
    big = big @ big                                        # the current stream is busy meanwhile
    side.wait_stream(torch.cuda.current_stream())
    got = step(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert c.take_status() == []


def test_graphs_that_share_a_cache():
    """Two captured calls of different sizes over one cache, whose lengths and
    contents change between their replays."""
    c, slots, ks, vs = filled([150, 90, 40], 16, 2, 64, torch.bfloat16, 13)
    g = torch.Generator().manual_seed(14)
    q1 = torch.randn((3, 8, 64), generator=g).bfloat16().cuda()
    q2 = torch.randn((60, 8, 64), generator=g).bfloat16().cuda()
    one, off, k, v = ints([0, 1, 2, 3]), ints([0, 20, 40, 60]), *(torch.randn((60, 2, 64), generator=g).bfloat16().cuda() for _ in range(2))
    freq = 100.0 ** (torch.arange(16, device="cuda") / -16)
    def decode():
        return c.attend(1, q1, one, slots)
    def chunk():
        turned = c.append_rotated(1, k, v, off, slots, freq, q=q2)
        return (*c.attend(1, turned, off, slots), *c.read(1, off, slots, 60))
    decode(), chunk()
    graphs = []
    for call in (decode, chunk):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        graphs.append((graph, got, call))
    for turn in range(4):
        k.normal_(generator=torch.Generator("cuda").manual_seed(turn))
        if turn == 2:
            c.free(slots, ints([70, 88, 25]))
        for graph, got, call in (graphs[::-1] if turn % 2 else graphs):
            for x in got:
                x.fill_(77)
            graph.replay()
            torch.cuda.synchronize()
            held = [x.clone() for x in got]
            for a, b in zip(held, call()):
                assert torch.equal(a, b)
    assert c.take_status() == []


def test_a_token_rotated_alone_is_the_token_of_the_chunk():
    """Chunks and single tokens at the same positions: the same bytes, and the
    same as the definition for the keys that come back."""
    rows = 37
    g = torch.Generator().manual_seed(15)
    k, v = (torch.randn((rows, 4, 128), generator=g).bfloat16().cuda() for _ in range(2))
    freq = 10000.0 ** (torch.arange(64, device="cuda") / -64)
    pair = []
    for cuts in ([rows], [1] * rows):
        c = kv.KvCache.create(1, 80, 4, 4, 128, 1, 80, bits=4)
        c.fork(ints([-1]), ints([0]), ints([0]), ints([0]), check=True)
        at = 0
        for n in cuts:
            c.extend(ints([0]), ints([at + n]), check=True)
            c.append_rotated(0, k[at:at + n], v[at:at + n], ints([0, n]), ints([0]), freq)
            at += n
        pair.append(c.read(0, ints([0, rows]), ints([0]), rows))
    for a, b in zip(*pair):
        assert torch.equal(a, b)
    want = rotated(k.double().cpu().numpy(), range(rows), freq.cpu().numpy())
    top = np.abs(want).reshape(rows, 4, 4, 32).max(-1)
    close(pair[0][0].double().cpu().numpy(), want, np.repeat(top, 32, -1).reshape(want.shape) / 3.5 + 2.0 ** -18, "keys")


def test_the_whole_range_of_lengths_in_one_call():
    """One token to thousands, none, and counts of none, in one call each way."""
    lengths = [1, 5000, 0, 2, 16, 17, 333, 1200]
    c, slots, ks, vs = filled(lengths, 16, 1, 64, torch.float16, 16)
    check(c, slots, ks, vs, [1, 1, 0, 1, 0, 1, 1, 1], 4, 17, torch.float16)
    check(c, slots, ks, vs, [1, 300, 0, 2, 0, 17, 33, 1], 4, 18, torch.float16)


def test_rotations_past_the_range():
    """Rotated keys that 32 bits do not hold are infinite, and so NaN in 4 bits; those
    that the 16-bit type alone does not hold are as large as codes get."""
    freq = torch.full((16,), np.pi / 4, device="cuda")
    for dtype, big in ((torch.bfloat16, 3.0e38), (torch.float16, 60000.0)):
        c = kv.KvCache.create(1, 4, 16, 1, 32, 1, 16, dtype, bits=4)
        c.fork(ints([-1]), ints([0]), ints([0]), ints([2]), check=True)
        k = torch.full((2, 1, 32), big, dtype=dtype, device="cuda")
        k[1] = 1.0
        c.append_rotated(0, k, k, ints([0, 2]), ints([0]), freq, positions=ints([1, 1]))
        got, v = c.read(0, ints([0, 2]), ints([0]), 2)
        if dtype is torch.bfloat16:
            assert torch.isnan(got[0]).all()
        else:
            assert (got[0, 0, :16] == 0).all() and (got[0, 0, 16:] == 6 * 2.0 ** 13).all()
        assert torch.isfinite(got[1]).all() and torch.isfinite(v).all()
    assert c.take_status() == []
