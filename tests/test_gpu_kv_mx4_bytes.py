"""Attention over caches in 4 bits whose bytes E appends never write, and whose
bytes E lie past 4 GiB: what it sees is what reads return, in the kernel of few
rows and in that of many."""
import math

import numpy as np
import pytest
import torch

from kv_reference import attention, attention_bounds, close
from paper_2609_13692_amd import kv
from test_gpu_kv_attention import DT, ints
from test_gpu_kv_mx4_attention import filled, set_byte

pytestmark = pytest.mark.gpu
TOP = {torch.bfloat16: 252, torch.float16: 140}           # the largest byte that is a number
BYTES = [0, 1, 2, 3, 50, 103, 104, 105, 126, 127, 128, 139, 140, 141, 142, 200, 250, 251, 252, 253, 254, 255]


def one_of_each_byte(name, dtype, dim):
    """A sequence of a token per byte, which all blocks of its keys (or values) have;
    its values (keys) have E = 127. And what reads return."""
    c, slots, _, _ = filled([len(BYTES)], 8, 1, dim, dtype, 21)
    for t, byte in enumerate(BYTES):
        for block in range(dim // 32):
            set_byte(c, "k_scale", slots.item(), t, 0, block, byte if name == "k" else 127)
            set_byte(c, "v_scale", slots.item(), t, 0, block, byte if name == "v" else 127)
    k, v = (x.double().cpu().numpy() for x in c.read(1, ints([0, len(BYTES)]), slots, len(BYTES)))
    for t, byte in enumerate(BYTES):
        for x, odd in ((k, name == "k"), (v, name == "v")):
            assert (np.isnan(x[t]) == (odd and byte > TOP[dtype])).all()
    return c, slots, k, v


def only(c, slots, t, q):
    """Attention that sees token t alone."""
    c.length[slots.item()] = t + 1
    out = c.attend(1, q.cuda(), ints([0, len(q)]), slots, causal=False, kv_begin=ints([t]), out_dtype=torch.float32)
    return [x.double().cpu().numpy() for x in out]


@pytest.mark.parametrize("count", [1, 70])
@pytest.mark.parametrize("dim", [32, 96, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_values_of_every_kind_of_byte(dtype, dim, count):
    """A row that sees one token returns its value. The weight that the product gets
    is 1 in 16 bits; the sum that it is divided by is one exponential of what m =
    lse log2(e) leaves when it is rounded (2^-24 lse), and that, its inverse and
    the product are off by 2^-22 at most together. Bfloat16's numbers below its
    smallest normal one, 2^-126, may be zeros, as they may in reads."""
    dtype = DT[dtype]
    c, slots, k, v = one_of_each_byte("v", dtype, dim)
    q = torch.randn((count, 2, dim), generator=torch.Generator().manual_seed(22)).to(dtype)
    for t, byte in enumerate(BYTES):
        out, lse = only(c, slots, t, q)
        want = np.broadcast_to(v[t, 0], out.shape)
        limit = (2.0 ** -24 * np.abs(lse[..., None]) + 2.0 ** -22) * np.abs(want)
        if dtype is torch.bfloat16:
            limit = np.where(np.abs(want) < 2.0 ** -126, 2.0 ** -126, limit)
        close(out, want, limit, f"value of byte {byte}")
        assert np.isfinite(lse).all()
    assert c.take_status() == []


@pytest.mark.parametrize("count", [1, 70])
@pytest.mark.parametrize("dim", [32, 96, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_keys_of_every_kind_of_byte(dtype, dim, count):
    """The logarithm of one weight is its score, of queries that make it one of a
    usual size. Bytes whose halves are below the smallest normal number of
    bfloat16 get no such queries: their keys may be zeros."""
    dtype = DT[dtype]
    c, slots, k, v = one_of_each_byte("k", dtype, dim)
    base = torch.randn((count, 2, dim), generator=torch.Generator().manual_seed(23))
    for t, byte in enumerate(BYTES):
        power = min(max(127 - byte, -13), 12) if dtype is torch.float16 else 0 if byte < 2 else 127 - byte
        q = (base * 2.0 ** power).to(dtype)
        out, lse = only(c, slots, t, q)
        if byte > TOP[dtype]:
            assert np.isnan(out).all() and np.isnan(lse).all()
            continue
        ref = attention(q.double().numpy(), k[t:t + 1], v[t:t + 1], 0, causal=False)
        bo, bl = attention_bounds(*ref, 1, dim, dtype, torch.float32)
        close(lse, ref[1], bl, f"score of byte {byte}")
        close(out, ref[0], bo, f"output under byte {byte}")
        if (dtype is torch.bfloat16 and byte >= 2) or byte >= 115:
            assert np.abs(ref[1]).max() > 2.0 ** -8           # what is compared is no rounding
    assert c.take_status() == []


@pytest.mark.parametrize("count", [1, 3, 100])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_bytes_above_the_range_reach_who_sees_them(dtype, dim, count):
    """Such a byte of a key makes rows NaN that see it, one of a value its 32
    dimensions; no other row, head or dimension changes."""
    dtype, length = DT[dtype], 150
    c, slots, _, _ = filled([length, 60], 16, 2, dim, dtype, 24)
    q = (torch.randn((count + 1, 4, dim), generator=torch.Generator().manual_seed(25)) * 1.5).to(dtype).cuda()
    off, slot = ints([0, count, count + 1]), slots[0].item()
    clean, clean_lse = c.attend(1, q, off, slots)
    for byte in (TOP[dtype] + 1, (TOP[dtype] + 256) // 2, 254, 255):
        for name, t, head, block in (("v", length - 1, 0, 0), ("v", length - 1 - count // 2, 1, dim // 32 - 1),
                                     ("k", length - 1 - count // 3, 1, 1), ("v", 3, 1, 0), ("k", 0, 0, dim // 32 - 1)):
            old = getattr(c, name + "_scale").clone()
            set_byte(c, name + "_scale", slot, t, head, block, byte)
            out, lse = c.attend(1, q, off, slots)
            want, want_lse = clean.clone(), clean_lse.clone()
            for j in range(max(0, t - (length - count)), count):
                rows = slice(2 * head, 2 * head + 2)
                if name == "v":
                    want[j, rows, 32 * block:32 * block + 32] = math.nan
                else:
                    want[j, rows], want_lse[j, rows] = math.nan, math.nan
            for a, b in ((out, want), (lse, want_lse)):
                assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a[~b.isnan()], b[~b.isnan()]), (byte, name, t, head, block)
            getattr(c, name + "_scale").copy_(old)
    assert c.take_status() == []


def test_bytes_past_four_gigabytes():
    """Scales a MiB apart from page to page, in two layers: those of pages from 4096
    on, and all of the second layer, lie past 32 bits of offset. Appends, reads, both
    attention kernels, a NaN, forks off partial pages, compaction and copies."""
    pages, page, heads, dim, filler, length = 4500, 16, 2, 64, 4300, 2395
    row, gap = dim // 32, 1 << 20
    raw = torch.full((2 * pages * gap,), 255, dtype=torch.uint8, device="cuda")
    shape, stride = (2, pages, page, heads, row), (pages * gap, gap, heads * row, row, 1)
    ke, ve = raw.as_strided(shape, stride), raw.as_strided(shape, stride, gap // 2)
    k, v = (torch.zeros((2, pages, page, heads, dim // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    i32 = dict(dtype=torch.int32, device="cuda")
    c = kv.KvCache(k, v, torch.full((3, pages), -1, **i32), torch.zeros(3, **i32), torch.zeros(pages, **i32),
                   torch.zeros(-(-pages // 64), dtype=torch.int64, device="cuda"), torch.zeros(1, **i32), ke, ve, torch.bfloat16)
    c.reset()
    c.fork(ints([-1, -1]), ints([2, 0]), ints([0, 0]), ints([filler * page, length]), check=True)
    first = c.table[0, 0].item()
    assert first * gap > 1 << 32
    small = kv.KvCache.create(2, 200, page, heads, dim, 3, 2500, bits=4)       # the same, in order
    small.fork(ints([-1]), ints([0]), ints([0]), ints([length]), check=True)
    g = torch.Generator("cuda").manual_seed(26)
    freq = 1000.0 ** (torch.arange(32, device="cuda") / -32)
    for layer in range(2):
        x, y = (torch.empty((length, heads, dim), device="cuda").normal_(generator=g).bfloat16() for _ in range(2))
        for to in (c, small):
            to.append_rotated(layer, x, y, ints([0, length]), ints([0]), freq)

    def compare(slots=(0,), nan=()):
        """Both caches, all layers; nan: those where a value is NaN."""
        for layer in range(2):
            n = [c.length[s].item() for s in slots]
            off = ints(np.concatenate([[0], np.cumsum(n)]))
            got, want = (x.read(layer, off, ints(slots), sum(n)) for x in (c, small))
            for a, b in zip(got, want):
                assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) and torch.equal(a.isnan(), b.isnan())
            assert got[1].isnan().any().item() == (layer in nan)
            for count in (1, 60):
                q = torch.empty((count * len(n), 4, dim), device="cuda").normal_(generator=g).bfloat16()
                cut = ints(count * i for i in range(len(n) + 1))
                got, want = (x.attend(layer, q, cut, ints(slots)) for x in (c, small))
                for a, b in zip(got, want):
                    assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) and torch.equal(a.isnan(), b.isnan())
                assert got[0].isnan().any().item() == (layer in nan)
    compare()
    kept = []
    for x in (c, small):
        at = (1, x.table[0, 140].item(), 5, 1, 0)
        kept.append((x.v_scale, at, x.v_scale[at].item()))
        x.v_scale[at] = 255
    compare(nan=(1,))
    for scales, at, byte in kept:
        scales[at] = byte
    for x in (c, small):                                       # a fork off a partial page, whose bytes are copied
        x.fork(ints([0]), ints([1]), ints([length - 3]), ints([length - 3]), check=True)
    compare((0, 1))
    assert c.table[1, length // page] != c.table[0, length // page]
    page_ids = ints([first + 1]), ints([0])
    c.copy(*page_ids, check=True)
    for x in (ke, ve):
        assert torch.equal(x[:, 0], x[:, first + 1])
    c.free(ints([2]), check=True)
    c.compact(check=True)
    assert c.table[0, 0] < 200
    compare((0, 1))
    assert c.take_status() == small.take_status() == []
