"""Caches whose dimensions lie in memory in other orders: layers inside the
pages, keys and values side by side in one buffer, heads outside the slots, gaps
between rows. Every call gives what it gives on the plain order, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2609_13692_amd import kv

pytestmark = pytest.mark.gpu

LAYERS, HEADS = 3, 2


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def plain(pages, page, dim, dtype):
    return [torch.zeros((LAYERS, pages, page, HEADS, dim), dtype=dtype, device="cuda") for _ in range(2)]


def layers_inside_pages(pages, page, dim, dtype):
    return [torch.zeros((pages, LAYERS, page, HEADS, dim), dtype=dtype, device="cuda").transpose(0, 1) for _ in range(2)]


def layers_inside_slots(pages, page, dim, dtype):
    return [torch.zeros((pages, page, LAYERS, HEADS, dim), dtype=dtype, device="cuda").permute(2, 0, 1, 3, 4)
            for _ in range(2)]


def side_by_side_rows(pages, page, dim, dtype):
    x = torch.zeros((LAYERS, pages, page, HEADS, 2, dim), dtype=dtype, device="cuda")
    return [x[..., 0, :], x[..., 1, :]]


def side_by_side_pages(pages, page, dim, dtype):
    x = torch.zeros((pages, LAYERS, 2, HEADS, page, dim), dtype=dtype, device="cuda")
    return [x[:, :, i].permute(1, 0, 3, 2, 4) for i in range(2)]


def gaps(pages, page, dim, dtype):
    x = torch.zeros((LAYERS, pages, page + 1, HEADS + 3, dim + 24), dtype=dtype, device="cuda")
    y = torch.zeros((LAYERS, pages, HEADS, page, dim + 8), dtype=dtype, device="cuda").transpose(2, 3)
    return [x[:, :, :page, 1:1 + HEADS, 16:16 + dim], y[..., :dim]]


ORDERS = [layers_inside_pages, layers_inside_slots, side_by_side_rows, side_by_side_pages, gaps]


def make(order, pages, page, dim, dtype, max_seqs, max_pages):
    k, v = order(pages, page, dim, dtype)
    i32 = dict(dtype=torch.int32, device="cuda")
    c = kv.KvCache(k, v, torch.full((max_seqs, max_pages), -1, **i32), torch.zeros(max_seqs, **i32),
                   torch.zeros(pages, **i32), torch.zeros(-(-pages // 64), dtype=torch.int64, device="cuda"),
                   torch.zeros(1, **i32))
    c.reset()
    return c


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("page,dim", [(1, 64), (4, 128), (16, 256), (64, 80), (128, 128)])
@pytest.mark.parametrize("order", ORDERS, ids=lambda f: f.__name__)
def test_orders(order, page, dim, dtype):
    lengths = [900, 33, 641, 1]
    need = sum(-(-n // page) for n in lengths)
    pages, max_pages = 2 * need + 20, -(-1000 // page)
    caches = [make(f, pages, page, dim, dtype, 6, max_pages) for f in (plain, order)]
    g = torch.Generator(device="cuda").manual_seed(page + dim)
    rows = torch.randn((sum(lengths), 2 * HEADS, dim), device="cuda", generator=g).to(dtype)
    off = np.concatenate([[0], np.cumsum(lengths)])
    q = torch.randn((700, 3 * HEADS, dim), device="cuda", generator=g).to(dtype)
    results = []
    for c in caches:
        # the first pages are used by a sequence that goes, so that pages move
        c.fork(ints([-1]), ints([5]), ints([0]), ints([25]), check=True)
        c.fork(ints([-1] * 4), ints(range(4)), ints([0] * 4), ints(lengths), check=True)
        for layer in range(LAYERS):
            c.append(layer, (1 + layer) * rows[:, :HEADS], rows[:, HEADS:], ints(off), ints(range(4)))
        c.fork(ints([0]), ints([4]), ints([777]), ints([790]), check=True)
        c.free(ints([5, 3]), check=True)
        live = c.compact(check=True)
        c.copy(ints([0]), ints([live]), check=True)
        got = [live, c.k.clone(), c.v.clone(), c.table.clone(), c.ref.clone(), c.free_bits.clone()]
        for layer in range(LAYERS):
            for counts, slots in (([1, 1, 1], [4, 1, 2]), ([300, 20, 130], [0, 4, 2]), ([9, 9], [2, 0])):
                o = ints(np.concatenate([[0], np.cumsum(counts)]))
                got += c.attend(layer, q[:sum(counts)], o, ints(slots))
        assert c.take_status() == []
        results.append(got)
    for x, y in zip(*results):
        assert x == y if isinstance(x, int) else torch.equal(x, y)
