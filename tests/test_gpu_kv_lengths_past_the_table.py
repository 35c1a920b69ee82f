"""Sequences whose length is more than their table has places for, or negative:
tokens go to their own places, or nowhere, and the length is reported. All
appends and reads, in 16 bits and in 4."""
import numpy as np
import pytest
import torch

from kv_reference import close
from mx4_reference import rotated
from paper_2609_13692_amd import kv
from test_gpu_kv_rotated import bound, frequencies, ints

pytestmark = pytest.mark.gpu
PAGE, PLACES = 4, 16                                   # of the tables below


def cache(bits, length, places=PLACES):
    """Two sequences of 16 tokens (`places` of room), the first of which then says
    that it has `length`; every byte of the pools is the same."""
    c = kv.KvCache.create(1, 20, PAGE, 2, 64, 2, places, bits=bits)
    c.fork(ints([-1, -1]), ints([0, 1]), ints([0, 0]), ints([16, 16]), check=True)
    if places > PLACES:
        c.extend(ints([0]), ints([length]), check=True)
    for x in pools(c):
        x.zero_()
    c.length[0] = length
    return c


def pools(c):
    return [x for x in (c.k, c.v, c.k_scale, c.v_scale) if x is not None]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("rotate", [False, True])
def test_newest_tokens_keep_their_places(bits, rotate):
    """Six tokens of a sequence of 18 in a table of 16 places: 12 to 15 are written,
    where a larger table has them, and 16 and 17 are not."""
    k, v, q = (torch.randn((6, 2, 64), device="cuda").bfloat16() for _ in range(3))
    freq = torch.tensor(frequencies(64), device="cuda")
    held = []
    for places in (PLACES, 40):
        c = cache(bits, 18, places)
        before = [x.clone() for x in pools(c)]
        if rotate:
            c.append_rotated(0, k, v, ints([0, 6]), ints([0]), freq, q=q)
        else:
            c.append(0, k, v, ints([0, 6]), ints([0]))
        assert c.take_status() == (["length"] if places == PLACES else [])
        written = {(c.table[0, p // PAGE].item(), p % PAGE) for p in range(12, 16 if places == PLACES else 18)}
        for x, old in zip(pools(c), before):
            changed = (x != old).any(-1).any(-1)[0]
            assert set(map(tuple, changed.nonzero().tolist())) <= written
        held.append(c.read(0, ints([0, 4]), ints([0]), 4, first=ints([12])))
        assert c.take_status() == []
    for a, b in zip(*held):
        assert torch.equal(a, b) and (a != 0).any()


@pytest.mark.parametrize("bits", [16, 4])
def test_newest_tokens_are_read_from_their_places(bits):
    """The newest six of 18 are tokens 12 to 15, and two that are not there."""
    c = cache(bits, 16)
    k, v = (torch.randn((16, 2, 64), device="cuda").bfloat16() for _ in range(2))
    c.append(0, k, v, ints([0, 16]), ints([0]))
    whole = c.read(0, ints([0, 16]), ints([0]), 16)
    assert c.take_status() == []
    c.length[0] = 18
    for first in (None, ints([12])):
        got = c.read(0, ints([0, 6]), ints([0]), 6, first=first)
        assert c.take_status() == ["length"]
        for x, y in zip(got, whole):
            assert torch.equal(x[:4], y[12:]) and (x[4:] == 0).all()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("length", [18, 2 ** 31 - 1, 0, -3])
def test_queries_turn_to_their_places(bits, length):
    """Token j of the n newest stands at length - n + j, whether or not there is
    such a place in the table."""
    c = cache(bits, length)
    before = [x.clone() for x in pools(c)]
    q = torch.randn((6, 2, 64), device="cuda").bfloat16()
    freq = frequencies(64)
    pos = np.arange(length - 6, length)
    x = q.double().cpu().numpy()
    y = rotated(x, pos, freq)
    off, slots = ints([0, 6]), ints([0])
    for k in (None, torch.randn((6, 2, 64), device="cuda").bfloat16()):
        got = c.append_rotated(0, k, k, off, slots, torch.tensor(freq, device="cuda"), q=q)
        close(got.double().cpu().numpy(), y, bound(x, y, freq, torch.bfloat16, False), "queries")
        assert c.take_status() == ([] if k is None else ["length"])
    if length != 18:
        for x, old in zip(pools(c), before):
            assert torch.equal(x, old)
