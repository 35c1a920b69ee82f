"""The largest numbers that rotated appends, caches in 4 bits and reads take."""
import pytest
import torch

from paper_2609_13692_amd import kv

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


@pytest.fixture
def room():
    """75 GB for one test, given back afterwards."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("less than 100 GB of device memory are free")
    yield
    torch.cuda.empty_cache()


def test_append_of_as_many_tokens_as_it_takes(room):
    """2^31 - 1 tokens of two sequences into 4 bits, rotated to their positions; some
    of all parts are those that a small cache has at the same positions."""
    lengths, page, dim = [1 << 30, (1 << 30) - 1], 1024, 32
    c = kv.KvCache.create(1, 1 << 21, page, 1, dim, 2, 1 << 30, torch.bfloat16, bits=4)
    c.fork(ints([-1, -1]), ints([0, 1]), ints([0, 0]), ints(lengths), check=True)
    k, v = (torch.randn((1, 1, dim), device="cuda").bfloat16() for _ in range(2))
    freq = 100.0 ** (torch.arange(8, device="cuda") / -8)
    total = sum(lengths)
    c.append_rotated(0, k.expand(total, 1, dim), v.expand(total, 1, dim), ints([0, lengths[0], total]), ints([0, 1]), freq)
    assert c.take_status() == []
    assert (c.v_scale.view(-1)[:total:4097] == c.v_scale.view(-1)[0]).all()
    small = kv.KvCache.create(1, 5, 16, 1, dim, 1, 80, torch.bfloat16, bits=4)
    small.fork(ints([-1]), ints([0]), ints([0]), ints([70]), check=True)
    for slot in (0, 1):
        for first in (0, 1000, (1 << 24) - 30, (1 << 29) + 12345, lengths[slot] - 70):
            small.append_rotated(0, k.expand(70, 1, dim), v.expand(70, 1, dim), ints([0, 70]), ints([0]), freq,
                                 positions=ints(range(first, first + 70)))
            got = c.read(0, ints([0, 70]), ints([slot]), 70, first=ints([first]))
            want = small.read(0, ints([0, 70]), ints([0]), 70)
            for a, b in zip(got, want):
                assert torch.equal(a, b) and a.any(), (slot, first)
    assert c.take_status() == [] and small.take_status() == []


def test_queries_of_as_many_tokens_as_it_takes(room):
    """2^31 - 1 rows of queries alone, every one at the position that it is given
    (which they share), in place of rows that they share: nothing else is written."""
    c = kv.KvCache.create(1, 1, 1, 1, 16, 1, 1, torch.bfloat16)
    total = (1 << 31) - 1
    freq = torch.full((8,), 0.5, device="cuda")
    positions = torch.full((total,), 3, dtype=torch.int32, device="cuda")
    q = torch.randn((1, 1, 16), device="cuda").bfloat16()
    out = torch.zeros((3, 1, 16), device="cuda", dtype=torch.bfloat16)
    c.append_rotated(0, None, None, None, None, freq, q=q.expand(total, 1, 16), q_out=out[1:2].expand(total, 1, 16),
                     positions=positions)
    want = c.append_rotated(0, None, None, None, None, freq, q=q, positions=ints([3]))
    assert torch.equal(out[1:2], want) and not out[0].any() and not out[2].any()
    assert c.take_status() == []
