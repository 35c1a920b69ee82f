"""The largest numbers that the paged cache's calls take."""
import pytest
import torch

from paper_2609_13692_amd import kv

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


@pytest.fixture
def room():
    """60 to 80 GB for one test, given back afterwards."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("less than 100 GB of device memory are free")
    yield
    torch.cuda.empty_cache()


def test_append_of_as_many_tokens_as_it_takes(room):
    """2^31 - 1 tokens, the most of a call, of two sequences of 2^30 and 2^30 - 1."""
    lengths, page = [1 << 30, (1 << 30) - 1], 1024
    c = kv.KvCache.create(1, 1 << 21, page, 1, 8, 2, 1 << 30, torch.float16)
    c.fork(ints([-1, -1]), ints([0, 1]), ints([0, 0]), ints(lengths), check=True)
    k, v = (torch.randn((1, 1, 8), device="cuda").half() for _ in range(2))
    total = sum(lengths)
    c.append(0, k.expand(total, 1, 8), v.expand(total, 1, 8), ints([0, lengths[0], total]), ints([0, 1]))
    assert c.take_status() == []
    for x, row in ((c.k, k), (c.v, v)):
        for first in range(0, 1 << 21, 1 << 17):
            same = (x[0, first:first + (1 << 17)] == row[0]).all(-1)
            if first + (1 << 17) == 1 << 21:
                assert not same[-1, -1] and not x[0, -1, -1].any()
                same[-1, -1] = True
            assert same.all()


def test_lists_of_as_many_sequences_as_they_take():
    """2^24 - 1 sequences forked, grown and freed in one call each."""
    n, pages = (1 << 24) - 1, (1 << 25) + 5
    c = kv.KvCache.create(1, pages, 1, 1, 8, n + 3, 2, torch.float16)
    dst = torch.randperm(n + 3, device="cuda", dtype=torch.int32)[:n].contiguous()
    none, one = torch.full((n,), -1, dtype=torch.int32, device="cuda"), torch.ones(n, dtype=torch.int32, device="cuda")
    assert c.fork(none, dst, torch.zeros_like(one), one, check=True) == pages - n
    assert torch.equal(c.table[dst.long(), 0], torch.arange(n, device="cuda", dtype=torch.int32))
    assert c.extend(dst, 2 * one, check=True) == pages - 2 * n
    assert torch.equal(c.table[dst.long(), 1], n + torch.arange(n, device="cuda", dtype=torch.int32))
    assert c.free(dst, one, check=True) == pages - n
    assert torch.equal(c.ref, (torch.arange(pages, device="cuda") < n).int()) and c.take_status() == []


def test_compaction_of_as_many_slots_as_there_can_be(room):
    slots = (1 << 31) - 1
    c = kv.KvCache.create(1, 200, 1, 1, 8, slots, 1, torch.float16)
    c.k.normal_()
    used = [0, 7, 1 << 30, slots - 2, slots - 1]
    c.fork(ints([-1] * 105), ints(list(range(100, 200)) + used), ints([0] * 105), ints([1] * 105), check=True)
    k = c.k.clone()
    c.free(ints(range(100, 200)), check=True)
    assert c.compact(check=True) == 5
    assert [int(c.table[s, 0]) for s in used] == [0, 1, 2, 3, 4] and c.ref.tolist() == [1] * 5 + [0] * 195
    assert torch.equal(c.k[:, :5], k[:, 100:105]) and c.take_status() == []


def test_merge_of_more_rows_than_one_launch_dimension_holds(room):
    """2^27 rows of 256 and some, in place: 2^32 threads and more."""
    rows = (1 << 27) + 9
    x = torch.empty((rows, 256), dtype=torch.bfloat16, device="cuda")
    x.copy_((torch.arange(rows, device="cuda") % 251)[:, None])
    lse = (torch.arange(rows, device="cuda") % 7).float()
    lse[::3] = -float("inf")
    want = lse.clone()
    out, total = kv.merge([x], [lse], out=x, lse=lse)
    assert out is x and torch.equal(total, want)
    for first in range(0, rows, 1 << 23):
        at = torch.arange(first, min(first + (1 << 23), rows), device="cuda")
        assert (out[first:first + (1 << 23)] == torch.where(at % 3 == 0, 0, at % 251)[:, None]).all()
