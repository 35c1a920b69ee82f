"""Page ids in tables that are no pages of the pool, or pages without
references: the page calls find them before they change anything, say so in
the status, and to a caller that asks."""
import pytest
import torch

from paper_2609_13692_amd import kv

pytestmark = pytest.mark.gpu

N_PAGES, PAGE = 90, 4


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


# tables short enough for checks inside the plan, and long ones
@pytest.fixture(params=[80, 40000], ids=["short", "long"])
def cache(request):
    c = kv.KvCache.create(2, N_PAGES, PAGE, 2, 16, 6, request.param)
    c.k.normal_()
    c.v.normal_()
    c.fork(ints([-1, -1, -1]), ints([0, 2, 5]), ints([0, 0, 0]), ints([70, 19, 30]), check=True)
    c.fork(ints([0]), ints([1]), ints([30]), ints([41]), check=True)
    c.free(ints([5]), check=True)
    return c


# no page, the first past the pool, far past it, and a page that is free
BAD = [-1, N_PAGES, 1 << 30, -(1 << 31), N_PAGES - 1]


def refused(c, call, *args):
    state = (c.k, c.v, c.table, c.length, c.ref, c.free_bits)
    before = [x.clone() for x in state]
    assert c.take_status() == []
    with pytest.raises(kv.MptError) as e:
        call(*args, check=True)
    assert e.value.name == "MPT_E_RANGE"
    assert c.take_status() == ["page"]
    call(*args)                                    # unasked: the same, and no exception
    assert c.take_status() == ["page"]
    for x, y in zip(before, state):
        assert torch.equal(x, y)


@pytest.mark.parametrize("bad", BAD)
def test_fork_that_copies_from_a_bad_page(cache, bad):
    cache.table[2, 4] = bad                        # tokens 16 .. 18
    refused(cache, cache.fork, ints([0, 2]), ints([3, 4]), ints([8, 18]), ints([20, 18]))


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("at", [0, 3])
def test_fork_that_shares_a_bad_page(cache, at, bad):
    cache.table[2, at] = bad
    refused(cache, cache.fork, ints([0, 2]), ints([3, 4]), ints([8, 16]), ints([20, 18]))
    # pages past those that are kept do not matter
    cache.fork(ints([2]), ints([3]), ints([4 * at]), ints([4 * at + 1]), check=True)
    assert cache.take_status() == []


@pytest.mark.parametrize("bad", BAD)
def test_growth_of_a_bad_page(cache, bad):
    cache.table[2, 4] = bad
    refused(cache, cache.extend, ints([0, 2]), ints([78, 20]))
    cache.extend(ints([0, 2]), ints([78, 19]), check=True)     # as long as it was: nothing is read
    assert cache.take_status() == []


@pytest.mark.parametrize("bad", BAD)
def test_free_of_a_bad_page(cache, bad):
    cache.table[2, 2] = bad
    refused(cache, cache.free, ints([0, 2]))
    refused(cache, cache.free, ints([0, 2]), ints([30, 8]))
    cache.free(ints([0, 2]), ints([30, 9]), check=True)        # the bad one is kept
    assert cache.take_status() == []


def test_a_page_loses_no_reference_that_it_does_not_have(cache):
    """Two tables list a page that counts one reference."""
    cache.table[2, 0] = cache.table[0, 17]
    cache.free(ints([0, 2]))
    assert cache.take_status() == ["page"]
    ref = cache.ref.tolist()
    assert min(ref) == 0
    free = [(int(cache.free_bits[p // 64]) >> p % 64) & 1 for p in range(N_PAGES)]
    assert free == [int(r == 0) for r in ref]


@pytest.mark.parametrize("bad", BAD + [1])
def test_compaction_of_a_bad_page(cache, bad):
    cache.free(ints([0]), ints([41]), check=True)
    cache.free(ints([1]), check=True)
    if bad == 1:                                   # a hole below the pages in use
        cache.free(ints([0]), ints([0]), check=True)
    cache.table[2, 2] = bad
    refused(cache, cache.compact)
