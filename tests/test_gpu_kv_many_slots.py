"""Page calls of caches with more slots than the plans mark by bits in LDS."""
import random

import pytest
import torch

from kv_reference import Pages
from paper_2609_13692_amd import kv

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def same(c, model):
    assert c.length.tolist() == model.length and c.ref.tolist() == model.ref
    table = c.table.tolist()
    assert all(row[:len(want)] == want for row, want in zip(table, model.rows) if want)


@pytest.mark.parametrize("slots", [1 << 16, (1 << 16) + 1, 80001])
@pytest.mark.parametrize("entries", [40, 1500])
def test_many_slots(slots, entries):
    """Calls one after the other on one workspace, with the last slots among
    theirs, and lists that are refused between them."""
    rng = random.Random(slots + entries)
    c, model = kv.KvCache.create(1, 20000, 2, 1, 8, slots, 8, torch.float16), Pages(20000, 2, slots)

    def refused(call, lists, name):
        before = [x.clone() for x in (c.table, c.length, c.ref, c.free_bits)]
        with pytest.raises(kv.MptError) as e:
            call(*[ints(x) for x in lists], check=True)
        assert e.value.name == name
        for x, y in zip(before, (c.table, c.length, c.ref, c.free_bits)):
            assert torch.equal(x, y)

    for turn in range(4):
        empty = [s for s in range(slots) if not model.length[s]]
        used = [s for s in range(slots) if model.length[s]]
        dst = rng.sample(empty[:-1], entries - 1) + [empty[-1]]
        src = [rng.choice(used) if used and rng.random() < 0.7 else -1 for _ in dst]
        keep = [rng.randint(0, model.length[s]) if s >= 0 else 0 for s in src]
        new = [k + rng.randint(1 if k == 0 else 0, 8 - k) for k in keep]
        refused(c.fork, (src, dst[:-1] + dst[:1], keep, new), "MPT_E_DUP")
        refused(c.fork, (src, dst[:-1] + [slots], keep, new), "MPT_E_RANGE")
        model.fork(src, dst, keep, new)
        assert c.fork(ints(src), ints(dst), ints(keep), ints(new), check=True) == len(model.free_ids())
        same(c, model)
        used = [s for s in range(slots) if model.length[s]]
        seqs = rng.sample(used, entries)
        new = [rng.randint(model.length[s], 8) for s in seqs]
        refused(c.extend, (seqs[:-1] + seqs[:1], [8] * entries), "MPT_E_DUP")
        refused(c.extend, (seqs[:-1] + [-1], [8] * entries), "MPT_E_RANGE")
        model.extend(seqs, new)
        assert c.extend(ints(seqs), ints(new), check=True) == len(model.free_ids())
        same(c, model)
        seqs = rng.sample(range(slots - 1), entries // 2) + [slots - 1]
        refused(c.free, (seqs + seqs[:1],), "MPT_E_DUP")
        refused(c.free, (seqs + [slots],), "MPT_E_RANGE")
        seqs = rng.sample(used, entries // 2)
        cut = [rng.randint(0, model.length[s]) for s in seqs]
        model.free(seqs, cut)
        assert c.free(ints(seqs), ints(cut), check=True) == len(model.free_ids())
        same(c, model)
    assert c.compact(check=True) == model.compact()
    same(c, model)
    assert set(c.take_status()) == {"duplicate", "slot"}
