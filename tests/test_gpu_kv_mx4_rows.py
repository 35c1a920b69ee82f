"""A cache in 4 bits: what appends write, reads give back and page calls move,
against the definition in 64 bits. Codes are equal to the last bit: the kernel's
64-bit rotations are off by less than 2^-48 of the largest element, and no input
lies that near to a border but on it (at position 0, where nothing is rounded)."""
import random

import numpy as np
import pytest
import torch

from mx4_reference import from_codes, packed, rotated, to_codes
from paper_2609_13692_amd import kv
from test_gpu_kv_rotated import DT, filled, frequencies, ints

pytestmark = pytest.mark.gpu


def stored(c, name, layer, slots, lengths, counts):
    """Packed codes and bytes E of the newest tokens."""
    pos = np.concatenate([np.arange(l - n, l) for l, n in zip(lengths, counts)])
    slot = np.repeat(slots.cpu().numpy(), counts)
    pages, at = torch.tensor(c.table.cpu().numpy()[slot, pos // c.page_size]).long().cuda(), torch.tensor(pos % c.page_size).cuda()
    return pos, [getattr(c, x)[layer, pages, at].cpu().numpy() for x in (name, name + "_scale")]


def check_codes(got, x, dtype, exact=True):
    code, scale, near = to_codes(x, dtype)
    assert exact or not ((near > 0) & (near < 2.0 ** -48)).any()
    assert np.array_equal(got[1], scale)
    assert np.array_equal(without_negative_zeros(got[0]), without_negative_zeros(packed(code)))


def without_negative_zeros(codes):
    """A zero's sign says nothing: inputs have zeros of both."""
    for bits in (0x0f, 0xf0):
        codes = np.where(codes & bits == 0x88 & bits, codes & (0xff ^ bits), codes)
    return codes


CASES = [
    # lengths, new tokens, heads, dim, page, rotated (0: a plain append), neighbours, heads first
    ([1], [1], 1, 32, 1, 0, False, True),
    ([1, 200, 33, 70, 64], [1, 5, 33, 0, 64], 2, 64, 16, 64, False, True),
    ([1, 200, 33, 70, 64], [1, 5, 33, 0, 64], 2, 64, 16, 32, True, False),
    ([130, 7], [40, 7], 3, 96, 1, 96, False, False),
    ([130, 7], [40, 7], 3, 96, 4, 48, False, True),
    ([90, 300], [90, 2], 8, 128, 16, 128, False, True),
    ([90, 300], [90, 2], 8, 128, 16, 128, True, False),
    ([90, 300], [90, 2], 8, 128, 16, 0, False, True),
    ([33, 70], [33, 1], 1, 256, 64, 256, False, True),
    ([33, 70], [33, 1], 5, 160, 8, 16, False, False),
    ([20], [20], 1, 224, 8, 224, True, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"h{c[2]}d{c[3]}p{c[4]}r{c[5]}{'n' if c[6] else ''}{'' if c[7] else 's'}")
def test_append_and_read(case, dtype):
    lengths, counts, heads, dim, page, rot, neighbours, first = case
    dtype = DT[dtype]
    c, slots = filled(lengths, page, heads, dim, dtype, heads_first=first, bits=4)
    for x in (c.k, c.v, c.k_scale, c.v_scale):
        x.fill_(0x5a)
    before = [x.clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]
    tokens = sum(counts)
    g = torch.Generator().manual_seed(dim + rot)
    fused = torch.randn((tokens, 2 * heads + 1, dim), generator=g) * torch.exp(4 * torch.randn((tokens, 1, dim // 32), generator=g)).repeat_interleave(32, -1)
    fused = fused.clamp(-60000, 60000).to(dtype).cuda()
    k, v = fused[:, :heads], fused[:, heads + 1:]
    off = np.concatenate([[0], np.cumsum(counts)])
    freq = frequencies(rot) if rot else None
    if rot:
        q = fused[:, heads:heads + 1]
        c.append_rotated(1, k, v, ints(off), slots, torch.tensor(freq, device="cuda"), q=q, interleaved=neighbours)
    else:
        c.append(1, k, v, ints(off), slots)
    assert c.take_status() == []
    pos, got_k = stored(c, "k", 1, slots, lengths, counts)
    _, got_v = stored(c, "v", 1, slots, lengths, counts)
    kd, vd = (x.double().cpu().numpy() for x in (k, v))
    check_codes(got_v, vd, dtype)
    check_codes(got_k, rotated(kd, pos, freq, neighbours) if rot else kd, dtype, exact=not rot)
    rk, rv = c.read(1, ints(off), slots, tokens)
    for r, got in ((rk, got_k), (rv, got_v)):
        assert np.array_equal(r.double().cpu().numpy(), from_codes(*got))
    # layer 0, and the other tokens, are as they were
    used = set()
    for n, s, l in zip(counts, slots.tolist(), lengths):
        used |= {(c.table[s, p // page].item(), p % page) for p in range(l - n, l)}
    for x, old in zip((c.k, c.v, c.k_scale, c.v_scale), before):
        changed = (x != old).any(-1).any(-1)
        assert not changed[0].any() and set(map(tuple, changed[1].nonzero().tolist())) <= used


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_borders_and_extremes(dtype):
    """Ties, the largest of 32 on either side of 7 2^e, the ends of the range of
    E, zeros, and blocks with a NaN or an infinity."""
    dtype = DT[dtype]
    rows = []
    for e in (-10, 0, 9):
        for top in (4.0, 5.0, 6.0, 7.0, np.nextafter(np.float32(7.0), np.float32(8.0)).item(), 7.0625):
            row = np.zeros(32)
            row[:9] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -2.5]
            row[9:18] = [0.2578125, 0.7421875, -1.2421875, 1.7578125, 2.515625, 3.484375, 4.96875, -5.03125, 0.2421875]
            row = np.clip(row, -top, top)
            row[31] = -top
            rows.append(row * 2.0 ** e)
    big, tiny = (3.3e38, 2.0 ** -126) if dtype is torch.bfloat16 else (65504.0, 2.0 ** -24)
    for top in (big, big / 2, tiny, 3 * tiny, 8 * tiny):
        rows.append(np.linspace(-top, top, 32))
    rows.append(np.zeros(32))
    rows.append(-np.zeros(32))
    for odd in (np.nan, np.inf, -np.inf):
        row = np.ones(32)
        row[13] = odd
        rows.append(row)
    x = torch.tensor(np.array(rows)).to(dtype).reshape(-1, 1, 32)
    n = len(rows)
    for rot in (False, True):
        c, slots = filled([n], 8, 1, 32, dtype, bits=4)
        if rot:                                             # at position 0 a rotation changes nothing
            c.append_rotated(0, x.cuda(), x.cuda(), ints([0, n]), slots, torch.ones(16, device="cuda"),
                             positions=ints([0] * n))
        else:
            c.append(0, x.cuda(), x.cuda(), ints([0, n]), slots)
        for name in ("k", "v"):
            _, got = stored(c, name, 0, slots, [n], [n])
            code, scale, _ = to_codes(x.double().numpy(), dtype)
            assert np.array_equal(got[1], scale)
            assert np.array_equal(without_negative_zeros(got[0]), without_negative_zeros(packed(code)))
        k, v = c.read(0, ints([0, n]), slots, n)
        assert torch.isnan(k[-3:]).all() and torch.isnan(v[-3:]).all() and torch.isfinite(k[:-3]).all()


def test_forks_cuts_and_moves_carry_codes_and_scales():
    """What sequences hold stays theirs through forks off partial pages, growth,
    frees, compaction and copies."""
    for page, heads, dim, first in ((1, 2, 64, True), (4, 3, 96, False), (16, 2, 128, True), (8, 1, 256, False), (8, 2, 32, True)):
        rng = random.Random(page)
        c = kv.KvCache.create(2, 900 // page, page, heads, dim, 8, 100, torch.bfloat16, heads_first=first, bits=4)
        held = {}

        def write(slot, a, b):
            """Tokens a .. b - 1 of a slot, in both layers."""
            if a == b:
                return []
            new = []
            for layer in range(2):
                x = torch.randn((b - a, heads, dim), device="cuda").bfloat16()
                c.append(layer, x, -x, ints([0, b - a]), ints([slot]))
                y = c.read(layer, ints([0, b - a]), ints([slot]), b - a)
                new.append(torch.stack(y))
            return [torch.stack(new)]

        def look():
            for slot, parts in held.items():
                want = torch.cat(parts, 2)
                n = want.shape[2]
                for layer in range(2):
                    k, v = c.read(layer, ints([0, n]), ints([slot]), n)
                    assert torch.equal(k, want[layer, 0]) and torch.equal(v, want[layer, 1])

        for step in range(40):
            free = [s for s in range(8) if s not in held]
            kind = rng.choice(["new", "fork", "fork", "grow", "cut", "free", "compact"])
            if kind == "new" and free:
                n = rng.randint(1, 60)
                c.fork(ints([-1]), ints(free[:1]), ints([0]), ints([n]), check=True)
                held[free[0]] = write(free[0], 0, n)
            elif kind == "fork" and free and held:
                src = rng.choice(list(held))
                whole = torch.cat(held[src], 2)
                keep = rng.randint(0, whole.shape[2])
                n = min(100, keep + rng.randint(0, 20))
                if n == 0:
                    continue
                c.fork(ints([src]), ints(free[:1]), ints([keep]), ints([n]), check=True)
                held[free[0]] = [whole[:, :, :keep]] + write(free[0], keep, n)
            elif kind == "grow" and held:
                slot = rng.choice(list(held))
                have = sum(x.shape[2] for x in held[slot])
                n = min(100, have + rng.randint(0, 20))
                c.extend(ints([slot]), ints([n]), check=True)
                held[slot] = held[slot] + write(slot, have, n)
            elif kind == "cut" and held:
                slot = rng.choice(list(held))
                whole = torch.cat(held[slot], 2)
                keep = rng.randint(1, whole.shape[2])
                c.free(ints([slot]), ints([keep]), check=True)
                held[slot] = [whole[:, :, :keep]]
            elif kind == "free" and held:
                slot = rng.choice(list(held))
                c.free(ints([slot]), check=True)
                del held[slot]
            elif kind == "compact":
                c.compact(check=True)
            look()
        a = c.ref.nonzero().flatten()[:1].int()
        b = (c.ref == 0).nonzero().flatten()[:1].int()
        c.copy(a, b, check=True)
        for x in (c.k, c.v, c.k_scale, c.v_scale):
            assert torch.equal(x[:, a.long()], x[:, b.long()])
        assert c.take_status() == []


def test_tokens_that_are_not_written_or_read():
    c, slots = filled([20, 20, 3], 8, 1, 64, torch.bfloat16, bits=4)
    c.fork(slots[:1], ints([4]), ints([16]), ints([16]), check=True)
    c.table[slots[1].item(), 2] = 10 ** 6
    before = [x.clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]
    k = torch.randn((15, 1, 64), device="cuda").bfloat16()
    c.append(0, k, k, ints([0, 6, 8, 13, 15]), torch.cat([slots, ints([77])]))
    assert set(c.take_status()) == {"slot", "length", "page", "shared page"}
    row = c.table.cpu().numpy()
    wrote = [(row[slots[0].item(), p // 8], p % 8) for p in (16, 17, 18, 19)] + [(row[slots[2].item(), 0], p) for p in (0, 1, 2)]
    for x, old in zip((c.k, c.v), before):
        changed = (x != old).any(-1).any(-1)
        assert sorted(map(tuple, changed[0].nonzero().tolist())) == sorted(wrote) and not changed[1].any()
    k, v = c.read(0, ints([0, 4, 6]), torch.cat([slots[1:2], ints([-3])]), 6)
    assert (k[2:] == 0).all() and (v[2:] == 0).all() and set(c.take_status()) == {"page", "slot"}


def test_a_captured_step():
    """Growth, append and read of a decode step, captured and replayed with the
    cache's own work between the replays."""
    c, slots = filled([30, 50], 8, 2, 128, torch.float16, max_len=80, bits=4)
    k, v = (torch.randn((2, 2, 128), device="cuda").half() for _ in range(2))
    freq, off = torch.tensor(frequencies(128), device="cuda"), ints([0, 1, 2])
    new_len, ko, vo = c.length[slots.long()].clone(), torch.empty_like(k), torch.empty_like(v)

    def step():
        new_len.add_(1)
        c.extend(slots, new_len)
        c.append_rotated(0, k, v, off, slots, freq)
        c.read(0, off, slots, 2, k_out=ko, v_out=vo)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(4):
        k.normal_()
        v.normal_()
        g.replay()
        torch.cuda.synchronize()
        got = ko.clone(), vo.clone()
        c.append_rotated(1, k, v, off, slots, freq)
        want = c.read(1, off, slots, 2)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        x = v.double().cpu().numpy()
        code, scale, _ = to_codes(x, torch.float16)
        assert np.array_equal(got[1].double().cpu().numpy(), from_codes(packed(code), scale))
    assert c.length[slots.long()].tolist() == [35, 55] and c.take_status() == []
