"""Infinite and NaN values that a row sees with a weight too small for the
cache's type, or for 32 bits: a sum with an infinity in it is infinite."""
import math

import numpy as np
import pytest
import torch

from kv_reference import attention, attention_bounds, close
from paper_2609_13692_amd import kv
from test_gpu_kv_attention import DT, check, filled, ints

pytestmark = pytest.mark.gpu

# lengths, new tokens, heads, kv heads, dim, page: one token, few and many rows, long contexts in groups
SHAPES = [([300, 41], [1, 1], 4, 1, 64, 16), ([500], [3], 4, 1, 128, 1), ([400, 90], [60, 77], 2, 1, 64, 16),
          ([1500, 700], [30, 64], 8, 1, 128, 16), ([333], [70], 4, 2, 256, 64), ([9000], [1], 4, 1, 128, 16),
          ([5000], [40], 1, 1, 128, 32)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("depth", [12.0, 70.0, 300.0], ids=["weight-e12", "weight-e70", "weight-e300"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"L{max(s[0])}q{max(s[1])}h{s[2]}k{s[3]}d{s[4]}p{s[5]}")
def test_infinities_under_small_weights(shape, depth, dtype):
    """Scores 0 up to a token, then lower or higher by `depth`; infinities and
    NaN in values on either side, so that their weights are e^-depth of the
    largest, before and after the running maximum moves."""
    lengths, counts, heads, kv_heads, dim, page = shape
    dt = DT[dtype]
    for turn, rising in enumerate((True, False)):
        c, slots, ks, vs = filled(lengths, page, kv_heads, dim, dt, 50 + turn)
        for i, n in enumerate(lengths):
            k = torch.zeros((n, kv_heads, dim))
            half = n // 2
            k[:half, :, 0] = 0.0 if rising else depth
            k[half:, :, 0] = depth if rising else 0.0
            v = torch.from_numpy(vs[i]).clone()
            low = 3 if rising else half + 2
            top = half + 5 if rising else 4
            v[low, :, 1] = math.inf
            v[low + 1, :, 2] = -math.inf
            v[low + 2, :, 3] = math.nan
            v[low, :, 4] = math.inf
            v[top, :, 4] = -math.inf
            v[top, :, 5] = math.inf
            v[low + 1, :, 6] = math.inf
            v[top + 1, :, 6] = math.inf
            ks[i], vs[i] = k.to(dt).double().numpy(), v.numpy()
            rows = torch.arange(n, device="cuda")
            page_of = c.table[int(slots[i])].long()[rows // page]
            c.k[1, page_of, rows % page] = k.to(dt).cuda()
            c.v[1, page_of, rows % page] = v.to(dt).cuda()
        q = torch.zeros((sum(counts), heads, dim), dtype=dt)
        q[:, :, 0] = 1.0
        off = np.concatenate([[0], np.cumsum(counts)]).astype(int)
        for how in (dict(scale=1.0), dict(scale=1.0, window=lengths[0] * 3 // 5), dict(scale=1.0, causal=False)):
            refs = [attention(q[a:b].double().numpy(), ks[i], vs[i], lengths[i] - counts[i], **how)
                    for i, (a, b) in enumerate(zip(off, off[1:]))]
            for out_dtype in (None, torch.float32):
                out, lse = c.attend(1, q.cuda(), ints(off), slots, out_dtype=out_dtype, **how)
                assert c.take_status() == []
                for i, (a, b) in enumerate(zip(off, off[1:])):
                    bo, bl = attention_bounds(*refs[i], lengths[i], dim, dt, out_dtype or dt)
                    bo = np.where(np.isfinite(refs[i][0]), bo, 0)
                    close(out[a:b].double().cpu().numpy(), refs[i][0], bo, f"out of entry {i}, {how}")
                    close(lse[a:b].double().cpu().numpy(), refs[i][1], bl, f"lse of entry {i}, {how}")


@pytest.mark.parametrize("counts", [[1], [70]], ids=["one", "many"])
@pytest.mark.parametrize("length", [150, 4000])
def test_rows_of_no_weight_and_rows_of_nan(length, counts):
    """Scores of minus infinity alone: zeros, whatever the values; NaN in a
    query: NaN in its row alone."""
    c, slots, ks, vs = filled([length], 16, 1, 64, torch.bfloat16, 60)
    rows = torch.arange(length, device="cuda")
    page_of = c.table[int(slots[0])].long()[rows // 16]
    c.k[1, page_of, rows % 16] = torch.cat([torch.full((length, 1, 1), -math.inf), torch.zeros((length, 1, 63))], 2).bfloat16().cuda()
    for t in (2, length - 90, length - 1):
        c.v[1, page_of[t], t % 16, 0, 3:40:2] = math.inf
        c.v[1, page_of[t], t % 16, 0, 4:40:2] = math.nan
    q = torch.zeros((counts[0], 4, 64), dtype=torch.bfloat16)
    q[:, :, 0] = 1.0
    q[-1, 2, 5] = math.nan
    for how in (dict(), dict(causal=False), dict(window=100)):
        for out_dtype in (None, torch.float32):
            out, lse = c.attend(1, q.cuda(), ints([0, counts[0]]), slots, out_dtype=out_dtype, **how)
            assert torch.isnan(out[-1, 2]).all() and torch.isnan(lse[-1, 2])
            out[-1, 2], lse[-1, 2] = 0, -math.inf
            assert not out.any() and (lse == -math.inf).all(), how


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_merged_infinities_under_small_weights(dtype):
    """Parts whose weights are e^-300 of the largest, or smaller than any."""
    o = [torch.randn((6, 64)).to(dtype) for _ in range(3)]
    lse = [torch.tensor([0.0, 300.0, 0.0, 5.0, -math.inf, math.nan]),
           torch.tensor([300.0, 0.0, 1e30, 5.0, 0.0, 0.0]), torch.tensor([0.0, 0.0, 0.0, 0.0, 0.0, 0.0])]
    o[0][:, 1] = math.inf
    o[1][:, 2] = -math.inf
    o[0][:, 3], o[1][:, 3] = math.inf, -math.inf
    o[2][:, 4] = math.nan
    got, total = kv.merge([x.cuda() for x in o], [x.cuda() for x in lse], out_dtype=torch.float32)
    got, total = got.cpu(), total.cpu()
    assert torch.isnan(got[5]).all() and torch.isnan(total[5])
    for row in range(5):
        there = [i for i in range(3) if lse[i][row] > -math.inf]
        for d in range(1, 5):
            want = sum(float(o[i][row, d]) for i in there if not math.isfinite(o[i][row, d]))
            have = float(got[row, d])
            if want == 0:
                assert math.isfinite(have), (row, d)
            else:
                assert have == want or (math.isnan(have) and math.isnan(want)), (row, d, have, want)
        assert torch.isfinite(got[row, 5:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES + [([130, 500], [1, 1], 4, 2, 256, 4), ([260], [40], 3, 1, 192, 16), ([90], [1], 2, 2, 80, 1),
                                            ([700], [50], 2, 1, 80, 16)],
                         ids=lambda s: f"L{max(s[0])}q{max(s[1])}h{s[2]}k{s[3]}d{s[4]}p{s[5]}")
def test_infinities_and_nan_anywhere(shape, dtype):
    """A few in every dimension, of either sign, and pages full of them, in
    tokens that all, some or no rows see."""
    lengths, counts, heads, kv_heads, dim, page = shape
    dt = DT[dtype]
    c, slots, ks, vs = filled(lengths, page, kv_heads, dim, dt, 70)
    g = torch.Generator().manual_seed(71)
    for i, n in enumerate(lengths):
        v = torch.from_numpy(vs[i]).clone()
        for x in (math.inf, -math.inf, math.nan):
            v[torch.rand(v.shape, generator=g) < 0.3 / n] = x
        v[n // 2, :, : dim // 2], v[n // 2 + 1, :, dim // 2: dim - 3] = -math.inf, math.nan
        v[n - 1, 0] = math.inf
        vs[i] = v.numpy()
        rows = torch.arange(n, device="cuda")
        c.v[1, c.table[int(slots[i])].long()[rows // page], rows % page] = v.to(dt).cuda()
    for how in (dict(), dict(window=lengths[0] // 3), dict(causal=False, softcap=8.0)):
        check(c, slots, ks, vs, counts, heads, 72, dt, **how)
        check(c, slots, ks, vs, counts, heads, 73, dt, out_dtype=torch.float32, **how)
