"""Rotated keys of a cache in 4 bits next to the smallest border of its codes."""
import numpy as np
import pytest
import torch

from mx4_reference import from_codes, packed, to_codes
from paper_2609_13692_amd import kv
from test_gpu_kv_rotated import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
def test_rounded_once_below_the_normal_numbers(interleaved):
    """A key whose rotation is x times the factor (no angle), so that in 64 bits it
    lies 2^-150 and more above, on, or below 2^-127, half of the smallest code: the
    32-bit numbers there are 2^-149 apart. And the border 3 2^-127 above it."""
    x = torch.zeros((2, 1, 32))
    x[0, 0, :16:2], x[0, 0, 1:16:2] = 2.0 ** -127, -2.0 ** -127
    x[1, 0, :16:2], x[1, 0, 1:16:2] = 3 * 2.0 ** -127, -3 * 2.0 ** -127
    x[:, 0, 16:] = x[:, 0, :16]
    x = x.bfloat16()
    assert (x.double()[0].abs() == 2.0 ** -127).all()
    one = np.float32(1)
    for factor in (one, np.nextafter(one, np.float32(2)), np.nextafter(one, np.float32(0)), np.float32(1 + 2.0 ** -22),
                   np.float32(1 - 2.0 ** -23), np.float32(1.5), np.float32(0.5)):
        c = kv.KvCache.create(1, 4, 16, 1, 32, 1, 16, bits=4)
        c.fork(ints([-1]), ints([0]), ints([0]), ints([2]), check=True)
        c.append_rotated(0, x.cuda(), x.cuda(), ints([0, 2]), ints([0]), torch.zeros(16, device="cuda"),
                         interleaved=interleaved, factor=float(factor))
        y = x.double().numpy() * float(factor)
        code, scale, _ = to_codes(y, torch.bfloat16)
        page = c.table[0, 0].item()
        assert np.array_equal(c.k_scale[0, page, :2].cpu().numpy(), scale) and (scale == 2).all()
        got = from_codes(c.k[0, page, :2].cpu().numpy(), scale)
        assert np.array_equal(got, from_codes(packed(code), scale)), factor
        assert c.take_status() == []
