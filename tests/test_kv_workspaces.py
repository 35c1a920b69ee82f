"""How many sizes of attention workspace a cache comes to hold: one for each that
its calls need."""
import ctypes

import pytest

from test_kv_abi import descriptor, lib  # noqa: F401
from test_kv_mx4_abi import descriptor4


@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 256])
@pytest.mark.parametrize("dtype", [0, 1, 3, 4])
@pytest.mark.parametrize("heads", [1, 2, 8])
def test_at_most_three_sizes(lib, dim, dtype, heads):  # noqa: F811
    make = descriptor4 if dtype >= 3 else descriptor
    row = dim // 2 if dtype >= 3 else dim
    how = dict(k_scale_stride=[8 * 16 * 100 * 32, 8 * 16 * 32, 8 * 32, 32], v_scale_stride=[8 * 16 * 100 * 32, 8 * 16 * 32, 8 * 32, 32]) \
        if dtype >= 3 else {}
    stride = [100 * 16 * heads * row, 16 * heads * row, heads * row, row]
    x = make(dtype=dtype, n_heads=heads, head_dim=dim, k_stride=stride, v_stride=stride, **how)
    p = ctypes.addressof(x)
    sizes = {lib.mpt_kv_attention_workspace_bytes(p, n, n * rows, heads * group) for n in (1, 3, 8, 32, 64, 65, 128, 257, 4096)
             for rows in (1, 2, 5, 8, 16, 17, 24, 32, 33, 48, 49, 64, 100, 128, 129, 300, 5000) for group in (1, 2, 7, 8)}
    assert 0 not in sizes and max(sizes) <= 68 << 20 and 1 <= len(sizes) <= 3, sorted(sizes)
