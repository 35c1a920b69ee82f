"""Reads of rows that leave one, two or three pieces to the last turn of a wave's
64 lanes, which still need the places of four tokens."""
import pytest

from test_gpu_kv_rows_in_runs import test_read_is_indexing as read_is_indexing

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 63, 60000])
@pytest.mark.parametrize("heads,dim", [(13, 40), (33, 16), (67, 8), (43, 24), (131, 8)])
@pytest.mark.parametrize("heads_first", [False, True])
def test_read_is_indexing_with_few_lanes_left(heads, dim, tokens, heads_first):
    """Pieces of a token: 65, 66, 67, 129 and 131."""
    assert 1 <= heads * (dim // 8) % 64 <= 3
    read_is_indexing(heads, dim, tokens, heads_first)
