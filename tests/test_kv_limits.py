"""Lists that no launch could apply are refused before anything is planned."""
import ctypes

import pytest

from paper_2609_13692_amd import mpt
from test_kv_abi import DUMMY, descriptor, lib  # noqa: F401


@pytest.mark.parametrize("n", [1 << 24, (1 << 31) - 1])
def test_lists_of_too_many_sequences(lib, n):  # noqa: F811
    d = descriptor(max_seqs=(1 << 31) - 1, max_pages=1)
    p, ws = ctypes.addressof(d), DUMMY
    need = lib.mpt_kv_workspace_bytes(p)
    assert lib.mpt_kv_fork(p, n, DUMMY, DUMMY, DUMMY, DUMMY, None, ws, need, None) == -1
    assert b"16777215" in lib.mpt_last_error()
    assert lib.mpt_kv_extend(p, n, DUMMY, DUMMY, None, ws, need, None) == -1
    assert lib.mpt_kv_free(p, n, DUMMY, None, None, ws, need, None) == -1
