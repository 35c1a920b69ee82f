"""Descriptor and argument checks of the paged cache's calls, before any
device call."""
import ctypes
import os

import pytest

from paper_2609_13692_amd import mpt

P = ctypes.c_void_p
DUMMY = 4096                # never dereferenced: every call below fails its host checks


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mpt.LIB_PATH):
        pytest.fail("libmpt.so is not built (run __graft_entry__.build())")
    return mpt.load()


def descriptor(**changes):
    d = mpt.KvDescriptor()
    for f in ("k", "v", "table", "length", "ref", "free_bits", "status"):
        setattr(d, f, DUMMY)
    d.dtype, d.n_layers, d.n_pages, d.page_size, d.n_heads, d.head_dim, d.max_seqs, d.max_pages = 0, 2, 100, 16, 8, 128, 10, 20
    d.k_stride[:] = d.v_stride[:] = [100 * 16 * 1024, 16 * 1024, 1024, 128]
    for f, x in changes.items():
        if f.endswith("_stride"):
            getattr(d, f)[:] = x
        else:
            setattr(d, f, x)
    return d


BAD = [dict(dtype=2), dict(dtype=-1), dict(n_layers=0), dict(n_pages=0), dict(n_pages=(1 << 26) + 1), dict(page_size=0),
       dict(page_size=12), dict(page_size=2048), dict(n_heads=0), dict(head_dim=4), dict(head_dim=100), dict(head_dim=264),
       dict(max_seqs=0), dict(max_pages=0), dict(max_pages=1 << 30), dict(k=None), dict(v=DUMMY + 8), dict(table=None),
       dict(length=None), dict(ref=None), dict(free_bits=None), dict(status=None), dict(k_stride=[0, 0, 4, 8]),
       dict(v_stride=[0, -8, 8, 8])]


@pytest.mark.parametrize("bad", BAD, ids=lambda b: next(iter(b.items())).__repr__())
def test_descriptors_that_are_refused(lib, bad):
    d = descriptor(**bad)
    p = ctypes.addressof(d)
    assert lib.mpt_kv_workspace_bytes(p) == 0
    assert lib.mpt_kv_attention_workspace_bytes(p, 1, 1, 8) == 0
    assert lib.mpt_kv_reset(p, None) == -1
    assert lib.mpt_kv_fork(p, 1, DUMMY, DUMMY, DUMMY, DUMMY, None, DUMMY, 1 << 30, None) == -1
    assert lib.mpt_kv_append(p, 0, 1, DUMMY, DUMMY, 1, DUMMY, 8, 8, DUMMY, 8, 8, None) == -1
    assert lib.mpt_kv_attention(p, 0, 1, DUMMY, DUMMY, 1, 8, DUMMY, 8, 8, DUMMY, 8, 8, 0, None, None, 1, 0, 0.0, 1.0,
                                DUMMY, 1 << 30, None) == -1
    assert b"cache" in lib.mpt_last_error()


def test_page_calls_check_lists_and_workspace(lib):
    d = descriptor()
    p, ws, need = ctypes.addressof(d), 4096, lib.mpt_kv_workspace_bytes(ctypes.addressof(d))
    assert 8 * 100 + 12 * 10 <= need < 8 * 100 + 12 * 10 + 4096 and need % 256 == 0
    assert lib.mpt_kv_workspace_bytes(None) == 0
    assert lib.mpt_kv_fork(p, 11, DUMMY, DUMMY, DUMMY, DUMMY, None, ws, need, None) == -1
    assert lib.mpt_kv_fork(p, -1, DUMMY, DUMMY, DUMMY, DUMMY, None, ws, need, None) == -1
    assert lib.mpt_kv_fork(p, 1, None, DUMMY, DUMMY, DUMMY, None, ws, need, None) == -1
    assert lib.mpt_kv_extend(p, 1, DUMMY, None, None, ws, need, None) == -1
    assert lib.mpt_kv_free(p, 1, None, None, None, ws, need, None) == -1
    assert lib.mpt_kv_copy(p, 101, DUMMY, DUMMY, None, ws, need, None) == -1
    for w, n in ((None, need), (ws + 8, need), (ws, need - 1)):
        assert lib.mpt_kv_fork(p, 1, DUMMY, DUMMY, DUMMY, DUMMY, None, w, n, None) == -6
        assert lib.mpt_kv_free(p, 1, DUMMY, None, None, w, n, None) == -6
        assert lib.mpt_kv_compact(p, None, w, n, None) == -6
        assert lib.mpt_kv_copy(p, 1, DUMMY, DUMMY, None, w, n, None) == -6
    assert b"needs" in lib.mpt_last_error()
    assert lib.mpt_kv_status(p, None, None) == -1


def test_append_and_attention_check_their_arguments(lib):
    d = descriptor()
    p = ctypes.addressof(d)
    ok = dict(layer=0, n=1, seqs=DUMMY, q_off=DUMMY, tokens=1, k=DUMMY, ks=[1024, 128], v=DUMMY, vs=[1024, 128])
    for bad in (dict(layer=2), dict(layer=-1), dict(n=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(seqs=None),
                dict(q_off=None), dict(k=None), dict(v=DUMMY + 2), dict(ks=[1024, 12]), dict(vs=[1, 8])):
        a = {**ok, **bad}
        assert lib.mpt_kv_append(p, a["layer"], a["n"], a["seqs"], a["q_off"], a["tokens"], a["k"], *a["ks"], a["v"], *a["vs"],
                                 None) == -1, bad
    assert lib.mpt_kv_append(p, 0, 0, None, None, 0, None, 8, 8, None, 8, 8, None) == 0
    need = lib.mpt_kv_attention_workspace_bytes(p, 1, 1, 32)
    assert need >= 256 and need % 256 == 0
    for n, t, h in ((-1, 1, 32), (65537, 1, 32), (1, -1, 32), (1, (1 << 30) + 1, 32), (1, 1 << 31, 32), (1, 1, 0), (1, 1, 12)):
        assert lib.mpt_kv_attention_workspace_bytes(p, n, t, h) == 0
    ok = dict(layer=0, n=1, seqs=DUMMY, q_off=DUMMY, tokens=1, heads=32, q=DUMMY, qs=[4096, 128], out=DUMMY, os=[4096, 128],
              out_dtype=0, window=0, softcap=0.0, scale=1.0, ws=4096, ws_bytes=need)

    def call(**bad):
        a = {**ok, **bad}
        return lib.mpt_kv_attention(p, a["layer"], a["n"], a["seqs"], a["q_off"], a["tokens"], a["heads"], a["q"], *a["qs"],
                                    a["out"], *a["os"], a["out_dtype"], None, None, 1, a["window"], a["softcap"], a["scale"],
                                    a["ws"], a["ws_bytes"], None)
    for bad in (dict(layer=2), dict(n=-1), dict(n=65537), dict(n=(1 << 20) + 1), dict(tokens=(1 << 30) + 1), dict(tokens=1 << 31), dict(heads=0), dict(heads=12), dict(seqs=None),
                dict(q_off=None), dict(q=None), dict(out=None), dict(q=DUMMY + 8), dict(out=DUMMY + 4), dict(qs=[4, 8]),
                dict(os=[8, 9]), dict(out_dtype=1), dict(out_dtype=3), dict(window=-1), dict(softcap=-1.0),
                dict(softcap=float("nan")), dict(softcap=float("inf")), dict(scale=float("nan")), dict(softcap=1e-30, scale=1e20)):
        assert call(**bad) == -1, bad
    for bad in (dict(ws=None), dict(ws=4096 + 16), dict(ws_bytes=need - 1)):
        assert call(**bad) == -6, bad
    assert call(n=0) == 0 and call(tokens=0) == 0
    assert lib.mpt_kv_attention_workspace_bytes(p, 25, 8250, 32) <= 68 << 20


def test_merge_checks_its_arguments(lib):
    parts, lses = (P * 2)(DUMMY, DUMMY), (P * 2)(DUMMY, DUMMY)
    ok = dict(n=2, rows=4, dim=64, parts=parts, lses=lses, t=2, out=8192, ot=0)

    def call(**bad):
        a = {**ok, **bad}
        return lib.mpt_kv_merge(a["n"], a["rows"], a["dim"], a["parts"], a["lses"], a["t"], a["out"], a["ot"], None, None)
    for bad in (dict(n=0), dict(n=17), dict(rows=-1), dict(dim=12), dict(dim=0), dict(dim=264), dict(t=3), dict(ot=-1),
                dict(parts=None), dict(lses=None), dict(out=None), dict(out=8200), dict(parts=(P * 2)(DUMMY, None)),
                dict(lses=(P * 2)(None, DUMMY)), dict(parts=(P * 2)(DUMMY, DUMMY + 8)), dict(out=DUMMY)):
        assert call(**bad) == -1, bad
    assert call(rows=0) == 0


def test_status_code_of_missing_pages(lib):
    assert lib.mpt_status_string(-10) == b"not enough free pages"
