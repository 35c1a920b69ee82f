"""Argument checks of rotated appends, of reads and of caches in 4 bits, before
any device call."""
import ctypes

import pytest
import torch

from paper_2609_13692_amd import kv, mpt
from test_kv_abi import DUMMY, descriptor, lib  # noqa: F401


def descriptor4(**changes):
    x = mpt.KvDescriptorMx4()
    own = {f: changes.pop(f) for f in list(changes) if "scale" in f}
    x.c = descriptor(**{"dtype": 3, **changes})
    x.k_scale = x.v_scale = DUMMY
    x.k_scale_stride[:] = x.v_scale_stride[:] = [100 * 16 * 32, 16 * 32, 32, 4]
    for f, y in own.items():
        if f.endswith("_stride"):
            getattr(x, f)[:] = y
        else:
            setattr(x, f, y)
    return x


@pytest.mark.parametrize("bad", [dict(dtype=5), dict(head_dim=120), dict(head_dim=16), dict(k_scale=None), dict(v_scale=None),
                                 dict(k_scale=DUMMY + 2), dict(v_scale_stride=[0, 512, 32, 2]), dict(k_scale_stride=[0, -4, 4, 4]),
                                 dict(k_stride=[0, 8, 16, 16]), dict(v_stride=[16, 16, 16, 24]), dict(table=None)],
                         ids=lambda b: repr(next(iter(b.items()))))
def test_descriptors_that_are_refused(lib, bad):  # noqa: F811
    x = descriptor4(**bad)
    p = ctypes.addressof(x)
    assert lib.mpt_kv_workspace_bytes(p) == 0 and b"cache" in lib.mpt_last_error()
    assert lib.mpt_kv_reset(p, None) == -1
    assert lib.mpt_kv_append(p, 0, 1, DUMMY, DUMMY, 1, DUMMY, 8, 8, DUMMY, 8, 8, None) == -1
    assert lib.mpt_kv_read(p, 0, 1, DUMMY, DUMMY, None, 1, DUMMY, 8, 8, DUMMY, 8, 8, None) == -1
    assert lib.mpt_kv_attention_workspace_bytes(p, 1, 1, 8) == 0


def test_descriptors_that_are_taken(lib):  # noqa: F811
    """Rows of scales of 1 to 8 bytes, aligned as an array without gaps has them."""
    for dim, address, row in ((32, DUMMY + 1, 1), (64, DUMMY + 2, 2), (96, DUMMY + 3, 3), (192, DUMMY + 2, 6), (256, DUMMY + 8, 8)):
        for dtype in (3, 4):
            x = descriptor4(dtype=dtype, head_dim=dim, k_stride=[dim * 8000, dim * 80, dim * 4, dim // 2], k_scale=address,
                            k_scale_stride=[row * 8000, row * 80, row * 4, row], v_scale_stride=[row * 8000, row * 80, row * 4, row])
            assert lib.mpt_kv_workspace_bytes(ctypes.addressof(x)) > 0, lib.mpt_last_error()
            if row & -row > 1:
                x.k_scale = DUMMY + 1
                assert lib.mpt_kv_workspace_bytes(ctypes.addressof(x)) == 0


@pytest.mark.parametrize("four", [False, True])
def test_rotated_append_and_read_check_their_arguments(lib, four):  # noqa: F811
    x = descriptor4() if four else descriptor()
    p = ctypes.addressof(x)
    good = dict(layer=0, n=1, seqs=DUMMY, q_off=DUMMY, tokens=1, k=DUMMY, ks=[1024, 128], v=DUMMY, vs=[1024, 128], heads=32,
                q=DUMMY, qs=[4096, 128], out=DUMMY + 64, os=[4096, 128], freq=DUMMY, position=None, dim=128, factor=1.0)

    def call(rotation=True, **bad):
        a = {**good, **bad}
        r = mpt.KvRotation(a["freq"], a["position"], a["dim"], 0, a["factor"])
        return lib.mpt_kv_append_rotated(p, a["layer"], a["n"], a["seqs"], a["q_off"], a["tokens"], a["k"], *a["ks"], a["v"],
                                         *a["vs"], ctypes.addressof(r) if rotation else None, a["heads"], a["q"], *a["qs"],
                                         a["out"], *a["os"], None)
    for bad in (dict(layer=2), dict(layer=-1), dict(n=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(seqs=None), dict(q_off=None),
                dict(k=None), dict(v=None), dict(q=None), dict(out=None), dict(k=DUMMY + 2), dict(v=DUMMY + 8), dict(q=DUMMY + 4),
                dict(out=DUMMY + 24), dict(ks=[4, 8]), dict(vs=[8, 9]), dict(qs=[8, 4]), dict(os=[12, 8]), dict(heads=0),
                dict(heads=65536), dict(freq=None), dict(dim=0), dict(dim=8), dict(dim=136), dict(dim=24), dict(dim=144),
                dict(dim=-16), dict(factor=float("inf")), dict(factor=float("nan")), dict(rotation=False),
                dict(out=DUMMY, os=[4096, 256])):
        assert call(**bad) == -1, bad
    assert call(tokens=0) == 0 and call(n=0) == 0 and call(k=None, v=None, q=None, out=None) == 0

    def read(layer=0, n=1, seqs=DUMMY, off=DUMMY, tokens=1, k=DUMMY, ks=(1024, 128), v=DUMMY, vs=(1024, 128)):
        return lib.mpt_kv_read(p, layer, n, seqs, off, None, tokens, k, *ks, v, *vs, None)
    for bad in (dict(layer=2), dict(n=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(seqs=None), dict(off=None), dict(k=DUMMY + 8),
                dict(v=DUMMY + 1), dict(ks=(4, 8)), dict(vs=(8, 12))):
        assert read(**bad) == -1, bad
    assert read(n=0) == 0 and read(tokens=0) == 0 and read(k=None, v=None) == 0


def test_caches_that_the_binding_refuses():
    z = lambda *shape, dtype=torch.uint8: torch.zeros(shape, dtype=dtype)  # noqa: E731
    rest = (z(2, 2, dtype=torch.int32), z(2, dtype=torch.int32), z(4, dtype=torch.int32), z(1, dtype=torch.int64), z(1, dtype=torch.int32))
    k, e = z(1, 4, 8, 2, 32), z(1, 4, 8, 2, 2)
    for error, args, kw in ((TypeError, (k, k), {}), (TypeError, (k, k), dict(k_scale=e, v_scale=e)),
                            (TypeError, (k, k), dict(k_scale=e, v_scale=e, dtype=torch.float32)),
                            (TypeError, (k.to(torch.int8), k.to(torch.int8)), dict(k_scale=e, v_scale=e, dtype=torch.float16)),
                            (ValueError, (k, k), dict(k_scale=e, dtype=torch.float16)),
                            (ValueError, (k, k), dict(k_scale=e, v_scale=e[..., :1], dtype=torch.float16)),
                            (ValueError, (k, k), dict(k_scale=e, v_scale=e.to(torch.int8), dtype=torch.float16)),
                            (ValueError, (k[..., :24], k[..., :24]), dict(k_scale=e, v_scale=e, dtype=torch.float16)),
                            (TypeError, (k.half(), k.half()), dict(dtype=torch.bfloat16)),
                            (ValueError, (k, k), dict(k_scale=e, v_scale=e, dtype=torch.float16))):     # not on a GPU
        with pytest.raises(error):
            kv.KvCache(*args, *rest, **kw)
    for kw in (dict(bits=8), dict(bits=4, head_dim=80)):
        with pytest.raises(ValueError):
            kv.KvCache.create(1, 4, 8, 2, kw.pop("head_dim", 64), 2, 16, **kw)
