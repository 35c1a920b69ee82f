"""Calls on a cache of another GPU than the current one: that GPU is the
current one while the library runs, and the caller's is again afterwards. The
library and the runtime's notion of a current GPU are stand-ins."""
import types

import pytest
import torch

from paper_2609_13692_amd import kv

HOME, OTHER = 0, 1
CALLS = ("reset", "status", "fork", "extend", "free", "compact", "copy", "append", "attention", "merge")


class Tensor:
    """What the binding asks of a device tensor on GPU OTHER."""

    def __init__(self, shape, dtype):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", OTHER)

    def get_device(self):
        return OTHER

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 4096

    def stride(self):
        return torch.empty(self.shape, device="meta").stride()


@pytest.fixture
def machine(monkeypatch):
    m = types.SimpleNamespace(current=HOME, ran=[])

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, m.current = m.current, self.index

        def __exit__(self, *_):
            m.current = self.before

    def call(name):
        def run(*args):
            m.ran.append((name, m.current))
            return 0
        return run
    m.lib = types.SimpleNamespace(**{"mpt_kv_" + n: call(n) for n in CALLS},
                                  mpt_kv_attention_workspace_bytes=lambda *a: 256)
    monkeypatch.setattr(kv, "load", lambda: m.lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: m.current, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: m.current)
    monkeypatch.setattr(torch.cuda, "device", Device)
    m.cache = object.__new__(kv.KvCache)
    m.cache.__dict__.update(_lib=m.lib, _p=0, _index=OTHER, _ws=None, _ws_at=256, _ws_bytes=256, _ws_stream=None,
                            _at_ws={256: Tensor([256], torch.uint8)}, _at_sizes={}, _scale=1.0, n_heads=2, head_dim=8,
                            dtype=torch.bfloat16, device=torch.device("cuda", OTHER))
    return m


def every_call(c, **how):
    ints = lambda n: Tensor([n], torch.int32)  # noqa: E731
    rows, out, lse = Tensor([3, 2, 8], torch.bfloat16), Tensor([3, 2, 8], torch.bfloat16), Tensor([3, 2], torch.float32)
    c.reset(**how)
    c.take_status(**how)
    c.fork(ints(1), ints(1), ints(1), ints(1), **how)
    c.extend(ints(1), ints(1), **how)
    c.free(ints(1), **how)
    c.compact(check=True, **how)
    c.copy(ints(1), ints(1), **how)
    c.append(0, rows, rows, ints(2), ints(1), **how)
    c.attend(0, rows, ints(2), ints(1), out=out, lse=lse, **how)
    kv.merge([rows], [lse], out=out, lse=lse, **how)


@pytest.mark.parametrize("current", [HOME, OTHER])
def test_calls_run_on_the_caches_gpu(machine, current):
    machine.current = current
    every_call(machine.cache)
    assert machine.ran == [(name, OTHER) for name in CALLS]
    assert machine.current == current


def test_streams_of_another_gpu_are_refused(machine):
    wrong = types.SimpleNamespace(cuda_stream=64, device_index=HOME, device=torch.device("cuda", HOME))
    one = Tensor([1], torch.int32)
    for call in (lambda: machine.cache.reset(stream=wrong), lambda: machine.cache.free(one, stream=wrong),
                 lambda: kv.merge([Tensor([1, 8], torch.float32)], [Tensor([1], torch.float32)],
                                  out=Tensor([1, 8], torch.float32), lse=Tensor([1], torch.float32), stream=wrong)):
        with pytest.raises(ValueError, match="GPU 1"):
            call()
    assert machine.ran == []
