"""Rotated appends and reads on a cache of another GPU than the current one, as
the other calls: that GPU is the current one while the library runs, streams and
tensors of another are refused. The library and the runtime are stand-ins."""
import types

import pytest
import torch

from test_kv_device import HOME, OTHER, Tensor, machine  # noqa: F401


@pytest.fixture
def both(machine):  # noqa: F811
    for name in ("mpt_kv_append_rotated", "mpt_kv_read"):
        setattr(machine.lib, name, lambda *a, name=name: machine.ran.append((name, machine.current)) or 0)
    return machine


def calls(c, **how):
    ints = lambda n: Tensor([n], torch.int32)  # noqa: E731
    rows, q = Tensor([3, 2, 8], torch.bfloat16), Tensor([3, 4, 8], torch.bfloat16)
    freq = Tensor([4], torch.float32)
    freq.dim = lambda: 1
    return (lambda: c.append_rotated(0, rows, rows, ints(2), ints(1), freq, q=q, q_out=q, **how),
            lambda: c.append_rotated(0, None, None, None, None, freq, q=q, q_out=q, positions=ints(3), **how),
            lambda: c.read(0, ints(2), ints(1), 3, k_out=rows, v_out=rows, **how))


@pytest.mark.parametrize("current", [HOME, OTHER])
def test_calls_run_on_the_caches_gpu(both, current):
    both.current = current
    for call in calls(both.cache):
        call()
    assert both.ran == [("mpt_kv_append_rotated", OTHER)] * 2 + [("mpt_kv_read", OTHER)]
    assert both.current == current


def test_streams_and_tensors_of_another_gpu_are_refused(both):
    wrong = types.SimpleNamespace(cuda_stream=64, device_index=HOME, device=torch.device("cuda", HOME))
    for call in calls(both.cache, stream=wrong):
        with pytest.raises(ValueError, match="GPU 1"):
            call()
    here = Tensor([1], torch.int32)
    here.get_device = lambda: HOME
    rows = Tensor([3, 2, 8], torch.bfloat16)
    freq = Tensor([4], torch.float32)
    freq.dim = lambda: 1
    with pytest.raises(ValueError, match="GPU 1"):
        both.cache.append_rotated(0, rows, rows, Tensor([2], torch.int32), here, freq)
    with pytest.raises(ValueError, match="GPU 1"):
        both.cache.read(0, Tensor([2], torch.int32), here, 3, k_out=rows, v_out=rows)
    freq.get_device = lambda: HOME
    with pytest.raises(ValueError, match="GPU 1"):
        both.cache.append_rotated(0, rows, rows, Tensor([2], torch.int32), Tensor([1], torch.int32), freq)
    assert both.ran == []
