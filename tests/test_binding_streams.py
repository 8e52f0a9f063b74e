"""Which device the binding's calls run on when it is not the current one.  No GPU is needed: the library and
CUDA's current device are stand-ins."""
import contextlib
import ctypes as C

import pytest
import torch

from paper_2605_14037_b200 import build as spkv_build


@pytest.fixture(scope="module")
def spkv():
    spkv_build.build()
    from paper_2605_14037_b200 import spkv as mod
    mod.lib()
    return mod


class Tensor:
    """As much of a device tensor as the binding looks at."""

    def __init__(self, shape, dtype, dev, ptr):
        self.shape, self.dtype, self.dev, self.ptr, self.is_cuda = torch.Size(shape), dtype, dev, ptr, True

    def get_device(self):
        return self.dev

    def data_ptr(self):
        return self.ptr

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True


@pytest.fixture
def two_devices(spkv, monkeypatch):
    """Device 0 is current; raw stream handles are 100 + device.  Yields (log of library calls, current device)."""
    now, log = [0], []

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], d
        yield
        now[0] = before

    class Library:
        def __getattr__(self, name):
            return lambda *args: log.append((name, now[0], args)) or 0

    monkeypatch.setattr(spkv, "_current_device", lambda: now[0])
    monkeypatch.setattr(spkv, "_raw_stream", lambda d: 100 + d)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: type("S", (), dict(cuda_stream=100 + now[0]))())
    monkeypatch.setattr(spkv, "lib", Library)
    return log


def raw(x):
    return x.value if isinstance(x, C.c_void_p) else x


def a_cache(spkv, dev):
    cache = spkv.Cache.__new__(spkv.Cache)
    cache.cfg = spkv.Config(1, 4, 4, 2, 128, 128, 64, 1024, 8, 0.5, spkv.FLAG_FORK, 0, None)
    cache.arena, cache.device, cache._h = Tensor((256,), torch.uint8, dev, 1 << 20), torch.device(f"cuda:{dev}"), None
    return cache


@pytest.mark.parametrize("dev", [0, 1])
def test_plan_and_fork_run_on_the_caches_device(spkv, two_devices, dev):
    cache = a_cache(spkv, dev)
    ids, plan = Tensor((2,), torch.int32, dev, 4096), Tensor((1 << 16,), torch.uint8, dev, 8192)
    assert cache.spkv_share_plan(ids, plan) is plan
    cache.spkv_seq_fork(0, [1, 2])
    for name, current, args in two_devices:
        assert current == dev and raw(args[-1]) == 100 + dev, name
    assert [c[0] for c in two_devices] == ["spkv_share_plan", "spkv_seq_fork"]


def test_a_plan_of_another_devices_tensors_is_refused(spkv, two_devices):
    cache = a_cache(spkv, 1)
    here = lambda d: (Tensor((2,), torch.int32, d, 4096), Tensor((1 << 16,), torch.uint8, d, 8192))
    for ids, plan in ((here(0)[0], here(1)[1]), (here(1)[0], here(0)[1])):
        with pytest.raises(ValueError):
            cache.spkv_share_plan(ids, plan)
    assert not two_devices
