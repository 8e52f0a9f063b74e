"""Where the binding's calls run and where their results come from: another device than the current one, another
stream than the current one.  The device tests need no GPU (the library and CUDA's current device are stand-ins)."""
import contextlib
import ctypes as C

import numpy as np
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


def test_a_stream_of_another_device_is_refused(spkv, two_devices):
    cache, stream = a_cache(spkv, 1), type("S", (), dict(device_index=0, cuda_stream=7))()
    ids, plan = Tensor((2,), torch.int32, 1, 4096), Tensor((1 << 16,), torch.uint8, 1, 8192)
    q = Tensor((2, 4, 128), torch.bfloat16, 1, 4096)
    nr = type("N", (), {})()
    for call in (lambda: cache.spkv_share_plan(ids, plan, stream=stream), lambda: cache.spkv_seq_fork(0, [1], stream=stream),
                 lambda: cache.spkv_decode_attention_shared(0, ids, q, plan, stream=stream),
                 lambda: spkv.spkv_norm_rope(nr, ids, q, q, stream=stream),
                 lambda: spkv.spkv_norm_rope_backward(nr, ids, q, q, q, q, stream=stream)):
        with pytest.raises(ValueError):
            call()
    assert not two_devices


# ---- on the GPU --------------------------------------------------------------------------------------
def pool_of(t):
    """The stream whose memory the tensor lies in."""
    at = t.data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"])


def forked(spkv, B=3, T0=900):
    from gpu_util import Workload
    from test_gpu_fork import feed, make
    cache = make(spkv, n_seqs=B + 1, max_context=2048)
    wl = Workload(2, T0, 1, 4, 2, (0.6, 1.0), cache.spkv_tau_logit())
    feed(cache, wl, 0, 0, 0, 0, T0)
    cache.spkv_seq_fork(0, range(1, B + 1))
    cache.check()
    gen = torch.Generator(device="cuda").manual_seed(3)
    return cache, torch.arange(1, B + 1, dtype=torch.int32, device="cuda"), torch.randn((B, 4, 128), generator=gen, device="cuda").bfloat16()


@pytest.mark.gpu
def test_results_come_from_the_memory_of_the_calls_stream(spkv):
    cache, ids, q = forked(spkv)
    plan = cache.spkv_share_plan(ids)
    w = torch.ones(128, device="cuda")
    nr = spkv.make_norm_rope(4, 2, wq=w, wk=w)
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    k = q[:, :2].contiguous()
    keep = [q.clone() for _ in range(8)]       # ... and the current stream has blocks of these sizes to give away
    del keep
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    res = [cache.spkv_share_plan(ids, stream=s), *cache.spkv_decode_attention_shared(0, ids, q, plan, want_lse=True, stream=s),
           *spkv.spkv_norm_rope(nr, pos, q, k, k, stream=s), *spkv.spkv_norm_rope_backward(nr, pos, q, k, q, k, k, stream=s)]
    s.synchronize()
    assert len(res) == 11 and all(pool_of(t) == s.cuda_stream for t in res)
    ref = [*cache.spkv_decode_attention_shared(0, ids, q, plan, want_lse=True),
           *spkv.spkv_norm_rope(nr, pos, q, k, k), *spkv.spkv_norm_rope_backward(nr, pos, q, k, q, k, k)]
    assert all(torch.equal(a, b) for a, b in zip(res[1:], ref))
    cache.check()


@pytest.mark.gpu
def test_a_plan_made_on_another_stream_is_not_cleared_behind_its_back(spkv):
    """The current stream is busy while another makes the plan: nothing the binding puts on the current one may
    reach the plan afterwards."""
    cache, ids, q = forked(spkv)
    want = cache.spkv_share_plan(ids).cpu().numpy().view(np.int32)[8:]
    assert want.any()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    plan = cache.spkv_share_plan(ids, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert np.array_equal(plan.cpu().numpy().view(np.int32)[8:], want)


@pytest.mark.gpu
def test_the_other_calls_results_too(spkv):
    cache, ids, q = forked(spkv)
    gen = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()
    T = 300
    k, v, qs, lg = rnd(T, 2, 128), rnd(T, 2, 128), rnd(T, 4, 128), torch.randn((T, 2), generator=gen, device="cuda")
    x, pred = rnd(3, 64), spkv.make_predictor(rnd(2, 64), torch.zeros(2, device="cuda"))
    keep = [torch.empty_like(t) for t in (q, qs, x) for _ in range(4)]     # blocks the current stream can give away
    del keep
    s = torch.cuda.Stream()
    torch.cuda.synchronize()

    def results(stream):
        r = [cache.spkv_score(pred, x, stream=stream), cache.spkv_decode_attention(0, ids, q, stream=stream),
             *cache.spkv_decode_attention_f32(0, ids, q, None, None, None, None, stream),
             cache.spkv_decode_attention_static(0, ids, q, stream=stream),
             spkv.spkv_softgate_forward(qs, k, v, lg, stream=stream),
             cache.spkv_cache_checkpoint(stream=stream), cache.spkv_prefill(0, 1, k, v, lg, qs, stream=stream)]
        cache.spkv_cache_rollback(r[-2], stream=stream)
        r.append(cache.spkv_decode_stack([pred], ids, x[None], q[None], k[None, :3], v[None, :3], stream=stream))
        cache.spkv_cache_rollback(r[-3], stream=stream)
        (stream or torch.cuda.current_stream()).synchronize()
        return r

    got = results(s)
    assert all(pool_of(t) == s.cuda_stream for t in got)
    assert all(torch.equal(a, b) for i, (a, b) in enumerate(zip(got, results(None))) if i != 6)
    cache.check()


@pytest.mark.gpu
def test_soft_gated_forward_waits_for_its_own_stream(spkv):
    """The device-side verdict is read behind the kernels of the stream the call was given."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    rnd = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()
    q, k, v, lg = rnd(500, 4, 128), rnd(500, 2, 128), rnd(500, 2, 128), torch.randn((500, 2), generator=gen, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
    spkv.spkv_softgate_forward(q, k, v, lg, stream=s)
    assert s.query(), "the call returned before its kernels had run"


@pytest.mark.gpu
def test_calls_with_results_given_do_not_reach_the_allocator(spkv):
    """Once a stream has its workspaces: row calls without weight gradients, plan, fork, reset and the shared-prefix call."""
    cache, ids, q = forked(spkv)
    nr = spkv.make_norm_rope(4, 2)
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    k = q[:, :2].contiguous()
    qo, out = torch.empty_like(q), torch.empty_like(q)
    ko, vo, lse = torch.empty_like(k), torch.empty_like(k), torch.empty(3, 4, device="cuda")
    plan = cache.spkv_share_plan(ids)

    def calls():
        spkv.spkv_norm_rope(nr, pos, q, k, k, qo, ko, vo)
        spkv.spkv_norm_rope_backward(nr, pos, q, k, q, k, k, qo, ko, vo, weight_grads=False)
        cache.spkv_cache_reset_seq(2)
        cache.spkv_seq_fork(0, [2])
        cache.spkv_share_plan(ids, plan)
        cache.spkv_decode_attention_shared(0, ids, q, plan, out=out, lse=lse)

    calls()
    torch.cuda.synchronize()
    count = lambda: (torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.mem_get_info()[0])
    before = count()
    for _ in range(5):
        calls()
    torch.cuda.synchronize()
    assert count() == before
    cache.check()
