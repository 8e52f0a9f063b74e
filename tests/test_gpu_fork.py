"""Sequences forked from one another: cache state against the oracle, page accounting, refusals."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import oracle
from gpu_util import D, Workload, assert_attn_close, compare_state, dev, load, to_dev_bf16

pytestmark = pytest.mark.gpu
W = 128


def make(spkv, n_seqs=5, Hq=4, Hkv=2, layers=1, pool=200, max_context=4096, w=W, flags=None, **kw):
    return spkv.Cache(layers, n_seqs, Hq, Hkv, max_context, pool, window=w, tau=0.5, device=dev(),
                      flags=spkv.FLAG_FORK if flags is None else flags, **kw)


def feed(cache, wl, layer, slot, j, lo, hi, chunk=None):
    """Tokens [lo, hi) of workload sequence j into slot (state only)."""
    step = chunk or max(hi - lo, 1)
    for a in range(lo, hi, step):
        b = min(hi, a + step)
        k, v = (to_dev_bf16(np.ascontiguousarray(x[a:b, j])) for x in (wl.K, wl.V))
        cache.spkv_prefill(layer, slot, k, v, torch.from_numpy(np.ascontiguousarray(wl.logit[a:b, j])).to(dev()))


def append(cache, wl, layer, slots, js, t):
    ids = torch.tensor(slots, dtype=torch.int32, device=dev())
    k, v = (to_dev_bf16(np.ascontiguousarray(x[t][js])) for x in (wl.K, wl.V))
    cache.spkv_append_evict(layer, ids, k, v, torch.from_numpy(np.ascontiguousarray(wl.logit[t][js])).to(dev()))


def unit(wl, parts, h, tl, w=W):
    """Oracle unit of KV head h after the token ranges parts = [(workload sequence, lo, hi), ...]."""
    u = oracle.Unit(w, D)
    for j, lo, hi in parts:
        if hi > lo:
            u.prefill(*(np.ascontiguousarray(x[lo:hi, j, h]) for x in (wl.K, wl.V)),
                      np.ascontiguousarray(wl.logit[lo:hi, j, h]), tl)
    return u


def used(cache):
    s = cache.spkv_cache_stats()
    assert s.pages_in_use + s.pages_free == cache.cfg.pool_pages
    return s.pages_in_use


@pytest.mark.parametrize("T0", [0, 1, 127, 128, 129, 192, 193, 700])
@pytest.mark.parametrize("rates", [(0.0, 1.0), (0.3, 0.7)])
def test_fork_equals_a_sequence_fed_on_its_own(T0, rates):
    spkv = load()
    cache = make(spkv)
    tl = cache.spkv_tau_logit()
    wl = Workload(T0 + 1, T0 + 150, 4, 4, 2, rates, tl)
    feed(cache, wl, 0, 0, 0, 0, T0, 97)
    before = used(cache)
    cache.spkv_seq_fork(0, [1, 3])
    tails = sum(len(unit(wl, [(0, 0, T0)], h, tl)) % 64 > 0 for h in range(2))
    assert used(cache) == before + 2 * tails          # full pages are shared, part-filled ones copied
    for s in (0, 1, 3):
        for h in range(2):
            compare_state(cache, 0, s, h, unit(wl, [(0, 0, T0)], h, tl))
    # each goes its own way, the source included: by single tokens and by a chunk
    for t in range(T0, T0 + 70):
        append(cache, wl, 0, [0, 1, 3], [0, 1, 2], t)
    feed(cache, wl, 0, 3, 2, T0 + 70, T0 + 150)
    cache.check()
    for s, j, hi in ((0, 0, T0 + 70), (1, 1, T0 + 70), (3, 2, T0 + 150)):
        for h in range(2):
            compare_state(cache, 0, s, h, unit(wl, [(0, 0, T0), (j, T0, hi)], h, tl))


@pytest.mark.parametrize("order", [(0, 1, 2), (2, 1, 0), (1, 0, 2)])
def test_pages_return_with_their_last_owner(order):
    spkv = load()
    cache = make(spkv, pool=60)
    tl = cache.spkv_tau_logit()
    wl = Workload(5, 900, 3, 4, 2, (0.4, 1.0), tl)
    for _ in range(3):                                  # refork after every round: no page is lost, none doubled
        feed(cache, wl, 0, 0, 0, 0, 800)
        cache.spkv_seq_fork(0, [1])
        feed(cache, wl, 0, 1, 1, 800, 860)
        cache.spkv_seq_fork(1, [2])                     # a fork of a fork
        feed(cache, wl, 0, 2, 2, 860, 900)
        parts = {0: [(0, 0, 800)], 1: [(0, 0, 800), (1, 800, 860)], 2: [(0, 0, 800), (1, 800, 860), (2, 860, 900)]}
        alive = [0, 1, 2]
        for s in order:
            cache.spkv_cache_reset_seq(s)
            alive.remove(s)
            for a in alive:
                for h in range(2):
                    compare_state(cache, 0, a, h, unit(wl, parts[a], h, tl))
        assert used(cache) == 0
    cache.check()
    # every page can be had again, each once
    feed(cache, wl, 0, 0, 0, 0, 900)
    cache.check()
    for h in range(2):
        compare_state(cache, 0, 0, h, unit(wl, [(0, 0, 900)], h, tl))


def test_many_destinations_layers_and_local_only_heads():
    """More destinations than one launch takes, two layers, a head without a page table, sinks."""
    spkv = load()
    local = [[0, 1, 0], [0, 0, 0]]
    cache = make(spkv, n_seqs=80, Hq=3, Hkv=3, layers=2, pool=1200, local_only=local, sink_tokens=4)
    tl = cache.spkv_tau_logit()
    wl = Workload(6, 400, 2, 3, 3, (0.5, 0.5, 0.0), tl)
    for l in range(2):
        feed(cache, wl, l, 7, l, 0, 400)
    dst = [s for s in range(80) if s != 7]
    cache.spkv_seq_fork(7, dst)
    cache.check()
    ln, t = cache.spkv_read_lengths(0)
    assert (t == 400).all() and (ln == ln[7]).all() and (ln[:, 1] == 0).all() and (ln[:, 2] == 4).all()
    for s in (0, 63, 64, 79):
        for l in range(2):
            for h in range(3):
                a, b = cache.spkv_read_kept(l, 7, h), cache.spkv_read_kept(l, s, h)
                assert all(np.array_equal(x, y) for x, y in zip(a, b))
                a, b = cache.spkv_read_window(l, 7, h), cache.spkv_read_window(l, s, h)
                assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_attention_and_prefill_of_a_fork_match_the_unforked_bits():
    spkv = load()
    cache, solo = make(spkv), make(spkv, flags=0)
    tl = cache.spkv_tau_logit()
    wl = Workload(7, 700, 2, 4, 2, (0.4, 0.9), tl)
    feed(cache, wl, 0, 0, 0, 0, 500)
    cache.spkv_seq_fork(0, [2])
    feed(solo, wl, 0, 2, 0, 0, 500)
    q = to_dev_bf16(np.ascontiguousarray(wl.q[500:700, 1]))
    k, v = (to_dev_bf16(np.ascontiguousarray(x[500:700, 1])) for x in (wl.K, wl.V))
    lg = torch.from_numpy(np.ascontiguousarray(wl.logit[500:700, 1])).to(dev())
    assert torch.equal(cache.spkv_prefill(0, 2, k, v, lg, q=q), solo.spkv_prefill(0, 2, k, v, lg, q=q))
    ids = torch.tensor([2], dtype=torch.int32, device=dev())
    assert torch.equal(cache.spkv_decode_attention(0, ids, q[-1:]), solo.spkv_decode_attention(0, ids, q[-1:]))
    cache.check()


def test_errors_on_the_device():
    spkv = load()
    cache = make(spkv, pool=8)
    tl = cache.spkv_tau_logit()
    wl = Workload(8, 330, 1, 4, 2, (1.0, 1.0), tl)
    feed(cache, wl, 0, 0, 0, 0, 330)                   # 202 kept per head: 4 pages each, the pool is empty
    cache.check()
    cache.spkv_seq_fork(0, [1])
    assert cache.spkv_status() == -5
    cache.spkv_clear_status()
    ln, t = cache.spkv_read_lengths(0)
    assert (ln[1] == 0).all() and (t[1] == 0).all()    # nothing half-made
    cache.spkv_cache_reset_seq(1)
    assert used(cache) == 8
    append(cache, Workload(9, 1, 1, 4, 2, (0.0, 0.0), tl), 0, [2], [0], 0)
    cache.spkv_seq_fork(0, [2])                         # not empty: left as it is
    assert cache.spkv_status() == -16
    cache.spkv_clear_status()
    ln, t = cache.spkv_read_lengths(0)
    assert (t[2] == 1).all() and (ln[2] == 0).all() and (ln[0] == 202).all()


def test_refusals():
    spkv = load()
    cache, plain = make(spkv), make(spkv, flags=0)

    def rc(c, src, dst):
        with pytest.raises(spkv.SpkvError) as e:
            c.spkv_seq_fork(src, dst)
        return e.value.code

    assert rc(cache, 0, [0]) == -1 and rc(cache, 0, [1, 1]) == -1 and rc(cache, 0, [5]) == -1 and rc(cache, 0, [-1]) == -1
    assert rc(cache, 5, [1]) == -1 and rc(cache, -1, [1]) == -1 and rc(plain, 0, [1]) == -3
    cache.spkv_seq_fork(0, [])
    assert spkv.lib().spkv_seq_fork(None, 0, None, 0, None) == -1
    assert spkv.lib().spkv_seq_fork(cache._h, 0, None, 1, None) == -1
    cache.check()


def test_checkpoint_rollback_and_attach():
    spkv = load()
    cache = make(spkv)
    tl = cache.spkv_tau_logit()
    wl = Workload(10, 600, 2, 4, 2, (0.6, 1.0), tl)
    feed(cache, wl, 0, 0, 0, 0, 500)
    save = cache.spkv_cache_checkpoint()
    before = used(cache)
    cache.spkv_seq_fork(0, [1, 2])
    feed(cache, wl, 0, 1, 1, 500, 560)
    cache.spkv_cache_rollback(save)                     # the forks are undone with everything else
    assert used(cache) == before
    cache.spkv_seq_fork(0, [4])
    feed(cache, wl, 0, 4, 1, 500, 600)
    arena = cache.arena.clone()
    again = spkv.Cache.attach(arena, cache.cfg)
    for h in range(2):
        compare_state(again, 0, 4, h, unit(wl, [(0, 0, 500), (1, 500, 600)], h, tl))
    again.spkv_cache_reset_seq(0)
    again.spkv_cache_reset_seq(4)
    assert used(again) == 0
    with pytest.raises(spkv.SpkvError):                 # the owner counts are part of the layout
        spkv.Cache.attach(arena, cache.cfg, flags=0)
    cache.check()


def test_debug_bounds_and_canaries():
    spkv = load()
    cache = make(spkv, flags=spkv.FLAG_FORK | spkv.FLAG_DEBUG_BOUNDS)
    tl = cache.spkv_tau_logit()
    wl = Workload(12, 500, 2, 4, 2, (0.6, 1.0), tl)
    feed(cache, wl, 0, 0, 0, 0, 400)
    cache.spkv_seq_fork(0, [1, 2])
    for t in range(400, 470):
        append(cache, wl, 0, [1, 2], [0, 1], t)
    for s in (0, 2, 1):
        cache.spkv_cache_reset_seq(s)
    cache.check()
    n = C.c_int32()
    assert spkv.lib().spkv_arena_canaries(C.byref(cache.cfg), None, 0, C.byref(n)) == 0 and n.value == 12
    assert used(cache) == 0


def test_fork_in_a_captured_graph():
    spkv = load()
    cache = make(spkv)
    tl = cache.spkv_tau_logit()
    wl = Workload(13, 420, 2, 4, 2, (0.6, 1.0), tl)
    feed(cache, wl, 0, 0, 0, 0, 300)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.spkv_cache_reset_seq(1)
        cache.spkv_seq_fork(0, [1])
    for hi in (340, 420):
        g.replay()
        for h in range(2):
            compare_state(cache, 0, 1, h, unit(wl, [(0, 0, 300 if hi == 340 else 340)], h, tl))
        feed(cache, wl, 0, 0, 0, 300 if hi == 340 else 340, hi)
    cache.check()


@pytest.mark.parametrize("T0,rates,w,local", [
    (100, (1.0, 0.5), 128, None),             # within the window: nothing kept yet
    (640, (0.0, 0.0), 512, None),             # nothing ever kept, a long ring
    (128 + 128 * 64, (1.0, 1.0), 128, None),  # 128 whole pages: more table entries than a warp takes
    (700, (1.0, 1.0), 128, [[1, 1]]),         # no page tables at all
    (1, (1.0, 1.0), 1, None),
])
def test_units_without_a_partly_filled_page(T0, rates, w, local):
    """No page is copied, so nothing but the block's own barrier stands between the look at the destination and its
    last write: every destination's ring, logits, table and owner counts are complete, time after time."""
    spkv = load()
    n = 64
    cache = make(spkv, n_seqs=n + 1, pool=2 * (T0 // 64 + 2), max_context=T0 + 64, w=w, local_only=local)
    tl = cache.spkv_tau_logit()
    wl = Workload(T0, T0, 1, 4, 2, rates, tl)
    feed(cache, wl, 0, 0, 0, 0, T0)
    ref = [unit(wl, [(0, 0, T0)], h, tl, w) for h in range(2)]
    pages = used(cache)
    assert pages == (0 if local else sum(len(u) // 64 for u in ref))
    kept, ring = ([read(0, 0, h) for h in range(2)] for read in (cache.spkv_read_kept, cache.spkv_read_window))
    for _ in range(5):
        cache.spkv_seq_fork(0, range(1, n + 1))
        cache.check()
        assert used(cache) == pages
        ln, t = cache.spkv_read_lengths(0)
        assert (t == T0).all() and (ln == ln[0]).all()
        for s in range(1, n + 1, 7):
            for h in range(2):
                for got, want in ((cache.spkv_read_kept(0, s, h), kept[h]), (cache.spkv_read_window(0, s, h), ring[h])):
                    assert all(np.array_equal(x, y) for x, y in zip(got, want))
        for s in range(1, n + 1):               # each counted itself in: no page goes back before the last of them
            cache.spkv_cache_reset_seq(s)
            if s % 16 == 0:
                assert used(cache) == pages
    if not local:
        for h in range(2):
            compare_state(cache, 0, 0, h, ref[h])
    cache.spkv_cache_reset_seq(0)
    assert used(cache) == 0
    cache.check()
