"""Decode attention of a batch with a common prefix: against the formula in 64 bits over the pairs the cache
holds (themselves compared with the oracle where sequences are forked), and against the per-sequence call."""
import math

import numpy as np
import pytest
import torch

from gpu_util import D, Workload, dev, load, to_dev_bf16
from paper_2605_14037_b200 import synth
from test_gpu_fork import append, feed, make, unit

pytestmark = pytest.mark.gpu
SC = 1 / math.sqrt(D)


def f64(bits):
    return synth.bf16_bits_to_f32(bits).astype(np.float64)


def reference(cache, layer, seq, h, q, scale=SC):
    """(out, sum of weights x |v|, lse, largest |q||k|) of the group's queries q [G, 128] float64"""
    kept, ring = cache.spkv_read_kept(layer, seq, h), cache.spkv_read_window(layer, seq, h)
    k, v = (np.concatenate([f64(kept[i]), f64(ring[i])]) for i in (1, 2))
    s = q @ k.T * scale
    m = s.max(-1, keepdims=True)
    p = np.exp(s - m)
    z = p.sum(-1, keepdims=True)
    return p @ v / z, p @ np.abs(v) / z, (m + np.log(z))[:, 0], (np.linalg.norm(q, axis=-1)[:, None] * np.linalg.norm(k, axis=-1)[None]).max()


def check(cache, layer, seqs, q_bits, out, lse, scale=SC, kv=None):
    """A weight is rounded to fp16 (2^-12 of it) or two bf16 terms (less); with the row sum kept in fp32 from the
    unrounded weights, the output is off by at most 2^-12 sum w|v|, then rounded to bf16: 8 significant
    bits, so half a step is up to 2^-8 of the value (torch.finfo(bfloat16).eps / 2).  Scores: 128 products
    added in fp32, 130 * 2^-24 |q||k| scale (and twice that as a relative error of a weight, on both
    sides of the quotient)."""
    G = q_bits.shape[1] // cache.cfg.n_kv_heads
    got, l = out.float().cpu().double().numpy(), lse.cpu().double().numpy()
    for b, s in enumerate(seqs):
        for h in range(cache.cfg.n_kv_heads):
            hs = slice(h * G, (h + 1) * G)
            ref, wv, rl, qk = reference(cache, layer, s, h, f64(q_bits[b, hs]), scale)
            es = 130 * 2.0 ** -24 * qk * scale
            err, tol = np.abs(got[b, hs] - ref), 2.0 ** -8 * np.abs(ref) + (2.0 ** -12 + 2.0 ** -18 + 2 * es) * wv + 1e-30
            assert (err <= tol).all(), (b, h, err.max(), (err / tol).max())
            assert (np.abs(l[b, hs] - rl) <= es + 2.0 ** -19 * (1 + np.abs(rl))).all(), (b, h, np.abs(l[b, hs] - rl).max())


def build(spkv, B, Hq, Hkv, T0, m, rates, seed=0, layers=1, flags=0, gain=1.0, pool=None, **kw):
    pool = pool or (Hkv * (T0 // 64 + 2) + B * Hkv * ((m + 128) // 64 + 3)) * layers
    cache = make(spkv, n_seqs=B + 1, Hq=Hq, Hkv=Hkv, layers=layers, pool=pool, max_context=T0 + m + 64,
                 flags=spkv.FLAG_FORK | flags, **kw)
    wl = Workload(seed, T0 + m, B, Hq, Hkv, rates, cache.spkv_tau_logit())
    if gain != 1.0:
        wl.V = synth.to_bf16_bits(synth.bf16_bits_to_f32(wl.V) * np.float32(gain))
    for l in range(layers):
        feed(cache, wl, l, 0, 0, 0, T0, 4096)
    cache.spkv_seq_fork(0, range(1, B + 1))
    for l in range(layers):
        for j in range(B):
            if m:
                feed(cache, wl, l, j + 1, j, T0, T0 + m)
    cache.check()
    ids = torch.arange(1, B + 1, dtype=torch.int32, device=dev())
    return cache, wl, ids


def queries(wl, t=-1):
    q = np.ascontiguousarray(wl.q[t])
    return q, to_dev_bf16(q)


def commons(cache, plan, layer=0):
    p = plan.cpu().numpy().view(np.int32)[8:].reshape(cache.cfg.n_layers, -1)[layer]
    return p[4:4 + 8 * cache.cfg.n_kv_heads:8]


@pytest.mark.parametrize("B,Hq,Hkv,T0,m,rates", [
    (2, 2, 2, 300, 1, (0.5, 1.0)),            # G = 1, few pages
    (2, 4, 2, 200, 0, (0.0, 0.3)),            # nothing in common: less than a page, or nothing kept
    (3, 6, 2, 1000, 70, (1.0, 0.1)),          # G = 3
    (7, 35, 7, 1500, 129, (0.4,) * 7),        # G = 5, odd head count
    (5, 16, 1, 3000, 40, (0.8,)),             # G = 16, one head
    (8, 32, 2, 2500, 33, (0.9, 0.05)),        # 128 rows exactly
    (9, 32, 2, 2500, 10, (0.9, 0.0)),         # 144 rows: the second slot in part
    (16, 32, 2, 2000, 200, (0.3, 0.6)),       # 256 rows exactly
    (23, 24, 2, 1800, 5, (0.7, 0.2)),         # 276 rows: a second row tile
    (64, 16, 2, 1200, 3, (0.5, 1.0)),         # 512 rows
    (4, 8, 2, 20000, 60, (1.0, 0.02)),        # long and short heads
])
def test_against_the_formula(B, Hq, Hkv, T0, m, rates):
    spkv = load()
    cache, wl, ids = build(spkv, B, Hq, Hkv, T0, m, rates, seed=B * 7 + T0)
    q, qd = queries(wl)
    plan = cache.spkv_share_plan(ids)
    ln, _ = cache.spkv_read_lengths(0)
    want = [len(unit(wl, [(0, 0, T0)], h, cache.spkv_tau_logit())) // 64 for h in range(Hkv)]
    assert commons(cache, plan).tolist() == want
    out, lse = cache.spkv_decode_attention_shared(0, ids, qd, plan, want_lse=True)
    cache.check()
    check(cache, 0, range(1, B + 1), q, out, lse)
    again, lse2 = cache.spkv_decode_attention_shared(0, ids, qd, plan, want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("B,Hq,Hkv", [(1024, 1, 1), (512, 4, 2), (64, 16, 16), (341, 48, 3)])
def test_the_largest_batches(B, Hq, Hkv):
    """1024 units (one piece of its own each), more query rows than a block of any KV head takes"""
    spkv = load()
    cache, wl, ids = build(spkv, B, Hq, Hkv, 700, 3, tuple(0.2 + 0.8 * (i % 2) for i in range(Hkv)), seed=B)
    q, qd = queries(wl)
    plan = cache.spkv_share_plan(ids)
    out, lse = cache.spkv_decode_attention_shared(0, ids, qd, plan, want_lse=True)
    cache.check()
    some = sorted({0, 1, B // 2, B - 2, B - 1, *range(0, B, max(1, B // 12))})
    check(cache, 0, [b + 1 for b in some], q[some], out[some], lse[some])
    lone = torch.empty_like(lse[some])   # (the per-sequence call takes fewer sequences at once)
    cache.spkv_decode_attention(0, ids[some].contiguous(), qd[some].contiguous(), lse=lone)
    # (each within 130 * 2^-24 |q| |k| scale of the formula, as in `check`; |q| |k| scale stays below 50 here)
    assert torch.isfinite(lse).all() and (lse[some] - lone).abs().max() < 2 * 130 * 2.0 ** -24 * 50 + 2.0 ** -17


def test_sequences_that_share_nothing_and_single_sequences():
    spkv = load()
    cache = make(spkv, n_seqs=4, flags=0)              # also without SPKV_FLAG_FORK
    wl = Workload(3, 500, 3, 4, 2, (0.5, 1.0), cache.spkv_tau_logit())
    for j in range(3):
        feed(cache, wl, 0, j, j, 0, 500 - 77 * j)
    q, qd = queries(wl)
    for seqs in ([0, 1, 2], [1]):
        ids = torch.tensor(seqs, dtype=torch.int32, device=dev())
        plan = cache.spkv_share_plan(ids)
        assert not commons(cache, plan).any()
        out, lse = cache.spkv_decode_attention_shared(0, ids, qd[:len(seqs)].contiguous(), plan, want_lse=True)
        check(cache, 0, seqs, q[:len(seqs)], out, lse)
    cache.check()


def test_empty_sequences_among_the_batch():
    """A sequence that has received nothing: zeros and -inf, as spkv_decode_attention gives."""
    spkv = load()
    cache, wl, ids = build(spkv, 2, 4, 2, 600, 5, (0.5, 1.0))
    cache.spkv_cache_reset_seq(2)
    q, qd = queries(wl)
    plan = cache.spkv_share_plan(ids)
    assert not commons(cache, plan).any()
    out, lse = cache.spkv_decode_attention_shared(0, ids, qd, plan, want_lse=True)
    check(cache, 0, [1], q[:1], out[:1], lse[:1])
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    cache.check()


def test_parent_and_nested_forks_in_one_batch():
    """The source decodes beside its forks, and a fork of a fork beside both: the common part is the shortest."""
    spkv = load()
    cache = make(spkv, n_seqs=6, pool=300)
    tl = cache.spkv_tau_logit()
    wl = Workload(4, 1500, 4, 4, 2, (0.5, 1.0), tl)
    feed(cache, wl, 0, 0, 0, 0, 1000)
    cache.spkv_seq_fork(0, [1])
    feed(cache, wl, 0, 1, 1, 1000, 1400)
    cache.spkv_seq_fork(1, [2, 3])
    feed(cache, wl, 0, 0, 0, 1000, 1100)
    feed(cache, wl, 0, 2, 2, 1400, 1500)
    q, qd = queries(wl)
    first = [len(unit(wl, [(0, 0, 1000)], h, tl)) // 64 for h in range(2)]
    second = [len(unit(wl, [(0, 0, 1000), (1, 1000, 1400)], h, tl)) // 64 for h in range(2)]
    for seqs, want in (([3, 0, 2, 1], first), ([2, 3], second), ([1, 3, 2], second)):
        ids = torch.tensor(seqs, dtype=torch.int32, device=dev())
        plan = cache.spkv_share_plan(ids)
        assert commons(cache, plan).tolist() == want
        n = len(seqs)
        out, lse = cache.spkv_decode_attention_shared(0, ids, qd[:n].contiguous(), plan, want_lse=True)
        check(cache, 0, seqs, q[:n], out, lse)
    cache.check()


def test_a_stale_plan_costs_time_not_the_result():
    spkv = load()
    cache, wl, ids = build(spkv, 3, 4, 2, 1500, 5, (0.5, 1.0), pool=400)
    q, qd = queries(wl)
    plan = cache.spkv_share_plan(ids)

    def run(seqs=(1, 2, 3)):
        i = torch.tensor(seqs, dtype=torch.int32, device=dev())
        out, lse = cache.spkv_decode_attention_shared(0, i, qd[:len(seqs)].contiguous(), plan, want_lse=True)
        check(cache, 0, seqs, q[:len(seqs)], out, lse)

    cache.spkv_cache_reset_seq(2)
    feed(cache, wl, 0, 2, 1, 0, 1400)                  # another sequence in its place, pages recycled
    run()
    cache.spkv_cache_reset_seq(1)                       # ... and in the first one's, shorter than the common part
    feed(cache, wl, 0, 1, 2, 0, 100)
    run()
    run((3, 2, 1))
    run((3, 2))                                         # a plan for another batch size
    cache.spkv_cache_reset_seq(1)
    cache.spkv_cache_reset_seq(2)
    cache.spkv_seq_fork(3, [1, 2])                      # longer common part than the plan's
    run()
    plan = torch.zeros_like(plan)                       # a plan that was never made
    run()
    cache.check()


def test_layers_growth_and_one_plan():
    """One plan for all layers while the sequences grow token by token; local-only head, window of 100."""
    spkv = load()
    cache, wl, ids = build(spkv, 4, 8, 2, 900, 4, (0.5, 1.0), layers=2, w=100, local_only=[[0, 0], [1, 0]])
    plan = cache.spkv_share_plan(ids)
    assert commons(cache, plan, 1)[0] == 0 and commons(cache, plan, 1)[1] > 0
    for t in range(100):
        for l in range(2):
            append(cache, wl, l, [1, 2, 3, 4], [0, 1, 2, 3], t)
            if t % 33 == 0:
                q, qd = queries(wl, t)
                out, lse = cache.spkv_decode_attention_shared(l, ids, qd, plan, want_lse=True)
                check(cache, l, range(1, 5), q, out, lse)
    cache.check()


@pytest.mark.parametrize("gain,flags", [(2.0 ** 21, 0), (2.0 ** -30, 0), (1.0, 2)])
def test_value_ranges(gain, flags):
    """Values past 2^20 and the PREFILL_PV_BF16 flag take the two-term product, tiny ones are rescaled."""
    spkv = load()
    cache, wl, ids = build(spkv, 9, 32, 2, 1500, 30, (0.5, 1.0), gain=gain, flags=flags)
    q, qd = queries(wl)
    out, lse = cache.spkv_decode_attention_shared(0, ids, qd, cache.spkv_share_plan(ids), want_lse=True)
    cache.check()
    check(cache, 0, range(1, 10), q, out, lse)


@pytest.mark.parametrize("B", [3, 20])
def test_large_scores(B):
    """Scores that grow along the sequence: the running maximum moves on every page."""
    spkv = load()
    cache = make(spkv, n_seqs=B + 1, Hq=16, Hkv=2, pool=200, max_context=4096)
    wl = Workload(8, 2000, B, 16, 2, (1.0, 0.5), cache.spkv_tau_logit())
    wl.K = synth.to_bf16_bits(synth.bf16_bits_to_f32(wl.K) * np.linspace(0.2, 12, 2000, dtype=np.float32)[:, None, None, None])
    feed(cache, wl, 0, 0, 0, 0, 1990)
    cache.spkv_seq_fork(0, range(1, B + 1))
    for j in range(B):
        feed(cache, wl, 0, j + 1, j, 1990, 2000)
    ids = torch.arange(1, B + 1, dtype=torch.int32, device=dev())
    q, qd = queries(wl)
    out, lse = cache.spkv_decode_attention_shared(0, ids, qd, cache.spkv_share_plan(ids), want_lse=True)
    cache.check()
    check(cache, 0, range(1, B + 1), q, out, lse)


def test_infinities_and_nans_stay_with_their_rows():
    spkv = load()
    cache, wl, ids = build(spkv, 3, 4, 2, 1200, 5, (1.0, 1.0))
    _, qd = queries(wl)
    plan = cache.spkv_share_plan(ids)
    clean = cache.spkv_decode_attention_shared(0, ids, qd, plan)
    bad = qd.clone()
    bad[1, 2, 7] = float("nan")
    out = cache.spkv_decode_attention_shared(0, ids, bad, plan)
    assert out[1, 2].isnan().all()
    keep = torch.ones((3, 4), dtype=torch.bool)
    keep[1, 2] = False
    assert torch.equal(out.cpu()[keep], clean.cpu()[keep])


@pytest.mark.parametrize("overlap", [False, True])
def test_decode_steps_in_a_graph_beside_the_per_sequence_call(overlap):
    """norm + rotation, append, shared attention for two layers, captured once and replayed, on a stream of its
    own: the same bits as the eager calls on a copy of the cache."""
    spkv = load()
    fl = spkv.FLAG_OVERLAP if overlap else 0
    cache, wl, ids = build(spkv, 6, 8, 2, 1000, 2, (0.5, 1.0), layers=2, flags=fl)
    twin = spkv.Cache.attach(cache.arena.clone(), cache.cfg)
    plan = cache.spkv_share_plan(ids)
    g = torch.Generator(device=dev()).manual_seed(1)
    nr = spkv.make_norm_rope(8, 2, wq=torch.ones(128, device=dev()), wk=torch.ones(128, device=dev()))
    qkv = torch.randn((2, 6, 12, 128), generator=g, device=dev()).bfloat16()
    lg = torch.randn((2, 6, 2), generator=g, device=dev())
    pos = torch.full((6,), 1002, dtype=torch.int32, device=dev())
    outs = [torch.empty((6, 8, 128), dtype=torch.bfloat16, device=dev()) for _ in range(2)]

    def step(c, outs):
        for l in range(2):
            q, k, v = spkv.spkv_norm_rope(nr, pos, qkv[l, :, :8], qkv[l, :, 8:10], qkv[l, :, 10:])
            c.spkv_note_foreign_work()
            c.spkv_append_evict(l, ids, k, v, lg[l])
            c.spkv_decode_attention_shared(l, ids, q, plan, out=outs[l])
        pos.add_(1)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        want = [torch.empty_like(o) for o in outs]
        step(twin, want)
        pos.sub_(1)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step(cache, outs)
        for i in range(5):
            if i:
                step(twin, want)
                pos.sub_(1)
            graph.replay()
            s.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), i
            qkv.mul_(0.9)
    cache.check()
    twin.check()
    for c in (cache,):
        out, lse = c.spkv_decode_attention_shared(0, ids, outs[0], plan, want_lse=True)
        check(c, 0, range(1, 7), spkv.bits_from_bf16(outs[0]), out, lse)


def test_the_batch_mixes_with_the_other_calls():
    """Shared, per-sequence and stack calls in turn on one cache and stream."""
    spkv = load()
    cache, wl, ids = build(spkv, 4, 8, 2, 800, 3, (0.5, 1.0), layers=2)
    plan = cache.spkv_share_plan(ids)
    q, qd = queries(wl)
    W1 = torch.randn((2, 64), device=dev()).bfloat16()
    preds = [spkv.make_predictor(W1, torch.zeros(2, device=dev()))] * 2
    rnd = lambda *s: torch.randn(s, device=dev()).bfloat16()
    for i in range(4):
        cache.spkv_decode_stack(preds, ids, rnd(2, 4, 64), rnd(2, 4, 8, 128), rnd(2, 4, 2, 128), rnd(2, 4, 2, 128))
        for l in range(2):
            out, lse = cache.spkv_decode_attention_shared(l, ids, qd, plan, want_lse=True)
            one = cache.spkv_decode_attention(l, ids, qd)
            check(cache, l, range(1, 5), q, out, lse)
            assert (out.float() - one.float()).abs().max() <= 2.0 ** -7 * 4
    cache.check()


def test_refusals():
    spkv = load()
    cache, wl, ids = build(spkv, 2, 4, 2, 300, 1, (0.5, 1.0))
    _, qd = queries(wl)
    plan = cache.spkv_share_plan(ids)
    l, h = spkv.lib(), cache._h
    out = torch.zeros_like(qd)
    ws = cache._workspace("x", l.spkv_decode_shared_workspace_bytes(cache.cfg, 2))
    p = lambda t: t.data_ptr()

    def call(layer=0, i=p(ids), B=2, q=p(qd), o=p(out), scale=SC, pl=p(plan), pb=plan.numel(), w=p(ws), wb=ws.numel()):
        return l.spkv_decode_attention_shared(h, layer, i, B, q, o, None, scale, pl, pb, w, wb, None)

    assert call() == 0
    assert call(layer=1) == -1 and call(layer=-1) == -1 and call(B=4) == -1 and call(B=-1) == -1 and call(i=None) == -1
    assert call(q=None) == -1 and call(q=p(qd) + 2) == -1 and call(o=p(out) + 8) == -1
    assert call(scale=0.0) == -1 and call(scale=-1.0) == -1 and call(scale=float("inf")) == -1 and call(scale=float("nan")) == -1
    assert call(pl=None) == -1 and call(pl=p(plan) + 4) == -1 and call(pb=plan.numel() - 1) == -7
    assert call(w=None) == -7 and call(w=p(ws) + 16) == -7 and call(wb=ws.numel() - 1) == -7
    assert call(B=0) == 0
    assert l.spkv_share_plan(h, p(ids), 0, p(plan), plan.numel(), None) == -1
    assert l.spkv_share_plan(h, None, 2, p(plan), plan.numel(), None) == -1
    assert l.spkv_share_plan(h, p(ids), 2, None, plan.numel(), None) == -1
    assert l.spkv_share_plan(h, p(ids), 2, p(plan), 8, None) == -7
    cache.check()
    bad = torch.tensor([1, 99], dtype=torch.int32, device=dev())        # found on the device, by plan and call
    cache.spkv_share_plan(bad, plan)
    assert cache.spkv_status() == -9
    cache.spkv_clear_status()
    o, lse = cache.spkv_decode_attention_shared(0, bad, qd, plan, want_lse=True)
    assert cache.spkv_status() == -9
    assert (o[1] == 0).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("B,Hq", [(2, 8), (33, 32)])
def test_long_shares(B, Hq):
    """More pages per block than the page-table entries a warp holds at once (32): 8 dense heads of 47000 tokens
    are 5900 pages, 40 and more per block; one and two slots of query rows."""
    spkv = load()
    cache = make(spkv, n_seqs=B + 1, Hq=Hq, Hkv=8, pool=8 * 740 + B * 8 * 4, max_context=48000)
    wl = Workload(21, 47000, 1, Hq, 8, (1.0,) * 8, cache.spkv_tau_logit(), with_q=False)
    feed(cache, wl, 0, 0, 0, 0, 47000, 8192)
    cache.spkv_seq_fork(0, range(1, B + 1))
    ids = torch.arange(1, B + 1, dtype=torch.int32, device=dev())
    plan = cache.spkv_share_plan(ids)
    rec = plan.cpu().numpy().view(np.int32)[8:]
    assert rec[0] > 32 and rec[1] <= 256
    q = synth.normal_bf16(np.random.default_rng(3), (B, Hq, D))
    out, lse = cache.spkv_decode_attention_shared(0, ids, to_dev_bf16(q), plan, want_lse=True)
    cache.check()
    for b in {0, B // 2, B - 1}:
        check(cache, 0, [b + 1], q[b:b + 1], out[b:b + 1], lse[b:b + 1])


@pytest.mark.parametrize("planned", [True, False])
def test_long_pieces_of_a_sequences_own(planned):
    """Sequences that share nothing and are long: with a plan their pages go in pieces, without one a block walks
    all 300 of a unit."""
    spkv = load()
    cache = make(spkv, n_seqs=2, Hq=4, Hkv=2, pool=1300, max_context=20000, flags=0)
    wl = Workload(22, 19000, 2, 4, 2, (1.0, 0.3), cache.spkv_tau_logit(), with_q=False)
    for j in range(2):
        feed(cache, wl, 0, j, j, 0, 19000, 8192)
    ids = torch.arange(2, dtype=torch.int32, device=dev())
    plan = cache.spkv_share_plan(ids)
    if not planned:
        plan.zero_()
    q = synth.normal_bf16(np.random.default_rng(4), (2, 4, D))
    out, lse = cache.spkv_decode_attention_shared(0, ids, to_dev_bf16(q), plan, want_lse=True)
    cache.check()
    check(cache, 0, [0, 1], q, out, lse)


@pytest.mark.parametrize("w", [1, 64, 65, 200])
@pytest.mark.parametrize("sinks", [0, 5])
def test_windows_and_sinks(w, sinks):
    spkv = load()
    cache, wl, ids = build(spkv, 4, 8, 2, 1000, 30, (0.4, 1.0), w=w, sink_tokens=sinks)
    q, qd = queries(wl)
    out, lse = cache.spkv_decode_attention_shared(0, ids, qd, cache.spkv_share_plan(ids), want_lse=True)
    cache.check()
    check(cache, 0, range(1, 5), q, out, lse)


def test_two_term_product_with_alternating_slots():
    """Values past 2^20 with at most 128 query rows: both slots of a block hold the same rows."""
    spkv = load()
    cache, wl, ids = build(spkv, 3, 8, 2, 1500, 30, (0.5, 1.0), gain=2.0 ** 21)
    q, qd = queries(wl)
    out, lse = cache.spkv_decode_attention_shared(0, ids, qd, cache.spkv_share_plan(ids), want_lse=True)
    cache.check()
    check(cache, 0, range(1, 4), q, out, lse)


def test_a_plan_of_another_cache():
    """Another layout's plan (heads without page tables) does not fit; the same layout's is checked like a stale one."""
    spkv = load()
    a, wl, ids = build(spkv, 3, 8, 2, 1500, 5, (0.5, 1.0), pool=300)
    b, _, _ = build(spkv, 3, 8, 2, 1500, 5, (0.5, 1.0), pool=300, local_only=[[1, 0]])
    c = make(spkv, n_seqs=4, Hq=8, Hkv=2, pool=300, max_context=1569)
    for j in range(3):
        feed(c, wl, 0, j + 1, j, 0, 900)
    q, qd = queries(wl)
    for cache in (b, c):
        out, lse = cache.spkv_decode_attention_shared(0, ids, qd, a.spkv_share_plan(ids), want_lse=True)
        cache.check()
        check(cache, 0, range(1, 4), q, out, lse)


def test_two_streams_in_turn():
    """Calls on two streams, ordered by events, on one cache and workspace."""
    spkv = load()
    cache, wl, ids = build(spkv, 6, 8, 2, 1200, 20, (0.5, 1.0))
    plan = cache.spkv_share_plan(ids)
    q, qd = queries(wl)
    want = cache.spkv_decode_attention_shared(0, ids, qd, plan)
    torch.cuda.synchronize()
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for i in range(6):
        with torch.cuda.stream(s[i & 1]):
            s[i & 1].wait_stream(s[1 - (i & 1)])
            outs.append(cache.spkv_decode_attention_shared(0, ids, qd, plan))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    cache.check()


def test_graphs_and_eager_calls_on_streams_of_their_own():
    """Graphs of a small batch captured on one stream, replayed at the same time on two, while eager calls of the whole
    batch make a larger workspace: nobody writes over anybody's parts."""
    spkv = load()
    cache, wl, ids = build(spkv, 24, 32, 2, 6000, 5, (0.8, 0.3))
    q, qd = queries(wl)
    plan, whole = cache.spkv_share_plan(ids[:4].contiguous()), cache.spkv_share_plan(ids)
    qs = [qd[:4].contiguous(), (qd[:4] * 0.5).contiguous()]
    few = ids[:4].contiguous()
    want = [cache.spkv_decode_attention_shared(0, few, x, plan) for x in qs]
    want_all = cache.spkv_decode_attention_shared(0, ids, qd, whole)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = x
            for _ in range(8):
                o = cache.spkv_decode_attention_shared(0, few, x, plan)
        graphs.append(g)
        outs.append(o)
    s = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(10):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, s):
            with torch.cuda.stream(st):
                g.replay()
        eager = [cache.spkv_decode_attention_shared(0, ids, qd, whole, stream=s[2]) for _ in range(4)]
        here = [cache.spkv_decode_attention_shared(0, few, x, plan) for x in qs]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs + here, want + want))
        assert all(torch.equal(e, want_all) for e in eager)
    cache.check()


def test_output_over_the_queries():
    spkv = load()
    cache, wl, ids = build(spkv, 6, 8, 2, 1200, 20, (0.5, 1.0))
    plan = cache.spkv_share_plan(ids)
    _, qd = queries(wl)
    want = cache.spkv_decode_attention_shared(0, ids, qd, plan)
    buf = qd.clone()
    cache.spkv_decode_attention_shared(0, ids, buf, plan, out=buf)
    assert torch.equal(buf, want)
    cache.check()


def test_binding_refusals():
    spkv = load()
    cache, wl, ids = build(spkv, 2, 4, 2, 300, 1, (0.5, 1.0))
    _, qd = queries(wl)
    plan = cache.spkv_share_plan(ids)
    for args in ((0, ids.long(), qd, plan), (0, ids, qd[:1], plan), (0, ids, qd.float(), plan), (0, ids[:1], qd, plan),
                 (0, ids, qd.transpose(0, 1).contiguous().transpose(0, 1), plan), (0, ids, qd, plan.view(torch.int32)),
                 (0, ids.cpu(), qd, plan), (0, ids, qd.cpu(), plan)):
        with pytest.raises(ValueError):
            cache.spkv_decode_attention_shared(*args)
    for kw in (dict(out=torch.empty_like(qd)[:1]), dict(lse=torch.empty((2, 4), device=dev(), dtype=torch.float64))):
        with pytest.raises(ValueError):
            cache.spkv_decode_attention_shared(0, ids, qd, plan, **kw)


@pytest.mark.parametrize("B,T0,m", [(2, 300, 1), (3, 1200, 40), (20, 4000, 3), (4, 100, 0)])
def test_range_checks_find_nothing_in_a_sound_cache(B, T0, m):
    """SPKV_FLAG_DEBUG_BOUNDS: shares of fewer pages than a warp has lanes, pieces of a unit's own pages, units without
    any -- no index that nobody uses is reported, and the results are those without the flag."""
    spkv = load()
    outs = []
    for flags in (0, spkv.FLAG_DEBUG_BOUNDS):
        cache, wl, ids = build(spkv, B, 16, 2, T0, m, (0.4, 1.0), seed=B, flags=flags)
        q, qd = queries(wl)
        plan = cache.spkv_share_plan(ids)
        outs.append(cache.spkv_decode_attention_shared(0, ids, qd, plan, want_lse=True))
        assert cache.spkv_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("B", [3, 20])
@pytest.mark.parametrize("wide", [False, True])
def test_roundings_of_weights_that_do_not_average_out(B, wide):
    """Keys of three scores, so that all weights of a kind are rounded alike: the largest, whose weight is exact, with
    values of zero, and two kinds whose fp16 weights are off by -1.87 and +1.80 times 2^-12 and whose values cancel.
    fp16 has 11 significant bits: a weight is off by up to 2^-11 of itself (finfo.eps / 2), hence the output by up
    to 2^-11 sum w|v|.  Two bf16 terms leave 2^-8 of 2^-8 of a weight.  A score is one exact product times
    log2(e) / sqrt(128), 3 roundings of 2^-24 of at most 2; exponential 2^-22, sums 2^-20: below 2^-18 together."""
    spkv = load()
    T0, big, plus, minus = 6000, 1.0, 0.486328125, 0.515625
    cache = make(spkv, n_seqs=B + 1, Hq=16, Hkv=2, pool=2 * (T0 // 64 + 2) + B * 8, max_context=T0 + 64,
                 flags=spkv.FLAG_FORK | (spkv.FLAG_PREFILL_PV_BF16 if wide else 0))
    wl = Workload(1, T0, 1, 16, 2, (1.0, 1.0), cache.spkv_tau_logit(), with_q=False)
    kind = np.arange(T0) % 64
    k = np.where(kind == 5, big, np.where(kind % 2 == 0, plus, minus)).astype(np.float32)
    n_plus, n_minus = (kind % 2 == 0).sum(), ((kind % 2 == 1) & (kind != 5)).sum()
    w = lambda x: np.exp(15.0 * (x - big) / math.sqrt(D))
    v = np.where(kind == 5, 0.0, np.where(kind % 2 == 0, 1.0, -n_plus * w(plus) / (n_minus * w(minus)))).astype(np.float32)
    keys = np.zeros((T0, 1, 2, D), np.float32)
    keys[..., 0] = k[:, None, None]
    wl.K, wl.V = synth.to_bf16_bits(keys), synth.to_bf16_bits(np.broadcast_to(v[:, None, None, None], keys.shape).copy())
    feed(cache, wl, 0, 0, 0, 0, T0)
    cache.spkv_seq_fork(0, range(1, B + 1))
    ids = torch.arange(1, B + 1, dtype=torch.int32, device=dev())
    q = np.zeros((B, 16, D), np.float32)
    q[..., 0] = 15.0
    q = synth.to_bf16_bits(q)
    out = cache.spkv_decode_attention_shared(0, ids, to_dev_bf16(q), cache.spkv_share_plan(ids))
    cache.check()
    ref, wv, _, _ = reference(cache, 0, 1, 0, f64(q[0, :8]))
    tol = 2.0 ** -8 * np.abs(ref) + ((2.0 ** -16 if wide else 2.0 ** -11) + 2.0 ** -18) * wv
    err = np.abs(out.double().cpu().numpy().reshape(B, 2, 8, D) - ref)
    assert np.abs(ref).max() < 2.0 ** -8 * wv.min(), "the values cancel"
    assert (err <= tol).all(), (err / wv).max() * 2 ** 12
