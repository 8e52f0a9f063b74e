"""Drafted trees: attention over cache and ancestors against the formula in 64 bits over the pairs the cache holds, and against
appending each node's path and decoding; accepted paths in the cache against the oracle and against single appends."""
import math

import numpy as np
import pytest
import torch

import oracle
from gpu_util import D, Workload, compare_state, dev, load, to_dev_bf16
from paper_2605_14037_b200 import synth

pytestmark = pytest.mark.gpu
SC = 1 / math.sqrt(D)


def f64(bits):
    return synth.bf16_bits_to_f32(np.asarray(bits)).astype(np.float64)


def host(t):
    return t.detach().cpu().view(torch.int16).numpy().view(np.uint16)


class Case:
    """A cache of sequences of the lengths `lens` (workload sequence j in slot j) and drafts of T nodes each."""

    def __init__(self, spkv, lens, Hq, Hkv, T, rates, w=128, seed=0, layers=1, parent="tree", n=None, flags=0, draft_rate=0.5, max_seqs=None,
                 pool=None, fused=False, tau=0.5, **kw):
        self.spkv, self.lens, self.Hq, self.Hkv, self.T, self.w, self.B = spkv, list(lens), Hq, Hkv, T, w, len(lens)
        B, G = self.B, Hq // Hkv
        pool = pool if pool is not None else layers * sum(Hkv * (t // 64 + 2) for t in lens) + 2 * B * Hkv * layers
        self.cache = spkv.Cache(layers, max_seqs or B, Hq, Hkv, max(lens) + 3 * T + 64, max(pool, 1), window=w, tau=tau,
                                device=dev(), flags=flags, **kw)
        self.tl = self.cache.spkv_tau_logit()
        rng = np.random.default_rng(seed)
        self.wl = [Workload(seed * 31 + l, max(max(lens), 1), B, Hq, Hkv, rates, self.tl, with_q=False) for l in range(layers)]
        for l in range(layers):
            for j, t in enumerate(lens):
                for a in range(0, t, 4096):
                    b = min(t, a + 4096)
                    k, v = (to_dev_bf16(np.ascontiguousarray(x[a:b, j])) for x in (self.wl[l].K, self.wl[l].V))
                    self.cache.spkv_prefill(l, j, k, v, torch.from_numpy(np.ascontiguousarray(self.wl[l].logit[a:b, j])).to(dev()))
        i = np.arange(T)
        if isinstance(parent, str):
            if parent == "chain":
                p = np.broadcast_to(i - 1, (B, T))
            elif parent == "forest":
                p = np.stack([[rng.integers(-1, x) if x else -1 for x in i] for _ in range(B)])
            else:
                p = np.stack([[max(0, x - 1 - rng.integers(0, min(x, 4))) if x else -1 for x in i] for _ in range(B)])
        else:
            p = np.asarray(parent)
        self.parent = np.ascontiguousarray(p, dtype=np.int32).reshape(B, T)
        self.n = np.full(B, T, np.int32) if n is None else np.asarray(n, np.int32)
        self.q, self.k, self.v = (synth.normal_bf16(rng, (B, T, h, D)) for h in (Hq, Hkv, Hkv))
        base = self.tl if math.isfinite(self.tl) else 0.0
        self.lg = synth.logits_with_keep_rate(rng, (B, T, Hkv), draft_rate, base).astype(np.float32)
        self.fused = fused
        self.ids = torch.arange(B, dtype=torch.int32, device=dev())
        self.to_device()

    def to_device(self):
        if self.fused:   # as views of one [B, T, Hq + 2 Hkv, 128] tensor
            f = to_dev_bf16(np.concatenate([self.q, self.k, self.v], 2))
            self.qd, self.kd, self.vd = f[:, :, :self.Hq], f[:, :, self.Hq:self.Hq + self.Hkv], f[:, :, self.Hq + self.Hkv:]
        else:
            self.qd, self.kd, self.vd = (to_dev_bf16(x) for x in (self.q, self.k, self.v))
        self.pd, self.nd = torch.from_numpy(self.parent).to(dev()), torch.from_numpy(self.n).to(dev())
        self.ld = torch.from_numpy(self.lg).to(dev())

    def path(self, b, i):
        line = []
        while i >= 0:
            line.append(i)
            i = int(self.parent[b, i])
        return line[::-1]

    def run(self, layer=0, ids=None, **kw):
        kw.setdefault("logits", self.ld)
        return self.cache.spkv_decode_attention_tree(layer, self.ids if ids is None else ids, self.qd, self.kd, self.vd, self.pd, self.nd,
                                                     want_lse=True, **kw)

    def reference(self, b, h, layer=0, seq=None, thr=None, sinks=0, local=False, scale=SC):
        """(out [n, G, D], sum w |v|, lse [n, G], largest |q| |k|, keys) of the nodes of tree b and KV head h"""
        seq = b if seq is None else seq
        thr = self.tl if thr is None else thr
        G, n = self.Hq // self.Hkv, int(self.n[b])
        kept, ring = self.cache.spkv_read_kept(layer, seq, h), self.cache.spkv_read_window(layer, seq, h)
        t = int(self.cache.spkv_read_lengths(layer)[1][seq, h])
        lines = [self.path(b, i) for i in range(n)]
        depth = np.array([len(x) - 1 for x in lines])
        pos = np.concatenate([kept[0], ring[0], t + depth])
        k, v = (np.concatenate([f64(kept[i]), f64(ring[i]), f64(x[b, :n, h])]) for i, x in ((1, self.k), (2, self.v)))
        stays = np.concatenate([np.ones(len(kept[0]), bool), (np.concatenate([ring[3], self.lg[b, :n, h]]) >= thr) | (pos[len(kept[0]):] < sinks)])
        if local:
            stays[:] = False
        m = len(pos) - n
        out, wv, lse = np.zeros((n, G, D)), np.zeros((n, G, D)), np.zeros((n, G))
        for i, line in enumerate(lines):
            see = np.zeros(len(pos), bool)
            see[:m] = True
            see[m + np.array(line)] = True
            see &= (pos > t + depth[i] - self.w) | stays
            q = f64(self.q[b, i, h * G:(h + 1) * G])
            with np.errstate(invalid="ignore"):
                s = q @ k[see].T * scale
                mx = s.max(-1, keepdims=True)
                p = np.exp(s - mx)
                z = p.sum(-1, keepdims=True)
                out[i], wv[i], lse[i] = p @ v[see] / z, p @ np.abs(v[see]) / z, (mx + np.log(z))[:, 0]
        qk = np.linalg.norm(f64(self.q[b, :n, h * G:(h + 1) * G]), axis=-1).max() * np.linalg.norm(k, axis=-1).max() if n else 0
        return out, wv, lse, qk, len(pos)

    def bounds(self, b, h, layer=0, seq=None, scale=SC, **kw):
        """Scores: 128 products added in fp32, es = 130 * 2^-24 |q| |k| scale (twice that as a relative error of a weight, on both
        sides of the quotient).  A weight is two bf16 terms: 8 bits each, 2^-16 of it; its exponential is within 2^-22.
        Products are added in fp32, 16 pairs and one term a step: off by up to a step's 2^-23 of the sum, 2 keys / 16 steps and as
        many for every part that is joined.  The result is rounded to bf16 by half a step, 2^-8 of the value."""
        ref, wv, rl, qk, keys = self.reference(b, h, layer, seq, scale=scale, **kw)
        es = 130 * 2.0 ** -24 * qk * scale
        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -16 + 2.0 ** -21 + 2 * es + (keys / 8 + 64) * 2.0 ** -23) * wv + 1e-30
        return tol, es + (keys / 8 + 64) * 2.0 ** -23 + 2.0 ** -20 * (1 + np.abs(rl))

    def check(self, out, lse, layer=0, seqs=None, scale=SC, trees=None, **kw):
        G = self.Hq // self.Hkv
        got, l = out.float().cpu().double().numpy(), lse.cpu().double().numpy()
        for b in range(self.B) if trees is None else trees:
            n = int(self.n[b])
            for h in range(self.Hkv):
                seq = None if seqs is None else seqs[b]
                ref, _, rl, _, _ = self.reference(b, h, layer, seq, scale=scale, **kw)
                hs = slice(h * G, (h + 1) * G)
                tol, el = self.bounds(b, h, layer, seq, scale=scale, **kw)
                err = np.abs(got[b, :n, hs] - ref)
                assert (err <= tol).all(), (b, h, err.max(), (err / tol).max())
                assert (np.abs(l[b, :n, hs] - rl) <= el).all(), (b, h, np.abs(l[b, :n, hs] - rl).max())


CASES = [
    # lens, Hq, Hkv, T, rates, w, more
    ((300,), 8, 2, 4, (0.5, 1.0), 128, {}),
    ((0, 1, 63, 64, 65), 4, 2, 3, (0.5, 1.0), 128, {}),              # nothing received yet, less than a window
    ((127, 128, 129, 130, 193), 6, 2, 9, (0.0, 0.4), 128, {}),       # around the window, G = 3
    ((1000, 40, 257), 2, 2, 1, (0.7, 0.1), 128, {}),                 # single tokens, G = 1
    ((700, 900), 16, 1, 8, (0.6,), 128, {"parent": "chain"}),        # G = 16: 128 query rows exactly
    ((700, 900), 16, 1, 9, (0.6,), 128, {"parent": "forest"}),       # a row more than a tile
    ((2000,), 40, 8, 13, (0.3,) * 8, 128, {}),                       # G = 5
    ((500, 90, 1300), 32, 2, 64, (0.9, 0.2), 128, {}),               # 1024 rows
    ((600, 50, 7), 8, 2, 64, (0.5, 0.2), 1, {"parent": "chain"}),    # a window of one pair: every ancestor has left it
    ((600, 5, 3, 0), 8, 2, 40, (0.5, 0.2), 16, {"parent": "chain"}), # drafts leave the window
    ((600, 45), 8, 2, 33, (0.5, 0.2), 5, {"parent": "forest", "draft_rate": 0.2}),
    ((900, 333), 4, 1, 17, (0.3,), 200, {}),                         # four ring pages, the last in part
    ((900, 64), 4, 1, 17, (0.3,), 64, {}),
    ((3000, 100, 1500, 2200, 5), 12, 4, 27, (0.9, 0.05, 0.0, 0.5), 128, {"n": (27, 1, 13, 0, 26), "parent": "forest"}),
    ((20000,), 8, 2, 16, (1.0, 0.02), 128, {}),                      # a long and a short head
    ((400,) * 40, 8, 2, 5, (0.4, 0.9), 128, {"fused": True}),
]


@pytest.mark.parametrize("lens,Hq,Hkv,T,rates,w,more", CASES)
def test_against_the_formula(lens, Hq, Hkv, T, rates, w, more):
    c = Case(load(), lens, Hq, Hkv, T, rates, w, seed=len(lens) * 100 + T, **more)
    before = c.cache.arena.clone()
    out, lse = c.run()
    c.cache.check()
    c.check(out, lse)
    again, lse2 = c.run()
    for b in range(c.B):
        n = int(c.n[b])
        assert torch.equal(out[b, :n], again[b, :n]) and torch.equal(lse[b, :n], lse2[b, :n])
    assert torch.equal(c.cache.arena, before), "the call only reads the cache"


@pytest.mark.parametrize("w,T,lens,sinks", [(128, 6, (500, 126, 30), 0), (4, 12, (90, 3, 0), 0), (1, 5, (70, 64), 3), (16, 20, (10, 333), 20)])
def test_equals_appending_the_path_and_decoding(w, T, lens, sinks):
    """Both sides are off by at most what `check` allows; held to the sum of the two."""
    c = Case(load(), lens, 6, 2, T, (0.5, 0.8), w, seed=T, parent="forest", sink_tokens=sinks, pool=200)
    out, lse = c.run()
    c.check(out, lse, sinks=sinks)
    saved = c.cache.spkv_cache_checkpoint()
    for i in range(T):
        for b in range(c.B):
            for x in c.path(b, i):
                c.cache.spkv_append_evict(0, c.ids[b:b + 1], *(a[b:b + 1, x].contiguous() for a in (c.kd, c.vd, c.ld)))
        l1 = torch.empty((c.B, c.Hq), device=dev())
        _, want = c.cache.spkv_decode_attention_f32(0, c.ids, c.qd[:, i].contiguous(), lse=l1)
        # |q| |k| scale < 30 for these normal rows: es < 2.4e-4; values below 6 in size
        tol = 2.0 ** -8 * want.abs() + 2 * (2.0 ** -16 + 2 * 2.4e-4 + 2.0 ** -16) * 6
        assert ((out[:, i].float() - want).abs() <= tol).all(), i
        assert ((lse[:, i] - l1).abs() <= 2 * 2.4e-4 + 2.0 ** -18).all()
        c.cache.spkv_cache_rollback(saved)
    c.cache.check()


def test_one_node_is_a_decode_step_after_its_append():
    c = Case(load(), (800, 128, 5, 0), 8, 2, 1, (0.5, 0.2), seed=4)
    out, lse = c.run()
    c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, c.ld)
    l1 = torch.empty((c.B, c.Hq), device=dev())
    _, want = c.cache.spkv_decode_attention_f32(0, c.ids, c.qd[:, 0].contiguous(), lse=l1)
    tol = 2.0 ** -8 * want.abs() + 2 * (2.0 ** -15 + 2 * 2.4e-4) * 6
    assert ((out[:, 0].float() - want).abs() <= tol).all() and ((lse[:, 0] - l1).abs() <= 2 * 2.4e-4 + 2.0 ** -18).all()
    c.cache.check()


def test_rows_of_absent_nodes_and_foreign_sequences_are_left_alone():
    c = Case(load(), (300, 40, 700), 8, 2, 10, (0.5, 0.2), n=(4, 0, 10), max_seqs=4)
    out, lse = torch.full((3, 10, 8, D), 7.0, dtype=torch.bfloat16, device=dev()), torch.full((3, 10, 8), 7.0, device=dev())
    c.run(out=out, lse=lse)
    c.cache.check()
    c.check(out, lse)
    assert (out[0, 4:] == 7).all() and (lse[0, 4:] == 7).all() and (out[1] == 7).all() and (lse[1] == 7).all()
    for bad in (-1, 4, 1 << 30):
        out.fill_(7), lse.fill_(7)
        c.run(out=out, lse=lse, ids=torch.tensor([0, bad, 2], dtype=torch.int32, device=dev()))
        assert c.cache.spkv_status() == -9
        c.cache.spkv_clear_status()
        c.check(out, lse)
        c.n[0] = 4
        out.fill_(7)
        c.nd = torch.tensor([4, 3, 10], dtype=torch.int32, device=dev())
        c.run(out=out, lse=lse, ids=torch.tensor([0, bad, 2], dtype=torch.int32, device=dev()))
        assert c.cache.spkv_status() == -9 and (out[1] == 7).all()
        c.cache.spkv_clear_status()
        c.nd = torch.from_numpy(c.n).to(dev())


def test_counts_and_parents_out_of_range():
    c = Case(load(), (300, 40), 4, 2, 6, (0.5, 0.2), parent="forest")
    good = c.parent.copy()
    for bad in (5, 6, 1 << 30, -2, -(1 << 31)):
        c.parent = good.copy()
        c.parent[1, 5] = bad
        c.to_device()
        c.parent[1, 5] = -1
        out, lse = c.run()
        assert c.cache.spkv_status() == -9, bad
        c.cache.spkv_clear_status()
        c.check(out, lse)
    c.parent = good
    for n, want in ((9, 6), (-3, 0)):
        c.n = np.array([6, n], np.int32)
        c.to_device()
        c.n[1] = want
        out, lse = c.run()
        assert c.cache.spkv_status() == -9
        c.cache.spkv_clear_status()
        c.check(out, lse)


def test_several_trees_on_one_sequence_and_layers():
    c = Case(load(), (500, 800), 8, 2, 7, (0.5, 0.2), layers=3, seed=9)
    for layer in (2, 0):
        out, lse = c.run(layer, ids=torch.tensor([1, 1], dtype=torch.int32, device=dev()))
        c.check(out, lse, layer=layer, seqs=[1, 1])
    c.cache.check()


def test_thresholds_sinks_and_local_heads():
    spkv = load()
    local = np.zeros((2, 4), bool)
    local[1, 2] = True
    c = Case(spkv, (40, 200), 8, 4, 20, (0.5, 0.2, 0.9, 0.4), w=8, layers=2, local_only=local, sink_tokens=12, parent="chain", seed=3)
    for layer in (0, 1):
        out, lse = c.run(layer)
        for b in range(2):
            for h in range(4):
                one = lambda t: t[:, :, 2 * h:2 * h + 2]
                ref, wv, rl, qk, keys = c.reference(b, h, layer, sinks=12, local=local[layer, h])
                err = np.abs(out[b, :, 2 * h:2 * h + 2].float().cpu().double().numpy() - ref)
                es = 130 * 2.0 ** -24 * qk * SC
                assert (err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -16 + 2.0 ** -21 + 2 * es + (keys / 8 + 64) * 2.0 ** -23) * wv).all(), (layer, b, h)
    # a head's own threshold, and a changed cache-wide one, hold for the pairs of window and path from now on
    c = Case(spkv, (300, 64), 8, 2, 24, (0.5, 0.5), w=8, parent="chain", seed=5)
    for tau in (0.05, 0.97, 0.0, 1.0):
        c.cache.spkv_set_tau(tau)
        out, lse = c.run()
        c.check(out, lse, thr=c.cache.spkv_tau_logit())
    c.cache.spkv_set_tau(0.5)
    c.cache.spkv_set_head_tau(0, -1, 0.9)
    out, lse = c.run()
    c.check(out, lse, thr=float(np.float32(math.log(0.9 / (1 - np.float32(0.9).astype(np.float64))))))


def test_without_logits():
    c = Case(load(), (300, 64), 8, 2, 16, (0.5, 0.5), w=16, parent="chain")
    a, la = c.run()
    b, lb = c.run(logits=None)
    assert torch.equal(a, b) and torch.equal(la, lb)
    c.cache.check()


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan, 3.3e38])
def test_what_a_node_does_not_see_does_not_touch_it(bad):
    """Infinities and NaN in keys and values of other branches, of pairs that left the node's window without
    being kept, of absent nodes, and behind the last pair of a ring page."""
    spkv = load()
    w = 8
    c = Case(spkv, (40, 3, 80), 8, 2, 12, (0.4, 0.4), w=w, parent="forest", n=(12, 9, 12), seed=2, draft_rate=0.3)
    bits = synth.to_bf16_bits(np.array([bad], np.float32))[0]
    clean_out, clean_lse = c.run()
    c.check(clean_out, clean_lse)
    bounds = {(b, h): c.bounds(b, h) for b in range(c.B) for h in range(2)}
    for b in range(c.B):
        for x in range(c.T):
            k0, v0 = c.k.copy(), c.v.copy()
            c.k[b, x, 0, 5] = bits
            c.v[b, x, 0, ::3] = bits
            c.to_device()
            out, lse = c.run()
            for i in range(int(c.n[b])):
                line = c.path(b, i)
                sees = x in line and (len(line) - 1 - line.index(x) < w or c.lg[b, x, 0] >= c.tl)
                if sees:
                    assert not torch.equal(out[b, i, :4], clean_out[b, i, :4]), (b, x, i)
                for hs, untouched in ((slice(0, 4), not sees), (slice(4, 8), True)):   # (the other KV head has nothing planted)
                    if untouched:   # both as near to the formula as `check` asks
                        err = (out[b, i, hs].float() - clean_out[b, i, hs].float()).abs().cpu().double().numpy()
                        el = (lse[b, i, hs] - clean_lse[b, i, hs]).abs().cpu().double().numpy()
                        assert (err <= 2 * bounds[b, hs.start // 4][0][i]).all() and (el <= 2 * bounds[b, hs.start // 4][1][i]).all(), (b, x, i)
            c.k, c.v = k0, v0
    c.cache.check()


@pytest.mark.parametrize("where", ["ring", "kept", "draft"])
def test_infinite_values_that_are_seen(where):
    """weight times infinity is infinity, of both signs NaN, whatever the other pairs hold"""
    spkv = load()
    c = Case(spkv, (400, 400), 8, 2, 5, (0.5, 0.5), seed=6, parent="chain")
    plant = np.random.default_rng(0)
    if where == "draft":
        c.v[0, 1, 0, 3], c.v[0, 1, 0, 4], c.v[0, 2, 0, 4], c.v[0, 3, 1, 7] = 0x7f80, 0x7f80, 0xff80, 0x7fc0
        c.to_device()
    else:
        spkv_cache = c.cache
        # through a fresh sequence: append pairs whose values are infinite, then enough others that they leave the window (kept)
        k = synth.normal_bf16(plant, (4, 2, 2, D))
        v = synth.normal_bf16(plant, (4, 2, 2, D))
        v[0, 0, 0, 3], v[0, 0, 0, 4], v[1, 0, 0, 4], v[2, 0, 1, 7] = 0x7f80, 0x7f80, 0xff80, 0x7fc0
        for x in range(4):
            spkv_cache.spkv_append_evict(0, c.ids, to_dev_bf16(k[x]), to_dev_bf16(v[x]), torch.full((2, 2), 9.0, device=dev()))
        if where == "kept":
            for x in range(130):
                r = to_dev_bf16(synth.normal_bf16(plant, (2, 2, D)))
                spkv_cache.spkv_append_evict(0, c.ids, r, r, torch.full((2, 2), -9.0, device=dev()))
    out, lse = c.run()
    got = out.float().cpu().double().numpy()
    for b in range(2):
        for h in range(2):
            with np.errstate(invalid="ignore"):
                ref = c.reference(b, h)[0]
            mine = got[b, :, 4 * h:4 * h + 4]
            assert np.array_equal(np.isnan(ref), np.isnan(mine)), (b, h)
            assert np.array_equal(ref == np.inf, mine == np.inf) and np.array_equal(ref == -np.inf, mine == -np.inf)
            ok = np.isfinite(ref)
            assert (np.abs(ref[ok] - mine[ok]) <= 2.0 ** -8 * np.abs(ref[ok]) + 0.01).all()
    assert (~np.isfinite(got)).any() and torch.isfinite(lse).all()
    c.cache.check()


def test_layouts_of_the_drafts():
    """views of a fused projection, head-major tensors, one row for all heads or tokens"""
    c = Case(load(), (300, 700), 8, 2, 6, (0.5, 0.2), seed=8)
    want, wl = c.run()
    c.fused = True
    c.to_device()
    assert not c.qd.is_contiguous()
    got, gl = c.run()
    assert torch.equal(want, got) and torch.equal(wl, gl)
    c.qd, c.kd, c.vd = (x.reshape(12, x.shape[2], D).transpose(0, 1).contiguous().transpose(0, 1).view(2, 6, x.shape[2], D) for x in (c.qd, c.kd, c.vd))
    got, gl = c.run()
    assert torch.equal(want, got) and torch.equal(wl, gl)
    c.k, c.v = c.k[:, :, :1].repeat(2, 2), c.v[:1, :1].repeat(2, 0).repeat(6, 1)
    c.kd, c.vd = to_dev_bf16(c.k[:, :, :1]).expand(-1, -1, 2, -1), to_dev_bf16(c.v[:1, :1]).expand(2, 6, -1, -1)
    out, lse = c.run()
    c.check(out, lse)


def test_scales():
    c = Case(load(), (900,), 8, 2, 6, (0.5, 0.2), seed=8)
    for scale in (1e-6, 0.5, 3.0):
        out, lse = c.run(sm_scale=scale)
        c.check(out, lse, scale=scale)


@pytest.mark.parametrize("B,Hq,Hkv,T", [(1024, 1, 1, 2), (64, 16, 16, 3), (341, 24, 3, 5), (128, 128, 8, 8)])
def test_the_largest_batches(B, Hq, Hkv, T):
    rng = np.random.default_rng(B)
    c = Case(load(), [int(x) for x in rng.integers(0, 260, B)], Hq, Hkv, T, tuple(0.2 + 0.8 * (i % 2) for i in range(Hkv)), w=64,
             n=rng.integers(0, T + 1, B), seed=B)
    out, lse = c.run()
    c.cache.check()
    c.check(out, lse, trees=sorted({0, 1, B // 2, B - 2, B - 1, *range(0, B, max(1, B // 12))}))


def test_one_long_sequence_among_many_short_ones():
    """shares of the long one in many blocks, and blocks that hold many short ones"""
    c = Case(load(), [30] * 50 + [30000] + [100] * 60, 4, 1, 3, (0.8,), seed=1)
    out, lse = c.run()
    c.cache.check()
    c.check(out, lse, trees=[0, 1, 25, 49, 50, 51, 80, 110])


def test_cuts_on_the_borders_of_short_units():
    """A long and a short sequence in turn, as many pairs of them as half the blocks, so that every second cut falls on the end of
    a short one: none is left out."""
    c = Case(load(), (19000, 1), 2, 1, 2, (1.0,), seed=3, max_seqs=296, pool=310)
    n = torch.cuda.get_device_properties(0).multi_processor_count
    ids = torch.tensor([0, 1] * n, dtype=torch.int32, device=dev())
    wide = lambda t: t.repeat(n, *[1] * (t.dim() - 1))
    want, wl = c.run()
    c.check(want, wl)
    out, lse = torch.full((2 * n, 2, 2, D), 7.0, dtype=torch.bfloat16, device=dev()), torch.full((2 * n, 2, 2), 7.0, device=dev())
    c.cache.spkv_decode_attention_tree(0, ids, wide(c.qd), wide(c.kd), wide(c.vd), wide(c.pd), wide(c.nd), wide(c.ld), out, lse)
    c.cache.check()
    # (the cuts differ from those of the two alone: rounding as in `bounds`)
    for b in range(2):
        tol, el = c.bounds(b, 0)
        assert ((out[b::2].float() - want[b].float()).abs().cpu().double().numpy() <= 2 * tol).all()
        assert ((lse[b::2] - wl[b]).abs().cpu().double().numpy() <= 2 * el).all()


def test_debug_bounds_and_overlap_caches():
    spkv = load()
    for flags in (spkv.FLAG_DEBUG_BOUNDS, spkv.FLAG_OVERLAP, spkv.FLAG_FORK):
        c = Case(spkv, (300, 700), 8, 2, 6, (0.5, 0.2), seed=8, flags=flags)
        out, lse = c.run()
        c.check(out, lse)
        c.cache.check()
        if flags == spkv.FLAG_OVERLAP:   # between hot-path launches of other layers' kind
            c.cache.spkv_append_evict(0, c.ids, *(a[:, 0].contiguous() for a in (c.kd, c.vd, c.ld)))
            out, lse = c.run()
            c.cache.spkv_append_evict(0, c.ids, *(a[:, 1].contiguous() for a in (c.kd, c.vd, c.ld)))
            c.cache.spkv_cache_stats()
            torch.cuda.synchronize()
            after = c.run()
            c.check(*after)
            c.cache.check()


# ---- accept --------------------------------------------------------------------------------------------
def walk(n, parent, tokens, target):
    if n <= 0:
        return [], -1
    line = [0]
    while True:
        nxt = [x for x in range(line[-1] + 1, n) if parent[x] == line[-1] and tokens[x] == target[line[-1]]]
        if not nxt:
            return line, int(target[line[-1]])
        line.append(nxt[0])


@pytest.mark.parametrize("B,T,vocab,kind", [(1, 1, 3, "tree"), (7, 8, 2, "tree"), (64, 64, 2, "forest"), (33, 64, 1, "chain"), (500, 33, 3, "tree"),
                                            (5, 32, 2, "wild")])
def test_accept(B, T, vocab, kind):
    spkv = load()
    rng = np.random.default_rng(B * T)
    i = np.arange(T)
    parent = {"chain": lambda: np.broadcast_to(i - 1, (B, T)), "forest": lambda: rng.integers(-1, np.maximum(i, 1) , (B, T)),
              "tree": lambda: np.maximum(0, i - 1 - rng.integers(0, 4, (B, T))) - (i == 0),
              "wild": lambda: rng.integers(-3, T + 3, (B, T))}[kind]().astype(np.int32)
    tokens, target = rng.integers(0, vocab, (2, B, T)).astype(np.int32)
    n = rng.integers(-1 if kind == "wild" else 0, T + 2 if kind == "wild" else T + 1, B).astype(np.int32)
    d = [torch.from_numpy(np.ascontiguousarray(x)).to(dev()) for x in (tokens, target, parent, n)]
    for counts in (n, None):
        path, n_path, nxt = (x.cpu().numpy() for x in spkv.spkv_tree_accept(d[0], d[1], d[2], None if counts is None else d[3]))
        for b in range(B):
            m = T if counts is None else max(0, min(T, int(n[b])))
            line, then = walk(m, np.where(parent[b] < i, parent[b], -1), tokens[b], target[b])
            assert n_path[b] == len(line) and nxt[b] == then and path[b].tolist() == line + [-1] * (T - len(line)), b
    if kind == "chain":
        same = spkv.spkv_tree_accept(d[0], d[1])
        assert np.array_equal(same[0].cpu().numpy(), path)


def test_accept_of_nothing():
    spkv = load()
    none = torch.empty((3, 0), dtype=torch.int32, device=dev())
    path, n_path, nxt = spkv.spkv_tree_accept(none, none)
    assert path.shape == (3, 0) and n_path.tolist() == [0] * 3 and nxt.tolist() == [-1] * 3
    assert spkv.spkv_tree_accept(none[:0], none[:0])[1].shape == (0,)


# ---- append --------------------------------------------------------------------------------------------
def units(c, layer, paths, thr=None):
    got = []
    for b in range(c.B):
        for h in range(c.Hkv):
            u = oracle.Unit(c.w, D)
            rows = [np.ascontiguousarray(np.concatenate([x[:c.lens[b], b, h], y[b, paths[b], h]]))
                    for x, y in ((c.wl[layer].K, c.k), (c.wl[layer].V, c.v), (c.wl[layer].logit, c.lg))]
            if len(rows[0]):
                u.prefill(*rows, c.tl if thr is None else thr)
            got.append((b, h, u))
    return got


@pytest.mark.parametrize("lens,T,w,more", [
    ((300, 128, 127, 0, 5), 8, 128, {}),
    ((300, 120, 64, 191, 192, 193), 64, 128, {"parent": "chain"}),
    ((300, 2, 0, 63, 64), 64, 4, {}),          # most of the path leaves the window at once
    ((300, 2, 0), 64, 1, {"draft_rate": 1.0}),
    ((70, 66, 65, 64), 63, 64, {"draft_rate": 0.9}),
    ((1000,) * 20, 5, 200, {"fused": True}),
])
def test_append_path_against_the_oracle(lens, T, w, more):
    c = Case(load(), lens, 4, 2, T, (0.5, 1.0), w, seed=T + w, **more)
    rng = np.random.default_rng(T)
    paths = [rng.permutation(T)[:rng.integers(0, T + 1)].tolist() for _ in lens]
    paths[0] = list(range(T))
    paths[-1] = [0] * T                        # the same node again and again
    if len(lens) > 3:
        paths[1] = []
    path = np.full((c.B, T), -1, np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    pd, nd = torch.from_numpy(path).to(dev()), torch.tensor([len(p) for p in paths], dtype=torch.int32, device=dev())
    before = c.cache.spkv_cache_stats()
    c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, c.ld, pd, nd)
    c.cache.check()
    pages = 0
    for b, h, u in units(c, 0, paths):
        compare_state(c.cache, 0, b, h, u)
        pages += (len(u) + 63) // 64
    stats = c.cache.spkv_cache_stats()
    assert stats.pages_in_use == pages and stats.pages_in_use + stats.pages_free == c.cache.cfg.pool_pages
    # what attention reads behind it: zeros behind the last row of a page, the largest value
    out, lse = c.run()
    c.check(out, lse)
    if T <= 8:
        q = to_dev_bf16(synth.normal_bf16(rng, (3, 4, D)))
        r = to_dev_bf16(synth.normal_bf16(rng, (3, 2, D)))
        o = c.cache.spkv_prefill(0, 0, r, r, torch.zeros((3, 2), device=dev()), q=q)
        assert torch.isfinite(o.float()).all()


def test_append_of_several_layers_at_once():
    spkv = load()
    c = Case(spkv, (200, 130, 7), 4, 2, 6, (0.5, 0.9), layers=4, seed=1)
    rng = np.random.default_rng(1)
    k, v = (synth.normal_bf16(rng, (3, c.B, c.T, 2, D)) for _ in "kv")
    lg = rng.normal(size=(3, c.B, c.T, 2)).astype(np.float32)
    path, n = torch.tensor([[0, 2, 5, -1, -1, -1], [0, 1, 2, 3, 4, 5], [-7] * 6], dtype=torch.int32, device=dev()), torch.tensor([3, 6, 0], dtype=torch.int32, device=dev())
    wide = to_dev_bf16(np.concatenate([k, v], 3))    # [3, B, T, 4, D]: views with strides of their own
    c.cache.spkv_append_path(1, c.ids, wide[:, :, :, :2], wide[:, :, :, 2:], torch.from_numpy(lg).to(dev()), path, n)
    c.cache.check()
    for layer in range(4):
        if layer:
            c.k, c.v, c.lg = k[layer - 1], v[layer - 1], lg[layer - 1]
        for b, h, u in units(c, layer, [[0, 2, 5], [0, 1, 2, 3, 4, 5], []] if layer else [[], [], []]):
            compare_state(c.cache, layer, b, h, u)


def test_append_path_as_an_append_of_several_tokens():
    c = Case(load(), (200, 130, 7), 4, 2, 6, (0.5, 0.9), seed=1)
    c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, c.ld)
    c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, c.ld, n_path=torch.tensor([2, 0, 6], dtype=torch.int32, device=dev()))
    c.cache.check()
    for b, h, u in units(c, 0, [[*range(6), 0, 1], [*range(6)], [*range(6)] * 2]):
        compare_state(c.cache, 0, b, h, u)


def test_append_path_with_sinks_local_heads_and_thresholds():
    spkv = load()
    local = np.array([[0, 1, 0]], bool)
    a, b = (Case(spkv, (3, 20, 9), 6, 3, 40, (0.5, 0.5, 0.5), w=8, local_only=local, sink_tokens=14, seed=7, parent="chain") for _ in "ab")
    for c in (a, b):
        c.cache.spkv_set_head_tau(0, 2, 0.8)
    a.cache.spkv_append_path(0, a.ids, a.kd, a.vd, a.ld)
    for x in range(40):
        b.cache.spkv_append_evict(0, b.ids, *(t[:, x].contiguous() for t in (b.kd, b.vd, b.ld)))
    for s in range(3):
        for h in range(3):
            for x, y in zip(a.cache.spkv_read_kept(0, s, h) + a.cache.spkv_read_window(0, s, h),
                            b.cache.spkv_read_kept(0, s, h) + b.cache.spkv_read_window(0, s, h)):
                assert np.array_equal(x, y), (s, h)
    a.cache.check()


@pytest.mark.parametrize("pool,max_context,code", [(1, 4096, -5), (2, 4096, -5), (50, 64, -6)])
def test_append_path_without_room_stores_what_fits(pool, max_context, code):
    spkv = load()

    def fresh():
        cache = spkv.Cache(1, 1, 1, 1, max_context, pool, window=2, tau=0.0, device=dev())
        return cache

    rng = np.random.default_rng(0)
    k, v = (to_dev_bf16(synth.normal_bf16(rng, (1, 64, 1, D))) for _ in "kv")
    lg, ids = torch.zeros((1, 64, 1), device=dev()), torch.zeros(1, dtype=torch.int32, device=dev())
    a, b = fresh(), fresh()
    for _ in range(3):
        a.spkv_append_path(0, ids, k, v, lg)
        for x in range(64):
            b.spkv_append_evict(0, ids, k[:, x].contiguous(), v[:, x].contiguous(), lg[:, x].contiguous())
    assert a.spkv_status() == b.spkv_status() == code
    for x, y in zip(a.spkv_read_kept(0, 0, 0) + a.spkv_read_window(0, 0, 0), b.spkv_read_kept(0, 0, 0) + b.spkv_read_window(0, 0, 0)):
        assert np.array_equal(x, y)


def test_append_path_entries_out_of_range():
    c = Case(load(), (200, 130), 4, 2, 40, (0.5, 0.9), seed=1)
    path = np.tile(np.arange(40, dtype=np.int32), (2, 1))
    path[0, 35], path[1, 2] = 40, -1
    c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, c.ld, torch.from_numpy(path).to(dev()))
    assert c.cache.spkv_status() == -9
    c.cache.spkv_clear_status()
    for b, h, u in units(c, 0, [[*range(35)], [0, 1]]):
        compare_state(c.cache, 0, b, h, u)
    c.cache.spkv_append_path(0, torch.tensor([-1, 2], dtype=torch.int32, device=dev()), c.kd, c.vd, c.ld)
    assert c.cache.spkv_status() == -9
    c.cache.spkv_clear_status()
    c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, c.ld, None, torch.tensor([-1, 41], dtype=torch.int32, device=dev()))
    assert c.cache.spkv_status() == -9
    for b, h, u in units(c, 0, [[*range(35)], [0, 1, *range(40)]]):
        compare_state(c.cache, 0, b, h, u)


# ---- a step, as it is used -----------------------------------------------------------------------------
def test_steps_equal_plain_decoding():
    """Ten steps of draft, tree attention, acceptance and commit give the state that single appends of the accepted tokens
    give, captured in a graph and replayed on its own outputs as well."""
    spkv = load()
    B, T, L = 3, 9, 2
    c, ref = (Case(spkv, (300, 127, 4), 8, 2, T, (0.5, 0.8), layers=L, seed=2, pool=400) for _ in "ab")
    rng = np.random.default_rng(5)
    k, v = (torch.empty((L, B, T, 2, D), dtype=torch.bfloat16, device=dev()) for _ in "kv")
    q = torch.empty((L, B, T, 8, D), dtype=torch.bfloat16, device=dev())
    lg = torch.empty((L, B, T, 2), device=dev())
    parent, tokens, target = (torch.empty((B, T), dtype=torch.int32, device=dev()) for _ in range(3))
    outs, lses = torch.empty_like(q), torch.empty((L, B, T, 8), device=dev())
    path, n_path, nxt = torch.empty((B, T), dtype=torch.int32, device=dev()), *(torch.empty(B, dtype=torch.int32, device=dev()) for _ in range(2))

    def step():
        for l in range(L):
            c.cache.spkv_decode_attention_tree(l, c.ids, q[l], k[l], v[l], parent, logits=lg[l], out=outs[l], lse=lses[l])
        spkv.spkv_tree_accept(tokens, target, parent, None, path, n_path, nxt)
        c.cache.spkv_append_path(0, c.ids, k, v, lg, path, n_path)

    def inputs():
        for t, heads in ((q, 8), (k, 2), (v, 2)):
            t.copy_(to_dev_bf16(synth.normal_bf16(rng, (L, B, T, heads, D))))
        lg.copy_(torch.from_numpy(rng.normal(size=(L, B, T, 2)).astype(np.float32)))
        p = np.maximum(0, np.arange(T) - 1 - rng.integers(0, 3, (B, T))) - (np.arange(T) == 0)
        for t, x in ((parent, p), (tokens, rng.integers(0, 2, (B, T))), (target, rng.integers(0, 2, (B, T)))):
            t.copy_(torch.from_numpy(x.astype(np.int32)))

    def reference_and_check():
        c.cache.check()
        line, n = path.cpu().numpy(), n_path.cpu().numpy()
        for i in range(int(n.max())):
            on = [b for b in range(B) if i < n[b]]
            ids = torch.tensor(on, dtype=torch.int32, device=dev())
            at = [int(line[b, i]) for b in on]
            for l in range(L):
                ref.cache.spkv_append_evict(l, ids, *(x[l][on, at].contiguous() for x in (k, v, lg)))
                if i + 1 == n.max():
                    continue
            for l in range(L):
                l1 = torch.empty((len(on), 8), device=dev())
                _, want = ref.cache.spkv_decode_attention_f32(l, ids, q[l][on, at].contiguous(), lse=l1)
                assert ((outs[l][on, at].float() - want).abs() <= 2.0 ** -8 * want.abs() + 2 * (2.0 ** -15 + 2 * 2.4e-4) * 6).all()
                assert ((lses[l][on, at] - l1).abs() <= 2 * 2.4e-4 + 2.0 ** -18).all()
        for l in range(L):
            for s in range(B):
                for h in range(2):
                    for x, y in zip(c.cache.spkv_read_kept(l, s, h) + c.cache.spkv_read_window(l, s, h),
                                    ref.cache.spkv_read_kept(l, s, h) + ref.cache.spkv_read_window(l, s, h)):
                        assert np.array_equal(x, y), (l, s, h)

    for _ in range(4):
        inputs()
        step()
        reference_and_check()
    graph = torch.cuda.CUDAGraph()
    inputs()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for _ in range(6):
        graph.replay()
        reference_and_check()
        inputs()


def test_two_streams_and_two_graphs_at_once():
    """Each call has a workspace of its own: eager on two streams, and captured graphs replayed side by side"""
    spkv = load()
    cs = [Case(spkv, (9000, 4000), 8, 2, 16, (0.9, 0.3), seed=s) for s in (1, 2)]
    want = [c.run() for c in cs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(5):
        got = [c.run(stream=s) for c, s in zip(cs, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, x in zip(got, want) for a, b in zip(g, x))
    # one cache read by two graphs at once
    c = cs[0]
    outs, graphs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.run())
        graphs.append(g)
    for _ in range(5):
        for o in outs:
            o[0].zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o[0], want[0][0]) and torch.equal(o[1], want[0][1]) for o in outs)
    c.cache.check()


def test_refusals():
    spkv = load()
    c = Case(spkv, (300, 40), 8, 2, 6, (0.5, 0.2))
    out = torch.full((2, 6, 8, D), 3.0, dtype=torch.bfloat16, device=dev())
    for kw in (dict(sm_scale=0.0), dict(sm_scale=float("nan")), dict(sm_scale=-1.0), dict(sm_scale=float("inf"))):
        with pytest.raises(spkv.SpkvError):
            c.run(out=out, **kw)
    with pytest.raises(spkv.SpkvError):
        c.run(layer=1, out=out)
    small = Case(spkv, (30, 4), 8, 2, 6, (0.5, 0.2), w=5)
    with pytest.raises(spkv.SpkvError):      # a node may leave another's window: the logits are needed
        small.run(logits=None)
    for name, bad in (("qd", c.qd[:, :, :4]), ("kd", c.kd.float()), ("vd", c.vd.transpose(0, 1)), ("pd", c.pd.long()), ("nd", c.nd[:1]),
                      ("kd", c.kd[..., :64]), ("pd", c.pd.cpu()), ("qd", c.qd.cpu())):
        good = getattr(c, name)
        setattr(c, name, bad)
        with pytest.raises(ValueError):
            c.run(out=out)
        setattr(c, name, good)
    odd = torch.zeros(2 * 6 * 2 * D + 4, dtype=torch.bfloat16, device=dev())[4:].view(2, 6, 2, D)
    with pytest.raises(spkv.SpkvError):      # rows that do not start on 16 bytes
        c.cache.spkv_decode_attention_tree(0, c.ids, c.qd, odd, c.vd, c.pd, out=out)
    with pytest.raises(spkv.SpkvError):
        c.cache.spkv_append_path(0, c.ids, odd, c.vd, c.ld)
    many = torch.zeros((2, 65, 8, D), dtype=torch.bfloat16, device=dev())
    with pytest.raises(spkv.SpkvError):      # more nodes than a tree may have
        c.cache.spkv_decode_attention_tree(0, c.ids, many, many[:, :, :2], many[:, :, :2])
    with pytest.raises(spkv.SpkvError):
        c.cache.spkv_append_path(0, c.ids, many[:, :, :2], many[:, :, :2], torch.zeros((2, 65, 2), device=dev()))
    for layer0, n in ((-1, 1), (1, 1), (0, 2)):
        with pytest.raises(spkv.SpkvError):
            c.cache.spkv_append_path(layer0, c.ids, c.kd[None].expand(n, -1, -1, -1, -1), c.vd[None].expand(n, -1, -1, -1, -1), c.ld[None].repeat(n, 1, 1, 1))
    with pytest.raises(ValueError):
        c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, c.ld[None])
    torch.cuda.synchronize()
    assert (out == 3).all() and c.cache.spkv_status() == 0
    # nothing to do
    c.cache.spkv_append_path(0, c.ids[:0], c.kd[:0], c.vd[:0], c.ld[:0])
    c.cache.spkv_append_path(0, c.ids, c.kd[:, :0], c.vd[:, :0], c.ld[:, :0])
    assert c.cache.spkv_decode_attention_tree(0, c.ids, c.qd[:, :0], c.kd[:, :0], c.vd[:, :0]).shape == (2, 0, 8, D)
    l, cfg = spkv.lib(), c.cache.cfg
    import ctypes as C
    assert l.spkv_decode_tree_workspace_bytes(C.byref(cfg), 2, 65) == 0 and l.spkv_decode_tree_workspace_bytes(None, 2, 6) == 0
    assert 0 < l.spkv_decode_tree_workspace_bytes(C.byref(cfg), 1, 1) <= l.spkv_decode_tree_workspace_bytes(C.byref(cfg), 2, 64)
    row = spkv.Rows(c.qd.data_ptr(), 1024, 128)
    r = C.addressof(row)
    need = l.spkv_decode_tree_workspace_bytes(C.byref(cfg), 2, 6)
    ws = torch.zeros(need + 256, dtype=torch.uint8, device=dev())
    call = lambda w, n: l.spkv_decode_attention_tree(c.cache._h, 0, c.ids.data_ptr(), 2, 6, None, None, r, r, r, None, out.data_ptr(), None, 0.1, w, n, None)
    assert call(None, need) == -7 and call(ws.data_ptr() + 16, need) == -7 and call(ws.data_ptr(), need - 1) == -7


def pool_of(t):
    """The stream whose memory the tensor lies in."""
    at = t.data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"])


def test_results_come_from_the_memory_of_the_calls_stream():
    spkv = load()
    c = Case(spkv, (300, 700), 8, 2, 6, (0.5, 0.2), seed=8)
    tokens = torch.zeros((2, 6), dtype=torch.int32, device=dev())
    x = torch.randn((4, 3000), device=dev())
    keep = [torch.empty_like(t) for t in (c.qd, tokens, x) for _ in range(8)]     # blocks the current stream can give away
    del keep
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    res = [*c.run(stream=s), *spkv.spkv_tree_accept(tokens, tokens, stream=s), *spkv.spkv_token_logprobs(x, tokens[:1, :4].t().contiguous(), top=2, stream=s)]
    s.synchronize()
    assert len(res) == 10 and all(pool_of(t) == s.cuda_stream for t in res)
    for a, b in zip(res, [*c.run(), *spkv.spkv_tree_accept(tokens, tokens), *spkv.spkv_token_logprobs(x, tokens[:1, :4].t().contiguous(), top=2)]):
        assert torch.equal(a, b)
    c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, c.ld, stream=s)
    s.synchronize()
    assert (c.cache.spkv_read_lengths(0)[1] == np.array([[306], [706]])).all()


def test_calls_with_results_given_do_not_reach_the_allocator():
    spkv = load()
    c = Case(spkv, (300, 700), 8, 2, 6, (0.5, 0.2), seed=8)
    out, lse = c.run()
    tokens = torch.zeros((2, 6), dtype=torch.int32, device=dev())
    path, n, nxt = spkv.spkv_tree_accept(tokens, tokens)
    x = torch.randn((4, 3000), device=dev())
    r = spkv.spkv_token_logprobs(x, top=2)
    none = torch.zeros(2, dtype=torch.int32, device=dev())

    def calls():
        c.cache.spkv_decode_attention_tree(0, c.ids, c.qd, c.kd, c.vd, c.pd, c.nd, c.ld, out, lse)
        spkv.spkv_tree_accept(tokens, tokens, None, None, path, n, nxt)
        c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, c.ld, path, none)
        spkv.spkv_token_logprobs(x, top=2, lse=r[0], entropy=r[2], top_ids=r[3], top_logp=r[4])

    calls()
    torch.cuda.synchronize()
    count = lambda: (torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.mem_get_info()[0])
    before = count()
    for _ in range(5):
        calls()
    torch.cuda.synchronize()
    assert count() == before
    c.cache.check()


@pytest.mark.parametrize("w,t", [(3, 0), (3, 7), (64, 200), (65, 64), (65, 131), (128, 127), (300, 299), (300, 1000), (4096, 5000)])
def test_windows_of_any_size(w, t):
    """rings of one to 64 pages, before and after they have gone round"""
    c = Case(load(), (t, max(0, t - 1)), 4, 1, 7, (0.4,), w, seed=w + t, parent="forest")
    out, lse = c.run()
    c.cache.check()
    c.check(out, lse)


@pytest.mark.parametrize("gain", [12.0, 60.0])
def test_large_scores(gain):
    """Scores of hundreds: the weights of a row live on a few keys, its maximum moves from page to page."""
    c = Case(load(), (3000, 500), 8, 2, 20, (0.9, 0.3), seed=4)
    c.q = synth.to_bf16_bits(synth.bf16_bits_to_f32(c.q) * np.float32(gain))
    c.to_device()
    out, lse = c.run()
    c.cache.check()
    c.check(out, lse)


def test_planted_page_indices_under_range_checks():
    """SPKV_FLAG_DEBUG_BOUNDS: an index in a page table that names no pool page is reported, nothing outside the arena is read or written"""
    spkv = load()
    c = Case(spkv, (700,), 4, 1, 6, (1.0,), seed=3, flags=spkv.FLAG_DEBUG_BOUNDS)
    n_ring = 2                                   # ring pages of the only unit: global pages 0 and 1; the pool's follow
    words = c.cache.arena.view(torch.int32)
    ln = int(c.cache.spkv_read_lengths(0)[0][0, 0])
    used = list(range(n_ring, n_ring + (ln + 63) // 64))
    head = words[:1 << 16].cpu().numpy()
    at = next(i for i in range(len(head) - len(used)) if head[i:i + len(used)].tolist() == used)
    words[at + 2] = 1                            # a ring page of the same arena: even an unchecked read would stay inside it
    c.run()
    assert c.cache.spkv_status() == -13
    c.cache.spkv_clear_status()
    words[at + len(used) - 1] = 0
    words[at + 2] = used[2]
    c.cache.spkv_append_path(0, c.ids, c.kd, c.vd, torch.full_like(c.ld, 9.0))
    assert c.cache.spkv_status() == (-13 if ln % 64 else 0)


# ---- trees of different sizes in several row tiles ---------------------------------------------------------
def ragged(B, top, seed):
    return [int(x) for x in np.random.default_rng(seed).integers(0, top, B)]


@pytest.mark.parametrize("lens,Hq,Hkv,T,n", [
    (ragged(13, 4000, 1), 20, 4, 27, [27, 26, 25, 1, 13, 0, 27, 3, 26, 9, 20, 27, 2]),           # a second tile of up to seven rows
    ([3000, 200, 9000, 0, 130, 700], 16, 1, 64, [0, 1, 8, 9, 33, 64]),                            # eight tiles, each shorter than the one before
    ([9000, 0, 65, 300, 2000], 16, 1, 64, [64, 8, 1, 7, 3]),                                      # one long tree: upper tiles of one unit
    ([3000, 200, 64, 0], 32, 2, 64, [8, 8, 3, 1]),                                                # upper tiles without a row
    ([20000, 20, 500], 32, 2, 64, [5, 64, 0]),                                                    # ... and those of a short sequence
    (ragged(60, 700, 2), 24, 3, 33, [int(x) for x in np.random.default_rng(3).integers(0, 34, 60)]),
    ([500, 30], 32, 2, 64, [0, 0]),
])
def test_trees_of_different_sizes_in_several_tiles(lens, Hq, Hkv, T, n):
    """T G > 128, and the tiles' lines of pages differ: blocks go to the tiles by their length.  Rows of absent nodes stay as they are."""
    rates = tuple(0.2 + 0.6 * (i % 2) for i in range(Hkv))
    c = Case(load(), lens, Hq, Hkv, T, rates, seed=len(lens) + T, n=n, parent="forest")
    out, lse = torch.full((c.B, T, Hq, D), 7.0, dtype=torch.bfloat16, device=dev()), torch.full((c.B, T, Hq), 7.0, device=dev())
    for byte in (None, 255):
        for ws in c.cache._tree_ws.values() if byte else ():
            ws.fill_(byte)       # (whatever the workspace holds)
        out.fill_(7), lse.fill_(7)
        c.run(out=out, lse=lse)
        c.cache.check()
        c.check(out, lse)
        for b in range(c.B):
            assert (out[b, n[b]:] == 7).all() and (lse[b, n[b]:] == 7).all(), b


# ---- infinities and NaN where the window's mask falls --------------------------------------------------------
def check_with_nonfinite(c, out, lse):
    """As Case.check, with `reference` infinite or NaN where a node sees such a value.  (|q| |k| scale < 30 for these normal rows.)"""
    G = c.Hq // c.Hkv
    got, l = out.float().cpu().double().numpy(), lse.cpu().double().numpy()
    seen = unseen = 0
    for b in range(c.B):
        for h in range(c.Hkv):
            with np.errstate(invalid="ignore"):
                ref, wv, rl, _, keys = c.reference(b, h)
            mine, ml = got[b, :int(c.n[b]), h * G:(h + 1) * G], l[b, :int(c.n[b]), h * G:(h + 1) * G]
            assert np.array_equal(np.isnan(ref), np.isnan(mine)), (b, h)
            assert np.array_equal(ref == np.inf, mine == np.inf) and np.array_equal(ref == -np.inf, mine == -np.inf), (b, h)
            ok, lok = np.isfinite(ref), np.isfinite(rl)
            tol = 2.0 ** -8 * np.abs(ref[ok]) + (2.0 ** -16 + 2.0 ** -21 + 2 * 2.4e-4 + (keys / 8 + 64) * 2.0 ** -23) * wv[ok] + 1e-30
            assert (np.abs(ref[ok] - mine[ok]) <= tol).all(), (b, h, np.abs(ref[ok] - mine[ok]).max())
            assert np.array_equal(np.isnan(rl), np.isnan(ml))
            assert (np.abs(rl[lok] - ml[lok]) <= 2.4e-4 + (keys / 8 + 64) * 2.0 ** -23 + 2.0 ** -20 * (1 + np.abs(rl[lok]))).all(), (b, h)
            seen, unseen = seen + (~ok).sum(), unseen + ok.sum()
    return seen, unseen


@pytest.mark.parametrize("what", ["v=inf", "v=nan", "k=inf", "k=nan"])
@pytest.mark.parametrize("w,t,clean", [(8, 40, 3), (8, 41, 5), (8, 0, 3), (70, 200, 66), (70, 0, 60), (130, 64, 122), (130, 300, 126)])
def test_pairs_that_leave_the_window_of_deep_nodes(w, t, clean, what):
    """Two pairs with a value or key that is not finite, not to be kept, and then `clean` others in the ring, before and after it has
    gone round: shallow nodes see them, deep ones do not."""
    spkv = load()
    c = Case(spkv, (t, t + 5, max(0, t - 1)), 6, 2, 12, (0.4, 0.4), w=w, parent="chain", seed=w + t + clean, draft_rate=0.3, pool=60)
    rng = np.random.default_rng(clean)
    bad = 0x7f80 if what.endswith("inf") else 0x7fc0
    for x in range(2 + clean):
        k, v = (synth.normal_bf16(rng, (3, 2, D)) for _ in "kv")
        if x < 2:
            (v if what[0] == "v" else k)[:, 0, 7 + x] = bad
        lg = torch.full((3, 2), -9.0 if x < 2 else float(9 * (x % 3 - 1)), device=dev())
        c.cache.spkv_append_evict(0, c.ids, to_dev_bf16(k), to_dev_bf16(v), lg)
    out, lse = c.run()
    c.cache.check()
    seen, unseen = check_with_nonfinite(c, out, lse)
    assert seen and unseen, "both kinds of nodes"
    assert torch.isfinite(out[:, :, 3:].float()).all(), "the other KV head"


@pytest.mark.parametrize("t", [0, 1, 63, 90, 127, 200, 333])
def test_what_an_earlier_sequence_left_behind(t):
    """NaN in ring slots that have not been written since the sequence was reset, and behind the last kept pair of a page"""
    spkv = load()
    c = Case(spkv, (500, 500), 6, 2, 5, (1.0, 1.0), seed=t + 1, parent="forest")
    rng = np.random.default_rng(t)
    nan = torch.full((500, 2, D), math.nan, dtype=torch.bfloat16, device=dev())
    for seq in range(2):
        c.cache.spkv_cache_reset_seq(seq)
        c.cache.spkv_prefill(0, seq, nan, nan, torch.full((500, 2), 9.0, device=dev()))
        c.cache.spkv_cache_reset_seq(seq)
    for seq in range(2):
        for a in range(0, t, 50):
            m = min(50, t - a)
            k, v = (to_dev_bf16(synth.normal_bf16(rng, (m, 2, D))) for _ in "kv")
            c.cache.spkv_prefill(0, seq, k, v, torch.from_numpy(rng.normal(size=(m, 2)).astype(np.float32)).to(dev()))
    out, lse = c.run()
    c.cache.check()
    seen, _ = check_with_nonfinite(c, out, lse)
    assert seen == 0
    c.check(out, lse)


# ---- weights that vanish -------------------------------------------------------------------------------------
def vanishing(spkv, T, low, plant, keys=9000, seed=1):
    """One sequence whose first `low` pairs score hundreds below the others (weights of e^-400 and less).  plant(V of those) -> None"""
    c = Case(spkv, (keys,), 8, 1, T, (1.0,), seed=seed, parent="chain")
    c.cache.spkv_cache_reset_seq(0)
    rng = np.random.default_rng(seed)
    e = np.where(rng.random(D) < 0.5, -1.0, 1.0).astype(np.float32)
    c.q[:] = synth.to_bf16_bits(8 * e)                                        # every query: scores 8 <e, k> / sqrt(128)
    K, V = synth.normal_bf16(rng, (keys, 1, D)), synth.normal_bf16(rng, (keys, 1, D))
    K[:low, 0] = synth.to_bf16_bits(-5 * e)                                   # -452
    plant(V[:low, 0])
    for a in range(0, keys, 3000):
        c.cache.spkv_prefill(0, 0, to_dev_bf16(K[a:a + 3000]), to_dev_bf16(V[a:a + 3000]), torch.full((len(K[a:a + 3000]), 1), 9.0, device=dev()))
    c.to_device()
    return c, e


BIG = int(synth.to_bf16_bits(np.array([3e38], np.float32))[0])


def check_rows(c, out):
    """infinite where the formula is; else within `bounds` (|q| |k| scale <= 8 sqrt(128) 5 sqrt(128) / sqrt(128))"""
    with np.errstate(invalid="ignore", over="ignore"):
        ref, wv, _, _, keys = c.reference(0, 0)
    mine = out[0].float().cpu().double().numpy()
    ok = np.isfinite(ref)
    assert np.array_equal(ref[~ok], mine[~ok])
    es = 130 * 2.0 ** -24 * 40 * math.sqrt(D)
    tol = 2.0 ** -8 * np.abs(ref[ok]) + (2.0 ** -16 + 2.0 ** -21 + 2 * es + (keys / 8 + 64) * 2.0 ** -23) * np.where(np.isfinite(wv[ok]), wv[ok], 0) + 1e-30
    assert (np.abs(mine[ok] - ref[ok]) <= tol).all(), (np.abs(mine[ok] - ref[ok]) - tol).max()
    return ok


@pytest.mark.parametrize("low", [64, 1000, 6000])
def test_finite_values_of_vanishing_weight_add_nothing(low):
    """... however large, in a range of their own or beside others; an infinite one comes through"""
    spkv = load()

    def large(v):
        v[5, 9], v[low // 2, 70] = BIG, BIG

    c, _ = vanishing(spkv, 4, low, large)
    out, lse = c.run()
    c.cache.check()
    assert check_rows(c, out).all()

    def infinite(v):
        large(v)
        v[7, 3], v[low - 1, 4], v[7, 90], v[8, 90] = 0x7f80, 0xff80, 0x7f80, 0x7f80

    c, _ = vanishing(spkv, 4, low, infinite)
    out, lse = c.run()
    c.cache.check()
    ok = check_rows(c, out)
    assert not ok[..., [3, 4, 90]].any() and ok.sum() == ok.size - 3 * ok.shape[0] * ok.shape[1]


@pytest.mark.parametrize("keys", [1, 100, 9000])
def test_finite_values_of_vanishing_weight_beside_an_infinite_one(keys):
    """the same among the drafts, whose page is then gone through key by key"""
    spkv = load()
    c, e = vanishing(spkv, 6, 0, lambda v: None, keys=keys)
    c.k[0, 1, 0] = synth.to_bf16_bits(-5 * e)
    c.v[0, 0, 0, 3], c.v[0, 1, 0, 9], c.v[0, 1, 0, 70], c.v[0, 1, 0, 4] = 0x7f80, BIG, BIG | 0x8000, 0xff80
    c.k[0, 0, 0] = synth.to_bf16_bits(e)                                      # (90: the largest weight of all)
    c.to_device()
    out, lse = c.run()
    c.cache.check()
    ok = check_rows(c, out)
    assert not ok[..., 3].any() and not ok[1:, :, 4].any() and ok[..., [9, 70]].all()


# ---- scores beyond a float32's whole numbers -------------------------------------------------------------------
@pytest.mark.parametrize("scale", [1e5, 3e7, 1e9, 3e10, 1e20, 1e30])
@pytest.mark.parametrize("sign", [1, -1, 0])
def test_scores_of_any_size(scale, sign):
    """Queries and keys of small whole numbers, whose products and sums are exact: a row's weights then are those of the pairs with its
    largest score, and their alike ones, whatever the scale.  sign: of all scores (0: both)"""
    spkv = load()
    rng = np.random.default_rng(int(math.log10(scale)) + sign)
    lens = (9000, 300, 2)
    c = Case(spkv, lens, 8, 2, 9, (1.0, 1.0), seed=3, parent="forest")
    whole = lambda *shape: synth.to_bf16_bits((rng.integers(-2, 3, shape) if sign == 0 else sign * rng.integers(1, 4, shape)).astype(np.float32))
    for b, t in enumerate(lens):
        c.cache.spkv_cache_reset_seq(b)
        for a in range(0, t, 4000):
            m = min(4000, t - a)
            c.cache.spkv_prefill(0, b, to_dev_bf16(whole(m, 2, D)), to_dev_bf16(synth.normal_bf16(rng, (m, 2, D))),
                                 torch.from_numpy(rng.normal(size=(m, 2)).astype(np.float32)).to(dev()))
    c.k = whole(*c.k.shape)
    c.q = synth.to_bf16_bits(rng.integers(1, 3, c.q.shape).astype(np.float32))
    c.to_device()
    scale = float(np.float32(scale))
    out, lse = c.run(sm_scale=scale)
    c.cache.check()
    for b in range(3):
        for h in range(2):
            ref, wv, rl, _, keys = c.reference(b, h, scale=scale)
            err = np.abs(out[b, :, 4 * h:4 * h + 4].float().cpu().double().numpy() - ref)
            assert (err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -16 + 2.0 ** -21 + (keys / 8 + 64) * 2.0 ** -23) * wv).all(), (b, h, err.max())
            assert (np.abs(lse[b, :, 4 * h:4 * h + 4].cpu().double().numpy() - rl) <= (keys / 8 + 64) * 2.0 ** -23 + 2.0 ** -20 * (1 + np.abs(rl))).all()
