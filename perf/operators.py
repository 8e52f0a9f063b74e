"""Operators next to the SP-KV cache, as cases that can be timed and checked one by one.

  norm_rope   what an attention layer does to its projected rows before the cache sees them: RMS
              norm of every query and key head, rotation by one or several position axes (time,
              height, width), values handed on -- out of the fused projection, in one pass
  norm_rope_grad   the backward pass of that: gradients of the rows and of the two norm weights
  shared      decode attention of a batch whose sequences were forked from one prefix: each query
              head attends over the prefix's kept pairs, what its own sequence kept since, and its
              window

`own = False` computes them in elementary torch operations in 32 bits (64 for angles and for long
sums), rounded once; `own = True` makes the calls of paper_2605_14037_b200.spkv.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
WINDOW, TAU, D_CACHE = 128, 0.5, 128
EPS = 1e-6


# ---- cases -------------------------------------------------------------------------------------
def _rows(op, name, n, hq, hkv, dtype="bf16", d=128, rot=128, axes=1, norm=True, interleaved=False, layout="fused",
          theta=500000.0, far=0):
    """One pass over the rows of n tokens.  layout: "fused" = views of one [n, (hq + 2 hkv) d]
    projection, "heads" = tensors of their own laid out [heads, n, d].  far: position of the first
    token (a decode step deep in a long context, a chunk of a long prompt)."""
    return {"name": name, "op": op, "n": n, "hq": hq, "hkv": hkv, "dtype": dtype, "d": d, "rot": rot, "axes": axes,
            "norm": norm, "interleaved": interleaved, "layout": layout, "theta": theta, "far": far}


def _shared(name, b, prefix, suffix, hq, hkv, mean):
    """b sequences forked from a prefix of `prefix` tokens, `suffix` tokens further on; KV head h of
    hkv keeps 2 mean (h + 0.5) / hkv of its pairs (at most all)."""
    return {"name": name, "op": "shared", "b": b, "prefix": prefix, "suffix": suffix, "hq": hq, "hkv": hkv, "mean": mean}


def listed():
    return [
        # one token of one small layer: the latency of a single-sequence decode step
        _rows("norm_rope", "rows decode 1", 1, 8, 2, far=4096),
        # a decode batch of 64 sequences, each deep in its own context
        _rows("norm_rope", "rows decode 64", 64, 32, 8, far=65536),
        # a prefill chunk
        _rows("norm_rope", "rows chunk 8192", 8192, 32, 8, far=24576),
        # patches of a short video: three axes, rotation only, adjacent pairs, small heads
        _rows("norm_rope", "rows video 4095", 4095, 16, 16, dtype="f16", d=64, rot=64, axes=3, norm=False,
              interleaved=True, theta=10000.0),
        # 32-bit rows in head-major order, half of each head rotated
        _rows("norm_rope", "rows f32 1001", 1001, 32, 8, dtype="f32", rot=64, layout="heads", far=100000),
        # training: one short odd sequence in 32 bits; image and text tokens; one long sequence
        _rows("norm_rope_grad", "grad f32 513", 513, 8, 2, dtype="f32", theta=10000.0),
        _rows("norm_rope_grad", "grad axes 4097", 4097, 32, 8, dtype="f16", axes=3),
        _rows("norm_rope_grad", "grad 32768", 32768, 32, 8),
        # two continuations of one short prompt
        _shared("shared 2 x 4096", 2, 4096, 1, 8, 2, 0.2),
        # parallel samples of a long prompt
        _shared("shared 16 x 32768", 16, 32768, 200, 32, 8, 0.15),
        # a wide model whose requests share a long document
        _shared("shared 8 x 65536", 8, 65536, 77, 64, 8, 0.2),
        # a full batch on a very long common context
        _shared("shared 64 x 131072", 64, 131072, 333, 32, 8, 0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rope", "norm_rope", "norm_rope_grad", "shared", "shared"])
    if op == "shared":
        hkv = rng.choice([2, 4, 8])
        c = _shared("", _log(rng, 2, 64), _log(rng, 300, 131072), _log(rng, 1, 400), hkv * rng.choice([1, 3, 4, 5, 8]),
                    hkv, round(rng.uniform(0.05, 0.3), 3))
        while c["b"] * c["hq"] * c["prefix"] * c["mean"] > 64 * 32 * 131072 * 0.1:   # no dearer than the largest listed
            c["prefix"] = c["prefix"] * 2 // 3
    else:
        hkv = rng.choice([1, 2, 4, 8])
        d = rng.choice([64, 80, 128, 128, 256])
        c = _rows(op, "", _log(rng, 1, 20000), hkv * rng.choice([1, 2, 4, 7]), hkv, rng.choice(["bf16", "bf16", "f16", "f32"]),
                  d, rng.choice([d, d, d // 32 * 16]), rng.choice([1, 1, 2, 3]), rng.random() < 0.75, rng.random() < 0.3,
                  rng.choice(["fused", "heads"]), rng.choice([10000.0, 500000.0]), rng.choice([0, _log(rng, 1, 1000000)]))
        while c["n"] * (c["hq"] + 2 * c["hkv"]) * c["d"] * BYTES[c["dtype"]] > 8192 * 48 * 128 * 2 * 3:
            c["n"] = c["n"] * 2 // 3
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _positions(c):
    """[axes, n] int32.  One axis: consecutive, or spread over the contexts of a decode batch.
    Several: frames of a 16-wide grid of patches (time, height, width)."""
    i = np.arange(c["n"], dtype=np.int64)
    if c["axes"] > 1:
        p = np.stack([i // 256, (i // 16) % 16, i % 16])[: c["axes"]]
    else:
        p = (i if c["n"] > 64 else i * 977 % 4096)[None]
    return torch.from_numpy((p + c["far"]).astype(np.int32)).to(DEV)


def _inv_freq(c):
    return c["theta"] ** (-np.arange(c["rot"] // 2, dtype=np.float64) * 2 / c["rot"])


def _axis(c):
    """Axis of each rotated pair: the axes take turns."""
    return (np.arange(c["rot"] // 2) % c["axes"]).astype(np.uint8)


def _row_inputs(c, seed):
    """Rows with the spread of a projection's output (a few heads much larger than others)."""
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    n, hq, hkv, d = c["n"], c["hq"], c["hkv"], c["d"]

    def rows(gain):
        if c["layout"] == "fused":
            x = torch.randn((n, hq + 2 * hkv, d), generator=g, device=DEV, dtype=torch.float32)
        else:
            x = torch.randn((hq + 2 * hkv, n, d), generator=g, device=DEV, dtype=torch.float32).transpose(0, 1)
        if gain:
            x *= torch.exp2(torch.randint(-1, 3, (1, hq + 2 * hkv, 1), generator=g, device=DEV).float())
        x = x.to(dt)
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]

    s = {"c": c, "pos": _positions(c)}
    s["q"], s["k"], s["v"] = rows(True)
    if c["op"] == "norm_rope_grad":
        s["gq"], s["gk"], s["gv"] = (t.contiguous() for t in rows(False))
    s["wq"], s["wk"] = ((1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(dt) if c["norm"] else None for _ in "qk")
    s["inv"] = torch.from_numpy(_inv_freq(c)).to(DEV)
    s["axis"] = torch.from_numpy(_axis(c).astype(np.int64)).to(DEV)
    return s


def _rates(c):
    return np.minimum(1.0, 2 * c["mean"] * (np.arange(c["hkv"]) + 0.5) / c["hkv"])


def _shared_inputs(c, seed):
    """Raw tokens: the prefix's K, V, logits [prefix, hkv, ...], each sequence's own [b, suffix, hkv, ...],
    and the queries of the newest token.  A logit >= 0 means utility >= 0.5, the threshold."""
    g = _gen(seed)
    b, n, m, hq, hkv = c["b"], c["prefix"], c["suffix"], c["hq"], c["hkv"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)

    rates = torch.from_numpy(_rates(c)).float().to(DEV)

    def logits(*shape):
        x = torch.rand(shape + (hkv,), generator=g, device=DEV)
        return torch.where(x < rates, 0.25 + x, -0.25 - x)

    s = {"c": c, "K": normal(n, hkv, D_CACHE), "V": normal(n, hkv, D_CACHE), "L": logits(n),
         "k": normal(b, m, hkv, D_CACHE), "v": normal(b, m, hkv, D_CACHE), "l": logits(b, m)}
    s["q"] = (1.5 * torch.randn((b, hq, D_CACHE), generator=g, device=DEV)).to(torch.bfloat16)
    return s


# ---- state -------------------------------------------------------------------------------------
def prepare(case, seed):
    if case["op"] != "shared":
        s = _row_inputs(case, seed)
        if own:
            from paper_2605_14037_b200 import spkv
            s["spkv"] = spkv
            s["plan"] = spkv.make_norm_rope(case["hq"], case["hkv"], head_dim=case["d"], dtype=DTYPES[case["dtype"]],
                                            wq=s["wq"], wk=s["wk"], norm=case["norm"], eps=EPS, rot_dim=case["rot"],
                                            inv_freq=_inv_freq(case), axis=_axis(case), n_axes=case["axes"],
                                            interleaved=case["interleaved"])
        return s
    s = _shared_inputs(case, seed)
    if own:
        s["cache"], s["ids"], s["plan"] = _cache(case, s)
        return {k: s[k] for k in ("c", "q", "cache", "ids", "plan")}
    return _compact(case, s)


def _compact(c, s):
    """The cache in plain tensors, as the plain form reads it: the pairs the prefix kept before the
    fork [hkv, N, 128] and, per sequence, those it can see since [b, hkv, M, 128], with their counts."""
    n, m = c["prefix"], c["suffix"]
    first = max(0, n - WINDOW)                       # positions from here on left (or sit in) a sequence's own window
    keep = s["L"][:first] >= 0                       # [first, hkv]
    tail_l = torch.cat([s["L"][None, first:].expand(c["b"], -1, -1), s["l"]], 1)
    see = tail_l >= 0                                # [b, n - first + m, hkv]
    see[:, max(0, see.shape[1] - WINDOW):] = True
    tk, tv = (torch.cat([x[None, first:].expand(c["b"], -1, -1, -1), y], 1) for x, y in ((s["K"], s["k"]), (s["V"], s["v"])))

    def pack(mask, *rows):
        """Rows where the mask holds, in order, padded with zeros: mask [..., t], rows [..., t, 128]."""
        count = mask.sum(-1)
        top = max(1, int(count.max()))
        order = torch.sort((~mask).to(torch.uint8), dim=-1, stable=True).indices[..., :top]
        live = torch.arange(top, device=DEV) < count[..., None]
        return [torch.gather(r, -2, order[..., None].expand(*order.shape, D_CACHE)) * live[..., None] for r in rows] + [live]

    out = {"c": c, "q": s["q"]}
    if first:
        out["K"], out["V"], out["live"] = pack(keep.t(), s["K"][:first].transpose(0, 1), s["V"][:first].transpose(0, 1))
    else:
        out["K"] = out["V"] = torch.zeros((c["hkv"], 1, D_CACHE), dtype=torch.bfloat16, device=DEV)
        out["live"] = torch.zeros((c["hkv"], 1), dtype=torch.bool, device=DEV)
    out["k"], out["v"], out["own_live"] = pack(see.transpose(1, 2), tk.transpose(1, 2), tv.transpose(1, 2))
    return out


def _cache(c, s):
    """The same pairs in the framework's cache: the prefix prefilled once into slot 0 in chunks, every
    sequence forked from it and continued by its own tokens."""
    from paper_2605_14037_b200 import spkv
    n, m, b, hkv = c["prefix"], c["suffix"], c["b"], c["hkv"]
    kept = int((s["L"] >= 0).sum()) // 64 + hkv
    cache = spkv.Cache(1, b + 1, c["hq"], hkv, n + m, kept + b * hkv * ((m + WINDOW) // 64 + 3), window=WINDOW, tau=TAU,
                       device=DEV, flags=spkv.FLAG_FORK)
    for i in range(0, n, 8192):
        cache.spkv_prefill(0, 0, *(x[i:i + 8192].contiguous() for x in (s["K"], s["V"], s["L"])))
    cache.spkv_seq_fork(0, range(1, b + 1))
    for j in range(b):
        cache.spkv_prefill(0, j + 1, *(x[j].contiguous() for x in (s["k"], s["v"], s["l"])))
    ids = torch.arange(1, b + 1, dtype=torch.int32, device=DEV)
    plan = cache.spkv_share_plan(ids)
    cache.check()
    return cache, ids, plan


# ---- one pass ----------------------------------------------------------------------------------
def run(s):
    op = s["c"]["op"]
    if own:
        if op == "norm_rope":
            return s["spkv"].spkv_norm_rope(s["plan"], s["pos"], s["q"], s["k"], s["v"])
        if op == "norm_rope_grad":
            return s["spkv"].spkv_norm_rope_backward(s["plan"], s["pos"], s["q"], s["k"], s["gq"], s["gk"], s["gv"])
        return s["cache"].spkv_decode_attention_shared(0, s["ids"], s["q"], s["plan"], want_lse=True)
    return {"norm_rope": _plain_rows, "norm_rope_grad": _plain_grad, "shared": _plain_shared}[op](s)


def _cos_sin(s):
    """[n, 1, rot / 2] each; the angle in 64 bits, as a far position times a frequency needs."""
    angle = s["pos"][s["axis"]].double() * s["inv"][:, None]
    return torch.cos(angle).t().float()[:, None], torch.sin(angle).t().float()[:, None]


def _turn(c, x, cos, sin):
    """Rotates the first rot dims of x [n, heads, d]."""
    r, h = c["rot"], c["rot"] // 2
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :h], x[..., h:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _unit(x):
    """(x / rms(x), 1 / rms(x)) of every row"""
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _plain_rows(s):
    c, dt = s["c"], s["q"].dtype
    cos, sin = _cos_sin(s)

    def head(x, w):
        x = x.float()
        if c["norm"]:
            x = _unit(x)[0] * w.float()
        return _turn(c, x, cos, sin).to(dt)

    return head(s["q"], s["wq"]), head(s["k"], s["wk"]), s["v"].clone(memory_format=torch.contiguous_format)


def _plain_grad(s):
    c, dt = s["c"], s["q"].dtype
    cos, sin = _cos_sin(s)

    def head(x, g, w):
        g = _turn(c, g.float(), cos, -sin)                       # the rotation's transpose
        if not c["norm"]:
            return g.to(dt), None
        u, r = _unit(x.float())
        dw = (g * u).sum((0, 1), dtype=torch.float64).float()
        g = g * w.float()
        return (r * (g - u * (g * u).mean(-1, keepdim=True))).to(dt), dw

    dq, dwq = head(s["q"], s["gq"], s["wq"])
    dk, dwk = head(s["k"], s["gk"], s["wk"])
    return dq, dk, s["gv"].clone(), dwq, dwk


def _plain_shared(s):
    c = s["c"]
    b, hq, hkv = c["b"], c["hq"], c["hkv"]
    q = s["q"].float().view(b, hkv, hq // hkv, D_CACHE) / math.sqrt(D_CACHE)
    kp, vp, kt, vt = (s[x].float() for x in ("K", "V", "k", "v"))
    sp = torch.einsum("bhgd,hnd->bhgn", q, kp).masked_fill_(~s["live"][None, :, None], -math.inf)
    st = torch.einsum("bhgd,bhmd->bhgm", q, kt).masked_fill_(~s["own_live"][:, :, None], -math.inf)
    top = torch.maximum(sp.amax(-1, keepdim=True), st.amax(-1, keepdim=True))
    sp, st = sp.sub_(top).exp_(), st.sub_(top).exp_()
    total = sp.sum(-1, keepdim=True) + st.sum(-1, keepdim=True)
    out = (torch.einsum("bhgn,hnd->bhgd", sp, vp) + torch.einsum("bhgm,bhmd->bhgd", st, vt)) / total
    return out.reshape(b, hq, D_CACHE).to(torch.bfloat16), (top + total.log()).reshape(b, hq)


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(c):
    if c["op"] == "shared":
        pre = float(np.sum(_rates(c))) * max(0, c["prefix"] - WINDOW)       # kept pairs of the prefix, all KV heads
        seen = min(WINDOW, c["prefix"] + c["suffix"])
        left = max(0, min(WINDOW, c["prefix"]) + c["suffix"] - WINDOW)
        tail = c["b"] * (float(np.sum(_rates(c))) * left + c["hkv"] * seen)
        rows = c["b"] * c["hq"]
        flops = 4 * D_CACHE * (c["b"] * pre + tail) * (c["hq"] // c["hkv"])
        return {"bytes": (pre + tail) * 4 * D_CACHE + rows * (4 * D_CACHE + 4), "flops": flops}
    e, d, n, qk, all_ = BYTES[c["dtype"]], c["d"], c["n"], c["hq"] + c["hkv"], c["hq"] + 2 * c["hkv"]
    rows = 2 * all_ if c["op"] == "norm_rope" else 2 * all_ + (qk if c["norm"] else 0)
    return {"bytes": n * d * e * rows + 4 * n * c["axes"], "flops": n * d * qk * (8 if c["op"] == "norm_rope" else 16)}


# ---- the same from the definitions in 64 bits ------------------------------------------------------
def exact(case, seed):
    if case["op"] == "shared":
        return _exact_shared(case, _shared_inputs(case, seed))
    s = _row_inputs(case, seed)
    with torch.enable_grad():
        x = [s[k].double().requires_grad_(case["op"] == "norm_rope_grad") for k in ("q", "k")]
        w = [s[k].double().requires_grad_(case["op"] == "norm_rope_grad") if case["norm"] else None for k in ("wq", "wk")]
        y = [_exact_head(case, s, a, b) for a, b in zip(x, w)]
        if case["op"] == "norm_rope":
            return y[0], y[1], s["v"].double()
        sum((a * s[g].double()).sum() for a, g in zip(y, ("gq", "gk"))).backward()
        return (x[0].grad, x[1].grad, s["gv"].double(), *(None if a is None else a.grad for a in w))


def _exact_head(case, s, x, w):
    """A pair of dims is a complex number; turning it by an angle is a product with exp(i angle)."""
    if case["norm"]:
        x = w * x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + EPS)
    r = case["rot"]
    lo, hi = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    phase = torch.stack([s["pos"][a].double() for a in _axis(case).tolist()], -1) * torch.from_numpy(_inv_freq(case)).to(DEV)
    z = torch.complex(lo, hi) * torch.polar(torch.ones_like(phase), phase)[:, None]
    lo, hi = z.real, z.imag
    y = torch.stack([lo, hi], -1).flatten(-2) if case["interleaved"] else torch.cat([lo, hi], -1)
    return torch.cat([y, x[..., r:]], -1)


def _exact_shared(c, s):
    """Query by query over the tokens themselves: a token is visible if its utility reaches the
    threshold or it is one of the last WINDOW of its sequence."""
    b, n, m, g = c["b"], c["prefix"], c["suffix"], c["hq"] // c["hkv"]
    out = torch.empty((b, c["hq"], D_CACHE), dtype=torch.float64, device=DEV)
    lse = torch.empty((b, c["hq"]), dtype=torch.float64, device=DEV)
    age = torch.arange(n + m - 1, -1, -1, device=DEV)
    for h in range(c["hkv"]):
        hs = slice(h * g, (h + 1) * g)
        for j in range(b):
            seen = torch.cat([s["L"][:, h], s["l"][j, :, h]]) >= 0
            at = torch.nonzero(seen | (age < WINDOW))[:, 0]
            k, v = (torch.cat([s[x][:, h], s[y][j, :, h]])[at].double() for x, y in (("K", "k"), ("V", "v")))
            z = s["q"][j, hs].double() @ k.t() * D_CACHE ** -0.5
            lse[j, hs] = torch.logsumexp(z, -1)
            out[j, hs] = torch.softmax(z, -1) @ v
    return out, lse
