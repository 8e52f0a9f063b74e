"""Operators of speculative decoding on the SP-KV cache, as cases that can be timed and checked one by one.

  tree    attention of a tree of drafted tokens over the cache: every node sees what its path from the root would
          have left it -- the pairs kept before, those of the window that are still in its own window or
          pass the threshold, and its ancestors
  logprobs  what a model's logits say of given tokens: their log probabilities, the rows' entropies and the likeliest
          alternatives
  accept  the path of a tree that the target's tokens confirm, and the token behind it
  step    a step as it is used: the drafts of the last tree that were accepted join the cache in every layer,
          then the new tree attends, layer by layer

`own = False` computes them in elementary torch operations in 32 bits, rounded once; `own = True` makes the calls of
paper_2605_14037_b200.spkv.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
D, TAU = 128, 0.5
VOCAB = 32000
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}


# ---- cases -------------------------------------------------------------------------------------
def _tree(name, b, ctx, nodes, hq, hkv, mean, shape="tree", ragged=False, window=128, op="tree", layers=1):
    """b sequences of ctx tokens (ragged: sequence j has ctx (j + 1) / b of them and fewer drafted nodes than the others),
    `nodes` drafted tokens each; KV head h of hkv keeps 2 mean (h + 0.5) / hkv of its pairs (at most all)."""
    return {"name": name, "op": op, "b": b, "ctx": ctx, "nodes": nodes, "hq": hq, "hkv": hkv, "mean": mean, "shape": shape,
            "ragged": ragged, "window": window, "layers": layers}


def _accept(name, b, nodes, shape="tree", ragged=False):
    return {"name": name, "op": "accept", "b": b, "nodes": nodes, "shape": shape, "ragged": ragged}


def _logprobs(name, rows, vocab, top, given=1, dtype="bf16", pad=0, scale=1.0):
    """rows of `vocab` logits (pad: behind each row, as a padded projection leaves them), `given` tokens of each looked up."""
    return {"name": name, "op": "logprobs", "rows": rows, "vocab": vocab, "top": top, "given": given, "dtype": dtype, "pad": pad,
            "scale": scale}


def listed():
    return [
        # four tokens guessed ahead in one short conversation of a small model
        _tree("tree 1 x 300, chain of 4", 1, 300, 4, 8, 2, 0.3, shape="chain"),
        # one user's very long document
        _tree("tree 1 x 131072, 16 nodes", 1, 131072, 16, 32, 8, 0.1),
        # a batch of long contexts, the tree as large as one tile of query rows
        _tree("tree 16 x 32768, 32 nodes", 16, 32768, 32, 32, 8, 0.15),
        # a full batch of chats
        _tree("tree 64 x 4096, 8 nodes", 64, 4096, 8, 32, 8, 0.2),
        # sequences and trees of all sizes, an odd group of query heads
        _tree("tree 13 x ragged 20000, 27 nodes", 13, 20000, 27, 20, 4, 0.25, ragged=True),
        # a wide model with the largest trees: many query rows a key
        _tree("tree 8 x 65536, 64 nodes", 8, 65536, 64, 64, 8, 0.15),
        # the rows of one small tree at an odd vocabulary, with alternatives; those of a large batch of trees
        _logprobs("logprobs 5 x 50257 f32, top 5", 5, 50257, 5, given=3, dtype="f32", scale=1.25),
        _logprobs("logprobs 768 x 128256, top 1", 768, 128256, 1),
        # one tree, and a large batch of the largest
        _accept("accept 1 x 8", 1, 8),
        _accept("accept 500 x 64, ragged", 500, 64, ragged=True),
        # a step of one sequence, and of a batch, over a few layers
        _tree("step 1 x 2000, 6 nodes", 1, 2000, 6, 8, 2, 0.3, op="step", layers=2),
        _tree("step 24 x 16384, 24 nodes", 24, 16384, 24, 32, 8, 0.15, op="step", layers=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    rows = c["b"] * c["hq"] * c["nodes"] * c["layers"]
    return rows * (c["ctx"] * c["mean"] + c["window"]), c["layers"] * c["b"] * c["hkv"] * c["ctx"]


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "logprobs", "logprobs", "accept", "step", "step"])
    shape, ragged = rng.choice(["tree", "tree", "chain"]), rng.random() < 0.4
    if op == "accept":
        c = _accept("", _log(rng, 1, 500), _log(rng, 2, 64), shape, ragged)
    elif op == "logprobs":
        c = _logprobs("", _log(rng, 1, 1000), _log(rng, 500, 200000), rng.choice([0, 1, 1, 5, 20]), rng.choice([1, 1, 4, 33]),
                      rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, 0, 7, 64]), rng.choice([1.0, 0.7]))
        while c["rows"] * c["vocab"] * BYTES[c["dtype"]] > 768 * 128256 * 2:
            c["rows"] = c["rows"] * 2 // 3
    else:
        hkv = rng.choice([1, 2, 4, 8])
        c = _tree("", _log(rng, 1, 64), _log(rng, 20, 131072), _log(rng, 1, 64), hkv * rng.choice([1, 3, 4, 5, 8, 16]), hkv,
                  round(rng.uniform(0.05, 0.4), 3), shape, ragged, rng.choice([32, 128, 128, 200]), op,
                  1 if op == "tree" else rng.choice([1, 2, 4]))
        top = [_cost(x) for x in listed() if x["op"] in ("tree", "step")]
        while any(v > max(t[i] for t in top) for i, v in enumerate(_cost(c))):   # no dearer than the largest listed
            c["ctx"] = c["ctx"] * 2 // 3
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------------------------
def _gen(seed, device=DEV):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed))
    return g


def _rates(c):
    return np.minimum(1.0, 2 * c["mean"] * (np.arange(c["hkv"]) + 0.5) / c["hkv"])


def _lengths(c):
    return [max(1, c["ctx"] * (j + 1) // c["b"]) if c["ragged"] else c["ctx"] for j in range(c["b"])]


def _nodes(c):
    n = [1 + (j * 7 + 3) % c["nodes"] if c["ragged"] else c["nodes"] for j in range(c["b"])]
    n[c["b"] // 2] = c["nodes"]
    return n


def _parents(c, g):
    """[b, nodes] on the host: node 0 is the newest token, every other node hangs on one of the few before it"""
    b, n = c["b"], c["nodes"]
    i = torch.arange(n)
    if c["shape"] == "chain":
        p = (i - 1).expand(b, n).clone()
    else:
        p = (i - 1 - (torch.rand((b, n), generator=g) * i.clamp(max=5)).long()).clamp(min=0)
        p[:, 0] = -1
    return p.to(torch.int32)


def _draft(c, seed):
    """Parents, node counts, drafted tokens and the target's token behind each node (three times in four that of
    one of the node's children)."""
    h = _gen(seed + 77, "cpu")
    b, n = c["b"], c["nodes"]
    parent = _parents(c, h)
    tokens = torch.randint(0, VOCAB, (b, n), generator=h, dtype=torch.int32)
    target = torch.randint(0, VOCAB, (b, n), generator=h, dtype=torch.int32)
    hit = torch.rand((b, n), generator=h) < 0.75
    for i in range(1, n):
        at = parent[:, i].long()[:, None]
        old = target.gather(1, at)
        target.scatter_(1, at, torch.where(hit.gather(1, at), tokens[:, i:i + 1], old))
    s = {"parent": parent, "tokens": tokens, "target": target, "n": torch.tensor(_nodes(c), dtype=torch.int32)}
    return {k: v.to(DEV) for k, v in s.items()}


def _scores(c, seed):
    """Logits as a model gives them: a few tokens far above the rest; one in sixteen of the vocabulary ruled out."""
    g = _gen(seed)
    n, v = c["rows"], c["vocab"]
    x = 2.5 * torch.randn((n, v + c["pad"]), generator=g, device=DEV)
    x[:, :v // 50] += 4.0
    x = torch.where(torch.rand((1, v + c["pad"]), generator=g, device=DEV) < 1 / 16, -math.inf, x).to(DTYPES[c["dtype"]])
    given = torch.randint(0, v, (n, c["given"]), generator=g, device=DEV, dtype=torch.int32)
    return {"c": c, "x": x[:, :v], "given": given}


def _raw(c, seed):
    """Raw tokens of the contexts (per layer, per sequence [t, hkv, 128]) and the drafts' rows.  A logit >= 0 means
    utility >= 0.5, the threshold."""
    g = _gen(seed)
    b, n, hq, hkv = c["b"], c["nodes"], c["hq"], c["hkv"]
    rates = torch.from_numpy(_rates(c)).float().to(DEV)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)

    def logits(*shape):
        x = torch.rand(shape + (hkv,), generator=g, device=DEV)
        return torch.where(x < rates, 0.25 + x, -0.25 - x)

    layers = []
    for _ in range(c["layers"]):
        one = {"K": [], "V": [], "L": []}
        for t in _lengths(c):
            one["K"].append(normal(t, hkv, D))
            one["V"].append(normal(t, hkv, D))
            one["L"].append(logits(t))
        # the drafts as an engine has them: views of one fused projection
        fused = normal(b, n, hq + 2 * hkv, D)
        fused[:, :, :hq] *= 1.5
        one.update(q=fused[:, :, :hq], k=fused[:, :, hq:hq + hkv], v=fused[:, :, hq + hkv:], l=logits(b, n))
        layers.append(one)
    s = {"c": c, "layers": layers, "new": _draft(c, seed)}
    if c["op"] == "step":
        s["old"] = _draft(c, seed + 1)
        s["old"].update(k=normal(c["layers"], b, n, hkv, D), v=normal(c["layers"], b, n, hkv, D), l=logits(c["layers"], b, n))
    return s


# ---- state -------------------------------------------------------------------------------------
def prepare(case, seed):
    if case["op"] in ("accept", "logprobs"):
        s = {"c": case, "new": _draft(case, seed)} if case["op"] == "accept" else _scores(case, seed)
        if own:
            from paper_2605_14037_b200 import spkv
            s["spkv"] = spkv
        return s
    s = _raw(case, seed)
    drafts = [{k: x[k] for k in ("q", "k", "v", "l")} for x in s["layers"]]
    out = {"c": case, "new": s["new"], "old": s.get("old"), "drafts": drafts}
    if own:
        out.update(_cache(case, s))
    else:
        out["cache"] = [_compact(case, x) for x in s["layers"]]
    return out


def _compact(c, x):
    """A layer's cache in plain tensors: the pairs kept [b, hkv, N, 128] with a mask of the live ones, and the last
    `window` pairs [b, hkv, window, 128] with logits and positions (before the start: not live)."""
    w, b, hkv, lens = c["window"], c["b"], c["hkv"], _lengths(c)
    kept = []
    for j, t in enumerate(lens):
        m = x["L"][j][:max(0, t - w)] >= 0
        kept.append(([x["K"][j][:len(m)][m[:, h], h] for h in range(hkv)], [x["V"][j][:len(m)][m[:, h], h] for h in range(hkv)]))
    top = max(1, max(len(k) for ks, _ in kept for k in ks))

    def zeros(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device=DEV)

    s = {"K": zeros(b, hkv, top, D), "V": zeros(b, hkv, top, D), "live": zeros(b, hkv, top, dtype=torch.bool),
         "rk": zeros(b, hkv, w, D), "rv": zeros(b, hkv, w, D), "rl": zeros(b, hkv, w, dtype=torch.float32)}
    for j, t in enumerate(lens):
        for h in range(hkv):
            k, v = kept[j][0][h], kept[j][1][h]
            s["K"][j, h, :len(k)], s["V"][j, h, :len(k)], s["live"][j, h, :len(k)] = k, v, True
        r = min(t, w)
        s["rk"][j, :, w - r:] = x["K"][j][t - r:].transpose(0, 1)
        s["rv"][j, :, w - r:] = x["V"][j][t - r:].transpose(0, 1)
        s["rl"][j, :, w - r:] = x["L"][j][t - r:].t()
    s["t"] = torch.tensor(lens, device=DEV)
    return s


def _cache(c, s):
    """The same pairs in the framework's cache, prefilled in chunks, and where the results go (rows of nodes that a
    ragged tree lacks are left as they are: zeros)."""
    from paper_2605_14037_b200 import spkv
    b, n, hq, hkv, w, lens = c["b"], c["nodes"], c["hq"], c["hkv"], c["window"], _lengths(c)
    pages = sum(int((x["L"][j] >= 0).sum()) for x in s["layers"] for j in range(b)) // 64 + c["layers"] * b * hkv * 3
    cache = spkv.Cache(c["layers"], b, hq, hkv, c["ctx"] + 2 * n + 64, pages, window=w, tau=TAU, device=DEV)
    for l, x in enumerate(s["layers"]):
        for j, t in enumerate(lens):
            for i in range(0, t, 8192):
                cache.spkv_prefill(l, j, *(x[a][j][i:i + 8192] for a in ("K", "V", "L")))
    cache.check()
    out = torch.zeros((c["layers"], b, n, hq, D), dtype=torch.bfloat16, device=DEV)
    return {"spkv": spkv, "cache": cache, "ids": torch.arange(b, dtype=torch.int32, device=DEV), "out": out,
            "lse": torch.zeros((c["layers"], b, n, hq), device=DEV),
            "before": cache.spkv_cache_checkpoint() if c["op"] == "step" else None}


# ---- one pass ----------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    c, new, old = s["c"], s.get("new"), s.get("old")
    if c["op"] == "accept":
        return s["spkv"].spkv_tree_accept(new["tokens"], new["target"], new["parent"], new["n"])
    if c["op"] == "logprobs":
        return s["spkv"].spkv_token_logprobs(s["x"], s["given"], top=c["top"], scale=c["scale"])
    cache, got = s["cache"], ()
    if c["op"] == "step":
        cache.spkv_cache_rollback(s["before"])           # (so that the step can be made again)
        path, n_path, nxt = s["spkv"].spkv_tree_accept(old["tokens"], old["target"], old["parent"], old["n"])
        cache.spkv_append_path(0, s["ids"], old["k"], old["v"], old["l"], path, n_path)
        got = (path, n_path, nxt)
    for l, x in enumerate(s["drafts"]):
        cache.spkv_decode_attention_tree(l, s["ids"], x["q"], x["k"], x["v"], new["parent"], new["n"], logits=x["l"],
                                         out=s["out"][l], lse=s["lse"][l])
    return (s["out"], s["lse"]) + got


def _run_plain(s):
    c, new, old = s["c"], s.get("new"), s.get("old")
    if c["op"] == "accept":
        return _plain_accept(c, new)
    if c["op"] == "logprobs":
        return _plain_logprobs(c, s["x"], s["given"])
    got = _plain_accept(c, old) if c["op"] == "step" else ()
    outs = [_plain_tree(c, s["cache"][l], x, new, None if old is None else (old, l) + got) for l, x in enumerate(s["drafts"])]
    return (torch.stack([o for o, _ in outs]), torch.stack([l for _, l in outs])) + got


def _plain_logprobs(c, x, given):
    """(log sum of exponentials, log probabilities of the given tokens, entropy, likeliest tokens, their log probabilities)"""
    z = x.float() * c["scale"]
    m = z.amax(1, keepdim=True)
    t = z - m
    e = t.exp()
    total = e.sum(1, dtype=torch.float64)
    weighed = (e * t.clamp(min=-1e4)).sum(1, dtype=torch.float64)
    lse = m[:, 0].double() + total.log()
    logp = z.gather(1, given.long()) - lse[:, None]
    at = torch.arange(z.shape[1], device=DEV)
    ids, tops = [], []
    for _ in range(c["top"]):
        best = z.amax(1, keepdim=True)
        i = torch.where(z == best, at, z.shape[1]).amin(1, keepdim=True)      # ties: the lowest
        ids.append(i)
        tops.append(best - lse[:, None])
        z = z.scatter(1, i, -math.inf)
    return (lse.float(), logp.float(), (total.log() - weighed / total).float(),
            torch.cat(ids, 1).int() if ids else None, torch.cat(tops, 1).float() if ids else None)


def _plain_accept(c, d):
    """(path [b, nodes], its length [b], the token behind it [b]); entries behind the path are -1"""
    b, n = d["tokens"].shape
    node = torch.arange(n, device=DEV)
    cur = torch.zeros((b, 1), dtype=torch.int64, device=DEV)
    alive = torch.ones((b, 1), dtype=torch.bool, device=DEV)
    path = torch.full((b, n), -1, dtype=torch.int32, device=DEV)
    for i in range(n):
        path[:, i:i + 1] = torch.where(alive, cur.int(), -1)
        fits = (d["parent"] == cur) & (d["tokens"] == d["target"].gather(1, cur)) & (node > cur) & (node < d["n"][:, None]) & alive
        first = torch.where(fits, node, n).amin(1, keepdim=True)
        alive = first < n
        cur = torch.where(alive, first, cur)
    length = (path >= 0).sum(1)
    return path, length.int(), d["target"].gather(1, cur)[:, 0]


def _plain_tree(c, z, x, new, commit):
    """One layer's attention.  Behind the kept pairs stand the window, the pairs committed just now (step) and the
    drafts; of those, a node at position p sees the ones of its path at positions > p - window or with a logit >= 0."""
    b, n, hq, hkv, w = c["b"], c["nodes"], c["hq"], c["hkv"], c["window"]
    t = z["t"]
    k, v, l = z["rk"], z["rv"], z["rl"]
    pos = t[:, None] - w + torch.arange(w, device=DEV)                        # [b, keys]
    live = pos >= 0
    if commit is not None:
        old, layer, path, length, _ = commit
        at = path.clamp(min=0).long()
        k, v = (torch.cat([a, old[m][layer].gather(1, at[:, :, None, None].expand(-1, -1, hkv, D)).transpose(1, 2)], 2)
                for a, m in ((k, "k"), (v, "v")))
        l = torch.cat([l, old["l"][layer].gather(1, at[:, :, None].expand(-1, -1, hkv)).transpose(1, 2)], 2)
        i = torch.arange(n, device=DEV)
        pos = torch.cat([pos, t[:, None] + i], 1)
        live = torch.cat([live, i < length[:, None]], 1)
        t = t + length
    # ancestors (and the node itself) of every node, and its depth
    up = torch.eye(n, dtype=torch.bool, device=DEV).expand(b, n, n).clone()
    for i in range(1, n):
        p = new["parent"][:, i].long()
        row = up.gather(1, p.clamp(min=0)[:, None, None].expand(-1, 1, n))[:, 0] & (p >= 0)[:, None]
        up[:, i] |= row
    depth = up.sum(-1) - 1                                                    # [b, n]
    k, v = (torch.cat([a, x[m].transpose(1, 2)], 2) for a, m in ((k, "k"), (v, "v")))
    l = torch.cat([l, x["l"].transpose(1, 2)], 2)
    pos = torch.cat([pos, t[:, None] + depth], 1)
    line = torch.cat([live[:, None].expand(-1, n, -1), up], 2)                # [b, n, keys] on the node's path
    near = pos[:, None] > (t[:, None] + depth)[:, :, None] - w                # [b, n, keys] in its window
    see = (line & near)[:, None] | (line[:, None] & (l >= 0)[:, :, None])     # [b, hkv, n, keys]
    q = x["q"].float().view(b, n, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4) / math.sqrt(D)   # [b, hkv, g, n, D]
    q = q.reshape(b, hkv, -1, D)

    def scores(keys, mask):
        return (q @ keys.float().transpose(-1, -2)).view(b, hkv, hq // hkv, n, -1).masked_fill_(~mask, -math.inf)

    far = scores(z["K"], z["live"][:, :, None, None])
    tail = scores(k, see[:, :, None])
    top = torch.maximum(far.amax(-1, keepdim=True), tail.amax(-1, keepdim=True))
    far, tail = far.sub_(top).exp_(), tail.sub_(top).exp_()
    total = far.sum(-1, keepdim=True) + tail.sum(-1, keepdim=True)
    out = far.flatten(2, 3) @ z["V"].float() + tail.flatten(2, 3) @ v.float()
    out = out.view(*total.shape[:-1], D) / total
    drawn = torch.arange(n, device=DEV) < new["n"][:, None]                   # [b, n]
    out = out.permute(0, 3, 1, 2, 4).reshape(b, n, hq, D) * drawn[:, :, None, None]
    lse = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(b, n, hq) * drawn[:, :, None]
    return out.to(torch.bfloat16), lse


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(c):
    if c["op"] == "accept":
        return {"bytes": c["b"] * (4 * 4 * c["nodes"] + 12), "flops": 2 * c["b"] * c["nodes"]}
    if c["op"] == "logprobs":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * BYTES[c["dtype"]] + c["rows"] * (8 + 8 * c["given"] + 8 * c["top"]), "flops": 6 * n}
    w, rates, g = c["window"], _rates(c), c["hq"] // c["hkv"]
    size = flops = 0.0
    for t, n in zip(_lengths(c), _nodes(c)):
        keys = float(np.sum(rates)) * max(0, t - w) + c["hkv"] * (min(t, w) + n)
        size += keys * 4 * D + n * c["hq"] * (4 * D + 4) + 4 * n
        flops += 4 * D * g * n * keys
        if c["op"] == "step":                            # an accepted pair or two: read, and written in place of another
            size += 2 * 2 * c["hkv"] * 4 * D
    return {"bytes": c["layers"] * size, "flops": c["layers"] * flops}


# ---- the same from the definitions in 64 bits ------------------------------------------------------
def exact(case, seed):
    if case["op"] == "accept":
        return None
    if case["op"] == "logprobs":
        s = _scores(case, seed)
        z = s["x"].double() * case["scale"]
        logp = torch.log_softmax(z, 1)
        top = logp.topk(case["top"], 1).values if case["top"] else None
        return (torch.logsumexp(z, 1), logp.gather(1, s["given"].long()), -torch.special.xlogy(logp.exp(), logp.exp()).sum(1), None, top)
    c, s = case, _raw(case, seed)
    w, g, n = c["window"], c["hq"] // c["hkv"], c["nodes"]
    out = torch.zeros((c["layers"], c["b"], n, c["hq"], D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((c["layers"], c["b"], n, c["hq"]), dtype=torch.float64, device=DEV)
    parents, counts = s["new"]["parent"].tolist(), s["new"]["n"].tolist()
    for b in range(c["b"]):
        taken = _walk({k: v[b].tolist() for k, v in s["old"].items() if k in ("parent", "tokens", "target", "n")}) if "old" in s else []
        # the nodes' paths: a path's tokens stand behind the context, one position after the other
        lines = []
        for i in range(counts[b]):
            lines.append((lines[parents[b][i]] if parents[b][i] >= 0 else []) + [i])
        for layer, x in enumerate(s["layers"]):
            K, V, L = (torch.cat([x[m][b], s["old"][m.lower()][layer, b][taken]]) if taken else x[m][b] for m in "KVL")
            t = len(K)
            for h in range(c["hkv"]):
                past = torch.nonzero((L[:, h] >= 0) | (torch.arange(t, device=DEV) > t - w))[:, 0]   # what any node may see
                hs = slice(h * g, (h + 1) * g)
                kp, vp = (torch.cat([a[past, h], x[m][b, :counts[b], h]]).double() for a, m in ((K, "k"), (V, "v")))
                z = torch.einsum("ngd,kd->ngk", x["q"][b, :counts[b], hs].double(), kp) * D ** -0.5
                see = torch.zeros((counts[b], len(kp)), dtype=torch.bool, device=DEV)
                loud_past, loud_new = L[past, h] >= 0, (x["l"][b, :, h] >= 0).tolist()
                for i, line in enumerate(lines):
                    p = t + len(line) - 1                                    # the node's own position
                    see[i, :len(past)] = loud_past | (past > p - w)
                    ok = [y for d, y in enumerate(line) if t + d > p - w or loud_new[y]]
                    see[i, len(past) + torch.tensor(ok, device=DEV)] = True
                z.masked_fill_(~see[:, None], -math.inf)
                lse[layer, b, :counts[b], hs] = torch.logsumexp(z, -1)
                out[layer, b, :counts[b], hs] = torch.softmax(z, -1) @ vp
    return (out, lse) + ((None, None, None) if "old" in s else ())


def _walk(d):
    """Node 0, then from node to node the first child whose token is the target's"""
    line, i = [0], 1
    while i < d["n"]:
        if d["parent"][i] == line[-1] and d["tokens"][i] == d["target"][line[-1]]:
            line.append(i)
        i += 1
    return line
