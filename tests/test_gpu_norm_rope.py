"""Per-head norm + position rotation and its backward pass against the formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

from gpu_util import dev, load

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
U = 2.0 ** -24          # half a step of float32


def inv_freq(rot, theta=10000.0):
    return theta ** (-np.arange(rot // 2) * 2.0 / max(rot, 1))


def rotate64(x, pos, inv, axis, rot, interleaved, scale, sign=1.0):
    """x [n, H, D] float64 -> rotated (first rot dims); also |lo| + |hi| of each element's pair."""
    y, mag = x.copy(), np.abs(x)
    if rot == 0:
        return y, mag
    ang = (pos[axis].astype(np.float64) * inv[:, None]).T[:, None]      # [n, 1, pairs]
    c, s = np.cos(ang), sign * np.sin(ang)
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = scale * (a * c - b * s), scale * (b * c + a * s)
    mag[..., lo] = mag[..., hi] = abs(scale) * (np.abs(a) + np.abs(b))
    return y, mag


class Case:
    """Seeded inputs of one call, in the layout asked for, and the formulas in float64."""

    def __init__(self, seed, n, hq, hkv, D=128, rot=None, dtype="bf16", axes=1, interleaved=False, norm=True, scale=1.0,
                 layout="fused", lo_pos=0, hi_pos=4096, weights=True, wdtype=None):
        rng = np.random.default_rng(seed)
        self.n, self.hq, self.hkv, self.D, self.dt = n, hq, hkv, D, DT[dtype]
        self.rot = D if rot is None else rot
        self.inter, self.scale, self.norm = interleaved, scale, norm
        self.pos = rng.integers(lo_pos, hi_pos, size=(axes, n), dtype=np.int64).astype(np.int32)
        self.inv = inv_freq(self.rot)
        self.axis = (np.arange(self.rot // 2) % axes).astype(np.uint8)
        H = hq + 2 * hkv
        gain = 2.0 ** rng.integers(-2, 4, size=(1, H, 1))
        x = torch.from_numpy(rng.standard_normal((n, H, D)) * gain).to(self.dt)
        g = torch.from_numpy(rng.standard_normal((n, H, D))).to(self.dt)
        self.x, self.g = self.place(x, layout), self.place(g, layout)
        wdt = DT[wdtype] if wdtype else self.dt
        self.w = [torch.from_numpy(1 + 0.3 * rng.standard_normal(D)).to(wdt).to(dev()) if weights else None for _ in "qk"]
        self.sides = {"q": norm in (True, "q"), "k": norm in (True, "k")}
        self.spkv = load()
        self.nr = self.spkv.make_norm_rope(hq, hkv, D, self.dt, self.w[0], self.w[1], norm=norm, eps=EPS, rot_dim=self.rot,
                                           inv_freq=self.inv, axis=self.axis, n_axes=axes, interleaved=interleaved, scale=scale)
        self.pos_d = torch.from_numpy(self.pos).to(dev())

    def place(self, x, layout):
        n, H, D = x.shape
        if layout == "heads":
            t = x.transpose(0, 1).contiguous().to(dev()).transpose(0, 1)
        elif layout == "padded":     # rows and tokens with gaps
            buf = torch.full((n, H + 1, D + 16), float("nan"), dtype=x.dtype, device=dev())
            t = buf[:, :H, 8 * 1:8 * 1 + D] if x.dtype != torch.float32 else buf[:, :H, 4:4 + D]
            t.copy_(x.to(dev()))
        else:
            t = x.contiguous().to(dev())
        return t[:, :self.hq], t[:, self.hq:self.hq + self.hkv], t[:, self.hq + self.hkv:]

    def w64(self, i):
        return np.ones(self.D) if self.w[i] is None else self.w[i].cpu().double().numpy()

    def half(self, y):
        """half a step of the result's type at y"""
        fi = torch.finfo(self.dt)
        return np.maximum(np.abs(y), fi.smallest_normal) * (fi.eps / 2)

    def forward64(self, i):
        x = self.x[i].cpu().double().numpy()
        if self.sides["qk"[i]]:
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * self.w64(i)
        return rotate64(x, self.pos, self.inv, self.axis, self.rot, self.inter, self.scale)

    def backward64(self, i):
        """dx, a bound on the size of what is added up for it, dw, the same for dw"""
        x, g = self.x[i].cpu().double().numpy(), self.g[i].cpu().double().numpy()
        g, mag = rotate64(g, self.pos, self.inv, self.axis, self.rot, self.inter, self.scale, -1.0)
        if not self.sides["qk"[i]]:
            return g, mag, None, None
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
        u, w = x * r, self.w64(i)
        dx = r * (w * g - u * (w * g * u).mean(-1, keepdims=True))
        size = r * (np.abs(w) * mag + np.abs(u) * (np.abs(w) * mag * np.abs(u)).mean(-1, keepdims=True))
        return dx, size, (g * u).sum((0, 1)), (mag * np.abs(u)).sum((0, 1))


# A result is rounded once (half a step of its type) after float32 work whose relative error, counted
# along the longest chain in units of 2^-24: sum of squares <= 16 fma + 5 adds + 2, halved by the root (12),
# rsqrt 4, x r w 2, sine / cosine 4 with their argument's rounding, rotation 2: below 32 for every case here,
# of |lo| + |hi|.  The backward adds the second row sum and three more products: below 80.
def check_forward(c, out):
    for i in range(2):
        ref, mag = c.forward64(i)
        got = out[i].cpu().double().numpy()
        err, tol = np.abs(got - ref), c.half(ref) + 32 * U * mag
        assert (err <= tol).all(), ("qk"[i], err.max(), (err - tol).max())
    if out[2] is not None:
        assert torch.equal(out[2], c.x[2])


def check_backward(c, res):
    for i in range(2):
        dx, size, dw, wsize = c.backward64(i)
        got = res[i].cpu().double().numpy()
        err, tol = np.abs(got - dx), c.half(dx) + 80 * U * size
        assert (err <= tol).all(), ("qk"[i], err.max(), (err - tol).max())
        if dw is None:
            assert res[3 + i] is None
        else:
            # a term's own error, then at most rows / 8 + 256 additions one after the other
            rows = c.n * (c.hq, c.hkv)[i]
            err, tol = np.abs(res[3 + i].cpu().double().numpy() - dw), (80 + rows / 8 + 256) * U * wsize
            assert res[3 + i].dtype == torch.float32 and (err <= tol).all(), ("qk"[i], err.max(), (err - tol).max())
    if res[2] is not None:
        assert torch.equal(res[2], c.g[2])


CASES = [
    dict(n=1, hq=8, hkv=2), dict(n=3, hq=5, hkv=1, layout="heads"), dict(n=64, hq=32, hkv=8, hi_pos=131072),
    dict(n=1, hq=1, hkv=1, D=16, dtype="f32"), dict(n=17, hq=3, hkv=3, D=16), dict(n=33, hq=2, hkv=1, D=48, rot=32),
    dict(n=257, hq=7, hkv=1, dtype="f16", axes=3, interleaved=True), dict(n=100, hq=4, hkv=4, D=80, rot=32, dtype="f16"),
    dict(n=129, hq=4, hkv=2, D=256, dtype="f32", rot=128), dict(n=50, hq=4, hkv=2, D=256, layout="padded"),
    dict(n=65, hq=6, hkv=2, D=64, dtype="f32", axes=2, interleaved=True, layout="padded"),
    dict(n=40, hq=4, hkv=2, D=192, axes=4, layout="heads"), dict(n=1300, hq=8, hkv=2, dtype="f32"),
    dict(n=5000, hq=8, hkv=2, norm=False), dict(n=30, hq=4, hkv=2, norm="q", wdtype="f32"),
    dict(n=30, hq=4, hkv=2, norm="k", weights=False, scale=1.25), dict(n=30, hq=4, hkv=2, rot=0),
    dict(n=77, hq=4, hkv=2, D=96, rot=96, dtype="f32", wdtype="bf16"), dict(n=9, hq=64, hkv=8, dtype="f16", rot=16),
    # from a block per token to a warp per token: eight, four, two warps a token, with and without heads for each
    dict(n=297, hq=3, hkv=1), dict(n=500, hq=40, hkv=5, interleaved=True, rot=64), dict(n=900, hq=17, hkv=2, dtype="f16", D=64),
    dict(n=2400, hq=5, hkv=3, D=32, dtype="f32"), dict(n=310, hq=2, hkv=2, D=240, rot=48, axes=2, interleaved=True),
    dict(n=1, hq=6, hkv=2, D=176, rot=96, interleaved=True, dtype="f16"),
    # several blocks a token, the last of them in part; a block a token with many heads
    dict(n=2, hq=64, hkv=63, dtype="f32"), dict(n=150, hq=37, hkv=7), dict(n=592, hq=19, hkv=9, D=80, rot=48, dtype="f16"),
    # two, four and eight warps a token
    dict(n=601, hq=40, hkv=5, interleaved=True, rot=64), dict(n=1200, hq=24, hkv=23, dtype="f32"),
    dict(n=888, hq=64, hkv=61, dtype="f32", D=112, rot=96),
]


@pytest.mark.parametrize("k", range(len(CASES)))
def test_forward(k):
    c = Case(k, **CASES[k])
    check_forward(c, c.spkv.spkv_norm_rope(c.nr, c.pos_d, *c.x))
    q, kk, v = c.spkv.spkv_norm_rope(c.nr, c.pos_d, c.x[0], c.x[1])      # without values
    assert v is None
    check_forward(c, (q, kk, None))


@pytest.mark.parametrize("k", range(len(CASES)))
def test_backward(k):
    c = Case(k, **CASES[k])
    a = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, c.x[0], c.x[1], *c.g)
    check_backward(c, a)
    b = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, c.x[0], c.x[1], *c.g)
    assert all(x is None and y is None or torch.equal(x, y) for x, y in zip(a, b)), "the same inputs, other bits"


@pytest.mark.parametrize("lo,hi", [(-5000, 5000), (10 ** 6, 2 * 10 ** 6), (2 ** 31 - 50, 2 ** 31 - 1), (-2 ** 31, -2 ** 31 + 50)])
def test_far_and_negative_positions(lo, hi):
    """The angle is reduced exactly: no position costs accuracy (float64 products of such positions with a
    frequency <= 1 are exact to 2^-22 of a radian, which the tolerance's 4 * 2^-24 does not cover, so
    the reference reduces its angles in long double)."""
    c = Case(3, n=40, hq=4, hkv=2, dtype="f32", lo_pos=lo, hi_pos=hi)
    two_pi = 2 * np.longdouble("3.14159265358979323846264338327950288")
    ang = c.pos[0].astype(np.longdouble)[:, None] * c.inv.astype(np.longdouble)[None]
    ang = np.asarray(ang - two_pi * np.floor(ang / two_pi), dtype=np.float64)
    out = c.spkv.spkv_norm_rope(c.nr, c.pos_d, *c.x)
    for i in range(2):
        x = c.x[i].cpu().double().numpy()
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * c.w64(i)
        a, b = x[..., :64], x[..., 64:]
        cs, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
        ref = np.concatenate([a * cs - b * sn, b * cs + a * sn], -1)
        mag = np.tile(np.abs(a) + np.abs(b), 2)
        assert (np.abs(out[i].cpu().double().numpy() - ref) <= c.half(ref) + 32 * U * mag).all()


def test_gradient_against_differences():
    """<dx, d> and <dw, e> against the central difference of the float32 forward along d and e.  The
    difference's own truncation is taken from the same difference in float64; its noise is the
    forward's error bound over the step."""
    c = Case(11, n=12, hq=3, hkv=2, dtype="f32", axes=2, D=64, rot=32)
    rng = np.random.default_rng(5)
    res = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, c.x[0], c.x[1], *c.g)
    h = 2.0 ** -7
    for i in range(2):
        x64, w64, g64 = c.x[i].cpu().double().numpy(), c.w64(i), c.g[i].cpu().double().numpy()
        for what in ("x", "w"):
            d = rng.choice([-1.0, 1.0], size=x64.shape if what == "x" else w64.shape)
            vals, ref, noise = [], [], 0.0
            for sgn in (1, -1):
                xt = torch.from_numpy(x64 + (sgn * h * d if what == "x" else 0)).float().to(dev())
                wt = torch.from_numpy(w64 + (sgn * h * d if what == "w" else 0)).float().to(dev())
                nr = c.spkv.make_norm_rope(c.hq, c.hkv, c.D, torch.float32, wt, wt, eps=EPS, rot_dim=c.rot, inv_freq=c.inv,
                                           axis=c.axis, n_axes=2)
                xs = [c.x[0], c.x[1]]
                xs[i] = xt
                vals.append((c.spkv.spkv_norm_rope(nr, c.pos_d, *xs)[i].cpu().double().numpy() * g64).sum())
                y = xt.cpu().double().numpy()
                y = y / np.sqrt((y * y).mean(-1, keepdims=True) + EPS) * wt.cpu().double().numpy()
                y, mag = rotate64(y, c.pos, c.inv, c.axis, c.rot, False, 1.0)
                ref.append((y * g64).sum())
                noise += (33 * U * mag * np.abs(g64)).sum()
            want = (res[i] if what == "x" else res[3 + i]).cpu().double().numpy()
            dx, size, dw, wsize = c.backward64(i)
            exact, own = ((dx * d).sum(), (81 * U * size).sum()) if what == "x" else ((dw * d).sum(), (400 * U * wsize).sum())
            trunc = abs((ref[0] - ref[1]) / (2 * h) - exact)
            scale = np.abs(dx if what == "x" else dw).sum()
            tol = noise / (2 * h) + trunc + own
            assert tol < 0.05 * scale, "the difference says something"
            assert abs((vals[0] - vals[1]) / (2 * h) - (want * d).sum()) <= tol


def test_rows_in_place():
    c = Case(7, n=70, hq=8, hkv=2)
    want = c.spkv.spkv_norm_rope(c.nr, c.pos_d, *c.x)
    q, k, v = (t.clone() for t in c.x)
    c.spkv.spkv_norm_rope(c.nr, c.pos_d, q, k, v, q, k, v)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, want[2])
    ref = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, c.x[0], c.x[1], *c.g)
    g = [t.clone() for t in c.g]
    c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, c.x[0], c.x[1], *g, dq=g[0], dk=g[1], dv=g[2])
    assert all(torch.equal(a, b) for a, b in zip(g, ref))
    xs = [t.clone() for t in c.x]                                    # ... and onto the forward's inputs
    c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, xs[0], xs[1], *c.g, dq=xs[0], dk=xs[1], dv=xs[2])
    assert torch.equal(xs[0], ref[0]) and torch.equal(xs[1], ref[1])


def test_only_the_rows_are_written():
    """Outputs with gaps: the gaps keep their contents."""
    c = Case(8, n=20, hq=3, hkv=2, layout="padded")
    buf = torch.full((20, 8, 160), 3.0, dtype=c.dt, device=dev())
    outs = buf[:, :3, 16:144], buf[:, 3:5, 16:144], buf[:, 5:7, 16:144]
    c.spkv.spkv_norm_rope(c.nr, c.pos_d, *c.x, *outs)
    check_forward(c, outs)
    gap = torch.ones((20, 8, 160), dtype=torch.bool)
    gap[:, :7, 16:144] = False
    assert (buf.cpu()[gap] == 3.0).all()


def test_rows_of_zeros_infinities_and_nans_stay_in_their_row():
    c = Case(9, n=6, hq=4, hkv=2)
    q = c.x[0].clone()
    q[1, 2] = 0
    q[2, 1, 5] = float("inf")
    q[3, 0, 70] = float("nan")
    clean = c.spkv.spkv_norm_rope(c.nr, c.pos_d, c.x[0], c.x[1])[0]
    out = c.spkv.spkv_norm_rope(c.nr, c.pos_d, q, c.x[1])[0]
    assert (out[1, 2] == 0).all() and out[2, 1].isnan().any() and out[3, 0].isnan().all()
    same = torch.ones((6, 4), dtype=torch.bool)
    same[1, 2] = same[2, 1] = same[3, 0] = False
    assert torch.equal(out.cpu()[same], clean.cpu()[same])


def test_offsets_past_32_bits():
    """Two tokens 2^31 + 2^12 elements apart."""
    spkv = load()
    stride = 2 ** 31 + 2 ** 12
    base = torch.empty(stride + 1024, dtype=torch.bfloat16, device=dev())
    rows = base.as_strided((2, 1, 128), (stride, 128, 1))
    kv = base.as_strided((2, 1, 128), (stride, 128, 1), 256)
    g = torch.Generator().manual_seed(3)
    a, b = torch.randn((2, 1, 128), generator=g).bfloat16(), torch.randn((2, 1, 128), generator=g).bfloat16()
    rows.copy_(a), kv.copy_(b)
    nr = spkv.make_norm_rope(1, 1, theta=500000.0)
    pos = torch.tensor([3, 9], dtype=torch.int32, device=dev())
    want = spkv.spkv_norm_rope(nr, pos, a.to(dev()), b.to(dev()))
    got = spkv.spkv_norm_rope(nr, pos, rows, kv, None, rows, kv)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_no_tokens_and_one_sided_calls():
    spkv = load()
    w = torch.ones(128, dtype=torch.float32, device=dev())
    nr = spkv.make_norm_rope(4, 2, wq=w, wk=w)
    e = [torch.empty((0, h, 128), dtype=torch.bfloat16, device=dev()) for h in (4, 2, 2)]
    pos = torch.empty(0, dtype=torch.int32, device=dev())
    assert [t.shape[0] for t in spkv.spkv_norm_rope(nr, pos, *e)] == [0, 0, 0]
    dw = spkv.spkv_norm_rope_backward(nr, pos, e[0], e[1], *e)[3:]
    assert all((t == 0).all() for t in dw)
    # queries alone (keys of another layer): the key side has no heads
    c = Case(4, n=21, hq=4, hkv=2)
    nr = spkv.make_norm_rope(4, 0, dtype=c.dt, wq=c.w[0], eps=EPS, norm="q", inv_freq=c.inv)
    none = torch.empty((21, 0, 128), dtype=c.dt, device=dev())
    full = spkv.spkv_norm_rope(c.nr, c.pos_d, *c.x)[0]
    assert torch.equal(spkv.spkv_norm_rope(nr, c.pos_d, c.x[0], none)[0], full)


def test_another_stream_and_a_captured_graph():
    c = Case(12, n=130, hq=8, hkv=2)
    want = c.spkv.spkv_norm_rope(c.nr, c.pos_d, *c.x)
    ref = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, c.x[0], c.x[1], *c.g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = c.spkv.spkv_norm_rope(c.nr, c.pos_d, *c.x)
        res = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, c.x[0], c.x[1], *c.g)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want)) and all(torch.equal(a, b) for a, b in zip(res, ref))
    x, g = [t.contiguous().clone() for t in c.x], [t.contiguous().clone() for t in c.g]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.spkv.spkv_norm_rope(c.nr, c.pos_d, *x)
        res = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, x[0], x[1], *g)
    for t in (*x, *g):
        t.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    want = c.spkv.spkv_norm_rope(c.nr, c.pos_d, *x)
    ref = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, x[0], x[1], *g)
    assert all(torch.equal(a, b) for a, b in zip(out, want)) and all(torch.equal(a, b) for a, b in zip(res, ref))


def test_captured_backward_passes_replayed_at_the_same_time():
    """Two graphs of one descriptor, captured on one stream and replayed on two beside eager calls on a third: the
    weight gradients' partial sums of each are its own."""
    c, d = Case(21, n=3000, hq=8, hkv=2), Case(22, n=2500, hq=8, hkv=2)
    calls = [lambda c=c: c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, c.x[0], c.x[1], *c.g),
             lambda: c.spkv.spkv_norm_rope_backward(c.nr, d.pos_d, d.x[0], d.x[1], *d.g)]
    want = [f() for f in calls]
    graphs, res = [], []
    for f in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r = f()
        graphs.append(graph)
        res.append(r)
    s = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        for r in res:
            for t in r:
                t.zero_()
        torch.cuda.synchronize()
        for graph, st in zip(graphs, s):
            with torch.cuda.stream(st):
                graph.replay()
        eager = [f() for f in calls]
        torch.cuda.synchronize()
        for a, b, w in zip(res, eager, want):
            assert all(torch.equal(x, z) and torch.equal(y, z) for x, y, z in zip(a, b, w))


def test_binding_refusals():
    spkv = load()
    nr = spkv.make_norm_rope(4, 2)
    pos = torch.zeros(5, dtype=torch.int32, device=dev())
    q, k = torch.zeros((5, 4, 128), dtype=torch.bfloat16, device=dev()), torch.zeros((5, 2, 128), dtype=torch.bfloat16, device=dev())
    for bad in ((pos.long(), q, k), (pos, q[:4], k), (pos, q.float(), k), (pos, q, k[:, :1]), (pos, q[..., :64], k),
                (pos, q.transpose(1, 2).contiguous().transpose(1, 2), k), (pos.cpu(), q, k), (pos, q.cpu(), k)):
        with pytest.raises(ValueError):
            spkv.spkv_norm_rope(nr, *bad)
    with pytest.raises(spkv.SpkvError):      # rows off the 16-byte grid
        odd = torch.zeros(5 * 4 * 128 + 8, dtype=torch.bfloat16, device=dev())[1:-7].view(5, 4, 128)
        spkv.spkv_norm_rope(nr, pos, odd, k)
    with pytest.raises(ValueError):
        spkv.make_norm_rope(4, 2, inv_freq=np.ones(3))


@pytest.mark.parametrize("graph", [False, True])
def test_rows_go_straight_into_an_overlapping_cache(graph):
    """SPKV_FLAG_OVERLAP: an append or decode behind the row call that writes its inputs waits for it.  All rows go
    through the same three buffers, the batch's own last among 9000, so that a launch which did not wait would
    find an earlier call's.  Against a twin that waits for the device between any two calls."""
    spkv = load()
    L, B, n, hq, hkv, T0 = 4, 8, 9000, 16, 4, 300
    gen = torch.Generator(device=dev()).manual_seed(5)
    rnd = lambda *shape: torch.randn(shape, generator=gen, device=dev())
    caches = [spkv.Cache(L, B, hq, hkv, 1024, L * B * hkv * 8, window=64, tau=0.5, device=dev(), flags=spkv.FLAG_OVERLAP)
              for _ in range(2)]
    for l in range(L):
        for s in range(B):
            k, v, lg = rnd(T0, hkv, 128).bfloat16(), rnd(T0, hkv, 128).bfloat16(), rnd(T0, hkv)
            for c in caches:
                c.spkv_prefill(l, s, k, v, lg)
    nr = spkv.make_norm_rope(hq, hkv)
    qkv = [rnd(n, hq + 2 * hkv, 128).bfloat16() for _ in range(L + 1)]
    lg = rnd(L, B, hkv)
    pos = torch.arange(n, dtype=torch.int32, device=dev())
    ids = torch.arange(B, dtype=torch.int32, device=dev())

    def step(c, q, k, v, outs, between):
        rows = lambda x: spkv.spkv_norm_rope(nr, pos, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q, k, v)
        for l in range(L):
            rows(qkv[l])
            between()
            c.spkv_append_evict(l, ids, k[-B:], v[-B:], lg[l])
            between()
            rows(qkv[l + 1])
            between()
            c.spkv_decode_attention(l, ids, q[-B:], out=outs[l])
            between()

    results = []
    for c, wait in zip(caches, (False, True)):
        bufs = [torch.zeros((n, h, 128), dtype=torch.bfloat16, device=dev()) for h in (hq, hkv, hkv)]
        once = torch.zeros((L, B, hq, 128), dtype=torch.bfloat16, device=dev())
        c.decode_workspace(B)
        torch.cuda.synchronize()
        if graph and not wait:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step(c, *bufs, once, lambda: None)
        outs = []
        for i in range(3):
            if wait:
                step(c, *bufs, once, torch.cuda.synchronize)
            elif graph:
                g.replay()
            else:
                step(c, *bufs, once, lambda: None)
            outs.append(once.clone())
            c.spkv_note_foreign_work()      # (the copy of the results)
        c.check()
        results.append(torch.stack(outs))
    assert torch.equal(*results) and results[0].abs().max() > 0
    for l in range(L):
        assert np.array_equal(caches[0].spkv_read_lengths(l)[0], caches[1].spkv_read_lengths(l)[0])
        for s in range(B):
            for h in range(hkv):
                for read in ("spkv_read_kept", "spkv_read_window"):
                    a, b = (getattr(c, read)(l, s, h) for c in caches)
                    assert all(np.array_equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("n", [3, 700])          # both forward kernels
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [("bf16", 128, 64), ("f32", 64, 16), ("f16", 96, 80), ("bf16", 48, 16), ("f32", 256, 0),
                                         ("bf16", 128, 128)])
def test_infinities_and_nans_stay_in_their_pair(n, interleaved, dtype, D, rot):
    """Dims from rot_dim on are not rotated: what is there neither reaches another dim nor changes; a rotated dim
    reaches its partner only.  Without norm, forward and backward, and values that are infinite in a normed row."""
    spkv, dt = load(), DT[dtype]
    gen = torch.Generator().manual_seed(D + rot)
    x = torch.randn((n, 5, D), generator=gen).to(dt).to(dev())
    pos = torch.arange(n, dtype=torch.int32, device=dev()) * 37 + 1
    partner = lambda d: d if d >= rot else d ^ 1 if interleaved else (d + rot // 2) % rot
    bad = x.clone()
    hit = torch.zeros(x.shape, dtype=torch.bool, device=dev())
    plant = [float("inf"), float("-inf"), float("nan"), -0.0]
    for i, d in enumerate(sorted({0, rot // 2, rot - 1, rot, rot + 1, rot + (D - rot) // 2, D - 1, D - 2})):
        if 0 <= d < D:
            t, h = i % n, i % 5
            bad[t, h, d] = plant[i % 4]
            hit[t, h, d] = hit[t, h, partner(d)] = True
    nr = spkv.make_norm_rope(4, 1, D, dt, norm=False, rot_dim=rot, interleaved=interleaved)
    calls = (lambda y: spkv.spkv_norm_rope(nr, pos, y[:, :4], y[:, 4:]),
             lambda y: spkv.spkv_norm_rope_backward(nr, pos, None, None, y[:, :4], y[:, 4:]))
    for call in calls:
        clean, got = (torch.cat(call(y)[:2], 1) for y in (x, bad))
        assert torch.equal(got[~hit], clean[~hit])
        bits = torch.int32 if dtype == "f32" else torch.int16
        rest, want = got[..., rot:].contiguous(), bad[..., rot:].contiguous()
        nan = want.isnan()
        assert torch.equal(rest.isnan(), nan)
        assert torch.equal(rest.view(bits)[~nan], want.view(bits)[~nan])        # bit for bit, -0 too
        assert (torch.isnan(got) | torch.isinf(got))[..., :rot].sum() <= 2 * (~torch.isfinite(bad))[..., :rot].sum()
    # an infinity in a normed row: 1 / sqrt(inf) = 0, so the row's other dims are zeros
    d = D - 1
    y = x.clone()
    y[n - 1, 2, d] = float("inf")
    nr = spkv.make_norm_rope(4, 1, D, dt, rot_dim=rot, interleaved=interleaved)
    got = spkv.spkv_norm_rope(nr, pos, y[:, :4], y[:, 4:])[0][n - 1, 2]
    others = torch.ones(D, dtype=torch.bool, device=dev())
    others[d] = others[partner(d)] = False
    assert got[d].isnan() and (got[others] == 0).all()


@pytest.mark.parametrize("hq,hkv", [(8, 2), (5, 1), (1, 1), (37, 7), (16, 16)])
@pytest.mark.parametrize("dtype,n", [("bf16", 9), ("f32", 1), ("f16", 900), ("bf16", 3000)])
def test_no_eps_and_head_counts_that_leave_lanes_idle(monkeypatch, hq, hkv, dtype, n):
    """eps = 0: a lane without a row must not bring 0 * (1 / 0) into the weight gradients of the rows there are."""
    monkeypatch.setitem(globals(), "EPS", 0.0)      # of the descriptor and of the formulas
    c = Case(hq + n, n, hq, hkv, dtype=dtype)
    assert c.nr.norm.eps == 0.0
    check_forward(c, c.spkv.spkv_norm_rope(c.nr, c.pos_d, *c.x))
    check_backward(c, c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, c.x[0], c.x[1], *c.g))


@pytest.mark.parametrize("n", [5, 1500])         # both forward kernels
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_broadcast_rows(n, dtype):
    """Rows that several tokens or heads share (stride 0), as inputs and as upstream gradients: the bits of the rows
    written out; a gradient is one per token and head."""
    c = Case(30 + n, n, 6, 2, dtype=dtype)
    x, g = [t[:1, :1] for t in c.x], [t[:, :1] for t in c.g]
    wide = lambda t, h: t.expand(n, h, c.D)
    for i, form in enumerate((lambda t, h: wide(t, h), lambda t, h: wide(t[:, :1], h) if t.shape[0] > 1 else wide(t, h))):
        xs, gs = [[form(t, h) for t, h in zip(ts, (6, 2, 2))] for ts in (x if i == 0 else [t[:, :1] for t in c.x], g)]
        full = [[t.contiguous() for t in ts] for ts in (xs, gs)]
        assert any(0 in t.stride() for t in xs) and any(0 in t.stride() for t in gs)
        a, b = c.spkv.spkv_norm_rope(c.nr, c.pos_d, *xs), c.spkv.spkv_norm_rope(c.nr, c.pos_d, *full[0])
        assert all(torch.equal(s, t) for s, t in zip(a, b))
        a = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, xs[0], xs[1], *gs)
        b = c.spkv.spkv_norm_rope_backward(c.nr, c.pos_d, full[0][0], full[0][1], *full[1])
        assert all(torch.equal(s, t) for s, t in zip(a, b))
        c2 = Case(30 + n, n, 6, 2, dtype=dtype)      # ... and the formulas
        c2.x, c2.g = tuple(full[0]), tuple(full[1])
        check_backward(c2, a)
