"""Log probabilities, entropies and top lists of rows of logits, against the formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

from gpu_util import dev, load

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def expect(x, given, top, scale):
    """x [n, v] float64 (already rounded to the type).  Order: NaN first, then descending, ties by index."""
    with np.errstate(all="ignore"):
        z = x * scale
        m = z.max(1, keepdims=True)
        ln = np.log(np.exp(z - m).sum(1))
        lse = np.where(np.isinf(m[:, 0]), m[:, 0], m[:, 0] + ln)
        # (relative to the maximum: next to the types' lowest value lse itself has no room for ln)
        logp = np.where(np.isinf(m), z - lse[:, None], z - m - ln[:, None])
        p = np.exp(logp)
        ent = -np.where(p == 0, 0, p * logp).sum(1)
        g = np.where((given >= 0) & (given < x.shape[1]), np.take_along_axis(logp, np.clip(given, 0, x.shape[1] - 1), 1), np.nan)
        order = np.lexsort((np.broadcast_to(np.arange(x.shape[1]), x.shape), -np.where(np.isnan(x), 0, x), ~np.isnan(x)), axis=1)[:, :top]
        ids = np.concatenate([order, np.full((len(x), max(0, top - x.shape[1])), -1)], 1)
        tl = np.concatenate([np.take_along_axis(logp, order, 1), np.full((len(x), max(0, top - x.shape[1])), np.nan)], 1)
    return lse, g, ent, ids, tl


def close(got, ref, tol):
    """(a value beyond float32 is an infinity there)"""
    got = got.cpu().double().numpy()
    with np.errstate(over="ignore"):
        ref = np.where(np.abs(ref) > 1e38, ref.astype(np.float32), ref)
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - ref) <= tol))
    assert not bad.any(), (got[bad][:4], ref[bad][:4], np.abs(got - ref)[bad].max())


def check(spkv, xt, given, top, scale=1.0, **kw):
    """A term of S is off by 2^-22 (the exponential) and 2^-23 times its exponent's size (the product with the scale, rounded;
    an exponent of t weighs 2^t, so t 2^t <= 0.54 of the largest term a term), sums by 2^-23 a step, 64 elements of a lane and 12 joins,
    in A likewise against sum 2^t |t|.  In nats, for lse, entropy and log probabilities, rel below; a log probability's own product and
    sums are rounded three times, 2^-24 of |x - m| scale and of itself."""
    lse, logp, ent, ids, tl = spkv.spkv_token_logprobs(xt, given, top=top, scale=scale, **kw)
    x = xt.float().cpu().double().numpy()
    g = np.zeros((len(x), 0), np.int64) if given is None else given.cpu().numpy().astype(np.int64)
    rl, rg, re, ri, rt = expect(x, g, top, scale)
    rel = 2.0 ** -22 + (0.54 + 2) * 2.0 ** -23 + 80 * 2.0 ** -23
    with np.errstate(all="ignore"):
        m = np.where(np.isfinite(x), x, -np.inf).max(1)
        size = np.where(np.isfinite(m), np.abs(m), 0) * scale
        spread = np.log(x.shape[1]) + 1
    close(lse, rl, rel + 2.0 ** -23 * (size + spread))
    close(ent, re, 2 * rel * (spread + 1) + 2.0 ** -22 * spread)
    if given is not None:
        close(logp, rg, rel + 2.0 ** -22 * (np.abs(np.where(np.isfinite(rg), rg, 0)) + spread))
    if top:
        assert np.array_equal(ids.cpu().numpy(), ri), (ids.cpu().numpy()[:, :5], ri[:, :5])
        close(tl, rt, rel + 2.0 ** -22 * (np.abs(np.where(np.isfinite(rt), rt, 0)) + spread))


def rows(n, v, dtype, seed, pad=0, off=0, gain=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (gain * torch.randn((n, v + pad + off), generator=g, device=dev())).to(TYPES[dtype])
    return x[:, off:off + v], torch.randint(-2, v + 2, (n, 3), generator=g, device=dev(), dtype=torch.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,v,top,pad,off", [
    (1, 1, 3, 0, 0), (3, 2, 1, 0, 0), (2, 31, 32, 0, 0), (5, 1000, 5, 0, 0), (2, 1023, 32, 1, 1), (2, 1024, 7, 0, 3), (3, 1025, 1, 5, 7),
    (4, 8191, 20, 2, 0), (3, 32000, 0, 0, 0), (7, 50257, 5, 0, 0), (2, 128256, 32, 64, 0), (40, 3001, 2, 3, 2), (1, 300001, 9, 0, 1),
])
def test_against_the_formulas(dtype, n, v, top, pad, off):
    spkv = load()
    x, given = rows(n, v, dtype, n * 7 + v, pad, off)
    check(spkv, x, given, top)
    check(spkv, x, given[:, :1].contiguous(), top, scale=0.7)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_masks_infinities_and_nan(dtype):
    spkv = load()
    x, given = rows(14, 5000, dtype, 1)
    low = torch.finfo(TYPES[dtype]).min
    x[0, ::2] = -math.inf
    x[1, 1:] = -math.inf                       # one token left
    x[2] = -math.inf                           # none
    x[3] = low                                 # all masked alike by the lowest value
    x[4, 17:] = low
    x[5, 4000] = math.inf
    x[6, [3, 4999]] = math.inf
    x[7, 2048] = math.nan
    x[8, 77], x[8, 78] = math.nan, math.inf
    x[9] = math.nan
    x[10] = 1.5                                # all alike
    x[11, 1024:2048] = x[11].float().max() + 1 # a whole chunk of ties
    x[12, 4999] = -torch.finfo(TYPES[dtype]).min   # the largest finite value
    x[13, :3000], x[13, 3000:] = 0.0, -0.0     # equal values
    for top in (1, 6, 32):
        check(spkv, x, given, top)
    for scale in (1e-5, 1e-2, 100.0):          # -infinity has probability 0 at every temperature
        check(spkv, x, given, 3, scale=scale)


def test_order_of_ascending_and_equal_logits():
    spkv = load()
    for x in (torch.arange(20000, device=dev()).float()[None], -torch.arange(20000, device=dev()).float()[None], torch.zeros((2, 9000), device=dev()),
              (torch.arange(30000, device=dev()) // 100 % 7).float()[None]):
        for top in (1, 5, 32):
            check(spkv, x * 1e-3, None, top)
            check(spkv, (x * 1e-3).bfloat16(), None, top)


def test_strides_past_32_bits_and_given_shapes():
    spkv = load()
    base, v = 1 << 31, 3000
    big = torch.empty(2 * base + v, dtype=torch.bfloat16, device=dev())
    x = big.as_strided((3, v), (base, 1))
    g = torch.Generator(device="cuda").manual_seed(3)
    for i in range(3):
        x[i] = torch.randn(v, generator=g, device=dev()).bfloat16()
    given = torch.randint(0, v, (3, 64), generator=g, device=dev(), dtype=torch.int32)
    check(spkv, x, given, 4)
    del big, x
    one = torch.randn((1, v), generator=g, device=dev())
    check(spkv, one.expand(5, v), given[:1].repeat(5, 1), 2)     # one row for all
    assert spkv.spkv_token_logprobs(one[:0], given[:0], top=2)[0].shape == (0,)


@pytest.mark.parametrize("dtype,n,v,top,pad,off", [
    ("f32", 20000, 1, 2, 0, 0), ("f16", 10007, 3, 4, 2, 1), ("f32", 3001, 2571, 3, 1, 1), ("bf16", 3001, 5121, 1, 0, 3), ("bf16", 6000, 1024, 0, 0, 0),
])
def test_pieces_that_begin_and_end_inside_rows(dtype, n, v, top, pad, off):
    """more chunks than the GPU has warps: several rows, and parts of rows, in a warp"""
    spkv = load()
    x, given = rows(n, v, dtype, n + v, pad, off)
    check(spkv, x, given, top, scale=1.3)


def test_many_rows_and_repeats_give_the_same_bits():
    spkv = load()
    x, given = rows(3000, 6007, "bf16", 5)
    a = spkv.spkv_token_logprobs(x, given, top=3)
    b = spkv.spkv_token_logprobs(x, given, top=3)
    assert all(torch.equal(s, t) or (torch.isnan(s) == torch.isnan(t)).all() for s, t in zip(a, b))
    check(spkv, x[::97], given[::97].contiguous(), 3)


def test_results_on_request_and_streams():
    spkv = load()
    x, given = rows(6, 4000, "f32", 2)
    full = spkv.spkv_token_logprobs(x, given, top=4)
    some = spkv.spkv_token_logprobs(x, want_entropy=False)
    assert some[1] is some[2] is some[3] is some[4] is None and torch.equal(some[0], full[0])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    on = spkv.spkv_token_logprobs(x, given, top=4, stream=s)
    s.synchronize()
    assert all(torch.equal(torch.nan_to_num(a, 9), torch.nan_to_num(b, 9)) for a, b in zip(full, on))
    out = [torch.empty_like(t) for t in full]
    got = spkv.spkv_token_logprobs(x, given, top=4, lse=out[0], logp=out[1], entropy=out[2], top_ids=out[3], top_logp=out[4])
    assert all(a is b for a, b in zip(got, out))
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(spkv.spkv_token_logprobs(x, given, top=4))
        graphs.append(g)
    for _ in range(3):
        for g, st in zip(graphs, (s, torch.cuda.Stream())):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(torch.nan_to_num(a, 9), torch.nan_to_num(b, 9)) for a, b in zip(full, o))


def test_acceptance_by_the_likeliest_token():
    """top ids of the nodes' logits are what spkv_tree_accept takes as the target"""
    spkv = load()
    x, _ = rows(2 * 6, 500, "bf16", 9)
    ids = spkv.spkv_token_logprobs(x, top=1)[3]
    target = ids.view(2, 6)
    tokens = torch.zeros((2, 6), dtype=torch.int32, device=dev())
    tokens[:, 1:] = target[:, :-1]
    tokens[1, 3] = 600
    path, n, nxt = spkv.spkv_tree_accept(tokens, target)
    assert n.tolist() == [6, 3] and nxt.tolist() == [int(target[0, 5]), int(target[1, 2])]


# ---- low and high temperatures ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("scale", [1e6, 1e8, 3e8, 3e9, 1e12, 1e20, 1e32, 1e34, 2e38, 3.4e38, 1e-30, 1e-42])
def test_rows_of_any_sign_at_any_scale(dtype, scale):
    """Rows whose maximum is negative, zero or positive: a scale admits every positive float32 (as float32 holds it), and the products
    of the scale and a logit may leave it."""
    spkv = load()
    x, given = rows(10, 5000, dtype, 11)
    x[0] -= 30                                  # every logit negative
    x[1] -= 30
    x[1, ::3] = -math.inf
    x[2] = -x[2].abs()
    x[2, 7] = 0.0                               # a maximum of zero
    x[3] = -x[3].abs()
    x[3, [9, 4000]] = 0.0                       # ... twice, the lowest value beside it
    x[3, 5:8] = torch.finfo(TYPES[dtype]).min
    x[4] = -20.0                                # all alike
    x[5, :3000] -= 6e4 if dtype == "f16" else 1e6   # pieces of the row far below the others
    x[6] -= 500
    x[7] = -torch.rand(5000, device=dev()) / 64 - 1 / 64
    x[8, 1:] = -math.inf                        # one token left, a negative one
    x[8, 0] = -3.0
    for top in (0, 3):
        check(spkv, x, given, top, scale=float(np.float32(scale)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_differences_beyond_float32(dtype):
    """logits of +-3e38: their difference leaves float32, its product with a small scale does not"""
    spkv = load()
    x, given = rows(4, 3000, dtype, 12)
    x[0] = torch.where(x[0] > 0, 3e38, -3e38)
    x[1] = x[1].clamp(-1, 1) * 3e38
    x[2, ::2] = -3e38
    x[3] = -3e38
    x[3, 100] = 1e38
    for scale in (1e-38, 3e-39, 1e-37):
        check(spkv, x, given, 4, scale=float(np.float32(scale)))


# ---- a fixed order -----------------------------------------------------------------------------------------
def bits(t):
    return t.view(torch.int32) if t.dtype == torch.float32 else t


@pytest.mark.parametrize("dtype,n,v,top", [("bf16", 3000, 6007, 3), ("f32", 700, 20011, 32), ("f16", 5, 128256, 1), ("f32", 20000, 100, 2)])
def test_repeats_give_the_same_bits_whatever_the_workspace_holds(dtype, n, v, top):
    spkv = load()
    x, given = rows(n, v, dtype, 6)
    first = spkv.spkv_token_logprobs(x, given, top=top)
    for byte in (0, 255, 0x7f):
        for ws in spkv._logprob_ws.values():
            ws.fill_(byte)
        again = spkv.spkv_token_logprobs(x, given, top=top)
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(first, again))
