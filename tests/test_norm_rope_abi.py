"""Argument checks of the norm + rotation entry points: no GPU is touched."""
import ctypes as C

import numpy as np
import pytest

from paper_2605_14037_b200 import build as spkv_build

FAKE = 1 << 20      # a 16-byte aligned address that is never read


@pytest.fixture(scope="module")
def spkv():
    spkv_build.build()
    from paper_2605_14037_b200 import spkv as mod
    mod.lib()
    return mod


def rope(spkv, rot=128, axes=1, inv=None, axis=None, scale=1.0, interleaved=0):
    inv = np.ones(max(rot // 2, 1)) if inv is None else np.asarray(inv, dtype=np.float64)
    r = spkv.Rope()
    rc = spkv.lib().spkv_rope_init(C.addressof(r), rot, interleaved, axes, scale, inv.ctypes.data,
                                   None if axis is None else np.asarray(axis, np.uint8).ctypes.data)
    return rc, r


def test_frequencies_as_fractions_of_a_turn(spkv):
    """2 pi f_i positions per turn: the 64-bit fraction is exact to 2^-63 turns, whole turns vanish."""
    f = [2 * np.pi * 0.25, 2 * np.pi * 3.5, -2 * np.pi * 0.25, 1.0, 1e-9, 0.0, 1e6, -1e-12]
    rc, r = rope(spkv, 16, inv=f)
    assert rc == 0
    two_pi = 2 * np.longdouble("3.14159265358979323846264338327950288")
    for p, x in enumerate(f):
        turns = np.longdouble(x) / two_pi
        want = turns - np.floor(turns)
        got = np.longdouble(int(r.turn[p])) / np.longdouble(2 ** 64)
        diff = abs(got - want)
        # the quotient is rounded to 64 significant bits: 2^-63 of its size, and the fraction is cut at 2^-64
        assert min(diff, abs(1 - diff)) <= 2.0 ** -62 * max(1.0, abs(float(turns))), (p, x)


@pytest.mark.parametrize("kw", [
    dict(rot=-16), dict(rot=8), dict(rot=272), dict(axes=0), dict(axes=5), dict(scale=float("nan")),
    dict(rot=16, inv=[1, 1, 1, float("inf"), 1, 1, 1, 1]), dict(rot=16, axes=2, axis=[0, 1, 2, 0, 1, 0, 1, 0]),
])
def test_rope_refusals(spkv, kw):
    assert rope(spkv, **kw)[0] == -1


def call(spkv, backward=False, n=5, pos=FAKE, rows=None, heads=(4, 2), ws=FAKE, ws_bytes=1 << 30, dwq=None, rp=None, v=None,
         v_out=None, **kw):
    d = dict(dtype=0, weight_dtype=0, head_dim=128, n_q_heads=heads[0], n_kv_heads=heads[1], norm=3, eps=1e-6)
    d.update(kw)
    norm = spkv.QkNorm(d["dtype"], d["weight_dtype"], d["head_dim"], d["n_q_heads"], d["n_kv_heads"], d["norm"], d["eps"], None, None)
    rp = rope(spkv)[1] if rp is None else rp
    good = spkv.Rows(FAKE, 512, 128)
    r = [C.byref(good)] * 4 if rows is None else [None if x is None else C.byref(spkv.Rows(*x)) for x in rows]
    l = spkv.lib()
    if backward:
        return l.spkv_norm_rope_backward(C.addressof(norm), C.addressof(rp), n, pos, r[0], r[1], r[0], r[1], v, r[2], r[3], v_out,
                                         dwq, None, ws, ws_bytes, None)
    return l.spkv_norm_rope(C.addressof(norm), C.addressof(rp), n, pos, r[0], r[1], v, r[2], r[3], v_out, None)


GOOD = (FAKE, 512, 128)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), -1), (dict(pos=None), -1), (dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(weight_dtype=7), -1),
    (dict(head_dim=8), -3), (dict(head_dim=272), -3), (dict(head_dim=100), -3), (dict(head_dim=64), -1),   # rot 128 > 64
    (dict(heads=(-1, 2)), -1), (dict(heads=(4, 5000)), -1), (dict(norm=4), -1), (dict(norm=-1), -1), (dict(eps=-1.0), -1),
    (dict(eps=float("nan")), -1), (dict(rows=[None, GOOD, GOOD, GOOD]), -1), (dict(rows=[GOOD, GOOD, GOOD, None]), -1),
    (dict(rows=[(0, 512, 128), GOOD, GOOD, GOOD]), -1), (dict(rows=[(FAKE + 2, 512, 128), GOOD, GOOD, GOOD]), -1),
    (dict(rows=[GOOD, (FAKE, 513, 128), GOOD, GOOD]), -1), (dict(rows=[GOOD, GOOD, (FAKE, 512, 4), GOOD]), -1),
    (dict(v=C.byref(C.c_int64())), -1),
])
def test_row_call_refusals(spkv, backward, kw, code):
    assert call(spkv, backward, **kw) == code


def test_workspace_and_null_arguments(spkv):
    l = spkv.lib()
    assert call(spkv, True, dwq=FAKE, ws=None) == -7
    assert call(spkv, True, dwq=FAKE, ws=FAKE + 4) == -7
    assert call(spkv, True, dwq=FAKE, ws_bytes=100) == -7
    assert call(spkv, True, dwq=FAKE, norm=2) == -1            # no query norm, no query weights
    assert call(spkv, n=0, pos=None) == 0                       # nothing to do
    assert call(spkv, heads=(0, 0)) == 0
    assert l.spkv_norm_rope(None, None, 1, None, *[None] * 6, None) == -1
    assert l.spkv_norm_rope_workspace_bytes(None) == 0
    rp = rope(spkv)[1]
    rp.axis[3] = 1
    assert call(spkv, rp=rp) == -1                              # an axis that does not exist
