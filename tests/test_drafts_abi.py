"""Argument checks of the calls for drafted tokens that take no cache: no GPU is touched."""
import pytest

from paper_2605_14037_b200 import build as spkv_build

FAKE = 1 << 20      # a 16-byte aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    spkv_build.build()
    from paper_2605_14037_b200 import spkv as mod
    return mod.lib()


def accept(lib, B=2, T=8, tokens=FAKE, target=FAKE, path=FAKE, n_path=FAKE, nxt=FAKE):
    return lib.spkv_tree_accept(B, T, None, None, tokens, target, path, n_path, nxt, None)


@pytest.mark.parametrize("kw", [dict(B=-1), dict(T=-1), dict(T=65), dict(tokens=None), dict(target=None), dict(path=None), dict(n_path=None), dict(nxt=None)])
def test_accept_refusals(lib, kw):
    assert accept(lib, **kw) == -1


def test_accept_of_no_sequences(lib):
    assert accept(lib, B=0, tokens=None, n_path=None) == 0


def logprobs(lib, dtype=0, n=4, v=100, x=FAKE, stride=100, scale=1.0, given=FAKE, n_given=1, n_top=1, lse=FAKE, ent=FAKE, logp=FAKE, ids=FAKE, tlp=FAKE,
             ws=FAKE, ws_bytes=1 << 30):
    return lib.spkv_token_logprobs(dtype, n, v, x, stride, scale, given, n_given, n_top, lse, ent, logp, ids, tlp, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(n=-1), -1), (dict(v=0), -1), (dict(x=None), -1), (dict(x=FAKE + 1), -1), (dict(dtype=2, x=FAKE + 2), -1),
    (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(given=None), -1),
    (dict(n_given=-1), -1), (dict(n_top=-1), -1), (dict(n_top=33), -3), (dict(n=1 << 20, n_given=1 << 12), -3), (dict(v=2 ** 31 - 1), -3),
    (dict(ws=None), -7), (dict(ws=FAKE + 8), -7), (dict(ws_bytes=10), -7),
])
def test_logprobs_refusals(lib, kw, code):
    assert logprobs(lib, **kw) == code


def test_logprobs_of_no_rows_and_workspace_sizes(lib):
    assert logprobs(lib, n=0, x=None, ws=None) == 0
    size = lib.spkv_logprobs_workspace_bytes
    assert size(0, 100, 0) >= 16 and size(10, 100000, 0) < size(10, 100000, 1) == size(10, 100000, 32) < size(20, 100000, 1)
    assert size(-1, 100, 0) == size(1, 0, 0) == size(1, 100, 33) == size(1, 100, -1) == 0


def test_calls_with_a_cache_refuse_a_missing_one(lib):
    assert lib.spkv_decode_attention_tree(None, 0, FAKE, 1, 1, None, None, FAKE, FAKE, FAKE, None, FAKE, None, 0.1, FAKE, 1 << 30, None) == -1
    assert lib.spkv_append_path(None, 0, 1, FAKE, 1, 1, None, None, FAKE, 0, FAKE, 0, FAKE, None) == -1


# ---- devices: the library and CUDA's current device are stand-ins (test_binding_streams.py) ------------------
from test_binding_streams import Tensor, a_cache, raw, two_devices  # noqa: E402,F401


@pytest.fixture(scope="module")
def spkv(lib):
    from paper_2605_14037_b200 import spkv as mod
    return mod


class Rows(Tensor):
    device = property(lambda self: f"cuda:{self.dev}")

    def stride(self, i=None):
        st, n = [], 1
        for x in reversed(self.shape):
            st.append(n)
            n *= x
        return tuple(reversed(st)) if i is None else st[::-1][i]

    def dim(self):
        return len(self.shape)


def drafts(dev):
    import torch
    t = lambda shape, dtype: Rows(shape, dtype, dev, 1 << 16)
    return dict(ids=t((2,), torch.int32), q=t((2, 3, 4, 128), torch.bfloat16), k=t((2, 3, 2, 128), torch.bfloat16), lg=t((2, 3, 2), torch.float32),
                tok=t((2, 3), torch.int32), n=t((2,), torch.int32), x=t((2, 50), torch.float32), f=t((2,), torch.float32), out=t((2, 3, 4, 128), torch.bfloat16))


def calls(spkv, cache, d, e=None, **kw):
    """The four calls; e: where one of each call's tensors comes from"""
    e = e or d
    return [lambda: cache.spkv_decode_attention_tree(0, d["ids"], d["q"], d["k"], e["k"], logits=d["lg"], out=d["out"], **kw),
            lambda: cache.spkv_append_path(0, d["ids"], d["k"], d["k"], e["lg"], **kw),
            lambda: spkv.spkv_tree_accept(d["tok"], e["tok"], None, None, d["tok"], d["n"], d["n"], **kw),
            lambda: spkv.spkv_token_logprobs(d["x"], lse=e["f"], want_entropy=False, **kw)]


@pytest.mark.parametrize("dev", [0, 1])
def test_calls_run_on_their_tensors_device(spkv, two_devices, monkeypatch, dev):
    cache = a_cache(spkv, dev)
    cache._tree_ws, cache._tree_bytes, cache.default_scale = {}, {(2, 3): 256}, 0.1
    monkeypatch.setattr(spkv, "_scratch", lambda store, n, d: Rows((n,), None, d, 4096))
    monkeypatch.setattr(spkv, "_logprob_bytes", {(2, 50, 0): 16})
    for call in calls(spkv, cache, drafts(dev)):
        call()
    assert [c[0] for c in two_devices] == ["spkv_decode_attention_tree", "spkv_append_path", "spkv_tree_accept", "spkv_token_logprobs"]
    for name, current, args in two_devices:
        assert current == dev and raw(args[-1]) == 100 + dev, name


def test_tensors_or_streams_of_another_device_are_refused(spkv, two_devices):
    cache, other = a_cache(spkv, 1), type("S", (), dict(device_index=0, cuda_stream=7))()
    cache._tree_ws, cache._tree_bytes, cache.default_scale = {}, {(2, 3): 256}, 0.1
    for call in calls(spkv, cache, drafts(1), drafts(0)) + calls(spkv, cache, drafts(0))[:2] + calls(spkv, cache, drafts(1), stream=other):
        with pytest.raises(ValueError):
            call()
    assert not two_devices


def test_top_lists_given_but_not_asked_for_are_refused(spkv, two_devices, monkeypatch):
    """(they would come back as they were)"""
    import torch
    monkeypatch.setattr(spkv, "_logprob_bytes", {(2, 50, 0): 16})
    x, f = drafts(0)["x"], drafts(0)["f"]
    for kw in (dict(top_ids=Rows((2, 5), torch.int32, 0, 4096)), dict(top_logp=Rows((2, 5), torch.float32, 0, 4096))):
        with pytest.raises(ValueError):
            spkv.spkv_token_logprobs(x, lse=f, want_entropy=False, **{"top_ids": Rows((2, 0), torch.int32, 0, 4096), **kw})
    assert not two_devices


def test_the_workspace_sizes_remembered_are_limited(spkv, two_devices, monkeypatch):
    import torch
    sizes = {}
    monkeypatch.setattr(spkv, "_logprob_bytes", sizes)
    monkeypatch.setattr(spkv, "_scratch", lambda store, n, d: Rows((n,), None, d, 4096))
    for n in range(1, 3000):
        spkv.spkv_token_logprobs(Rows((n, 50), torch.float32, 0, 4096), lse=Rows((n,), torch.float32, 0, 4096), want_entropy=False)
    assert 0 < len(sizes) <= 1024
