"""ctypes binding of libspkv.so: the same entry points as include/spkv.h.

Argument marshalling only -- every step of the path runs in the CUDA kernels of the
library.  PyTorch supplies device memory and streams.  There is no CPU fallback: if
the library cannot be loaded, importing this module raises.

Low level: ``lib()`` returns the ctypes handle with prototypes set; the ``spkv_*``
functions below mirror the C names and accept torch tensors.
High level: ``Cache`` owns an arena tensor and workspaces and forwards to them.
"""
from __future__ import annotations

import ctypes as C
import functools
import inspect
import math
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libspkv.so")

SPKV_OK = 0
ERRORS = {
    -1: "SPKV_E_INVALID", -2: "SPKV_E_ARENA_TOO_SMALL", -3: "SPKV_E_UNSUPPORTED", -4: "SPKV_E_CUDA",
    -5: "SPKV_E_POOL_EXHAUSTED", -6: "SPKV_E_CONTEXT_OVERFLOW", -7: "SPKV_E_WORKSPACE",
    -8: "SPKV_E_TIMEOUT", -9: "SPKV_E_BOUNDS", -10: "SPKV_E_SCRATCH_LIMIT", -11: "SPKV_E_ORDER_DECODE",
    -12: "SPKV_E_ORDER_APPEND", -13: "SPKV_E_BOUNDS_PAGE", -14: "SPKV_E_CANARY", -15: "SPKV_E_ATTACH", -16: "SPKV_E_FORK",
}


FLAG_OVERLAP = 1          # SPKV_FLAG_OVERLAP
FLAG_PREFILL_PV_BF16 = 2  # SPKV_FLAG_PREFILL_PV_BF16
FLAG_DEBUG_BOUNDS = 4      # SPKV_FLAG_DEBUG_BOUNDS
FLAG_FORK = 8              # SPKV_FLAG_FORK


class Config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("max_seqs", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("window", C.c_int32),
                ("page_tokens", C.c_int32), ("max_context", C.c_int32), ("pool_pages", C.c_int64),
                ("tau", C.c_float), ("flags", C.c_int32), ("sink_tokens", C.c_int32),
                ("h_local_only", C.c_void_p)]


class Predictor(C.Structure):
    _fields_ = [("kind", C.c_int32), ("d_in", C.c_int32), ("hidden", C.c_int32),
                ("reserved", C.c_int32), ("d_W1", C.c_void_p), ("d_b1", C.c_void_p),
                ("d_W2", C.c_void_p), ("d_b2", C.c_void_p)]


class Stats(C.Structure):
    _fields_ = [("units", C.c_int64), ("pairs_seen", C.c_int64), ("pairs_kept", C.c_int64),
                ("pairs_in_window", C.c_int64), ("pairs_evicted", C.c_int64),
                ("gates_open", C.c_int64), ("pages_in_use", C.c_int64), ("pages_free", C.c_int64),
                ("bytes_resident", C.c_int64), ("density_all", C.c_double),
                ("density_cache", C.c_double)]


BF16, F16, F32 = 0, 1, 2          # SPKV_BF16 / SPKV_F16 / SPKV_F32
_DTYPE = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}
NORM_Q, NORM_K = 1, 2             # SPKV_NORM_Q / SPKV_NORM_K
MAX_ROW_DIM, MAX_AXES = 256, 4    # SPKV_MAX_ROW_DIM / SPKV_MAX_AXES
MAX_DRAFT, MAX_TOP = 64, 32       # SPKV_MAX_DRAFT / SPKV_MAX_TOP


class Rows(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class Rope(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("n_axes", C.c_int32), ("scale", C.c_float),
                ("turn", C.c_uint64 * (MAX_ROW_DIM // 2)), ("axis", C.c_uint8 * (MAX_ROW_DIM // 2))]


class QkNorm(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("weight_dtype", C.c_int32), ("head_dim", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("norm", C.c_int32), ("eps", C.c_float), ("d_wq", C.c_void_p),
                ("d_wk", C.c_void_p)]


class SpkvError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {ERRORS.get(code, code)} ({lib().spkv_error_string(code).decode()})")


_lib = None


def lib():
    """Loads libspkv.so (fails loudly when it is missing) and declares prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} not found: build it with "
                          "`python -m paper_2605_14037_b200.build` (there is no fallback path)")
    l = C.CDLL(_LIB_PATH)
    vp, i32, sz, f32 = C.c_void_p, C.c_int32, C.c_size_t, C.c_float
    cfgp, pp = C.POINTER(Config), C.POINTER(Predictor)
    protos = {
        "spkv_arena_bytes": (C.c_int, [cfgp, C.POINTER(sz)]),
        "spkv_cache_create": (C.c_int, [cfgp, vp, sz, vp, C.POINTER(vp)]),
        "spkv_cache_attach": (C.c_int, [cfgp, vp, sz, vp, C.POINTER(vp)]),
        "spkv_cache_checkpoint_bytes": (sz, [vp]),
        "spkv_cache_checkpoint": (C.c_int, [vp, vp, sz, vp]),
        "spkv_cache_rollback": (C.c_int, [vp, vp, sz, vp]),
        "spkv_note_foreign_work": (C.c_int, [vp]),
        "spkv_safe_steps": (C.c_int, [vp, vp, i32, vp, C.POINTER(C.c_int64)]),
        "spkv_safe_steps_from_lengths": (C.c_int, [cfgp, vp, vp, C.c_int64, C.c_int64, C.POINTER(C.c_int64)]),
        "spkv_arena_canaries": (C.c_int, [cfgp, C.POINTER(sz), i32, C.POINTER(i32)]),
        "spkv_cache_destroy": (C.c_int, [vp]),
        "spkv_cache_reset_seq": (C.c_int, [vp, i32, vp]),
        "spkv_set_tau": (C.c_int, [vp, f32]),
        "spkv_set_head_tau": (C.c_int, [vp, i32, i32, f32, vp]),
        "spkv_score": (C.c_int, [vp, pp, vp, i32, vp, vp, vp]),
        "spkv_append_evict": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, vp]),
        "spkv_score_append_evict": (C.c_int, [vp, i32, pp, vp, i32, vp, vp, vp, vp, vp]),
        "spkv_decode_workspace_bytes": (sz, [cfgp, i32]),
        "spkv_decode_attention": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, f32, vp, sz, vp]),
        "spkv_stream_read": (C.c_int, [vp, sz, vp, vp, vp]),
        "spkv_wait_selftest": (C.c_int, [vp, C.c_longlong, vp, vp]),
        "spkv_decode_attention_f32": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, vp, f32, vp, sz, vp]),
        "spkv_decode_attention_static": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, f32, vp]),
        "spkv_seq_fork": (C.c_int, [vp, i32, vp, i32, vp]),
        "spkv_share_plan_bytes": (sz, [cfgp]),
        "spkv_share_plan": (C.c_int, [vp, vp, i32, vp, sz, vp]),
        "spkv_decode_shared_workspace_bytes": (sz, [cfgp, i32]),
        "spkv_decode_attention_shared": (C.c_int, [vp, i32, vp, i32, vp, vp, vp, f32, vp, sz, vp, sz, vp]),
        "spkv_decode_tree_workspace_bytes": (sz, [cfgp, i32, i32]),
        "spkv_decode_attention_tree": (C.c_int, [vp, i32, vp, i32, i32] + [vp] * 8 + [f32, vp, sz, vp]),
        "spkv_append_path": (C.c_int, [vp, i32, i32, vp, i32, i32, vp, vp, vp, C.c_int64, vp, C.c_int64, vp, vp]),
        "spkv_tree_accept": (C.c_int, [i32, i32] + [vp] * 8),
        "spkv_logprobs_workspace_bytes": (sz, [i32, i32, i32]),
        "spkv_token_logprobs": (C.c_int, [i32, i32, i32, vp, C.c_int64, f32, vp, i32, i32] + [vp] * 6 + [sz, vp]),
        "spkv_prefill_workspace_bytes": (sz, [cfgp, i32]),
        "spkv_prefill": (C.c_int, [vp, i32, i32, i32, vp, vp, vp, vp, vp, f32, vp, sz, vp]),
        "spkv_rope_init": (C.c_int, [vp, i32, i32, i32, f32, vp, vp]),
        "spkv_norm_rope": (C.c_int, [vp, vp, i32] + [vp] * 8),
        "spkv_norm_rope_workspace_bytes": (sz, [vp]),
        "spkv_norm_rope_backward": (C.c_int, [vp, vp, i32] + [vp] * 12 + [sz, vp]),
        "spkv_softgate_workspace_bytes": (sz, [i32, i32, i32]),
        "spkv_softgate_forward": (C.c_int, [i32, i32, i32, i32, vp, vp, vp, vp, f32, f32, f32, i32, vp, vp, vp, sz,
                                            vp, vp]),
        "spkv_decode_step_staging_bytes": (sz, [cfgp, i32, i32]),
        "spkv_decode_step_host": (C.c_int, [vp, i32, pp, vp, i32, vp, vp, vp, vp, vp, f32, vp, sz, vp]),
        "spkv_decode_step_host_flush": (C.c_int, [vp, vp]),
        "spkv_decode_stack_staging_bytes": (sz, [cfgp, i32, i32]),
        "spkv_decode_stack_host": (C.c_int, [vp, vp, vp, i32, vp, vp, vp, vp, vp, f32, vp, sz, vp]),
        "spkv_decode_stack_workspace_bytes": (sz, [cfgp, i32]),
        "spkv_decode_stack": (C.c_int, [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, f32, vp, sz, vp]),
        "spkv_status": (C.c_int, [vp, vp]),
        "spkv_clear_status": (C.c_int, [vp, vp]),
        "spkv_cache_stats": (C.c_int, [vp, vp, C.POINTER(Stats)]),
        "spkv_read_lengths": (C.c_int, [vp, i32, vp, vp, vp]),
        "spkv_read_kept": (C.c_int, [vp, i32, i32, i32, vp, vp, vp, i32, C.POINTER(i32), vp]),
        "spkv_read_window": (C.c_int, [vp, i32, i32, i32, vp, vp, vp, vp, C.POINTER(i32), vp]),
        "spkv_tau_logit": (f32, [vp]),
        "spkv_error_string": (C.c_char_p, [C.c_int]),
    }
    for name, (res, args) in protos.items():
        fn = getattr(l, name)
        fn.restype, fn.argtypes = res, args
    _lib = l
    return l


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on_device(dev, fn, *args):
    """fn(*args, dev's current stream) with `dev` current (the caller's current device is put back)"""
    if dev == _current_device():
        return fn(*args, _raw_stream(dev))
    with torch.cuda.device(dev):
        return fn(*args, _raw_stream(dev))


def _under(stream, dev, call, *args):
    """call(*args) with `stream` current: what the call allocates -- results, plan, workspace -- then comes from that
    stream's memory.  (A block of another stream's may still have work in flight there.)"""
    if stream.device_index != dev:
        raise ValueError("the stream is on another device than the call's tensors")
    with torch.cuda.stream(stream):
        return call(*args)


def _on_its_stream(call):
    """A call that allocates results or workspaces, with the stream given to it made current (see _under)."""
    at = list(inspect.signature(call).parameters).index("stream")

    @functools.wraps(call)
    def run(*args, **kw):
        stream = args[at] if len(args) > at else kw.get("stream")
        if stream is None:
            return call(*args, **kw)
        with torch.cuda.stream(stream):
            return call(*args, **kw)
    return run


_capturing = torch.cuda.is_current_stream_capturing


def _scratch(store, nbytes, dev):
    """Workspace of one call on `dev`'s current stream: kept in `store` per stream (calls on two streams may run at
    once), replaced when it is too small.  A call that is being captured gets one from its graph's memory pool, which
    no other graph and no eager call uses."""
    if dev != _current_device():
        with torch.cuda.device(dev):
            return _scratch(store, nbytes, dev)
    if _capturing():
        return torch.empty(nbytes, dtype=torch.uint8, device=f"cuda:{dev}")
    key = (dev, _raw_stream(dev))
    ws = store.get(key)
    if ws is None or ws.numel() < nbytes:
        ws = store[key] = torch.empty(nbytes, dtype=torch.uint8, device=f"cuda:{dev}")
    return ws


def _ptr(t, dtype=None):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensor, contiguous"
    if dtype is not None:
        assert t.dtype == dtype, (t.dtype, dtype)
    return C.c_void_p(t.data_ptr())


def _check(rc, where):
    if rc != SPKV_OK:
        raise SpkvError(rc, where)


def make_predictor(W1, b1, W2=None, b2=None) -> Predictor:
    """Linear predictor (W1 [Hkv,d_in], b1 [Hkv]) or two-layer perceptron
    (W1 [hidden,d_in], b1 [hidden], W2 [Hkv,hidden], b2 [Hkv]); bf16 weights, f32 biases."""
    p = Predictor()
    p.kind = 0 if W2 is None else 1
    p.d_in = W1.shape[1]
    p.hidden = 0 if W2 is None else W1.shape[0]
    p.d_W1, p.d_b1 = _ptr(W1, torch.bfloat16), _ptr(b1, torch.float32)
    p.d_W2 = _ptr(W2, torch.bfloat16) if W2 is not None else None
    p.d_b2 = _ptr(b2, torch.float32) if b2 is not None else None
    p._keep = (W1, b1, W2, b2)
    return p


class Cache:
    """An SP-KV cache inside one torch-owned arena tensor, plus the workspaces the
    attention calls need.  Methods carry the names of the C entry points."""

    def __init__(self, n_layers, max_seqs, n_q_heads, n_kv_heads, max_context, pool_pages,
                 window=128, tau=0.5, device="cuda:0", head_dim=128, page_tokens=64, sink_tokens=0,
                 flags=0, local_only=None):
        """local_only: optional [n_layers, n_kv_heads] array, non-zero = that head is declared
        local-only (window attention, no page table, not scored by the fused append)."""
        import numpy as np
        self._local_only = None
        if local_only is not None:
            self._local_only = np.ascontiguousarray(np.asarray(local_only) != 0, dtype=np.uint8)
            assert self._local_only.shape == (n_layers, n_kv_heads)
        self.cfg = Config(n_layers, max_seqs, n_q_heads, n_kv_heads, head_dim, window, page_tokens,
                          max_context, pool_pages, tau, flags, sink_tokens,
                          self._local_only.ctypes.data if self._local_only is not None else None)
        self.device = torch.device(device)
        n = C.c_size_t()
        _check(lib().spkv_arena_bytes(C.byref(self.cfg), C.byref(n)), "spkv_arena_bytes")
        self.arena_bytes = n.value
        with torch.cuda.device(self.device):
            self.arena = torch.empty(self.arena_bytes, dtype=torch.uint8, device=self.device)
            h = C.c_void_p()
            _check(lib().spkv_cache_create(C.byref(self.cfg), _ptr(self.arena), self.arena_bytes,
                                           _stream(), C.byref(h)), "spkv_cache_create")
        self._h = h
        self._ws, self._shared_ws, self._shared_bytes, self._tree_ws, self._tree_bytes = {}, {}, {}, {}, {}
        self.G = n_q_heads // n_kv_heads
        self.default_scale = 1.0 / math.sqrt(head_dim)

    @classmethod
    def attach(cls, arena, cfg, tau=None, flags=None, local_only=None):
        """A Cache over an arena tensor that already holds one (a copy of another cache's arena):
        spkv_cache_attach.  `cfg` is the Config the arena was created with; tau / flags override;
        local_only as at creation (it is part of the layout and has to be given again)."""
        import numpy as np
        self = cls.__new__(cls)
        self.cfg = Config.from_buffer_copy(cfg)
        self._local_only = None
        if local_only is not None:
            self._local_only = np.ascontiguousarray(np.asarray(local_only) != 0, dtype=np.uint8)
            assert self._local_only.shape == (cfg.n_layers, cfg.n_kv_heads)
        self.cfg.h_local_only = self._local_only.ctypes.data if self._local_only is not None else None
        if tau is not None:
            self.cfg.tau = tau
        if flags is not None:
            self.cfg.flags = flags
        self.device = arena.device
        self.arena, self.arena_bytes = arena, arena.numel()
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().spkv_cache_attach(C.byref(self.cfg), _ptr(arena), arena.numel(), _stream(), C.byref(h)),
                   "spkv_cache_attach")
        self._h, self._ws, self._shared_ws, self._shared_bytes, self._tree_ws, self._tree_bytes = h, {}, {}, {}, {}, {}
        self.G = self.cfg.n_q_heads // self.cfg.n_kv_heads
        self.default_scale = 1.0 / math.sqrt(self.cfg.head_dim)
        return self

    @_on_its_stream
    def spkv_cache_checkpoint(self, buf=None, stream=None):
        """Saves metadata + ring pages into `buf` (allocated when None); returns the buffer."""
        n = lib().spkv_cache_checkpoint_bytes(self._h)
        if buf is None:
            buf = torch.empty(n, dtype=torch.uint8, device=self.device)
        _check(lib().spkv_cache_checkpoint(self._h, _ptr(buf), buf.numel(), _stream(stream)), "spkv_cache_checkpoint")
        return buf

    def spkv_cache_rollback(self, buf, stream=None):
        _check(lib().spkv_cache_rollback(self._h, _ptr(buf), buf.numel(), _stream(stream)), "spkv_cache_rollback")

    def spkv_note_foreign_work(self):
        _check(lib().spkv_note_foreign_work(self._h), "spkv_note_foreign_work")

    def spkv_safe_steps(self, seq_ids=None, stream=None) -> int:
        """Decode steps the listed sequences (host ints; None = all) can take before the pool or a
        page table could run out, every evicted pair assumed kept."""
        import numpy as np
        ids = np.ascontiguousarray(np.asarray([] if seq_ids is None else seq_ids, dtype=np.int32))
        out = C.c_int64()
        _check(lib().spkv_safe_steps(self._h, ids.ctypes.data if ids.size else None, int(ids.size),
                                     _stream(stream), C.byref(out)), "spkv_safe_steps")
        return int(out.value)

    def close(self):
        if getattr(self, "_h", None):
            lib().spkv_cache_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- workspaces (zero-filled once, as the C interface asks) -----------------------
    def _workspace(self, kind, nbytes):
        ws = self._ws.get(kind)
        if ws is None or ws.numel() < nbytes:
            ws = torch.zeros(max(nbytes, 256), dtype=torch.uint8, device=self.device)
            self._ws[kind] = ws
        return ws

    def decode_workspace(self, B):
        return self._workspace("decode", lib().spkv_decode_workspace_bytes(C.byref(self.cfg), B))

    # -- hot path -----------------------------------------------------------------------
    @_on_its_stream
    def spkv_score(self, pred, x, logits=None, flags=None, stream=None):
        n_tok = x.shape[0]
        if logits is None:
            logits = torch.empty((n_tok, self.cfg.n_kv_heads), dtype=torch.float32, device=x.device)
        _check(lib().spkv_score(self._h, C.byref(pred), _ptr(x, torch.bfloat16), n_tok,
                                _ptr(logits, torch.float32), _ptr(flags, torch.uint8),
                                _stream(stream)), "spkv_score")
        return logits

    def spkv_append_evict(self, layer, seq_ids, k, v, logits, stream=None):
        _check(lib().spkv_append_evict(self._h, layer, _ptr(seq_ids, torch.int32), seq_ids.numel(),
                                       _ptr(k, torch.bfloat16), _ptr(v, torch.bfloat16),
                                       _ptr(logits, torch.float32), _stream(stream)),
               "spkv_append_evict")

    def spkv_score_append_evict(self, layer, pred, seq_ids, x, k, v, logits_out=None, stream=None):
        _check(lib().spkv_score_append_evict(
            self._h, layer, C.byref(pred), _ptr(seq_ids, torch.int32), seq_ids.numel(),
            _ptr(x, torch.bfloat16), _ptr(k, torch.bfloat16), _ptr(v, torch.bfloat16),
            _ptr(logits_out, torch.float32), _stream(stream)), "spkv_score_append_evict")

    @_on_its_stream
    def spkv_decode_attention(self, layer, seq_ids, q, out=None, lse=None, sm_scale=None,
                              stream=None):
        B = seq_ids.numel()
        if out is None:
            out = torch.empty_like(q)
        ws = self.decode_workspace(B)
        _check(lib().spkv_decode_attention(
            self._h, layer, _ptr(seq_ids, torch.int32), B, _ptr(q, torch.bfloat16),
            _ptr(out, torch.bfloat16), _ptr(lse, torch.float32),
            self.default_scale if sm_scale is None else sm_scale, _ptr(ws), ws.numel(),
            _stream(stream)), "spkv_decode_attention")
        return out

    @_on_its_stream
    def spkv_decode_attention_f32(self, layer, seq_ids, q, out=None, out_f32=None, lse=None, sm_scale=None,
                                  stream=None):
        """spkv_decode_attention that also returns the rows before their rounding to bf16;
        returns (out bf16, out float32)."""
        B = seq_ids.numel()
        if out is None:
            out = torch.empty_like(q)
        if out_f32 is None:
            out_f32 = torch.empty(q.shape, dtype=torch.float32, device=q.device)
        ws = self.decode_workspace(B)
        _check(lib().spkv_decode_attention_f32(
            self._h, layer, _ptr(seq_ids, torch.int32), B, _ptr(q, torch.bfloat16),
            _ptr(out, torch.bfloat16), _ptr(out_f32, torch.float32), _ptr(lse, torch.float32),
            self.default_scale if sm_scale is None else sm_scale, _ptr(ws), ws.numel(),
            _stream(stream)), "spkv_decode_attention_f32")
        return out, out_f32

    @_on_its_stream
    def spkv_decode_attention_static(self, layer, seq_ids, q, out=None, lse=None, sm_scale=None,
                                     stream=None):
        """Same result as spkv_decode_attention, for callers that may not allocate device
        memory: the scratch is a fixed array inside the library (no workspace tensor)."""
        B = seq_ids.numel()
        if out is None:
            out = torch.empty_like(q)
        _check(lib().spkv_decode_attention_static(
            self._h, layer, _ptr(seq_ids, torch.int32), B, _ptr(q, torch.bfloat16),
            _ptr(out, torch.bfloat16), _ptr(lse, torch.float32),
            self.default_scale if sm_scale is None else sm_scale, _stream(stream)),
            "spkv_decode_attention_static")
        return out

    def spkv_share_plan(self, seq_ids, plan=None, stream=None):
        """The plan a batch with a common prefix decodes by (a device tensor; one for all layers and steps of
        the same sequences)."""
        dev = self.arena.get_device()
        if stream is not None:
            return _under(stream, dev, self.spkv_share_plan, seq_ids, plan)
        if plan is None:
            plan = torch.empty(lib().spkv_share_plan_bytes(C.byref(self.cfg)), dtype=torch.uint8, device=f"cuda:{dev}")
        if seq_ids.get_device() != dev or plan.get_device() != dev:
            raise ValueError("all tensors of a call live on the cache's device")
        _check(_on_device(dev, lib().spkv_share_plan, self._h, _ptr(seq_ids, torch.int32), seq_ids.numel(),
                          _ptr(plan, torch.uint8), plan.numel()), "spkv_share_plan")
        return plan

    def spkv_decode_attention_shared(self, layer, seq_ids, q, plan, out=None, lse=None, sm_scale=None, want_lse=False,
                                     stream=None):
        """spkv_decode_attention with the pages that all sequences have in common read once for the batch.
        Returns out, or (out, lse) with want_lse."""
        B, cfg = seq_ids.shape[0], self.cfg
        shape = (B, cfg.n_q_heads, cfg.head_dim)
        dev = q.get_device()
        if stream is not None:
            return _under(stream, dev, self.spkv_decode_attention_shared, layer, seq_ids, q, plan, out, lse, sm_scale, want_lse)

        def check(t, dtype, want):
            if t.dtype is not dtype or t.shape != want or t.get_device() != dev or not t.is_contiguous():
                raise ValueError(f"expected a contiguous {dtype} tensor {tuple(want)} on the cache's device, got "
                                 f"{t.dtype} {tuple(t.shape)} on {t.device}")

        check(q, torch.bfloat16, shape)
        check(seq_ids, torch.int32, (B,))
        check(plan, torch.uint8, plan.shape)
        if out is None:
            out = torch.empty_like(q)
        else:
            check(out, torch.bfloat16, shape)
        if lse is not None:
            check(lse, torch.float32, shape[:2])
        elif want_lse:
            lse = q.new_empty(B, cfg.n_q_heads, dtype=torch.float32)
        if dev < 0 or dev != self.arena.get_device():
            raise ValueError("all tensors of a call live on the cache's device")
        nbytes = self._shared_bytes.get(B)
        if nbytes is None:
            nbytes = self._shared_bytes[B] = lib().spkv_decode_shared_workspace_bytes(C.byref(cfg), B)
        ws = _scratch(self._shared_ws, nbytes, dev)
        rc = _on_device(dev, lib().spkv_decode_attention_shared, self._h, layer, seq_ids.data_ptr(), B, q.data_ptr(),
                        out.data_ptr(), None if lse is None else lse.data_ptr(),
                        self.default_scale if sm_scale is None else sm_scale, plan.data_ptr(), plan.numel(), ws.data_ptr(),
                        ws.numel())
        if rc:
            raise SpkvError(rc, "spkv_decode_attention_shared")
        return (out, lse) if want_lse else out

    def spkv_decode_attention_tree(self, layer, seq_ids, q, k, v, parent=None, n_nodes=None, logits=None, out=None, lse=None,
                                   sm_scale=None, want_lse=False, stream=None):
        """Attention of drafted nodes over the cache and their ancestors.  q [B, T, n_q_heads, 128], k, v
        [B, T, n_kv_heads, 128] (views of one fused projection too), parent [B, T] int32 (None: chains), n_nodes
        [B] int32 (None: T each), logits [B, T, n_kv_heads] (may be None while T <= window).  Returns out
        [B, T, n_q_heads, 128], or (out, lse) with want_lse."""
        dev = q.get_device()
        if stream is not None:
            return _under(stream, dev, self.spkv_decode_attention_tree, layer, seq_ids, q, k, v, parent, n_nodes, logits, out,
                          lse, sm_scale, want_lse)
        cfg = self.cfg
        B, T = q.shape[0], q.shape[1]
        hq, hkv = cfg.n_q_heads, cfg.n_kv_heads
        if dev < 0 or dev != self.arena.get_device():
            raise ValueError("all tensors of a call live on the cache's device")
        rows = (Rows * 3)()
        _THREE_ROWS.pack_into(rows, 0, *_draft_rows(q, B, T, hq, dev, "q"), *_draft_rows(k, B, T, hkv, dev, "k"),
                              *_draft_rows(v, B, T, hkv, dev, "v"))
        at = C.addressof(rows)
        ptrs = (_dense(seq_ids, torch.int32, (B,), dev), _dense(n_nodes, torch.int32, (B,), dev),
                _dense(parent, torch.int32, (B, T), dev), _dense(logits, torch.float32, (B, T, hkv), dev))
        out, at_out = _result(q, out, torch.bfloat16, (B, T, hq, 128), dev)
        at_lse = None
        if lse is not None or want_lse:
            lse, at_lse = _result(q, lse, torch.float32, (B, T, hq), dev)
        nbytes = self._tree_bytes.get((B, T))
        if nbytes is None:
            nbytes = self._tree_bytes[B, T] = max(256, lib().spkv_decode_tree_workspace_bytes(C.byref(cfg), B, T))
        ws = _scratch(self._tree_ws, nbytes, dev)
        rc = _on_device(dev, lib().spkv_decode_attention_tree, self._h, layer, ptrs[0], B, T, ptrs[1], ptrs[2], at, at + _ROW,
                        at + 2 * _ROW, ptrs[3], at_out, at_lse, self.default_scale if sm_scale is None else sm_scale,
                        ws.data_ptr(), ws.numel())
        if rc:
            raise SpkvError(rc, "spkv_decode_attention_tree")
        return (out, lse) if want_lse else out

    def spkv_append_path(self, layer0, seq_ids, k, v, logits, path=None, n_path=None, stream=None):
        """Appends n_path[b] nodes path[b] (None: 0, 1, 2, ...) of every sequence: k, v [B, T, n_kv_heads, 128] and logits
        [B, T, n_kv_heads] of layer0, or [n, B, T, ...] of n layers from layer0 on."""
        dev = k.get_device()
        if stream is not None:
            return _under(stream, dev, self.spkv_append_path, layer0, seq_ids, k, v, logits, path, n_path)
        if dev < 0 or dev != self.arena.get_device():
            raise ValueError("all tensors of a call live on the cache's device")
        hkv = self.cfg.n_kv_heads
        n = 1
        strides = (0, 0)
        if k.dim() == 5:
            n = k.shape[0]
            if v.dim() != 5 or v.shape[0] != n or logits.dim() != 4 or logits.shape[0] != n:
                raise ValueError("k, v and logits of several layers: [n, B, T, ...] each")
            if n > 1:
                strides = (k.stride(0), v.stride(0))
            if n == 0:
                return
            k, v = k[0], v[0]
        elif logits.dim() != 3:
            raise ValueError("k, v and logits of one layer: [B, T, ...] each")
        B, T = k.shape[0], k.shape[1]
        rows = (Rows * 2)()
        _TWO_ROWS.pack_into(rows, 0, *_draft_rows(k, B, T, hkv, dev, "k"), *_draft_rows(v, B, T, hkv, dev, "v"))
        at = C.addressof(rows)
        lg = _dense(logits, torch.float32, (n, B, T, hkv) if logits.dim() == 4 else (B, T, hkv), dev)
        _check(_on_device(dev, lib().spkv_append_path, self._h, layer0, n, _dense(seq_ids, torch.int32, (B,), dev), B, T,
                          _dense(path, torch.int32, (B, T), dev), _dense(n_path, torch.int32, (B,), dev), at, strides[0],
                          at + _ROW, strides[1], lg), "spkv_append_path")

    @_on_its_stream
    def spkv_prefill(self, layer, seq, k, v, logits, q=None, out=None, sm_scale=None, stream=None):
        Cn = k.shape[0]
        if q is not None and out is None:
            out = torch.empty_like(q)
        ws = self._workspace("prefill", lib().spkv_prefill_workspace_bytes(C.byref(self.cfg), Cn))
        _check(lib().spkv_prefill(
            self._h, layer, seq, Cn, _ptr(q, torch.bfloat16), _ptr(k, torch.bfloat16),
            _ptr(v, torch.bfloat16), _ptr(logits, torch.float32), _ptr(out, torch.bfloat16),
            self.default_scale if sm_scale is None else sm_scale, _ptr(ws), ws.numel(),
            _stream(stream)), "spkv_prefill")
        return out

    @_on_its_stream
    def spkv_decode_step_host(self, layer, pred, seq_ids, h_x, h_q, h_k, h_v, h_out, sm_scale=None,
                              stream=None):
        """Host (pinned) tensors in, host tensor out; enqueues the copies (on the cache's own
        copy streams) and the kernels.  h_out is complete after spkv_decode_step_host_flush()
        and a synchronisation of the stream."""
        B = seq_ids.numel()
        nbytes = lib().spkv_decode_step_staging_bytes(C.byref(self.cfg), B, pred.d_in)
        old = self._ws.get("staging")
        if old is not None and old.numel() < nbytes:   # growing: drain the pipeline that uses the old one
            self.spkv_decode_step_host_flush(stream)
            torch.cuda.synchronize(self.device)
        st = self._workspace("staging", nbytes)
        for t in (h_x, h_q, h_k, h_v, h_out):
            assert not t.is_cuda and t.is_contiguous() and t.dtype == torch.bfloat16
        _check(lib().spkv_decode_step_host(
            self._h, layer, C.byref(pred), _ptr(seq_ids, torch.int32), B,
            C.c_void_p(h_x.data_ptr()), C.c_void_p(h_q.data_ptr()), C.c_void_p(h_k.data_ptr()),
            C.c_void_p(h_v.data_ptr()), C.c_void_p(h_out.data_ptr()),
            self.default_scale if sm_scale is None else sm_scale, _ptr(st), st.numel(),
            _stream(stream)), "spkv_decode_step_host")

    @_on_its_stream
    def spkv_decode_stack(self, preds, seq_ids, x, q, k, v, out=None, logits_out=None, lse=None, sm_scale=None,
                          stream=None):
        """One decode step of all layers from device tensors [L, B, ...]: the appends of every layer in
        one launch, decode attention of every layer in one persistent launch."""
        B, L = seq_ids.numel(), self.cfg.n_layers
        assert len(preds) == L and q.shape[0] == L
        arr = (Predictor * L)(*preds)
        if out is None:
            out = torch.empty_like(q)
        ws = self._workspace("decode_stack", lib().spkv_decode_stack_workspace_bytes(C.byref(self.cfg), B))
        _check(lib().spkv_decode_stack(
            self._h, C.cast(arr, C.c_void_p), _ptr(seq_ids, torch.int32), B, _ptr(x, torch.bfloat16),
            _ptr(q, torch.bfloat16), _ptr(k, torch.bfloat16), _ptr(v, torch.bfloat16), _ptr(out, torch.bfloat16),
            _ptr(logits_out, torch.float32), _ptr(lse, torch.float32),
            self.default_scale if sm_scale is None else sm_scale, _ptr(ws), ws.numel(), _stream(stream)),
            "spkv_decode_stack")
        return out

    @_on_its_stream
    def spkv_decode_stack_host(self, preds, seq_ids, h_x, h_q, h_k, h_v, h_out, sm_scale=None, stream=None):
        """One decode step of all layers from host (pinned) tensors [L, B, ...]; enqueues four
        copies in, the 2 L kernels and one copy out on the stream."""
        B, L = seq_ids.numel(), self.cfg.n_layers
        assert len(preds) == L
        arr = (Predictor * L)(*preds)
        nbytes = lib().spkv_decode_stack_staging_bytes(C.byref(self.cfg), B, preds[0].d_in)
        st = self._workspace("stack_staging", nbytes)
        for t in (h_x, h_q, h_k, h_v, h_out):
            assert not t.is_cuda and t.is_contiguous() and t.dtype == torch.bfloat16 and t.shape[0] == L
        _check(lib().spkv_decode_stack_host(
            self._h, C.cast(arr, C.c_void_p), _ptr(seq_ids, torch.int32), B,
            C.c_void_p(h_x.data_ptr()), C.c_void_p(h_q.data_ptr()), C.c_void_p(h_k.data_ptr()),
            C.c_void_p(h_v.data_ptr()), C.c_void_p(h_out.data_ptr()),
            self.default_scale if sm_scale is None else sm_scale, _ptr(st), st.numel(),
            _stream(stream)), "spkv_decode_stack_host")

    def spkv_decode_step_host_flush(self, stream=None):
        """Makes the stream wait for the output copy of the last spkv_decode_step_host call."""
        _check(lib().spkv_decode_step_host_flush(self._h, _stream(stream)), "spkv_decode_step_host_flush")

    # -- maintenance / introspection ---------------------------------------------------
    def spkv_cache_reset_seq(self, seq, stream=None):
        _check(lib().spkv_cache_reset_seq(self._h, seq, _stream(stream)), "spkv_cache_reset_seq")

    def spkv_seq_fork(self, src, dst, stream=None):
        """Makes the empty sequences `dst` (host ints) continuations of sequence src (FLAG_FORK caches)."""
        import numpy as np
        dev = self.arena.get_device()
        if stream is not None:
            return _under(stream, dev, self.spkv_seq_fork, src, dst)
        ids = np.ascontiguousarray(np.asarray(list(dst), dtype=np.int32))
        _check(_on_device(dev, lib().spkv_seq_fork, self._h, int(src), ids.ctypes.data if ids.size else None, int(ids.size)),
               "spkv_seq_fork")

    def spkv_set_tau(self, tau):
        _check(lib().spkv_set_tau(self._h, tau), "spkv_set_tau")

    def spkv_set_head_tau(self, layer, kv_head, tau, stream=None):
        """Threshold of one (layer, KV head) (kv_head = -1: the whole layer); NaN clears it."""
        _check(lib().spkv_set_head_tau(self._h, layer, kv_head, tau, _stream(stream)), "spkv_set_head_tau")

    def spkv_tau_logit(self) -> float:
        return float(lib().spkv_tau_logit(self._h))

    def spkv_status(self, stream=None) -> int:
        return int(lib().spkv_status(self._h, _stream(stream)))

    def spkv_clear_status(self, stream=None):
        _check(lib().spkv_clear_status(self._h, _stream(stream)), "spkv_clear_status")

    def check(self):
        _check(self.spkv_status(), "device status")

    def spkv_cache_stats(self, stream=None) -> Stats:
        s = Stats()
        _check(lib().spkv_cache_stats(self._h, _stream(stream), C.byref(s)), "spkv_cache_stats")
        return s

    def spkv_read_lengths(self, layer, stream=None):
        import numpy as np
        shape = (self.cfg.max_seqs, self.cfg.n_kv_heads)
        ln, t = np.empty(shape, np.int32), np.empty(shape, np.int32)
        _check(lib().spkv_read_lengths(self._h, layer, ln.ctypes.data, t.ctypes.data,
                                       _stream(stream)), "spkv_read_lengths")
        return ln, t

    def spkv_read_kept(self, layer, seq, kvh, stream=None):
        """(positions int32 [n], K bits uint16 [n,128], V bits uint16 [n,128])"""
        import numpy as np
        n = C.c_int32()
        _check(lib().spkv_read_kept(self._h, layer, seq, kvh, None, None, None, 0, C.byref(n),
                                    _stream(stream)), "spkv_read_kept")
        cap = n.value
        pos = np.empty(cap, np.int32)
        k = np.empty((cap, 128), np.uint16)
        v = np.empty((cap, 128), np.uint16)
        _check(lib().spkv_read_kept(self._h, layer, seq, kvh, pos.ctypes.data, k.ctypes.data,
                                    v.ctypes.data, cap, C.byref(n), _stream(stream)),
               "spkv_read_kept")
        return pos, k, v

    def spkv_read_window(self, layer, seq, kvh, stream=None):
        """(positions [n], K bits [n,128], V bits [n,128], logits f32 [n]), ascending position"""
        import numpy as np
        w = self.cfg.window
        pos = np.empty(w, np.int32)
        k = np.empty((w, 128), np.uint16)
        v = np.empty((w, 128), np.uint16)
        lg = np.empty(w, np.float32)
        n = C.c_int32()
        _check(lib().spkv_read_window(self._h, layer, seq, kvh, pos.ctypes.data, k.ctypes.data,
                                      v.ctypes.data, lg.ctypes.data, C.byref(n), _stream(stream)),
               "spkv_read_window")
        n = n.value
        return pos[:n], k[:n], v[:n], lg[:n]


@_on_its_stream
def spkv_stream_read(buf, passes=5, stream=None):
    """Read-only HBM rate in GB/s: streams the uint8 tensor `buf` through spkv_stream_read
    `passes` times (after one warm-up pass), timed with CUDA events on the launching stream."""
    sink = torch.zeros(2, dtype=torch.int64, device=buf.device)   # checksum, page counter
    status = torch.zeros(1, dtype=torch.int32, device=buf.device)
    nbytes = buf.numel() // 32768 * 32768
    call = lambda: _check(lib().spkv_stream_read(_ptr(buf), nbytes, _ptr(sink), _ptr(status), _stream(stream)),
                          "spkv_stream_read")
    call()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(passes):
        call()
    e1.record()
    e1.synchronize()
    if int(status.item()) != 0:
        raise SpkvError(int(status.item()), "spkv_stream_read")
    return nbytes * passes / (e0.elapsed_time(e1) * 1e-3) / 1e9


class NormRope:
    """Descriptor of an attention layer's per-head norm and position rotation (make_norm_rope)."""

    def __init__(self, norm, rope, dtype, keep):
        self.norm, self.rope, self.dtype, self._keep = norm, rope, dtype, keep
        self._n, self._r = C.addressof(norm), C.addressof(rope)
        self.heads, self.head_dim, self.n_axes = (norm.n_q_heads, norm.n_kv_heads), norm.head_dim, rope.n_axes
        self.weights_on = next((w.get_device() for w in keep if w is not None), None)
        self.forward, self.backward = lib().spkv_norm_rope, lib().spkv_norm_rope_backward
        self.workspace_bytes = lib().spkv_norm_rope_workspace_bytes(self._n)
        self._ws = {}


def make_norm_rope(n_q_heads, n_kv_heads, head_dim=128, dtype=torch.bfloat16, wq=None, wk=None, norm=True, eps=1e-6,
                   rot_dim=None, theta=10000.0, inv_freq=None, axis=None, n_axes=1, interleaved=False, scale=1.0):
    """norm: True (queries and keys), False, "q" or "k"; wq, wk [head_dim] device tensors of one type or None
    (ones), read at every call.  inv_freq [rot_dim / 2] (default theta^(-2 i / rot_dim)) and axis
    [rot_dim / 2] (the position axis of each pair) are host sequences."""
    import numpy as np
    rot_dim = head_dim if rot_dim is None else rot_dim
    inv = np.ascontiguousarray(theta ** (-np.arange(rot_dim // 2) * 2.0 / max(rot_dim, 1)) if inv_freq is None
                               else inv_freq, dtype=np.float64)
    ax = None if axis is None else np.ascontiguousarray(axis, dtype=np.uint8)
    if inv.shape != (rot_dim // 2,) or (ax is not None and ax.shape != inv.shape):
        raise ValueError("inv_freq and axis take one entry per rotated pair")
    rope = Rope()
    _check(lib().spkv_rope_init(C.addressof(rope), rot_dim, int(bool(interleaved)), n_axes, scale, inv.ctypes.data,
                                None if ax is None else ax.ctypes.data), "spkv_rope_init")
    for w in (wq, wk):
        if w is not None and (w.shape != (head_dim,) or (wq is not None and w.dtype != wq.dtype)):
            raise ValueError("norm weights are [head_dim] tensors of one type")
    if wq is not None and wk is not None and wq.device != wk.device:
        raise ValueError("norm weights live on one device")
    wd = next((w.dtype for w in (wq, wk) if w is not None), torch.float32)
    which = {True: NORM_Q | NORM_K, False: 0, "q": NORM_Q, "k": NORM_K}[norm]
    d = QkNorm(_DTYPE[dtype], _DTYPE[wd], head_dim, n_q_heads, n_kv_heads, which, eps, _ptr(wq), _ptr(wk))
    return NormRope(d, rope, dtype, (wq, wk))


# The row calls are made once per layer and token batch, often for a handful of rows: what the binding does
# around the launch is kept to a few microseconds (one check per tensor, all views packed at once).
_TWO_ROWS, _THREE_ROWS, _SIX_ROWS, _EIGHT_ROWS = (struct.Struct("Qqq" * n) for n in (2, 3, 6, 8))
_ROW = C.sizeof(Rows)


def _row(nr, t, heads, n, dev, what):
    """(pointer, token stride, head stride) of a [n, heads, head_dim] tensor of any token and head stride."""
    D = nr.head_dim
    if t.dtype is not nr.dtype or t.shape != (n, heads, D):
        raise ValueError(f"{what}: expected {nr.dtype} [{n}, {heads}, {D}], got {t.dtype} {tuple(t.shape)}")
    if t.get_device() != dev:
        raise ValueError("all tensors of a call live on one device")
    st = t.stride()
    if st[2] != 1 or dev < 0:
        raise ValueError(f"{what}: a device tensor whose rows are contiguous")
    return t.data_ptr(), st[0] if n > 1 else 0, st[1] if heads > 1 else 0   # (the stride of a single entry says nothing)


def _row_out(nr, like, t, heads, n, dev, what):
    """(tensor, its row view) of a result: the caller's, or a contiguous one made here"""
    if t is not None:
        return t, _row(nr, t, heads, n, dev, what)
    D = nr.head_dim
    t = like.new_empty(n, heads, D)   # (separate sizes: 0.4 us less than a tuple)
    return t, (t.data_ptr(), heads * D, D)


def _draft_rows(t, B, T, heads, dev, what):
    """(pointer, token stride, head stride) of a bf16 [B, T, heads, 128] tensor whose tokens b T + i are evenly spaced"""
    if t.dtype is not torch.bfloat16 or t.shape != (B, T, heads, 128):
        raise ValueError(f"{what}: expected bfloat16 [{B}, {T}, {heads}, 128], got {t.dtype} {tuple(t.shape)}")
    if t.get_device() != dev:
        raise ValueError("all tensors of a call live on one device")
    st = t.stride()
    tok = st[1] if T > 1 else st[0] if B > 1 else 0
    if st[3] != 1 or (B > 1 and T > 1 and st[0] != T * tok):
        raise ValueError(f"{what}: rows are contiguous and tokens evenly spaced")
    return t.data_ptr(), tok, st[2] if heads > 1 else 0


def _dense(t, dtype, shape, dev):
    """Pointer of a contiguous tensor of this type, shape and device (None: null)"""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"expected a contiguous {dtype} tensor {tuple(shape)} on device {dev}, got {t.dtype} {tuple(t.shape)} "
                         f"on {t.device}")
    return t.data_ptr()


def _result(like, t, dtype, shape, dev):
    """(tensor, its pointer) of a result: the caller's, or one made here"""
    if t is None:
        t = like.new_empty(shape, dtype=dtype)
        return t, t.data_ptr()
    return t, _dense(t, dtype, shape, dev)


def _positions(nr, pos, dev):
    """(n_tok, pointer) of an int32 [n_tok] or [n_axes, n_tok] device tensor"""
    n = pos.shape[-1]
    if pos.dtype is not torch.int32 or not pos.is_contiguous() or pos.numel() != nr.n_axes * n:
        raise ValueError(f"positions: contiguous int32 [{nr.n_axes}, n_tok] on the device")
    if pos.get_device() != dev or (nr.weights_on is not None and nr.weights_on != dev):
        raise ValueError("all tensors of a call live on one device")
    return n, pos.data_ptr()


def spkv_norm_rope(nr, positions, q, k, v=None, q_out=None, k_out=None, v_out=None, stream=None):
    """Norm + rotation of q [n_tok, n_q_heads, head_dim] and k [n_tok, n_kv_heads, head_dim] (any strides;
    e.g. views of one fused projection), v handed on.  Returns (q_out, k_out, v_out), contiguous
    tensors unless given; v_out is None without v."""
    dev = q.get_device()
    if stream is not None:
        return _under(stream, dev, spkv_norm_rope, nr, positions, q, k, v, q_out, k_out, v_out)
    n, pos = _positions(nr, positions, dev)
    hq, hkv = nr.heads
    rq, rk = _row(nr, q, hq, n, dev, "q"), _row(nr, k, hkv, n, dev, "k")
    q_out, oq = _row_out(nr, q, q_out, hq, n, dev, "q_out")
    k_out, ok = _row_out(nr, q, k_out, hkv, n, dev, "k_out")
    io = (Rows * 6)()
    at = C.addressof(io)
    if v is None:
        v_out = None
        _SIX_ROWS.pack_into(io, 0, *rq, *rk, 0, 0, 0, *oq, *ok, 0, 0, 0)
        av = av_out = None
    else:
        v_out, ov = _row_out(nr, q, v_out, hkv, n, dev, "v_out")
        _SIX_ROWS.pack_into(io, 0, *rq, *rk, *_row(nr, v, hkv, n, dev, "v"), *oq, *ok, *ov)
        av, av_out = at + 2 * _ROW, at + 5 * _ROW
    rc = _on_device(dev, nr.forward, nr._n, nr._r, n, pos, at, at + _ROW, av, at + 3 * _ROW, at + 4 * _ROW, av_out)
    if rc:
        raise SpkvError(rc, "spkv_norm_rope")
    return q_out, k_out, v_out


def spkv_norm_rope_backward(nr, positions, q, k, q_grad, k_grad, v_grad=None, dq=None, dk=None, dv=None,
                            weight_grads=True, stream=None):
    """Gradients of spkv_norm_rope: q, k its input rows (None for a side without norm), q_grad, k_grad,
    v_grad those of its outputs.  Returns (dq, dk, dv, dwq, dwk); dwq, dwk float32, None for a
    side without norm or weight_grads=False; dv None without v_grad."""
    dev = q_grad.get_device()
    if stream is not None:
        return _under(stream, dev, spkv_norm_rope_backward, nr, positions, q, k, q_grad, k_grad, v_grad, dq, dk, dv, weight_grads)
    n, pos = _positions(nr, positions, dev)
    (hq, hkv), D, normed = nr.heads, nr.head_dim, nr.norm.norm
    none = (0, 0, 0)
    xq = _row(nr, q, hq, n, dev, "q") if normed & NORM_Q else none
    xk = _row(nr, k, hkv, n, dev, "k") if normed & NORM_K else none
    gq, gk = _row(nr, q_grad, hq, n, dev, "q_grad"), _row(nr, k_grad, hkv, n, dev, "k_grad")
    dq, yq = _row_out(nr, q_grad, dq, hq, n, dev, "dq")
    dk, yk = _row_out(nr, q_grad, dk, hkv, n, dev, "dk")
    gv = yv = none
    if v_grad is None:
        dv = None
    else:
        gv = _row(nr, v_grad, hkv, n, dev, "v_grad")
        dv, yv = _row_out(nr, q_grad, dv, hkv, n, dev, "dv")
    dwq = q_grad.new_empty(D, dtype=torch.float32) if weight_grads and normed & NORM_Q else None
    dwk = q_grad.new_empty(D, dtype=torch.float32) if weight_grads and normed & NORM_K else None
    ws, ws_bytes = None, 0
    if dwq is not None or dwk is not None:
        ws_bytes = nr.workspace_bytes
        scratch = _scratch(nr._ws, ws_bytes, dev)   # (alive until the launch is made)
        ws = scratch.data_ptr()
    io = (Rows * 8)()
    at = C.addressof(io)
    _EIGHT_ROWS.pack_into(io, 0, *xq, *xk, *gq, *gk, *gv, *yq, *yk, *yv)
    rc = _on_device(dev, nr.backward, nr._n, nr._r, n, pos, at, at + _ROW, at + 2 * _ROW, at + 3 * _ROW,
                    at + 4 * _ROW if v_grad is not None else None, at + 5 * _ROW, at + 6 * _ROW,
                    at + 7 * _ROW if v_grad is not None else None, None if dwq is None else dwq.data_ptr(),
                    None if dwk is None else dwk.data_ptr(), ws, ws_bytes)
    if rc:
        raise SpkvError(rc, "spkv_norm_rope_backward")
    return dq, dk, dv, dwq, dwk


def spkv_tree_accept(tokens, target, parent=None, n_nodes=None, path=None, n_path=None, next=None, stream=None):
    """The nodes of each tree that the target confirms: tokens, target [B, T] int32 (target: what the target model puts
    behind each node), parent [B, T] int32 (None: chains), n_nodes [B] int32 (None: T).  Returns (path [B, T], n_path [B],
    next [B]), int32."""
    dev = tokens.get_device()
    if stream is not None:
        return _under(stream, dev, spkv_tree_accept, tokens, target, parent, n_nodes, path, n_path, next)
    if dev < 0 or tokens.dim() != 2:
        raise ValueError("tokens: a device tensor [B, T]")
    B, T = shape = tokens.shape
    i32 = torch.int32
    ptrs = (_dense(n_nodes, i32, (B,), dev), _dense(parent, i32, shape, dev), _dense(tokens, i32, shape, dev),
            _dense(target, i32, shape, dev))
    path, at_path = _result(tokens, path, i32, shape, dev)
    n_path, at_n = _result(tokens, n_path, i32, (B,), dev)
    next, at_next = _result(tokens, next, i32, (B,), dev)
    rc = _on_device(dev, lib().spkv_tree_accept, B, T, *ptrs, at_path, at_n, at_next)
    if rc:
        raise SpkvError(rc, "spkv_tree_accept")
    return path, n_path, next


_logprob_ws, _logprob_bytes = {}, {}


def spkv_token_logprobs(logits, given=None, top=0, scale=1.0, lse=None, logp=None, entropy=None, top_ids=None, top_logp=None,
                        want_entropy=True, stream=None):
    """Of rows of logits [n, vocab] (bf16, fp16 or fp32; rows contiguous, any row stride): log sum of exponentials, log probabilities
    of the tokens given [n, m] int32 (outside the vocabulary: NaN), entropy, and the `top` largest with their log
    probabilities, all of scale * logits.  Returns (lse [n], logp [n, m], entropy [n], top_ids [n, top], top_logp
    [n, top]); None for what is not asked for."""
    dev = logits.get_device()
    if stream is not None:
        return _under(stream, dev, spkv_token_logprobs, logits, given, top, scale, lse, logp, entropy, top_ids, top_logp, want_entropy)
    if dev < 0 or logits.dim() != 2 or logits.dtype not in _DTYPE or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits: bf16, fp16 or fp32 rows [n, vocab] on the device, each contiguous")
    n, vocab = logits.shape
    f32, i32 = torch.float32, torch.int32
    m = 0 if given is None else given.shape[-1]
    at_given = _dense(given, i32, (n, m), dev)
    lse, at_lse = _result(logits, lse, f32, (n,), dev)
    at_logp = at_entropy = at_ids = at_top = None
    if given is not None or logp is not None:
        logp, at_logp = _result(logits, logp, f32, (n, m), dev)
    if want_entropy or entropy is not None:
        entropy, at_entropy = _result(logits, entropy, f32, (n,), dev)
    if top > 0 or top_ids is not None or top_logp is not None:
        top_ids, at_ids = _result(logits, top_ids, i32, (n, top), dev)
        top_logp, at_top = _result(logits, top_logp, f32, (n, top), dev)
    ws_bytes = _logprob_bytes.get((n, vocab, top))
    if ws_bytes is None:
        if len(_logprob_bytes) >= 1024:      # (row counts vary from call to call)
            _logprob_bytes.clear()
        ws_bytes = _logprob_bytes[n, vocab, top] = max(16, lib().spkv_logprobs_workspace_bytes(n, vocab, top))
    ws = _scratch(_logprob_ws, ws_bytes, dev)
    rc = _on_device(dev, lib().spkv_token_logprobs, _DTYPE[logits.dtype], n, vocab, logits.data_ptr(),
                    logits.stride(0) if n > 1 else 0, scale, at_given, m, top, at_lse, at_entropy, at_logp, at_ids, at_top,
                    ws.data_ptr(), ws.numel())
    if rc:
        raise SpkvError(rc, "spkv_token_logprobs")
    return lse, logp, entropy, top_ids, top_logp


_softgate_ws = {}


@_on_its_stream
def spkv_softgate_forward(q, k, v, logits, window=128, alpha=0.0, tau=0.5, sm_scale=None, flags=0, out=None,
                          want_lse=False, stream=None, status=None):
    """Soft-gated whole-sequence forward (Eq. 6 / Eq. 7; see spkv.h).  q [T,Hq,128], k, v [T,Hkv,128]
    bf16, logits [T,Hkv] float32 on one device -> out [T,Hq,128] bf16 (and lse [T,Hq] float32).
    status: an int32 device tensor of one zero that receives the device-side verdict; when given,
    the call does not synchronise and the caller reads it; otherwise the call waits and raises."""
    T, Hq, Hkv = q.shape[0], q.shape[1], k.shape[1]
    if out is None:
        out = torch.empty_like(q)
    lse = torch.empty((T, Hq), dtype=torch.float32, device=q.device) if want_lse else None
    nbytes = lib().spkv_softgate_workspace_bytes(T, Hq, Hkv)
    ws = _softgate_ws.get(q.device)
    if ws is None or ws.numel() < nbytes:
        ws = _softgate_ws[q.device] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=q.device)
    own_status = status is None
    if own_status:
        status = torch.zeros(1, dtype=torch.int32, device=q.device)
    _check(lib().spkv_softgate_forward(
        T, Hq, Hkv, window, _ptr(q, torch.bfloat16), _ptr(k, torch.bfloat16), _ptr(v, torch.bfloat16),
        _ptr(logits, torch.float32), alpha, tau, 1.0 / math.sqrt(q.shape[2]) if sm_scale is None else sm_scale,
        flags, _ptr(out, torch.bfloat16), _ptr(lse), _ptr(ws), ws.numel(), _ptr(status), _stream(stream)),
        "spkv_softgate_forward")
    if own_status:
        code = int(status.item())      # synchronises: the status word is the call's device-side verdict
        if code != 0:
            raise SpkvError(code, "spkv_softgate_forward (device)")
    return (out, lse) if want_lse else out


@_on_its_stream
def spkv_wait_selftest(buf, limit_clocks, stream=None):
    """Runs the library's bounded-wait error path once (see spkv.h); returns the four status
    words [code, drained, clocks waited, data in place] as a list."""
    status = torch.zeros(4, dtype=torch.int32, device=buf.device)
    _check(lib().spkv_wait_selftest(_ptr(buf), int(limit_clocks), _ptr(status), _stream(stream)),
           "spkv_wait_selftest")
    return status.cpu().tolist()


def bf16_from_bits(bits, device):
    """numpy uint16 bit patterns -> torch.bfloat16 tensor on `device` (same bits)."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.view(torch.bfloat16).to(device)


def bits_from_bf16(t):
    """torch.bfloat16 tensor -> numpy uint16 bit patterns."""
    import numpy as np
    return t.detach().contiguous().cpu().view(torch.int16).numpy().view(np.uint16)
