"""ctypes binding of libmixattn.so: the same calls as include/mixattn.h.

Argument marshalling only.  Device tensors are torch tensors (torch supplies
device memory and streams); host arrays are numpy int32 arrays or sequences.
There is no fallback: if the library is missing the import fails, and a call
on a host-only context that needs the GPU returns MIXATTN_ERR_CUDA.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from typing import Optional, Sequence

import numpy as np

FULL, SLIDING = 0, 1
F32, BF16 = 0, 1
KV_NATIVE, KV_FP8_E4M3 = 0, 1

OK = 0
ERR_INVALID_ARG = -1
ERR_INVALID_LAYOUT = -2
ERR_NOT_OWNER = -3
ERR_OUT_OF_PAGES = -4
ERR_EMPTY_CONTEXT = -5
ERR_BAD_SEQ = -6
ERR_UNSUPPORTED = -7
ERR_CUDA = -8
ERR_TOO_LARGE = -9

K_APPEND, K_DECODE_FULL, K_DECODE_SLIDING, K_COMBINE, K_PREFILL_FULL, K_PREFILL_SLIDING, K_GATHER, K_FORK, K_READ, K_SELECT = range(10)
K_SHARED, K_MERGE, K_ROPE, K_ADJUST = range(10, 14)
MIN_SHARED_TOKENS, MIN_SAVED_BYTES = 128, 56000000
MAX_RULE_TOKENS, MAX_RULE_BIASES = (1 << 20) - 1, 2047

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmixattn.so")


class LayerDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("window", C.c_int32), ("kv_owner_layer", C.c_int32)]


class Config(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32),
        ("layers", C.POINTER(LayerDesc)),
        ("n_q_heads", C.c_int32),
        ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32),
        ("dtype", C.c_int32),
        ("max_seqs", C.c_int32),
        ("page_size", C.c_int32),
        ("n_pages", C.c_int32),
        ("max_seq_len", C.c_int32),
        ("free_order", C.POINTER(C.c_int32)),
        ("softmax_scale", C.c_float),
        ("device", C.c_int32),
        ("arena", C.c_void_p),
        ("arena_bytes", C.c_size_t),
        ("chunk_scratch_tokens", C.c_int32),
        ("kv_format", C.c_int32),
    ]


class RopeDesc(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("halves", C.c_int32), ("theta", C.c_double),
                ("inv_freq", C.POINTER(C.c_double)), ("scale", C.c_float)]


class LogitRules(C.Structure):
    _fields_ = [
        ("tokens", C.c_void_p),
        ("token_stride", C.c_int64),
        ("max_tokens", C.c_int32),
        ("n_tokens", C.c_void_p),
        ("n_prompt", C.c_void_p),
        ("repetition", C.c_void_p),
        ("frequency", C.c_void_p),
        ("presence", C.c_void_p),
        ("temperature", C.c_void_p),
        ("bias_tokens", C.c_void_p),
        ("bias_values", C.c_void_p),
        ("n_bias", C.c_int32),
        ("allowed", C.c_void_p),
        ("allowed_stride", C.c_int64),
        ("n_allowed", C.c_int32),
        ("allowed_rows", C.c_void_p),
    ]


class Rope:
    """A rotary embedding (mixattn_rope): `rotary_dim` channels, pairs (2p, 2p + 1) or, with `halves`,
    (p, p + rotary_dim / 2), turned by position * theta^(-2p / rotary_dim), or by position * inv_freq[p]."""

    def __init__(self, rotary_dim: int, theta: float = 10000.0, inv_freq=None, halves: bool = False, scale: float = 1.0):
        self._freq = None
        if inv_freq is not None:
            self._freq = np.array(inv_freq, dtype=np.float64)
            if self._freq.shape != (rotary_dim // 2,):
                raise MixAttnError(ERR_INVALID_ARG, "Rope: one frequency per pair of channels")
        elif 2 <= rotary_dim <= 1024 and 1.0 < theta < float("inf"):      # (formed once; anything else is the call's to refuse)
            self._freq = np.float64(theta) ** (-2.0 * np.arange(rotary_dim // 2) / rotary_dim)
        self.desc = RopeDesc(int(rotary_dim), int(bool(halves)), float(theta),
                             None if self._freq is None else self._freq.ctypes.data_as(C.POINTER(C.c_double)), float(scale))
        self.ref = C.byref(self.desc)


def _load() -> C.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2409_15012_b200.build` "
            "(there is no fallback implementation)")
    lib = C.CDLL(_LIB_PATH)
    i32, p32, vp = C.c_int32, C.POINTER(C.c_int32), C.c_void_p
    cfgp = C.POINTER(Config)
    sig = {
        "mixattn_arena_bytes": [cfgp, C.POINTER(C.c_size_t)],
        "mixattn_cache_bytes": [cfgp, C.POINTER(C.c_size_t)],
        "mixattn_create": [cfgp, C.POINTER(vp)],
        "mixattn_destroy": [vp],
        "mixattn_seq_reset": [vp, i32],
        "mixattn_append_kv": [vp, i32, i32, p32, p32, vp, vp, vp],
        "mixattn_append_kv_rope": [vp, i32, i32, p32, p32, vp, vp, C.c_float, vp],
        "mixattn_decode": [vp, i32, i32, p32, vp, vp, vp],
        "mixattn_decode_static_scratch": [vp, i32, i32, p32, vp, vp, vp],
        "mixattn_decode_layers": [vp, i32, i32, i32, p32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), vp, p32],
        "mixattn_attend_chunk": [vp, i32, i32, p32, p32, vp, vp, vp, vp, vp],
        "mixattn_prefill": [vp, i32, i32, p32, p32, vp, vp, vp, vp, vp],
        "mixattn_get_len": [vp, i32, i32, p32],
        "mixattn_get_block_table": [vp, i32, p32, i32, p32],
        "mixattn_get_n_free_pages": [vp, p32],
        "mixattn_get_ring_state": [vp, i32, i32, p32, p32],
        "mixattn_locate": [vp, i32, i32, i32, p32, p32],
        "mixattn_debug_read_kv": [vp, i32, i32, i32, vp, vp],
        "mixattn_debug_read_kv_fp8": [vp, i32, i32, i32, vp, vp, vp, vp],
        "mixattn_get_device_status": [vp, p32],
        "mixattn_set_layer_scores": [vp, i32, C.c_float, C.POINTER(C.c_float)],
        "mixattn_fork_seqs": [vp, i32, p32, p32, vp],
        "mixattn_get_stored": [vp, i32, i32, p32, p32],
        "mixattn_read_kv": [vp, i32, i32, p32, p32, p32, vp, vp, vp],
        "mixattn_beam_select": [vp, i32, i32, i32, i32, vp, C.c_int64, vp, vp, i32, i32, vp, vp, vp, vp],
        "mixattn_decode_shared": [vp, i32, i32, vp, vp, vp, vp],
        "mixattn_set_prefix_sharing": [vp, i32],
        "mixattn_set_share_min_bytes": [vp, C.c_int64],
        "mixattn_get_distinct_tokens": [vp, i32, i32, p32, C.POINTER(C.c_int64)],
        "mixattn_rope_qkv": [vp, i32, i32, vp, vp, vp, C.POINTER(RopeDesc), vp, C.c_int64, vp, C.c_int64, vp, C.c_int64, i32,
                             vp, vp, vp, vp],
        "mixattn_adjust_logits": [vp, i32, i32, i32, vp, C.c_int64, i32, vp, C.c_int64, C.POINTER(LogitRules), vp],
        "mixattn_set_split_tokens": [vp, i32],
        "mixattn_set_chunk_gather_reuse": [vp, i32],
        "mixattn_set_chunk_ring_direct": [vp, i32],
        "mixattn_profile_enable": [vp, i32],
        "mixattn_profile_read": [vp, i32, p32, C.POINTER(C.c_float)],
        "mixattn_get_launch_count": [vp, C.POINTER(C.c_int64)],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = C.c_int
    lib.mixattn_strerror.argtypes = [C.c_int]
    lib.mixattn_strerror.restype = C.c_char_p
    return lib


lib = _load()
EXPORTS = [
    "mixattn_arena_bytes", "mixattn_cache_bytes", "mixattn_create", "mixattn_destroy",
    "mixattn_seq_reset", "mixattn_append_kv", "mixattn_append_kv_rope", "mixattn_decode", "mixattn_decode_static_scratch", "mixattn_decode_layers", "mixattn_prefill",
    "mixattn_attend_chunk", "mixattn_set_layer_scores", "mixattn_fork_seqs", "mixattn_read_kv", "mixattn_beam_select",
    "mixattn_decode_shared", "mixattn_set_prefix_sharing", "mixattn_set_share_min_bytes", "mixattn_get_distinct_tokens", "mixattn_rope_qkv", "mixattn_adjust_logits",
    "mixattn_get_stored",
    "mixattn_get_len", "mixattn_get_block_table", "mixattn_get_n_free_pages",
    "mixattn_get_ring_state", "mixattn_locate", "mixattn_debug_read_kv", "mixattn_debug_read_kv_fp8",
    "mixattn_get_device_status", "mixattn_set_split_tokens", "mixattn_set_chunk_gather_reuse",
    "mixattn_set_chunk_ring_direct",
    "mixattn_profile_enable",
    "mixattn_profile_read", "mixattn_get_launch_count", "mixattn_strerror",
]


_torch = None


def _get_torch():
    """torch, imported on first use (host-only contexts never need it)."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


class MixAttnError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {lib.mixattn_strerror(code).decode()} ({code})")
        self.code = code


def strerror(code: int) -> str:
    return lib.mixattn_strerror(code).decode()


def _i32(a) -> np.ndarray:
    try:
        b = np.ascontiguousarray(a, dtype=np.int32)
    except OverflowError:
        raise MixAttnError(ERR_INVALID_ARG, "sequence of integers") from None
    if isinstance(a, np.ndarray) and a.dtype.kind in "iu" and a.dtype != np.int32 and not np.array_equal(a, b):   # (it wraps)
        raise MixAttnError(ERR_INVALID_ARG, "sequence of integers")
    return b


def _p32(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.POINTER(C.c_int32))


def _ints(a):
    """(ctypes int32 array, length) of a host sequence of whole numbers; short lists are a step of a
    generation loop's cost, and this is several times faster than going through numpy.  What is not
    one whole number per entry (a nested sequence, say) is refused."""
    b = None
    if type(a) is list:
        try:
            b = array("i", a)
        except TypeError:
            pass
        except OverflowError:
            raise MixAttnError(ERR_INVALID_ARG, "sequence of integers") from None
    if b is None:
        x = np.asarray(a)
        if x.ndim != 1 or x.dtype.kind not in "iufb":
            raise MixAttnError(ERR_INVALID_ARG, "sequence of integers")
        b = x.astype(np.int32)
        if not np.array_equal(b, x):
            raise MixAttnError(ERR_INVALID_ARG, "sequence of integers")
    n = len(b)
    return ((C.c_int32 * n).from_buffer(b) if n else (C.c_int32 * 1)()), n


def _ints_at(a):
    """(address, length, owner of the memory) of a host sequence of whole numbers, for the calls that take addresses."""
    if type(a) is list:
        try:
            b = array("i", a)
        except (TypeError, OverflowError):      # (_ints refuses the latter)
            pass
        else:
            at, n = b.buffer_info()
            return at, n, b
    b, n = _ints(a)
    return C.addressof(b), n, b


def _dev(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _stream(stream) -> Optional[int]:
    if stream is None:
        return None
    return int(getattr(stream, "cuda_stream", stream))


def make_config(layout: Sequence, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: int,
                max_seqs: int, n_pages: int, max_seq_len: int = 0, free_order=None,
                softmax_scale: float = 0.0, device: int = -1, page_size: int = 16,
                chunk_scratch_tokens: int = 0, kv_format: int = KV_NATIVE):
    """Returns (Config, keepalive): keepalive owns the arrays the struct points to."""
    layers = (LayerDesc * max(1, len(layout)))()
    for i, (kind, window, owner) in enumerate(layout):
        layers[i] = LayerDesc(int(kind), int(window), int(owner))
    fo = None if free_order is None else _i32(free_order)
    cfg = Config(len(layout), layers, n_q_heads, n_kv_heads, head_dim, dtype, max_seqs, page_size,
                 n_pages, max_seq_len, _p32(fo), float(softmax_scale), device, None, 0,
                 int(chunk_scratch_tokens), int(kv_format))
    return cfg, (layers, fo)


def arena_bytes(cfg: Config) -> int:
    out = C.c_size_t(0)
    rc = lib.mixattn_arena_bytes(C.byref(cfg), C.byref(out))
    if rc:
        raise MixAttnError(rc, "mixattn_arena_bytes")
    return out.value


def cache_bytes(cfg: Config) -> int:
    out = C.c_size_t(0)
    rc = lib.mixattn_cache_bytes(C.byref(cfg), C.byref(out))
    if rc:
        raise MixAttnError(rc, "mixattn_cache_bytes")
    return out.value


class Context:
    """Owns a mixattn_ctx and (on a GPU) the torch tensor that backs its arena.

    Methods have the names of the C calls without the prefix and raise
    MixAttnError on a non-zero status (`rc_*` variants return the status).
    """

    def __init__(self, layout, n_q_heads, n_kv_heads, head_dim, dtype, max_seqs, n_pages,
                 max_seq_len=0, free_order=None, softmax_scale=0.0, device=-1, chunk_scratch_tokens=0,
                 kv_format=KV_NATIVE):
        self.cfg, self._keep = make_config(layout, n_q_heads, n_kv_heads, head_dim, dtype, max_seqs,
                                           n_pages, max_seq_len, free_order, softmax_scale, device,
                                           chunk_scratch_tokens=chunk_scratch_tokens, kv_format=kv_format)
        self.arena = None
        self._like = self._ints_like = None      # empty tensors that results are allocated like
        if device >= 0:
            torch = _get_torch()
            nbytes = arena_bytes(self.cfg)
            self.arena = torch.empty(nbytes, dtype=torch.uint8, device=f"cuda:{device}")
            self._like = torch.empty(0, dtype=torch.bfloat16 if dtype == BF16 else torch.float32, device=self.arena.device)
            self._ints_like = torch.empty(0, dtype=torch.int32, device=self.arena.device)
            self._device, self._current_stream = device, torch._C._cuda_getCurrentRawStream   # (a handle, without an object)
            self.cfg.arena = self.arena.data_ptr()
            self.cfg.arena_bytes = nbytes
        h = C.c_void_p()
        rc = lib.mixattn_create(C.byref(self.cfg), C.byref(h))
        if rc:
            raise MixAttnError(rc, "mixattn_create")
        self.h = h
        self.n_q_heads, self.n_kv_heads, self.head_dim, self.dtype = n_q_heads, n_kv_heads, head_dim, dtype

    def close(self):
        if getattr(self, "h", None):
            lib.mixattn_destroy(self.h)
            self.h = None
        self.arena = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _empty(self, like, shape, handle):
        """like.new_empty(shape), its memory taken from the stream that the call's kernels run on: a block
        that was let go on another stream may still be written to there."""
        if (handle or 0) == self._current_stream(self._device):
            return like.new_empty(shape)
        cuda = _get_torch().cuda
        on = cuda.ExternalStream(handle, device=self._device) if handle else cuda.default_stream(self._device)
        with cuda.stream(on):
            return like.new_empty(shape)

    # -- calls -------------------------------------------------------------
    def rc_append_kv(self, layer, seq_ids, n_new=None, k=None, v=None, stream=None) -> int:
        s = _i32(seq_ids)
        n = None if n_new is None else _i32(n_new)
        if n is not None and len(n) != len(s):
            return ERR_INVALID_ARG
        return lib.mixattn_append_kv(self.h, layer, len(s), _p32(s), _p32(n), _dev(k), _dev(v), _stream(stream))

    def append_kv(self, layer, seq_ids, n_new=None, k=None, v=None, stream=None):
        rc = self.rc_append_kv(layer, seq_ids, n_new, k, v, stream)
        if rc:
            raise MixAttnError(rc, "mixattn_append_kv")

    def rc_append_kv_rope(self, layer, seq_ids, n_new, k, v, rope_theta, stream=None) -> int:
        s = _i32(seq_ids)
        n = None if n_new is None else _i32(n_new)
        if n is not None and len(n) != len(s):
            return ERR_INVALID_ARG
        return lib.mixattn_append_kv_rope(self.h, layer, len(s), _p32(s), _p32(n), _dev(k), _dev(v),
                                          float(rope_theta), _stream(stream))

    def append_kv_rope(self, layer, seq_ids, n_new, k, v, rope_theta, stream=None):
        rc = self.rc_append_kv_rope(layer, seq_ids, n_new, k, v, rope_theta, stream)
        if rc:
            raise MixAttnError(rc, "mixattn_append_kv_rope")

    def rc_decode(self, layer, seq_ids, q, out, stream=None) -> int:
        s, n = _ints(seq_ids)
        return lib.mixattn_decode(self.h, layer, n, s, _dev(q), _dev(out), _stream(stream))

    def decode(self, layer, seq_ids, q, out, stream=None):
        rc = self.rc_decode(layer, seq_ids, q, out, stream)
        if rc:
            raise MixAttnError(rc, "mixattn_decode")

    def rc_decode_static_scratch(self, layer, seq_ids, q, out, stream=None) -> int:
        """mixattn_decode_static_scratch: decode whose split partials live in the
        library's static device array instead of the arena workspace."""
        s = _i32(seq_ids)
        return lib.mixattn_decode_static_scratch(self.h, layer, len(s), _p32(s), _dev(q), _dev(out),
                                                 _stream(stream))

    def rc_decode_shared(self, layer, seq_ids, q, out, stream=None) -> int:
        s, n, _own = _ints_at(seq_ids)
        return lib.mixattn_decode_shared(self.h, layer, n, s, _dev(q), _dev(out), _stream(stream))

    def decode_shared(self, layer, seq_ids, q, out, stream=None):
        """decode() that reads pages shared by several of the sequences (forks of one prompt) once for all."""
        rc = self.rc_decode_shared(layer, seq_ids, q, out, stream)
        if rc:
            raise MixAttnError(rc, "mixattn_decode_shared")

    def set_prefix_sharing(self, enable: bool):
        """decode() and decode_layers() go the way of decode_shared() (off at first)."""
        rc = lib.mixattn_set_prefix_sharing(self.h, 1 if enable else 0)
        if rc:
            raise MixAttnError(rc, "mixattn_set_prefix_sharing")

    def set_share_min_bytes(self, nbytes: int):
        """Bytes of keys and values that a shared decode has to save (bf16 contexts); < 0 = automatic, 0 = always."""
        rc = lib.mixattn_set_share_min_bytes(self.h, int(nbytes))
        if rc:
            raise MixAttnError(rc, "mixattn_set_share_min_bytes")

    def get_distinct_tokens(self, layer, seq_ids) -> int:
        """Cached tokens that a decode_shared() of these sequences reads where it shares prefixes."""
        s, n = _ints(seq_ids)
        out = C.c_int64()
        rc = lib.mixattn_get_distinct_tokens(self.h, layer, n, s, C.byref(out))
        if rc:
            raise MixAttnError(rc, "mixattn_get_distinct_tokens")
        return out.value

    def _rows(self, t, heads):
        """(pointer, elements between tokens) of a [tokens, heads, head_dim] tensor whose head vectors lie
        one after the other; None if it is not one of this context."""
        if t is None:
            return None, 0
        d = self.head_dim
        shape = t.shape
        if len(shape) != 3 or shape[1] != heads or shape[2] != d or t.dtype is not self._like.dtype or t.get_device() != self._device:
            return None
        a, b, c = t.stride()
        if c != 1 or (heads > 1 and b != d):
            return None
        return t.data_ptr(), a

    def rope_qkv(self, layer, seq_ids, n_new, rope, q=None, k=None, v=None, store=False, first_pos=None, out=True, stream=None):
        """Rotates q [tokens, Hq, D] and k [tokens, Hkv, D] (views of one projection are fine) at their
        positions (default: behind what the cache holds) and returns (q, k, v) as dense tensors, None for
        what was not given; with `store`, k and v are appended to the cache instead of being returned.
        `out`: False if nothing is to be returned, or a triple of dense tensors (or None) to write to.
        The new tensors belong to `stream` (default: the default stream)."""
        def refuse():
            raise MixAttnError(ERR_INVALID_ARG, "mixattn_rope_qkv")
        s, m, _own_s = _ints_at(seq_ids)
        n = p = None
        tokens = m
        if n_new is not None:
            n, mn, _own_n = _ints_at(n_new)
            if mn != m:
                refuse()
            tokens = sum(_own_n[:mn])
        if first_pos is not None:
            p, mp, _own_p = _ints_at(first_pos)
            if mp != m:
                refuse()
        if self._like is None:
            if q is not None or k is not None or v is not None or not store:
                raise MixAttnError(ERR_CUDA, "mixattn_rope_qkv")
            rc = lib.mixattn_rope_qkv(self.h, layer, m, s, n, p, rope.ref, None, 0, None, 0, None, 0, 1, None, None, None, None)
            if rc:
                raise MixAttnError(rc, "mixattn_rope_qkv")
            return None, None, None
        hq, hkv, d = self.n_q_heads, self.n_kv_heads, self.head_dim
        rq, rk, rv = self._rows(q, hq), self._rows(k, hkv), self._rows(v, hkv)
        if rq is None or rk is None or rv is None:
            refuse()
        if (q is not None and q.shape[0] != tokens) or (k is not None and k.shape[0] != tokens) or (v is not None and v.shape[0] != tokens):
            refuse()
        stream = _stream(stream)
        outs = [None, None, None]
        if out is True:
            if q is not None:
                outs[0] = self._empty(self._like, (tokens, hq, d), stream)
            if not store:
                if k is not None:
                    outs[1] = self._empty(self._like, (tokens, hkv, d), stream)
                if v is not None:
                    outs[2] = self._empty(self._like, (tokens, hkv, d), stream)
        elif out is not None and out is not False:
            if type(out) not in (list, tuple) or len(out) != 3:
                refuse()
            outs = list(out)
            for t, h in zip(outs, (hq, hkv, hkv)):
                if t is not None and (self._rows(t, h) is None or t.shape[0] != tokens or not t.is_contiguous()):
                    refuse()
        rc = lib.mixattn_rope_qkv(self.h, layer, m, s, n, p, rope.ref, rq[0], rq[1], rk[0], rk[1], rv[0], rv[1], 1 if store else 0,
                                  _dev(outs[0]), _dev(outs[1]), _dev(outs[2]), stream)
        if rc:
            raise MixAttnError(rc, "mixattn_rope_qkv")
        return tuple(outs)

    def pointer_table(self, tensors):
        """Host array of device pointers, one per layer (None -> NULL), for mixattn_decode_layers.
        `tensors` maps a layer index to a tensor, or is a sequence indexed by layer."""
        n = self.cfg.n_layers
        arr = (C.c_void_p * n)()
        for l in range(n):
            t = tensors.get(l) if isinstance(tensors, dict) else tensors[l]
            arr[l] = None if t is None else int(t.data_ptr())
        return arr

    def rc_decode_layers(self, layer_begin, layer_end, seq_ids, q_tab, k_tab, v_tab, out_tab, stream=None):
        """mixattn_decode_layers with pointer tables from pointer_table(); returns (status, layers_done)."""
        s = _i32(seq_ids)
        done = C.c_int32(0)
        rc = lib.mixattn_decode_layers(self.h, layer_begin, layer_end, len(s), _p32(s), q_tab, k_tab, v_tab, out_tab,
                                       _stream(stream), C.byref(done))
        return rc, done.value

    def decode_layers(self, layer_begin, layer_end, seq_ids, q_tab, k_tab, v_tab, out_tab, stream=None):
        rc, _ = self.rc_decode_layers(layer_begin, layer_end, seq_ids, q_tab, k_tab, v_tab, out_tab, stream)
        if rc:
            raise MixAttnError(rc, "mixattn_decode_layers")

    def rc_prefill(self, layer, seq_ids, seq_lens, q, k, v, out, stream=None) -> int:
        (s, n), (lens, m) = _ints(seq_ids), _ints(seq_lens)
        if n != m:
            return ERR_INVALID_ARG
        return lib.mixattn_prefill(self.h, layer, n, s, lens, _dev(q), _dev(k), _dev(v), _dev(out), _stream(stream))

    def prefill(self, layer, seq_ids, seq_lens, q, k, v, out, stream=None):
        rc = self.rc_prefill(layer, seq_ids, seq_lens, q, k, v, out, stream)
        if rc:
            raise MixAttnError(rc, "mixattn_prefill")

    def rc_attend_chunk(self, layer, seq_ids, seq_lens, q, k, v, out, stream=None) -> int:
        (s, n), (lens, m) = _ints(seq_ids), _ints(seq_lens)
        if n != m:
            return ERR_INVALID_ARG
        return lib.mixattn_attend_chunk(self.h, layer, n, s, lens, _dev(q), _dev(k), _dev(v), _dev(out), _stream(stream))

    def attend_chunk(self, layer, seq_ids, seq_lens, q, k, v, out, stream=None):
        rc = self.rc_attend_chunk(layer, seq_ids, seq_lens, q, k, v, out, stream)
        if rc:
            raise MixAttnError(rc, "mixattn_attend_chunk")

    def rc_set_layer_scores(self, layer, softcap=0.0, slopes=None) -> int:
        a = None
        if slopes is not None:
            a = np.ascontiguousarray(slopes, dtype=np.float32)
            if a.shape != (self.n_q_heads,):
                return ERR_INVALID_ARG
            a = a.ctypes.data_as(C.POINTER(C.c_float))
        return lib.mixattn_set_layer_scores(self.h, layer, float(softcap), a)

    def set_layer_scores(self, layer, softcap=0.0, slopes=None):
        """Caps the layer's scores (softcap * tanh(s / softcap)) and / or biases them by distance
        (- slopes[h] * (i - j), one slope per query head); the defaults restore plain scores."""
        rc = self.rc_set_layer_scores(layer, softcap, slopes)
        if rc:
            raise MixAttnError(rc, "mixattn_set_layer_scores")

    def rc_fork_seqs(self, src, dst, stream=None) -> int:
        (s, n), (d, m) = _ints(src), _ints(dst)
        if n != m:
            return ERR_INVALID_ARG
        return lib.mixattn_fork_seqs(self.h, n, s, d, _stream(stream))

    def fork_seqs(self, src, dst, stream=None):
        """Every sequence dst[i] becomes a copy of what src[i] was before the call (all at once)."""
        (s, n), (d, m) = _ints(src), _ints(dst)
        rc = lib.mixattn_fork_seqs(self.h, n, s, d, _stream(stream)) if n == m else ERR_INVALID_ARG
        if rc:
            raise MixAttnError(rc, "mixattn_fork_seqs")

    def read_kv(self, layer, seq_ids, first_pos=None, n_tokens=None, stream=None):
        """Returns (K, V), the cached tokens [sum n_tokens, Hkv, D] of the sequences, oldest first
        (default: everything stored).  The tensors belong to `stream` (default: the default stream)."""
        s, m = _ints(seq_ids)
        p = n = None
        if first_pos is not None:
            p, mp = _ints(first_pos)
            if mp != m:
                raise MixAttnError(ERR_INVALID_ARG, "mixattn_read_kv")
        if n_tokens is not None:
            n, mn = _ints(n_tokens)
            if mn != m:
                raise MixAttnError(ERR_INVALID_ARG, "mixattn_read_kv")
        if n is not None:
            rows = sum([max(0, x) for x in n[:m]])
        elif p is not None:
            rows = sum([max(0, self.get_len(layer, seq) - first) for seq, first in zip(s[:m], p[:m])])
        else:
            stored = (C.c_int32 * (m or 1))()
            rc = lib.mixattn_get_stored(self.h, layer, m, s, stored)
            if rc:
                raise MixAttnError(rc, "mixattn_read_kv")
            rows = sum(stored) if m else 0
        if self._like is None:
            raise MixAttnError(ERR_CUDA, "mixattn_read_kv")
        hkv, d = self.n_kv_heads, self.head_dim
        stream = _stream(stream)
        kv = self._empty(self._like, (2, rows, hkv, d), stream)
        at = kv.data_ptr()
        rc = lib.mixattn_read_kv(self.h, layer, m, s, p, n, at, at + rows * hkv * d * (2 if self.dtype == BF16 else 4), stream)
        if rc:
            raise MixAttnError(rc, "mixattn_read_kv")
        return kv.unbind(0)

    def get_stored(self, layer, seq_ids):
        """Tokens the layer's cache holds of each sequence: its length, or at most the window."""
        s, n = _ints(seq_ids)
        out = (C.c_int32 * max(n, 1))()
        rc = lib.mixattn_get_stored(self.h, layer, n, s, out)
        if rc:
            raise MixAttnError(rc, "mixattn_get_stored")
        return out[:n]

    def rc_beam_select(self, logits, scores, n_out, out_scores, out_beams, out_tokens, finished=None, eos_token=0,
                       stream=None) -> int:
        """logits [groups, beams, vocab] (fp32 or bf16, last dimension dense, rows evenly spaced)."""
        torch = _get_torch()
        o = logits.shape[0] * n_out
        for t, dt in ((out_scores, torch.float32), (out_beams, torch.int32), (out_tokens, torch.int32)):
            if t.dtype is not dt or t.numel() != o or not t.is_contiguous() or t.get_device() != self.cfg.device:
                return ERR_INVALID_ARG
        return self._beam_select(logits, scores, n_out, out_scores.data_ptr(), out_beams.data_ptr(), out_tokens.data_ptr(),
                                 finished, eos_token, stream)

    def _beam_select(self, logits, scores, n_out, out_scores, out_beams, out_tokens, finished, eos_token, stream) -> int:
        torch = _get_torch()
        g, b, v = logits.shape
        sg, sb, sv = logits.stride()
        dt = logits.dtype
        if dt is torch.bfloat16:
            dt = BF16
        elif dt is torch.float32:
            dt = F32
        else:
            return ERR_INVALID_ARG
        if b == 1:
            sb = sg                              # one beam per group: the groups are the rows
        if g * b <= 1:
            sb = v
        if (v > 1 and sv != 1) or (g > 1 and sg != b * sb):
            return ERR_INVALID_ARG
        dev = self.cfg.device
        if logits.get_device() != dev or scores.get_device() != dev or (finished is not None and finished.get_device() != dev):
            return ERR_INVALID_ARG               # a tensor of the host or of another device
        if scores.dtype is not torch.float32 or scores.numel() != g * b or not scores.is_contiguous():
            return ERR_INVALID_ARG
        if finished is not None and (finished.dtype is not torch.uint8 or finished.numel() != g * b or
                                     not finished.is_contiguous()):
            return ERR_INVALID_ARG
        return lib.mixattn_beam_select(self.h, g, b, v, dt, logits.data_ptr(), sb, scores.data_ptr(), _dev(finished),
                                       eos_token, n_out, out_scores, out_beams, out_tokens, _stream(stream))

    def beam_select(self, logits, scores, n_out, finished=None, eos_token=0, stream=None):
        """The n_out best continuations of every group: (scores fp32, beams int32, tokens int32),
        [groups, n_out] each.  The tensors belong to `stream` (default: the default stream)."""
        if self._ints_like is None or n_out < 1:
            raise MixAttnError(ERR_INVALID_ARG if n_out < 1 else ERR_CUDA, "mixattn_beam_select")
        g = logits.shape[0]
        stream = _stream(stream)
        out = self._empty(self._ints_like, (3, g, n_out), stream)
        at, step = out.data_ptr(), 4 * g * n_out
        rc = self._beam_select(logits, scores, n_out, at, at + step, at + 2 * step, finished, eos_token, stream)
        if rc:
            raise MixAttnError(rc, "mixattn_beam_select")
        s, b, t = out.unbind(0)      # (while the kernel runs)
        return s.view(_get_torch().float32), b, t

    def rc_adjust_logits(self, logits, out=None, tokens=None, n_tokens=None, n_prompt=None, repetition=None, frequency=None,
                         presence=None, temperature=None, bias_tokens=None, bias_values=None, allowed=None, allowed_rows=None,
                         stream=None) -> int:
        torch = _get_torch()
        if self._like is None:
            return ERR_CUDA
        out = logits if out is None else out
        if logits.dim() != 2 or out.shape != logits.shape:
            return ERR_INVALID_ARG
        types = {torch.bfloat16: BF16, torch.float32: F32}
        rows, vocab = logits.shape
        dev = self._device
        r = LogitRules()

        def matrix(t, dtype):       # rows of a tensor, its last dimension dense: (pointer, elements between rows), or None
            if t.dim() != 2 or (dtype is not None and t.dtype is not dtype) or t.get_device() != dev or (t.shape[1] > 1 and t.stride(1) != 1):
                return None
            # (a single row or an expanded one has no stride of its own to check)
            return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1]

        strides = []
        for t in (logits, out):
            at = matrix(t, None)
            if t.dtype not in types or at is None:
                return ERR_INVALID_ARG
            strides.append(at[1])
        for name, t, dtype in (("n_tokens", n_tokens, torch.int32), ("n_prompt", n_prompt, torch.int32), ("repetition", repetition, torch.float32),
                               ("frequency", frequency, torch.float32), ("presence", presence, torch.float32),
                               ("temperature", temperature, torch.float32), ("allowed_rows", allowed_rows, torch.int32)):
            if t is not None:
                if t.dtype is not dtype or t.shape != (rows,) or not t.is_contiguous() or t.get_device() != dev:
                    return ERR_INVALID_ARG
                setattr(r, name, t.data_ptr())
        if tokens is not None and tokens.dim() == 2 and tokens.shape[1] == 0:    # (empty lists)
            tokens, r.n_tokens, r.n_prompt = None, None, None
        if tokens is not None:
            at = matrix(tokens, torch.int32)
            if at is None or tokens.shape[0] != rows:
                return ERR_INVALID_ARG
            r.tokens, r.token_stride = at
            r.max_tokens = tokens.shape[1]
        if (bias_tokens is None) != (bias_values is None):
            return ERR_INVALID_ARG
        if bias_tokens is not None:
            for t, dtype in ((bias_tokens, torch.int32), (bias_values, torch.float32)):
                if t.dtype is not dtype or t.dim() != 2 or t.shape != (rows, bias_tokens.shape[1]) or not t.is_contiguous() or t.get_device() != dev:
                    return ERR_INVALID_ARG
            r.bias_tokens, r.bias_values, r.n_bias = bias_tokens.data_ptr(), bias_values.data_ptr(), bias_tokens.shape[1]
        if allowed is not None:
            at = matrix(allowed, torch.int32)
            # (a set of no masks has no address, which would read as no set at all)
            if at is None or allowed.shape[1] < (vocab + 31) // 32 or (rows > 0 and allowed.shape[0] == 0):
                return ERR_INVALID_ARG
            r.allowed, r.allowed_stride = at
            r.n_allowed = allowed.shape[0]
        return lib.mixattn_adjust_logits(self.h, rows, vocab, types[logits.dtype], logits.data_ptr(), strides[0], types[out.dtype],
                                         out.data_ptr(), strides[1], C.byref(r), _stream(stream))

    def adjust_logits(self, logits, out=None, **rules):
        """Penalties for the tokens of a row's list, biases, temperature and grammar masks on logits [rows, vocab], in
        place or into `out`.  Rules, all optional: tokens int32 [rows, n] with n_tokens and n_prompt int32
        [rows]; repetition, frequency, presence, temperature fp32 [rows]; bias_tokens int32 and bias_values
        fp32 [rows, n]; allowed int32 [masks, words] (bit t % 32 of word t // 32) with allowed_rows int32 [rows];
        stream (default: the default stream)."""
        rc = self.rc_adjust_logits(logits, out, **rules)
        if rc:
            raise MixAttnError(rc, "mixattn_adjust_logits")

    def seq_reset(self, seq):
        rc = lib.mixattn_seq_reset(self.h, seq)
        if rc:
            raise MixAttnError(rc, "mixattn_seq_reset")

    def get_len(self, layer, seq) -> int:
        out = C.c_int32()
        rc = lib.mixattn_get_len(self.h, layer, seq, C.byref(out))
        if rc:
            raise MixAttnError(rc, "mixattn_get_len")
        return out.value

    def get_block_table(self, seq):
        n = C.c_int32()
        rc = lib.mixattn_get_block_table(self.h, seq, None, 0, C.byref(n))
        if rc:
            raise MixAttnError(rc, "mixattn_get_block_table")
        buf = np.zeros(max(1, n.value), dtype=np.int32)
        rc = lib.mixattn_get_block_table(self.h, seq, _p32(buf), n.value, C.byref(n))
        if rc:
            raise MixAttnError(rc, "mixattn_get_block_table")
        return buf[:n.value].tolist()

    def get_n_free_pages(self) -> int:
        out = C.c_int32()
        rc = lib.mixattn_get_n_free_pages(self.h, C.byref(out))
        if rc:
            raise MixAttnError(rc, "mixattn_get_n_free_pages")
        return out.value

    def get_ring_state(self, layer, seq):
        a, b = C.c_int32(), C.c_int32()
        rc = lib.mixattn_get_ring_state(self.h, layer, seq, C.byref(a), C.byref(b))
        if rc:
            raise MixAttnError(rc, "mixattn_get_ring_state")
        return a.value, b.value

    def locate(self, layer, seq, pos):
        a, b = C.c_int32(), C.c_int32()
        rc = lib.mixattn_locate(self.h, layer, seq, pos, C.byref(a), C.byref(b))
        if rc:
            raise MixAttnError(rc, "mixattn_locate")
        return a.value, b.value

    def debug_read_kv(self, layer, seq, pos):
        """Returns (K, V) as torch CPU tensors [Hkv, D] in the context dtype."""
        import torch
        dt = torch.bfloat16 if self.dtype == BF16 else torch.float32
        k = torch.empty(self.n_kv_heads, self.head_dim, dtype=dt)
        v = torch.empty_like(k)
        rc = lib.mixattn_debug_read_kv(self.h, layer, seq, pos, k.data_ptr(), v.data_ptr())
        if rc:
            raise MixAttnError(rc, "mixattn_debug_read_kv")
        return k, v

    def debug_read_kv_fp8(self, layer, seq, pos):
        """Quantised storage: (k_codes, k_exp, v_codes, v_exp) as numpy arrays: uint8 [Hkv, D]
        codes and int32 [Hkv] shared exponents."""
        kc = np.zeros((self.n_kv_heads, self.head_dim), dtype=np.uint8)
        vc = np.zeros_like(kc)
        kx = np.zeros(self.n_kv_heads, dtype=np.int32)
        vx = np.zeros_like(kx)
        rc = lib.mixattn_debug_read_kv_fp8(self.h, layer, seq, pos, kc.ctypes.data, kx.ctypes.data,
                                           vc.ctypes.data, vx.ctypes.data)
        if rc:
            raise MixAttnError(rc, "mixattn_debug_read_kv_fp8")
        return kc, kx, vc, vx

    def get_device_status(self) -> int:
        out = C.c_int32()
        rc = lib.mixattn_get_device_status(self.h, C.byref(out))
        if rc:
            raise MixAttnError(rc, "mixattn_get_device_status")
        return out.value

    def set_split_tokens(self, tokens: int):
        rc = lib.mixattn_set_split_tokens(self.h, tokens)
        if rc:
            raise MixAttnError(rc, "mixattn_set_split_tokens")

    def set_chunk_gather_reuse(self, enable: bool):
        """Layers that share a cache gather the same rows for a chunk: copy them once per run of
        such calls (the caller keeps k / v unchanged between them)."""
        rc = lib.mixattn_set_chunk_gather_reuse(self.h, 1 if enable else 0)
        if rc:
            raise MixAttnError(rc, "mixattn_set_chunk_gather_reuse")

    def set_chunk_ring_direct(self, enable: bool):
        """Sliding-window chunk calls read the ring in place where its window is a whole number of
        128-key tiles (on by default); off = they copy the cached keys like every other chunk call."""
        rc = lib.mixattn_set_chunk_ring_direct(self.h, 1 if enable else 0)
        if rc:
            raise MixAttnError(rc, "mixattn_set_chunk_ring_direct")

    def profile_enable(self, enable: bool):
        rc = lib.mixattn_profile_enable(self.h, 1 if enable else 0)
        if rc:
            raise MixAttnError(rc, "mixattn_profile_enable")

    def profile_read(self, kernel_class: int):
        n, ms = C.c_int32(), C.c_float()
        rc = lib.mixattn_profile_read(self.h, kernel_class, C.byref(n), C.byref(ms))
        if rc:
            raise MixAttnError(rc, "mixattn_profile_read")
        return n.value, ms.value

    def get_launch_count(self) -> int:
        out = C.c_int64()
        rc = lib.mixattn_get_launch_count(self.h, C.byref(out))
        if rc:
            raise MixAttnError(rc, "mixattn_get_launch_count")
        return out.value
