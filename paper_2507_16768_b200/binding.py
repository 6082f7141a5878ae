"""Thin ctypes binding of the C ABI in ``include/wg.h``.

Argument marshalling only: every step of the path runs in the library's CUDA kernels.
Device buffers are ``torch`` tensors (PyTorch is used for device memory and streams); host
arrays are numpy.  There is no CPU fallback: if ``libwg.so`` has not been built, importing
this module fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libwg.so")

WG_OK = 0
WG_ERR_ARG = -1
WG_ERR_GRAMMAR = -2
WG_ERR_CAPACITY = -3
WG_ERR_TOKEN_REJECTED = -4
WG_ERR_CUDA = -5
WG_ERR_EMPTY_MASK = -6
WG_ERR_STATE = -7

WG_DTYPE_BF16 = 0
WG_DTYPE_FP32 = 1
WG_DTYPE_FP16 = 2
WG_KV_BF16 = 0
WG_KV_FP16 = 1
WG_KV_E4M3 = 2
WG_KV_INT8 = 3
WG_KV_MAX_HEAD_DIM = 256
WG_USE_CACHE = 0
WG_NO_CACHE = 1
WG_RESTART_ON_DONE = 2
WG_CACHE_DENSE = 0
WG_CACHE_COMPACT = 1
WG_BEAM_NORM_ALLOWED = 0
WG_BEAM_NORM_FULL = 1
WG_BEAM_NORM_NONE = 2
WG_BEAM_MAX_BEAMS = 32
WG_BEAM_MAX_OUT = 64
WG_ENTRY_ALLOWS = 0
WG_ENTRY_DENIES = 1

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2507_16768_b200.build` "
        "(nvcc, sm_100a). This package has no CPU fallback.")

_lib = C.CDLL(LIB_PATH)


class WgStats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in (
        "cache_hits", "cache_misses", "masks_built", "rows_uncached", "tokens_rejected",
        "empty_masks", "bad_states", "cache_entries", "cache_bytes")]

    def as_dict(self):
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


class _WgKvCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)] + \
        [(n, C.c_int32) for n in ("storage", "n_blocks", "block_size", "n_heads", "head_dim")]


class _WgRope(C.Structure):
    _fields_ = [("table", C.c_void_p)] + [(n, C.c_int32) for n in ("n_pos", "rot_dim", "interleaved")]


_vp, _i32, _i64, _u32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32
_SIGNATURES = {
    "wg_load_vocab": (_i32, [_vp, _vp, _i32, _i32, C.POINTER(_vp)]),
    "wg_vocab_free": (None, [_vp]),
    "wg_compile_grammar": (_i32, [_vp, _i32, _vp, _i32, _vp, _i32, _vp, _i32, _i32, C.POINTER(_vp)]),
    "wg_grammar_free": (None, [_vp]),
    "wg_grammar_minimize": (_i32, [_vp, C.POINTER(_vp)]),
    "wg_template_compile": (_i32, [_vp, _i32, _vp, _i32, _vp, _i32, _vp, _i32, _i32, C.POINTER(_vp)]),
    "wg_template_info": (_i32, [_vp, C.POINTER(_i32), C.POINTER(_i32), C.POINTER(_i32)]),
    "wg_template_instantiate": (_i32, [_vp, C.POINTER(_vp), _i32, C.POINTER(_vp)]),
    "wg_template_free": (None, [_vp]),
    "wg_grammar_save": (_i32, [_vp, _vp, C.c_size_t, C.POINTER(C.c_size_t)]),
    "wg_grammar_load": (_i32, [C.c_char_p, C.c_size_t, C.POINTER(_vp)]),
    "wg_regex_to_optree": (_i32, [C.c_char_p, _i32, C.POINTER(_vp)]),
    "wg_optree_sizes": (_i32, [_vp, C.POINTER(_i32), C.POINTER(_i32), C.POINTER(_i32),
                               C.POINTER(_i32), C.POINTER(_i32)]),
    "wg_optree_copy": (_i32, [_vp, _vp, _vp, _vp, _vp]),
    "wg_optree_free": (None, [_vp]),
    "wg_compile_regex": (_i32, [C.c_char_p, _i32, C.POINTER(_vp)]),
    "wg_compile_regex_fragment": (_i32, [C.c_char_p, _i32, C.POINTER(_vp)]),
    "wg_regex_error": (C.c_char_p, []),
    "wg_grammar_info": (_i32, [_vp, C.POINTER(_i32), C.POINTER(_i32), C.POINTER(_i32),
                               C.POINTER(_i32), C.POINTER(C.c_uint64)]),
    "wg_grammar_step": (_i32, [_vp, _i32, _i32]),
    "wg_grammar_forced_token": (_i32, [_vp, _i32, C.POINTER(_i32), C.POINTER(_i32)]),
    "wg_ctx_create": (_i32, [_vp, _i32, _i32, C.POINTER(_vp)]),
    "wg_ctx_create_ex": (_i32, [_vp, _i32, _i32, _i32, C.c_size_t, C.POINTER(_vp)]),
    "wg_ctx_free": (None, [_vp]),
    "wg_cache_entry_read": (_i32, [_vp, _i32, _i32, C.POINTER(_i32), C.POINTER(_i32), _vp, _i32,
                                   C.POINTER(_i64), _vp]),
    "wg_ctx_add_grammar": (_i32, [_vp, _vp, C.POINTER(_i32)]),
    "wg_ctx_remove_grammar": (_i32, [_vp, _i32]),
    "wg_cache_prewarm": (_i32, [_vp, _i32, _vp]),
    "wg_cache_clear": (_i32, [_vp, _vp]),
    "wg_get_stats": (_i32, [_vp, C.POINTER(WgStats), _vp]),
    "wg_reset_stats": (_i32, [_vp, _vp]),
    "wg_mask_cache_lookup": (_i32, [_vp, _vp, _vp, _i32, _vp, _vp]),
    "wg_build_masks": (_i32, [_vp, _vp, _vp, _i32, _vp, _i64, _u32, _vp]),
    "wg_apply_mask": (_i32, [_vp, _i32, _i64, _vp, _i64, _i32, _i32, _vp, _vp, _vp]),
    "wg_apply_workspace_bytes": (C.c_size_t, [_i32]),
    "wg_apply_mask_noalloc": (_i32, [_vp, _i32, _i64, _vp, _i64, _i32, _i32, _vp, _vp]),
    "wg_advance": (_i32, [_vp, _vp, _vp, _vp, _i32, _vp, _u32, _vp]),
    "wg_decode_step": (_i32, [_vp, _vp, _vp, _i32, _vp, _i32, _i64, _vp, _i64, _vp, _vp, _u32, _vp]),
    "wg_decode_step_shard": (_i32, [_vp, _vp, _vp, _i32, _vp, _i32, _i64, _vp, _i64, _i32, _i32, _vp,
                                    _u32, _vp]),
    "wg_advance_keys": (_i32, [_vp, _vp, _vp, _vp, _i32, _vp, _vp, _u32, _vp]),
    "wg_step_graph_create": (_i32, [_vp, _vp, _vp, _i32, _vp, _i32, _i64, _vp, _i64, _vp, _vp, _u32,
                                    C.POINTER(_vp)]),
    "wg_step_graph_launch": (_i32, [_vp, _vp]),
    "wg_step_graph_free": (None, [_vp]),
    "wg_decode_step_host": (_i32, [_vp, _vp, _vp, _i32, _vp, _vp, _i32, _i64, _vp, _i64, _vp, _vp,
                                   _vp, _u32, _vp]),
    "wg_beam_create": (_i32, [_i32, _i32, _i32, _i32, C.POINTER(_vp)]),
    "wg_beam_free": (None, [_vp]),
    "wg_beam_select": (_i32, [_vp, _vp, _i32, _i64, _vp, _i64, _vp, _vp, _i32, _i32, _i32, _i32, _i32,
                              _vp, _vp, _vp, _vp]),
    "wg_beam_step": (_i32, [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _i32, _i64, _vp, _i64, _i32, _vp,
                            _vp, _vp, _u32, _vp]),
    "wg_beam_backtrack": (_i32, [_vp, _vp, _i32, _i32, _i32, _vp, _vp]),
    "wg_kv_pool_create": (_i32, [_i32, _i32, _i32, C.POINTER(_vp)]),
    "wg_kv_pool_free": (None, [_vp]),
    "wg_kv_pool_refs": (_vp, [_vp]),
    "wg_kv_pool_load": (_i32, [_vp, _vp, _vp]),
    "wg_kv_pool_n_free": (_i32, [_vp, C.POINTER(_i32), _vp]),
    "wg_kv_extend": (_i32, [_vp, _vp, _i64, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _i32, _vp, _vp]),
    "wg_kv_shrink": (_i32, [_vp, _vp, _i64, _i32, _vp, _vp, _i32, _vp, _vp]),
    "wg_kv_reorder": (_i32, [_vp, _vp, _i64, _i32, _vp, _vp, _i32, _i32, _vp, _i32, _vp, _vp, _vp, _vp]),
    "wg_rope_frequencies": (_i32, [_i32] + [C.c_double] * 5 + [_vp]),
    "wg_rope_table": (_i32, [_vp, _i32, _i32, C.c_double, _vp, _vp]),
    "wg_kv_write": (_i32, [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _i32, _vp, _vp]),
    "wg_kv_read": (_i32, [_vp, _vp, _i64, _i32, _vp, _i32, _vp, _vp, _vp, _i32, _i32, _vp]),
    "wg_attend_create": (_i32, [_i32, _i32, _i32, _i32, C.POINTER(_vp)]),
    "wg_attend_free": (None, [_vp]),
    "wg_kv_attend": (_i32, [_vp, _vp, _vp, _i64, _vp, _i64, _vp, _i32, _i32, _vp, _i64, _i32, _vp, _i32, _vp, _vp, _vp, _i32,
                            C.c_float, _i32, _i32, _vp]),
    "wg_ctx_set_timing": (_i32, [_vp, _i32]),
    "wg_ctx_get_timing": (_i32, [_vp, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                 C.POINTER(_i64)]),
    "wg_ctx_count_build_work": (_i32, [_vp, _i32]),
    "wg_get_build_work": (_i32, [_vp, C.POINTER(_i64), C.POINTER(_i64), C.POINTER(_i64), _vp]),
    "wg_strerror": (C.c_char_p, [_i32]),
    "wg_last_cuda_error": (_i32, []),
    "wg_kernel_launch_count": (_i64, []),
}
for _name, (_res, _args) in _SIGNATURES.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args

EXPORTED = tuple(_SIGNATURES)


class WgError(RuntimeError):
    def __init__(self, status: int, where: str):
        msg = _lib.wg_strerror(int(status)).decode()
        if status == WG_ERR_CUDA:
            msg += f" (cudaError {_lib.wg_last_cuda_error()})"
        super().__init__(f"{where}: {msg} [{status}]")
        self.status = int(status)


def _check(status: int, where: str) -> None:
    if status != WG_OK:
        raise WgError(status, where)


def _np_ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _device_of(ctx):
    """Index of the device a context (or None: any device) lives on."""
    return None if ctx is None else getattr(ctx, "device", None)


def _dev_ptr(t, dtype=None, what: str = "tensor", device=None):
    """Raw device pointer of a torch CUDA tensor (None passes through)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if dtype is not None and t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise TypeError(f"{what} has dtype {t.dtype}")
    if device is not None and t.device.index != device:
        raise ValueError(f"{what} lives on cuda:{t.device.index}, the context on cuda:{device}")
    return C.c_void_p(t.data_ptr())


def _vec(t, n: int, dtype, what: str, device=None):
    """Pointer of a contiguous 1-D device array that holds at least ``n`` elements: the kernels
    index these arrays by row number without any further check."""
    if t is None:
        return None
    p = _dev_ptr(t, dtype, what, device)
    if t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous 1-D tensor")
    if t.numel() < n:
        raise ValueError(f"{what} holds {t.numel()} elements, the batch has {n} rows")
    return p


def _mat(t, rows: int, cols: int, dtype, what: str, device=None):
    """(pointer, row stride) of a 2-D device array with unit inner stride that holds at least
    ``rows`` rows of ``cols`` elements."""
    p = _dev_ptr(t, dtype, what, device)
    _, stride = _rows(t, what)
    if t.shape[0] < rows or t.shape[1] < cols:
        raise ValueError(f"{what} is {tuple(t.shape)}, at least ({rows}, {cols}) is needed")
    return p, stride


def _stream_ptr(stream):
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def kernel_launch_count() -> int:
    return int(_lib.wg_kernel_launch_count())


class Vocab:
    """wg_load_vocab: copies a CSR vocabulary (numpy, host) to the current device."""

    def __init__(self, offsets: np.ndarray, data: np.ndarray, eos_id: int):
        self._offsets = np.ascontiguousarray(offsets, np.uint32)
        self._data = np.ascontiguousarray(data, np.uint8)
        self.V = int(self._offsets.shape[0] - 1)
        self.W = (self.V + 31) // 32
        self.eos_id = int(eos_id)
        h = _vp()
        _check(_lib.wg_load_vocab(_np_ptr(self._offsets), _np_ptr(self._data), self.V, self.eos_id,
                                  C.byref(h)), "wg_load_vocab")
        self.handle = h
        import torch
        self.device = torch.cuda.current_device()     # wg_load_vocab uploads to the current device

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.wg_vocab_free(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


class RegexTree:
    """The operator tree of a regular expression as flat arrays (wg_regex_to_optree)."""

    def __init__(self, pattern):
        if isinstance(pattern, str):
            pattern = pattern.encode("utf-8")
        h = _vp()
        rc = _lib.wg_regex_to_optree(pattern, len(pattern), C.byref(h))
        if rc != WG_OK:
            raise WgError(rc, "wg_regex_to_optree: " + _lib.wg_regex_error().decode())
        try:
            n = [_i32() for _ in range(5)]
            _check(_lib.wg_optree_sizes(h, *[C.byref(x) for x in n]), "wg_optree_sizes")
            self.nodes = np.zeros((n[0].value, 8), np.int32)
            self.children = np.zeros(n[1].value, np.int32)
            self.sets = np.zeros((n[2].value, 9), np.uint32)
            self.data = np.zeros(n[3].value, np.uint8)
            self.root = n[4].value
            _check(_lib.wg_optree_copy(h, _np_ptr(self.nodes), _np_ptr(self.children),
                                       _np_ptr(self.sets), _np_ptr(self.data)), "wg_optree_copy")
        finally:
            _lib.wg_optree_free(h)

    @property
    def n_nodes(self) -> int:
        return int(self.nodes.shape[0])


class Grammar:
    """wg_compile_grammar: lowers a flat operator tree to a byte-level table (host side).

    ``Grammar.from_regex(pattern)`` goes through wg_compile_regex instead.
    """

    def __init__(self, flat=None, _handle=None):
        if _handle is None:
            nodes = np.ascontiguousarray(flat.nodes, np.int32)
            children = np.ascontiguousarray(flat.children, np.int32)
            sets = np.ascontiguousarray(flat.sets, np.uint32)
            data = np.ascontiguousarray(flat.data, np.uint8)
            _handle = _vp()
            _check(_lib.wg_compile_grammar(_np_ptr(nodes), nodes.shape[0], _np_ptr(children),
                                           children.shape[0], _np_ptr(sets), sets.shape[0],
                                           _np_ptr(data), data.shape[0], int(flat.root),
                                           C.byref(_handle)), "wg_compile_grammar")
        h = _handle
        self.handle = h
        n, s, d, c, hs = _i32(), _i32(), _i32(), _i32(), C.c_uint64()
        _check(_lib.wg_grammar_info(h, C.byref(n), C.byref(s), C.byref(d), C.byref(c), C.byref(hs)),
               "wg_grammar_info")
        self.n_states, self.start_state, self.done_state = n.value, s.value, d.value
        self.n_classes, self.content_hash = c.value, hs.value

    @classmethod
    def from_regex(cls, pattern, fragment: bool = False) -> "Grammar":
        """wg_compile_regex, or wg_compile_regex_fragment for a template argument."""
        if isinstance(pattern, str):
            pattern = pattern.encode("utf-8")
        h = _vp()
        fn = _lib.wg_compile_regex_fragment if fragment else _lib.wg_compile_regex
        rc = fn(pattern, len(pattern), C.byref(h))
        if rc != WG_OK:
            raise WgError(rc, "wg_compile_regex: " + _lib.wg_regex_error().decode())
        return cls(_handle=h)

    def save(self) -> bytes:
        """wg_grammar_save: the compiled table as a blob for wg_grammar_load."""
        need = C.c_size_t()
        _lib.wg_grammar_save(self.handle, None, 0, C.byref(need))
        buf = C.create_string_buffer(need.value)
        _check(_lib.wg_grammar_save(self.handle, buf, need.value, C.byref(need)), "wg_grammar_save")
        return buf.raw

    @classmethod
    def load(cls, blob: bytes) -> "Grammar":
        h = _vp()
        _check(_lib.wg_grammar_load(blob, len(blob), C.byref(h)), "wg_grammar_load")
        return cls(_handle=h)

    def minimized(self) -> "Grammar":
        """wg_grammar_minimize: the same language with equivalent states merged."""
        h = _vp()
        _check(_lib.wg_grammar_minimize(self.handle, C.byref(h)), "wg_grammar_minimize")
        return Grammar(_handle=h)

    def step(self, state: int, symbol: int) -> int:
        return int(_lib.wg_grammar_step(self.handle, int(state), int(symbol)))

    def forced_token(self, state: int):
        """(token id, next state) if ``state`` belongs to a token-level Write, else None."""
        tok, nxt = _i32(), _i32()
        if _lib.wg_grammar_forced_token(self.handle, int(state), C.byref(tok), C.byref(nxt)):
            return tok.value, nxt.value
        return None

    def step_token(self, state: int, token: int, symbols) -> int:
        """Host-side state after a whole token (``symbols`` = its bytes, or [256] for EOS)."""
        forced = self.forced_token(state)
        if forced is not None:
            return forced[1] if token == forced[0] else 0
        return self.walk(state, symbols)

    def walk(self, state: int, symbols) -> int:
        for s in symbols:
            state = self.step(state, s)
        return state

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.wg_grammar_free(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


class Template:
    """wg_template_compile: an operator tree with holes, lowered once; ``instantiate`` splices
    one compiled grammar per argument into the holes (wg_template_instantiate)."""

    def __init__(self, flat):
        nodes = np.ascontiguousarray(flat.nodes, np.int32)
        children = np.ascontiguousarray(flat.children, np.int32)
        sets = np.ascontiguousarray(flat.sets, np.uint32)
        data = np.ascontiguousarray(flat.data, np.uint8)
        h = _vp()
        _check(_lib.wg_template_compile(_np_ptr(nodes), nodes.shape[0], _np_ptr(children),
                                        children.shape[0], _np_ptr(sets), sets.shape[0],
                                        _np_ptr(data), data.shape[0], int(flat.root), C.byref(h)),
               "wg_template_compile")
        self.handle = h
        n, k, a = _i32(), _i32(), _i32()
        _check(_lib.wg_template_info(h, C.byref(n), C.byref(k), C.byref(a)), "wg_template_info")
        self.n_states, self.n_holes, self.n_args = n.value, k.value, a.value

    def instantiate(self, args) -> Grammar:
        args = list(args)
        arr = (_vp * max(1, len(args)))(*[g.handle for g in args])
        h = _vp()
        _check(_lib.wg_template_instantiate(self.handle, arr, len(args), C.byref(h)),
               "wg_template_instantiate")
        return Grammar(_handle=h)

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.wg_template_free(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


class Context:
    """wg_ctx: device tables, the mask cache and per-batch scratch."""

    def __init__(self, vocab: Vocab, cache_capacity: int, max_batch: int,
                 cache_mode: int = WG_CACHE_DENSE, arena_bytes: int = 0):
        self.vocab = vocab
        self.max_batch = int(max_batch)
        self.device = vocab.device
        h = _vp()
        if cache_mode == WG_CACHE_DENSE and not arena_bytes:
            _check(_lib.wg_ctx_create(vocab.handle, int(cache_capacity), int(max_batch),
                                      C.byref(h)), "wg_ctx_create")
        else:
            _check(_lib.wg_ctx_create_ex(vocab.handle, int(cache_capacity), int(max_batch),
                                         int(cache_mode), int(arena_bytes), C.byref(h)),
                   "wg_ctx_create_ex")
        self.handle = h

    def cache_entry(self, grammar_id: int, state: int, stream=None):
        """wg_cache_entry_read: (kind, sorted token ids, device bytes) of one compact cache
        entry, or None when the state is not cached."""
        kind, n, nbytes = _i32(), _i32(), _i64()
        ids = np.zeros(self.vocab.V, np.int32)
        _check(_lib.wg_cache_entry_read(self.handle, int(grammar_id), int(state), C.byref(kind),
                                        C.byref(n), _np_ptr(ids), ids.shape[0], C.byref(nbytes),
                                        _stream_ptr(stream)), "wg_cache_entry_read")
        if kind.value < 0:
            return None
        return kind.value, ids[:n.value].copy(), int(nbytes.value)

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.wg_ctx_free(self.handle)
            self.handle = None

    def __del__(self):
        self.close()

    def add_grammar(self, grammar: Grammar) -> int:
        gid = _i32()
        _check(_lib.wg_ctx_add_grammar(self.handle, grammar.handle, C.byref(gid)),
               "wg_ctx_add_grammar")
        return gid.value

    def remove_grammar(self, grammar_id: int) -> None:
        """Frees the grammar's tables and cached masks; the id goes to a grammar added later."""
        _check(_lib.wg_ctx_remove_grammar(self.handle, int(grammar_id)), "wg_ctx_remove_grammar")

    def cache_prewarm(self, grammar_id: int, stream=None) -> None:
        _check(_lib.wg_cache_prewarm(self.handle, int(grammar_id), _stream_ptr(stream)),
               "wg_cache_prewarm")

    def cache_clear(self, stream=None) -> None:
        _check(_lib.wg_cache_clear(self.handle, _stream_ptr(stream)), "wg_cache_clear")

    def stats(self, stream=None) -> dict:
        st = WgStats()
        _check(_lib.wg_get_stats(self.handle, C.byref(st), _stream_ptr(stream)), "wg_get_stats")
        return st.as_dict()

    def set_timing(self, enable: bool) -> None:
        _check(_lib.wg_ctx_set_timing(self.handle, int(bool(enable))), "wg_ctx_set_timing")

    def get_timing(self) -> dict:
        """Summed kernel milliseconds of the steps recorded since the last read."""
        b, a, n = C.c_double(), C.c_double(), _i64()
        _check(_lib.wg_ctx_get_timing(self.handle, C.byref(b), C.byref(a), C.byref(n)),
               "wg_ctx_get_timing")
        return {"build_ms": b.value, "apply_ms": a.value, "steps": int(n.value)}

    def count_build_work(self, enable: bool) -> None:
        _check(_lib.wg_ctx_count_build_work(self.handle, int(bool(enable))),
               "wg_ctx_count_build_work")

    def build_work(self, stream=None) -> dict:
        """Work counted by the build kernel's counting variant since the last reset_stats."""
        q, l, m = _i64(), _i64(), _i64()
        _check(_lib.wg_get_build_work(self.handle, C.byref(q), C.byref(l), C.byref(m),
                                      _stream_ptr(stream)), "wg_get_build_work")
        return {"tokens_walked": q.value, "table_lookups": l.value, "mask_words_read": m.value}

    def reset_stats(self, stream=None) -> None:
        _check(_lib.wg_reset_stats(self.handle, _stream_ptr(stream)), "wg_reset_stats")


def _logits_dtype(logits) -> int:
    import torch
    if logits.dtype == torch.bfloat16:
        return WG_DTYPE_BF16
    if logits.dtype == torch.float32:
        return WG_DTYPE_FP32
    raise TypeError(f"logits must be bfloat16 or float32, not {logits.dtype}")


def _rows(t, what: str):
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{what} must be 2-D with unit inner stride")
    return t.shape[0], t.stride(0)


def wg_mask_cache_lookup(ctx: Context, gid, sid, slot, stream=None) -> None:
    import torch
    B, dev = gid.shape[0], _device_of(ctx)
    _check(_lib.wg_mask_cache_lookup(ctx.handle, _vec(gid, B, torch.int32, "gid", dev),
                                     _vec(sid, B, torch.int32, "sid", dev), B,
                                     _vec(slot, B, torch.int32, "slot", dev), _stream_ptr(stream)),
           "wg_mask_cache_lookup")


def wg_build_masks(ctx: Context, gid, sid, bitmask, flags: int = WG_USE_CACHE, stream=None) -> None:
    import torch
    B, dev = bitmask.shape[0], _device_of(ctx)
    mask, stride = _mat(bitmask, B, ctx.vocab.W, (torch.int32, torch.uint32), "bitmask", dev)
    _check(_lib.wg_build_masks(ctx.handle, _vec(gid, B, torch.int32, "gid", dev),
                               _vec(sid, B, torch.int32, "sid", dev), B, mask, stride,
                               int(flags), _stream_ptr(stream)), "wg_build_masks")


def _apply_args(logits, bitmask, V: int, argmax_out):
    """Checked (logits pointer, dtype, stride, mask pointer, mask stride, B, token pointer)."""
    import torch
    if logits.dim() != 2:
        raise ValueError("logits must be 2-D with unit inner stride")
    B, V = logits.shape[0], int(V)
    dev = logits.device.index if logits.is_cuda else None
    lp, stride = _mat(logits, B, V, None, "logits", dev)
    mp, mstride = _mat(bitmask, B, (V + 31) // 32, (torch.int32, torch.uint32), "bitmask", dev)
    return lp, _logits_dtype(logits), stride, mp, mstride, B, V, \
        _vec(argmax_out, B, torch.int32, "argmax_out", dev), dev


def wg_apply_mask(logits, bitmask, V: int, argmax_out=None, workspace=None, stream=None) -> None:
    lp, dtype, stride, mp, mstride, B, V, tok, dev = _apply_args(logits, bitmask, V, argmax_out)
    ws = _dev_ptr(workspace, None, "workspace", dev)
    if argmax_out is not None:
        need = wg_apply_workspace_bytes(B)
        if workspace is None or not workspace.is_contiguous() or \
                workspace.numel() * workspace.element_size() < need:
            raise ValueError(f"workspace must be a contiguous device buffer of {need} bytes")
    _check(_lib.wg_apply_mask(lp, dtype, stride, mp, mstride, B, V, tok, ws, _stream_ptr(stream)),
           "wg_apply_mask")


WG_NOALLOC_MAX_ROWS = 4096


def wg_apply_mask_noalloc(logits, bitmask, V: int, argmax_out, stream=None) -> None:
    """Mask + greedy argmax for callers that may not allocate device memory.

    Same results as ``wg_apply_mask`` with ``argmax_out``; the scratch is a fixed 32 KB array
    inside the library, so at most ``WG_NOALLOC_MAX_ROWS`` rows per call, and calls that can
    overlap on the GPU must not be issued (they share that array).
    """
    if argmax_out is None:
        raise ValueError("argmax_out is required")
    lp, dtype, stride, mp, mstride, B, V, tok, _ = _apply_args(logits, bitmask, V, argmax_out)
    _check(_lib.wg_apply_mask_noalloc(lp, dtype, stride, mp, mstride, B, V, tok,
                                      _stream_ptr(stream)), "wg_apply_mask_noalloc")


def wg_apply_workspace_bytes(B: int) -> int:
    return int(_lib.wg_apply_workspace_bytes(int(B)))


def wg_advance(ctx: Context, gid, sid, token, status=None, flags: int = 0, stream=None) -> None:
    import torch
    B, dev = gid.shape[0], _device_of(ctx)
    _check(_lib.wg_advance(ctx.handle, _vec(gid, B, torch.int32, "gid", dev),
                           _vec(sid, B, torch.int32, "sid", dev),
                           _vec(token, B, torch.int32, "token", dev), B,
                           _vec(status, B, torch.int32, "status", dev), int(flags),
                           _stream_ptr(stream)), "wg_advance")


def _step_args(ctx: Context, gid, sid, logits, n_cols: int, bitmask, token_out, status):
    """The checked arrays of one decode step over ``logits.shape[0]`` rows."""
    import torch
    if logits.dim() != 2:
        raise ValueError("logits must be 2-D with unit inner stride")
    B, dev = logits.shape[0], _device_of(ctx)
    lp, stride = _mat(logits, B, n_cols, None, "logits", dev)
    mp, mstride = _mat(bitmask, B, ctx.vocab.W, (torch.int32, torch.uint32), "bitmask", dev)
    return (_vec(gid, B, torch.int32, "gid", dev), _vec(sid, B, torch.int32, "sid", dev), B, lp,
            _logits_dtype(logits), stride, mp, mstride,
            _vec(token_out, B, torch.int32, "token_out", dev),
            _vec(status, B, torch.int32, "status", dev))


def wg_decode_step(ctx: Context, gid, sid, logits, bitmask, token_out, status=None,
                   flags: int = WG_USE_CACHE, stream=None) -> None:
    """One decode step.  With ``token_out`` None the step only masks (no argmax, no advance): the
    caller samples from the masked logits and calls ``wg_advance``."""
    g, s, B, lp, dtype, stride, mp, mstride, tok, st = _step_args(
        ctx, gid, sid, logits, ctx.vocab.V, bitmask, token_out, status)
    if tok is None and (st is not None or int(flags) & WG_RESTART_ON_DONE):
        raise ValueError("a step without token_out advances nothing: no status, no WG_RESTART_ON_DONE")
    _check(_lib.wg_decode_step(ctx.handle, g, s, B, lp, dtype, stride, mp, mstride, tok, st,
                               int(flags), _stream_ptr(stream)), "wg_decode_step")


WG_SHARD_ALIGN = 8192


def wg_decode_step_shard(ctx: Context, gid, sid, logits_shard, bitmask, v_begin: int, v_end: int,
                         best_keys, flags: int = WG_USE_CACHE, stream=None) -> None:
    """The decode step on the vocabulary slice [v_begin, v_end); ``best_keys`` (int64, B) gets
    the packed per-row maxima to be MAX-reduced over the GPUs that hold the other slices."""
    import torch
    g, s, B, lp, dtype, stride, mp, mstride, _, _ = _step_args(
        ctx, gid, sid, logits_shard, max(int(v_end) - int(v_begin), 0), bitmask, None, None)
    _check(_lib.wg_decode_step_shard(
        ctx.handle, g, s, B, lp, dtype, stride, mp, mstride, int(v_begin), int(v_end),
        _vec(best_keys, B, torch.int64, "best_keys", _device_of(ctx)), int(flags),
        _stream_ptr(stream)), "wg_decode_step_shard")


def wg_advance_keys(ctx: Context, gid, sid, best_keys, token_out, status=None, flags: int = 0,
                    stream=None) -> None:
    import torch
    B, dev = gid.shape[0], _device_of(ctx)
    _check(_lib.wg_advance_keys(ctx.handle, _vec(gid, B, torch.int32, "gid", dev),
                                _vec(sid, B, torch.int32, "sid", dev),
                                _vec(best_keys, B, torch.int64, "best_keys", dev), B,
                                _vec(token_out, B, torch.int32, "token_out", dev),
                                _vec(status, B, torch.int32, "status", dev), int(flags),
                                _stream_ptr(stream)), "wg_advance_keys")


class StepPlan:
    """A wg_decode_step call with everything but the logits marshalled once.

    The per-call work of the binding (pointer extraction, dtype and shape checks) costs more
    than a small decode step takes on the GPU; a plan does it once for buffers that stay put
    (ids, states, bitmask, tokens, status) and only takes the logits tensor per call.
    """

    def __init__(self, ctx: Context, gid, sid, bitmask, token_out, status=None,
                 flags: int = WG_USE_CACHE, stream=None):
        import torch
        self._keep = (ctx, gid, sid, bitmask, token_out, status)
        self.B, dev = bitmask.shape[0], _device_of(ctx)
        if gid.shape[0] != self.B or sid.shape[0] != self.B or token_out.shape[0] != self.B:
            raise ValueError("gid, sid, token_out and bitmask disagree on the batch size")
        self._ctx = ctx.handle
        self._V, self._device = ctx.vocab.V, dev
        self._gid = _vec(gid, self.B, torch.int32, "gid", dev)
        self._sid = _vec(sid, self.B, torch.int32, "sid", dev)
        self._mask, self._mstride = _mat(bitmask, self.B, ctx.vocab.W, (torch.int32, torch.uint32),
                                         "bitmask", dev)
        self._tok = _vec(token_out, self.B, torch.int32, "token_out", dev)
        self._status = _vec(status, self.B, torch.int32, "status", dev)
        self._flags = int(flags)
        self._stream = _stream_ptr(stream)
        self._dtypes = {torch.bfloat16: WG_DTYPE_BF16, torch.float32: WG_DTYPE_FP32}
        self._fn = _lib.wg_decode_step

    def __call__(self, logits) -> None:
        if logits.dim() != 2 or logits.shape[0] != self.B or logits.shape[1] < self._V \
                or logits.stride(1) != 1 or not logits.is_cuda \
                or (self._device is not None and logits.device.index != self._device):
            raise ValueError("logits must be a tensor [B, V] with unit inner stride on the "
                             "context's device")
        rc = self._fn(self._ctx, self._gid, self._sid, self.B, logits.data_ptr(),
                      self._dtypes[logits.dtype], logits.stride(0), self._mask, self._mstride,
                      self._tok, self._status, self._flags, self._stream)
        if rc != WG_OK:
            raise WgError(rc, "wg_decode_step")


class StepGraph:
    """wg_step_graph: one decode step recorded as a CUDA graph for fixed buffers."""

    def __init__(self, ctx: Context, gid, sid, logits, bitmask, token_out, status=None,
                 flags: int = WG_USE_CACHE):
        self._keep = (ctx, gid, sid, logits, bitmask, token_out, status)
        g, s, B, lp, dtype, stride, mp, mstride, tok, st = _step_args(
            ctx, gid, sid, logits, ctx.vocab.V, bitmask, token_out, status)
        if tok is None:
            raise ValueError("token_out is required")
        h = _vp()
        _check(_lib.wg_step_graph_create(ctx.handle, g, s, B, lp, dtype, stride, mp, mstride, tok, st,
                                         int(flags), C.byref(h)), "wg_step_graph_create")
        self.handle = h
        self._launch = _lib.wg_step_graph_launch

    def launch(self, stream=None) -> None:
        rc = self._launch(self.handle, _stream_ptr(stream))
        if rc != WG_OK:
            raise WgError(rc, "wg_step_graph_launch")

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.wg_step_graph_free(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


def wg_decode_step_host(ctx: Context, gid, sid, logits_host, logits_dev, bitmask, token_dev,
                        token_host, status=None, flags: int = WG_USE_CACHE, stream=None) -> None:
    """logits_host / token_host are CPU tensors (pinned for asynchronous copies)."""
    g, s, B, lp, dtype, stride, mp, mstride, tok, st = _step_args(
        ctx, gid, sid, logits_dev, ctx.vocab.V, bitmask, token_dev, status)
    if tok is None:
        raise ValueError("token_dev is required")
    if logits_host.is_cuda or token_host.is_cuda or not logits_host.is_contiguous() \
            or not token_host.is_contiguous():
        raise TypeError("logits_host and token_host must be contiguous CPU tensors")
    if logits_host.dim() != 2 or logits_host.shape[0] < B or logits_host.shape[1] != ctx.vocab.V \
            or logits_host.dtype != logits_dev.dtype:
        raise ValueError("logits_host must hold B rows of V elements of the device dtype")
    if token_host.numel() < B or token_host.element_size() != 4:
        raise ValueError("token_host must hold B 32-bit integers")
    _check(_lib.wg_decode_step_host(
        ctx.handle, g, s, B, C.c_void_p(logits_host.data_ptr()), lp, dtype, stride, mp, mstride,
        tok, C.c_void_p(token_host.data_ptr()), st, int(flags), _stream_ptr(stream)),
        "wg_decode_step_host")


_torch_c = None      # torch._C, looked up once (an import statement is 65 ns at every call)


def _on_stream(stream, device: int):
    """The raw stream of a call whose arrays are on ``device``: the given one, else the device's current one (asked
    for by number: making a stream object costs more than a small launch).  A launch goes to the current
    device, and a default stream has the same handle on all of them, so that device has to be the current one."""
    global _torch_c
    if _torch_c is None:
        import torch
        _torch_c = torch._C
    if _torch_c._cuda_getDevice() != device:
        raise ValueError(f"the call's arrays are on cuda:{device}, which is not the current device")
    if stream is not None:
        return stream.cuda_stream
    return _torch_c._cuda_getCurrentRawStream(device)


# ---- constrained beam search ---------------------------------------------------------------------
class Beam:
    """wg_beam: scratch of the selection for up to ``max_requests`` requests of ``max_beams`` beams."""

    def __init__(self, V: int, max_requests: int, max_beams: int, max_out: Optional[int] = None):
        import torch
        self.V, self.max_requests, self.max_beams = int(V), int(max_requests), int(max_beams)
        self.max_out = int(max_beams if max_out is None else max_out)
        self.device = torch.cuda.current_device()
        h = _vp()
        _check(_lib.wg_beam_create(self.V, self.max_requests, self.max_beams, self.max_out, C.byref(h)),
               "wg_beam_create")
        self.handle = h

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.wg_beam_free(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


def _beam_rows(n_beam: int, rows: int):
    n_beam = int(n_beam)
    if n_beam < 1 or rows < 1 or rows % n_beam:
        raise ValueError(f"{rows} rows are no whole number of requests of {n_beam} beams")
    return rows // n_beam, n_beam


def _beam_out(t, n_req: int, dtype, what: str, device):
    """(pointer, entries per request) of a contiguous [n_req, n_out] output."""
    p = _dev_ptr(t, dtype, what, device)
    if t.dim() != 2 or not t.is_contiguous() or t.shape[0] != n_req:
        raise ValueError(f"{what} must be a contiguous tensor of {n_req} rows")
    return p, int(t.shape[1])


class BeamPlan:
    """A wg_beam_select call with everything but the logits marshalled once (see ``StepPlan``).

    ``score`` (and ``finished``) hold one entry per row, ``score_out``, ``parent_out`` and ``token_out``
    are ``[n_req, n_out]``; the arrays are kept and read or written by every call.  Without ``stream``
    a call goes to the stream that is current when it is made.
    """

    def __init__(self, beam: Beam, n_beam: int, score, score_out, parent_out, token_out, bitmask=None,
                 finished=None, eos_id: int = 0, norm: int = WG_BEAM_NORM_ALLOWED, stream=None):
        import torch
        self._keep = (score, score_out, parent_out, token_out, bitmask, finished)
        dev = beam.device
        rows = int(score.numel())
        self.n_req, self.n_beam = _beam_rows(n_beam, rows)
        self.rows, self._V, self._device = rows, beam.V, dev
        so, n_out = _beam_out(score_out, self.n_req, torch.float32, "score_out", dev)
        po, n_p = _beam_out(parent_out, self.n_req, torch.int32, "parent_out", dev)
        to, n_t = _beam_out(token_out, self.n_req, torch.int32, "token_out", dev)
        if not n_out == n_p == n_t:
            raise ValueError("score_out, parent_out and token_out disagree on the candidates per request")
        mask, mstride = (None, 0) if bitmask is None else \
            _mat(bitmask, rows, (beam.V + 31) // 32, (torch.int32, torch.uint32), "bitmask", dev)
        if finished is not None and not 0 <= int(eos_id) < beam.V:
            raise ValueError(f"eos_id {eos_id} is not in the vocabulary")
        self._beam = beam                # (its handle is asked for at every call: none once it is closed)
        self._tail = (mask, mstride, _vec(score, rows, torch.float32, "score", dev),
                      _vec(finished, rows, torch.int32, "finished", dev), int(eos_id), self.n_req,
                      self.n_beam, n_out, int(norm), so, po, to)
        self._stream = stream
        self._dtypes = {torch.bfloat16: WG_DTYPE_BF16, torch.float32: WG_DTYPE_FP32}
        self._fn = _lib.wg_beam_select

    def __call__(self, logits) -> None:
        if logits.dim() != 2 or logits.shape[0] != self.rows or logits.shape[1] < self._V \
                or logits.stride(1) != 1 or not logits.is_cuda or logits.device.index != self._device:
            raise ValueError("logits must be a tensor [rows, V] with unit inner stride on the beam's device")
        if logits.dtype not in self._dtypes:
            raise TypeError(f"logits must be bfloat16 or float32, not {logits.dtype}")
        rc = self._fn(self._beam.handle, logits.data_ptr(), self._dtypes[logits.dtype], logits.stride(0), *self._tail,
                      _on_stream(self._stream, self._device))
        if rc != WG_OK:
            raise WgError(rc, "wg_beam_select")


def wg_beam_select(beam: Beam, n_beam: int, logits, score, score_out, parent_out, token_out, bitmask=None,
                   finished=None, eos_id: int = 0, norm: int = WG_BEAM_NORM_ALLOWED, stream=None) -> None:
    """One selection: the best candidates of every request over its beams and the vocabulary."""
    BeamPlan(beam, n_beam, score, score_out, parent_out, token_out, bitmask, finished, eos_id, norm, stream)(logits)


def wg_beam_step(beam: Beam, ctx: Context, n_beam: int, gid, sid, score, logits, bitmask, parent_out, token_out,
                 status=None, norm: int = WG_BEAM_NORM_ALLOWED, flags: int = WG_USE_CACHE, stream=None) -> None:
    """One decode step of a beam search under grammars: masks, selection, and the rows' grammars, states
    and scores after it (in place)."""
    import torch
    g, s, rows, lp, dtype, stride, mp, mstride, tok, st = _step_args(
        ctx, gid, sid, logits, ctx.vocab.V, bitmask, token_out, status)
    if tok is None or parent_out is None:
        raise ValueError("parent_out and token_out are required")
    n_req, n_beam = _beam_rows(n_beam, rows)
    dev = _device_of(ctx)
    if beam.device != dev:
        raise ValueError(f"the beam's scratch is on cuda:{beam.device}, the context on cuda:{dev}")
    _check(_lib.wg_beam_step(beam.handle, ctx.handle, g, s, _vec(score, rows, torch.float32, "score", dev), n_req,
                             n_beam, lp, dtype, stride, mp, mstride, int(norm),
                             _vec(parent_out, rows, torch.int32, "parent_out", dev), tok, st, int(flags),
                             _on_stream(stream, dev)), "wg_beam_step")


def wg_beam_backtrack(token, parent, out, stream=None) -> None:
    """``token``, ``parent``: [n_steps, n_req, n_beam] as the steps returned them; ``out``:
    [n_req, n_beam, n_steps], the sequence of every final beam."""
    import torch
    shape, dev, int32 = token.shape, token.device.index, torch.int32
    if len(shape) != 3 or parent.shape != shape:
        raise ValueError("token and parent must be [n_steps, n_req, n_beam]")
    T, R, K = shape
    if out.shape != (R, K, T):
        raise ValueError(f"out must be [{R}, {K}, {T}]")
    for t, what in ((token, "token"), (parent, "parent"), (out, "out")):
        if not t.is_cuda or t.dtype is not int32:
            raise TypeError(f"{what} must be an int32 CUDA tensor")
        if t.device.index != dev or not t.is_contiguous():
            raise ValueError(f"{what} must be contiguous, all on one device")
    _check(_lib.wg_beam_backtrack(token.data_ptr(), parent.data_ptr(), T, R, K, out.data_ptr(),
                                  _on_stream(stream, dev)), "wg_beam_backtrack")


# ---- block tables of a paged cache ---------------------------------------------------------------
class _PoolHandle:
    """Owns the library's pool object: freed when neither the pool nor a view of its counts is left."""

    def __init__(self, n_blocks: int, block_size: int, max_seqs: int):
        self.value = None
        h = _vp()
        _check(_lib.wg_kv_pool_create(n_blocks, block_size, max_seqs, C.byref(h)), "wg_kv_pool_create")
        self.value = h

    def __del__(self):
        if self.value and _lib is not None:
            _lib.wg_kv_pool_free(self.value)
            self.value = None


class _DeviceArray:
    """A library-owned int32 array for ``torch.as_tensor``, which makes a view of it and keeps this
    object, and with it the memory, for as long as the view lives."""

    def __init__(self, owner, ptr: int, n: int):
        self._owner = owner
        self.__cuda_array_interface__ = {"data": (ptr, False), "shape": (n,), "typestr": "<i4", "version": 2}


class KvPool:
    """wg_kv_pool: the blocks of a paged cache, counted by the table rows that name them.

    ``ref`` is an int32 [n_blocks] view of the counts, to be read only."""

    def __init__(self, n_blocks: int, block_size: int, max_seqs: int):
        import torch
        self.n_blocks, self.block_size, self.max_seqs = int(n_blocks), int(block_size), int(max_seqs)
        self.device = torch.cuda.current_device()
        self._owner = _PoolHandle(self.n_blocks, self.block_size, self.max_seqs)
        self.handle = self._owner.value
        self.ref = torch.as_tensor(_DeviceArray(self._owner, _lib.wg_kv_pool_refs(self.handle), self.n_blocks),
                                   device=f"cuda:{self.device}")

    def load(self, ref, stream=None) -> None:
        """Sets the counts from an int32 device tensor (a saved ``ref``)."""
        import torch
        _check(_lib.wg_kv_pool_load(self.handle, _vec(ref, self.n_blocks, torch.int32, "ref", self.device),
                                    _on_stream(stream, self.device)), "wg_kv_pool_load")

    def n_free(self, stream=None) -> int:
        n = _i32()
        _check(_lib.wg_kv_pool_n_free(self.handle, C.byref(n), _on_stream(stream, self.device)), "wg_kv_pool_n_free")
        return n.value


class SlotMap:
    """Where a step's tokens go: ``cu`` [n_seq + 1], and per token ``slot`` (int64), ``pos`` and ``seq``."""

    def __init__(self, n_seq: int, n_tokens: int, device=None):
        import torch
        dev = torch.device("cuda", torch.cuda.current_device() if device is None else int(device))
        self.n_seq, self.n_tokens, self.device = int(n_seq), int(n_tokens), dev.index
        self.cu = torch.zeros(self.n_seq + 1, dtype=torch.int32, device=dev)
        self.slot = torch.full((self.n_tokens,), -1, dtype=torch.int64, device=dev)
        self.pos = torch.full((self.n_tokens,), -1, dtype=torch.int32, device=dev)
        self.seq = torch.full((self.n_tokens,), -1, dtype=torch.int32, device=dev)
        self._args = tuple(C.c_void_p(t.data_ptr()) for t in (self.cu, self.slot, self.pos, self.seq)) \
            + (self.n_tokens,)


class KvPlanes:
    """The cache arrays that follow a reorder: CUDA tensors ``[n_blocks, block_size, ...]``, contiguous
    (e.g. the keys and the values of every layer, and their scales)."""

    def __init__(self, planes, block_size: int):
        import torch
        self.planes = list(planes)
        self.block_size = int(block_size)
        if not self.planes:
            raise ValueError("no planes")
        self.device = self.planes[0].device.index
        self.n_blocks = int(self.planes[0].shape[0])
        rows = []
        for i, t in enumerate(self.planes):
            if not t.is_cuda or t.device.index != self.device:
                raise ValueError(f"plane {i} is not on cuda:{self.device}")
            if t.dim() < 2 or not t.is_contiguous() or t.shape[0] != self.n_blocks \
                    or t.shape[1] != self.block_size:
                raise ValueError(f"plane {i} must be contiguous [n_blocks, block_size, ...]")
            rows.append([t.data_ptr(), t.numel() // (self.n_blocks * self.block_size) * t.element_size()])
        self._table = torch.tensor(rows, dtype=torch.int64).to(f"cuda:{self.device}")
        self._args = (C.c_void_p(self._table.data_ptr()), len(rows))


class KvTables:
    """Block tables ``table`` [n_seq, max_blocks] and lengths ``lens`` [n_seq] (int32, updated in place)
    over a pool; ``status`` [n_seq] gets the calls' per-sequence results.  Pointers are taken once: the
    tensors must stay where they are."""

    def __init__(self, pool: KvPool, table, lens, status=None):
        import torch
        dev = pool.device
        self._i32 = torch.int32
        self.pool, self.table, self.lens, self.status, self.device = pool, table, lens, status, dev
        self.n_seq = int(table.shape[0])
        if self.n_seq > pool.max_seqs:
            raise ValueError(f"{self.n_seq} sequences, the pool takes {pool.max_seqs}")
        tp, stride = _mat(table, self.n_seq, 1, torch.int32, "table", dev)
        self._head = (pool.handle, tp, stride, int(table.shape[1]),
                      _vec(lens, self.n_seq, torch.int32, "lens", dev))
        self._status = _vec(status, self.n_seq, torch.int32, "status", dev)

    def _rows(self, t, what):
        if not t.is_cuda or t.dtype != self._i32 or not t.is_contiguous() or t.numel() != self.n_seq \
                or t.device.index != self.device:
            raise ValueError(f"{what} must be a contiguous int32 tensor of {self.n_seq} entries on "
                             f"cuda:{self.device}")
        return t.data_ptr()

    def extend(self, n_new, slots: SlotMap, stream=None) -> None:
        """wg_kv_extend: room for ``n_new`` [n_seq] more tokens; ``slots`` says where they go."""
        if slots.n_seq != self.n_seq or slots.device != self.device:
            raise ValueError("slots were made for another batch or device")
        rc = _lib.wg_kv_extend(*self._head, self._rows(n_new, "n_new"), self.n_seq, *slots._args, self._status,
                               _on_stream(stream, self.device))
        if rc != WG_OK:
            raise WgError(rc, "wg_kv_extend")

    def shrink(self, keep, status=None, stream=None) -> None:
        """wg_kv_shrink: cuts the sequences to ``keep`` [n_seq] tokens.  ``status``, where given, gets
        WG_ERR_ARG for a ``keep`` outside 0 .. the sequence's length (which is then left alone)."""
        st = self._rows(status, "status") if status is not None else None
        rc = _lib.wg_kv_shrink(*self._head, self._rows(keep, "keep"), self.n_seq, st, _on_stream(stream, self.device))
        if rc != WG_OK:
            raise WgError(rc, "wg_kv_shrink")

    def reorder(self, parent, planes: Optional[KvPlanes] = None, copy_src=None, copy_dst=None,
                stream=None) -> None:
        """wg_kv_reorder: ``parent`` [n_req, n_beam] as a selection returned it."""
        if parent.dim() != 2:
            raise ValueError("parent must be [n_req, n_beam]")
        if planes is not None and (planes.block_size != self.pool.block_size or planes.n_blocks < self.pool.n_blocks
                                   or planes.device != self.device):
            raise ValueError("planes were made for another pool")
        n_req, n_beam = parent.shape
        rc = _lib.wg_kv_reorder(*self._head, self._rows(parent, "parent"), n_req, n_beam,
                                *((None, 0) if planes is None else planes._args),
                                None if copy_src is None else self._rows(copy_src, "copy_src"),
                                None if copy_dst is None else self._rows(copy_dst, "copy_dst"), self._status,
                                _on_stream(stream, self.device))
        if rc != WG_OK:
            raise WgError(rc, "wg_kv_reorder")


# ---- what a paged cache holds --------------------------------------------------------------------
class Rope:
    """The cosines and sines of rotary positions 0 .. n_pos - 1 (wg_rope_table), on the current device; ready for every
    stream when the constructor returns.

    The first ``rot_dim`` dimensions of a head are rotated in pairs (i, i + rot_dim / 2), or (2i, 2i + 1) if
    ``interleaved``.  For contexts longer than the model was trained on, ``factor`` slows the rotation down: all of it,
    or, with ``original`` (the positions trained on), ``low`` and ``high``, only that of pairs that turn less than ``high`` times
    within ``original`` positions (those below ``low`` in full).  ``magnitude`` multiplies what is rotated."""

    def __init__(self, n_pos: int, rot_dim: int, base: float = 10000.0, interleaved: bool = False, factor: float = 1.0,
                 low: float = 0.0, high: float = 0.0, original: float = 0.0, magnitude: float = 1.0):
        import torch
        self.n_pos, self.rot_dim, self.interleaved = int(n_pos), int(rot_dim), bool(interleaved)
        if self.rot_dim < 16 or self.rot_dim % 16:
            raise ValueError(f"rot_dim must be a multiple of 16, not {rot_dim}")
        if self.n_pos < 1:
            raise ValueError(f"{n_pos} positions")
        freq = np.zeros(self.rot_dim // 2, np.float64)
        if self.rot_dim > WG_KV_MAX_HEAD_DIM:
            raise ValueError(f"rot_dim is at most {WG_KV_MAX_HEAD_DIM}")
        _check(_lib.wg_rope_frequencies(self.rot_dim, float(base), float(factor), float(original), float(low), float(high),
                                        _np_ptr(freq)), "wg_rope_frequencies")
        self.frequencies = freq
        self.device = torch.cuda.current_device()
        self.table = torch.empty((self.n_pos, self.rot_dim), dtype=torch.float32, device=f"cuda:{self.device}")
        _check(_lib.wg_rope_table(_np_ptr(freq), self.rot_dim // 2, self.n_pos, float(magnitude),
                                  _dev_ptr(self.table), _stream_ptr(None)), "wg_rope_table")
        torch.cuda.current_stream().synchronize()
        self._struct = _WgRope(self.table.data_ptr(), self.n_pos, self.rot_dim, int(self.interleaved))
        self._arg = C.addressof(self._struct)


_model_dtypes = {}      # filled when torch is there (see _on_stream)
_float32 = None


def _model_dtype(t, what: str) -> int:
    global _float32
    if not _model_dtypes:
        import torch
        _float32 = torch.float32
        _model_dtypes.update({torch.bfloat16: WG_DTYPE_BF16, torch.float16: WG_DTYPE_FP16})
    kind = _model_dtypes.get(t.dtype)
    if kind is None:
        raise TypeError(f"{what} must be bfloat16 or float16, not {t.dtype}")
    return kind


def _heads(t, n: int, heads: int, dim: int, dtype, device: int, what: str):
    """(pointer, elements from token to token) of a [n, heads, dim] array whose tokens are whole: 16-byte aligned rows
    of heads * dim elements without gaps, any distance apart."""
    if t.dtype is not dtype:
        raise TypeError(f"{what} must be a CUDA tensor of {dtype}")
    if t.get_device() != device:
        raise ValueError(f"{what} must be on cuda:{device}, as the cache is")
    if t.shape != (n, heads, dim):
        raise ValueError(f"{what} must be [{n}, {heads}, {dim}], not {list(t.shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1 or (s1 != dim and heads > 1):
        raise ValueError(f"the heads of a token of {what} must follow each other without gaps")
    if n < 2:
        s0 = heads * dim
    p = t.data_ptr()
    if p & 15 or s0 & 7 or s0 < heads * dim:
        raise ValueError(f"the tokens of {what} must begin at multiples of 16 bytes and not overlap")
    return p, s0


class KvCache:
    """wg_kv_cache: keys and values, ``[n_blocks, block_size, n_heads, head_dim]`` contiguous CUDA tensors of bfloat16,
    float16, float8_e4m3fn or int8, the last two with float32 scales ``[n_blocks, block_size, n_heads]``.

    The tensors are kept and must stay where they are.  ``planes`` are the same arrays for ``KvTables.reorder``."""

    def __init__(self, keys, values, key_scale=None, value_scale=None):
        import torch
        storages = {torch.bfloat16: WG_KV_BF16, torch.float16: WG_KV_FP16, torch.float8_e4m3fn: WG_KV_E4M3, torch.int8: WG_KV_INT8}
        if keys.dtype not in storages or values.dtype is not keys.dtype:
            raise TypeError("keys and values must both be bfloat16, float16, float8_e4m3fn or int8")
        if keys.dim() != 4 or tuple(values.shape) != tuple(keys.shape):
            raise ValueError("keys and values must both be [n_blocks, block_size, n_heads, head_dim]")
        self.n_blocks, self.block_size, self.n_heads, self.head_dim = (int(n) for n in keys.shape)
        if self.head_dim < 16 or self.head_dim % 16 or self.head_dim > WG_KV_MAX_HEAD_DIM:
            raise ValueError(f"head_dim must be a multiple of 16 up to {WG_KV_MAX_HEAD_DIM}, not {self.head_dim}")
        if min(self.n_blocks, self.block_size, self.n_heads) < 1:
            raise ValueError("an empty cache")
        self.storage, self.dtype = storages[keys.dtype], keys.dtype
        narrow = self.storage >= WG_KV_E4M3
        if (key_scale is not None) != narrow or (value_scale is not None) != narrow:
            raise ValueError("8-bit caches, and no others, have key_scale and value_scale")
        self.device = keys.device.index
        for t, what in ((keys, "keys"), (values, "values"), (key_scale, "key_scale"), (value_scale, "value_scale")):
            if t is None:
                continue
            if not t.is_cuda or t.device.index != self.device or not t.is_contiguous() or t.data_ptr() & 15:
                raise ValueError(f"{what} must be contiguous, 16-byte aligned, and on the keys' CUDA device")
            if what.endswith("scale") and (t.dtype is not torch.float32 or tuple(t.shape) != tuple(keys.shape[:3])):
                raise ValueError(f"{what} must be float32 [n_blocks, block_size, n_heads]")
        self.keys, self.values, self.key_scale, self.value_scale = keys, values, key_scale, value_scale
        ptr = [None if t is None else t.data_ptr() for t in (keys, values, key_scale, value_scale)]
        self._struct = _WgKvCache(*ptr, self.storage, self.n_blocks, self.block_size, self.n_heads, self.head_dim)
        self._arg = C.addressof(self._struct)
        self._planes = None

    @classmethod
    def empty(cls, n_blocks: int, block_size: int, n_heads: int, head_dim: int, dtype) -> "KvCache":
        """A cache of zeros on the current device."""
        import torch
        shape = (int(n_blocks), int(block_size), int(n_heads), int(head_dim))
        planes = [torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(2)]
        if dtype in (torch.float8_e4m3fn, torch.int8):
            planes += [torch.ones(shape[:3], dtype=torch.float32, device="cuda") for _ in range(2)]
        return cls(*planes)

    @property
    def planes(self) -> "KvPlanes":
        if self._planes is None:
            self._planes = KvPlanes([t for t in (self.keys, self.values, self.key_scale, self.value_scale) if t is not None],
                                    self.block_size)
        return self._planes

    def write(self, k, v, slots: SlotMap, rope: Optional[Rope] = None, q=None, q_out=None, status=None, stream=None) -> None:
        """wg_kv_write: the tokens of ``slots`` into the cache.  ``k``, ``v`` are ``[n_tokens, n_heads, head_dim]`` (views into
        a fused projection will do), ``q`` and ``q_out`` ``[n_tokens, query heads, head_dim]``; without ``q_out`` the queries
        are rotated in place; without ``rope`` nothing is rotated.  ``status`` [n_tokens] gets WG_ERR_ARG for slots outside the cache and positions outside ``rope``."""
        n, dev, dtype = slots.n_tokens, self.device, k.dtype
        kind = _model_dtype(k, "k")
        if self.storage <= WG_KV_FP16 and dtype is not self.dtype:
            raise TypeError(f"k is {dtype}, the cache holds {self.dtype}")
        if slots.device != dev:
            raise ValueError(f"slots live on cuda:{slots.device}, the cache on cuda:{dev}")
        kp, ks = _heads(k, n, self.n_heads, self.head_dim, dtype, dev, "k")
        vp, vs = _heads(v, n, self.n_heads, self.head_dim, dtype, dev, "v")
        qp = qs = op = os_ = None
        heads = 0
        if q is not None:
            heads = int(q.shape[1]) if q.dim() == 3 else 0
            if heads < 1:
                raise ValueError("q must be [n_tokens, query heads, head_dim]")
            qp, qs = _heads(q, n, heads, self.head_dim, dtype, dev, "q")
            op, os_ = (qp, qs) if q_out is None else _heads(q_out, n, heads, self.head_dim, dtype, dev, "q_out")
        elif q_out is not None:
            raise ValueError("q_out without q")
        if rope is not None:
            if rope.device != dev:
                raise ValueError(f"rope lives on cuda:{rope.device}, the cache on cuda:{dev}")
            if rope.rot_dim > self.head_dim:
                raise ValueError(f"rope rotates {rope.rot_dim} dimensions, a head has {self.head_dim}")
        if status is not None:
            import torch
            status = _vec(status, n, torch.int32, "status", dev)
        _, slot, pos, _ = slots._args[:4]
        rc = _lib.wg_kv_write(self._arg, kp, ks, vp, vs, qp, qs or 0, op, os_ or 0, heads, kind,
                              None if rope is None else rope._arg, slot, pos, n, status, _on_stream(stream, dev))
        if rc != WG_OK:
            raise WgError(rc, "wg_kv_write")

    def _check_tables(self, tables: "KvTables") -> None:
        pool = tables.pool
        if pool.block_size != self.block_size or pool.n_blocks > self.n_blocks or tables.device != self.device:
            raise ValueError("tables were made for another cache")

    def read(self, tables: "KvTables", cu, k_out=None, v_out=None, stream=None) -> None:
        """wg_kv_read: position p of sequence s goes to row ``cu[s] + p`` of ``k_out`` and ``v_out``, contiguous
        ``[rows, n_heads, head_dim]`` of bfloat16, float16 or float32.  ``cu``: int32 [n_seq + 1], the sums of the lengths."""
        import torch
        self._check_tables(tables)
        outs = [t for t in (k_out, v_out) if t is not None]
        if not outs:
            raise ValueError("neither k_out nor v_out")
        kinds = {torch.bfloat16: WG_DTYPE_BF16, torch.float16: WG_DTYPE_FP16, torch.float32: WG_DTYPE_FP32}
        dtype, rows, dev = outs[0].dtype, int(outs[0].shape[0]), self.device
        if dtype not in kinds:
            raise TypeError(f"outputs must be bfloat16, float16 or float32, not {dtype}")
        for t in outs:
            if not t.is_cuda or t.dtype is not dtype or t.device.index != dev or not t.is_contiguous() \
                    or tuple(t.shape) != (rows, self.n_heads, self.head_dim) or t.data_ptr() & 15:
                raise ValueError("outputs must be alike: contiguous [rows, n_heads, head_dim], 16-byte aligned, on the cache's device")
        _, table, stride, max_blocks, lens = tables._head
        rc = _lib.wg_kv_read(self._arg, table, stride, max_blocks, lens, tables.n_seq,
                             _vec(cu, tables.n_seq + 1, torch.int32, "cu", dev), None if k_out is None else k_out.data_ptr(),
                             None if v_out is None else v_out.data_ptr(), kinds[dtype], rows, _on_stream(stream, dev))
        if rc != WG_OK:
            raise WgError(rc, "wg_kv_read")


class Attend:
    """wg_attend: scratch of the attention over a paged cache, for up to ``max_tokens`` tokens a call."""

    def __init__(self, max_tokens: int, n_q_heads: int, n_heads: int, head_dim: int):
        import torch
        self.max_tokens, self.n_q_heads, self.n_heads, self.head_dim = int(max_tokens), int(n_q_heads), int(n_heads), int(head_dim)
        self.device = torch.cuda.current_device()
        self.scale = max(1, self.head_dim) ** -0.5
        h = _vp()
        _check(_lib.wg_attend_create(self.max_tokens, self.n_q_heads, self.n_heads, self.head_dim, C.byref(h)), "wg_attend_create")
        self.handle = h

    def close(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.wg_attend_free(self.handle)
            self.handle = None

    def __del__(self):
        self.close()

    def __call__(self, q, cache: KvCache, tables: KvTables, out, slots: Optional[SlotMap] = None, scale: Optional[float] = None,
                 window: int = 0, group: int = 1, lse=None, stream=None) -> None:
        """wg_kv_attend: ``q`` and ``out`` are ``[n_tokens, n_q_heads, head_dim]``, ``lse`` float32 ``[n_tokens, n_q_heads]``.

        With ``slots`` (the map that placed the step's tokens) row t is token t of the map; without, row t is the last
        token of sequence t.  ``scale`` is 1 / sqrt(head_dim) if it is not given.  ``group``: so many neighbouring tokens, the beams of a
        request or the drafted tokens of a sequence, read what their tables have in common together."""
        cache._check_tables(tables)
        dev = self.device
        if cache.device != dev or cache.n_heads != self.n_heads or cache.head_dim != self.head_dim:
            raise ValueError("the scratch was made for another device, number of heads or head size")
        n = tables.n_seq if slots is None else slots.n_tokens
        if slots is None and q.shape[0] <= n:
            n = int(q.shape[0])
        if n > self.max_tokens:
            raise ValueError(f"{n} tokens, the scratch takes {self.max_tokens}")
        if slots is not None and (slots.device != dev or slots.n_seq != tables.n_seq):
            raise ValueError("slots were made for another batch or device")
        dtype, kind = q.dtype, _model_dtype(q, "q")
        if cache.storage <= WG_KV_FP16 and dtype is not cache.dtype:
            raise TypeError(f"q is {dtype}, the cache holds {cache.dtype}")
        qp, qs = _heads(q, n, self.n_q_heads, self.head_dim, dtype, dev, "q")
        op, os_ = _heads(out, n, self.n_q_heads, self.head_dim, dtype, dev, "out")
        if lse is not None:
            if lse.dtype is not _float32 or lse.get_device() != dev or lse.shape != (n, self.n_q_heads) or not lse.is_contiguous():
                raise ValueError(f"lse must be a contiguous float32 tensor [{n}, {self.n_q_heads}] on cuda:{dev}")
            lse = lse.data_ptr()
        _, table, stride, max_blocks, lens = tables._head
        _, slot, pos, seq = (None,) * 4 if slots is None else slots._args[:4]
        rc = _lib.wg_kv_attend(self.handle, cache._arg, qp, qs, op, os_, lse, kind, self.n_q_heads, table, stride, max_blocks, lens,
                               tables.n_seq, seq, pos, slot, n, self.scale if scale is None else float(scale), int(window),
                               int(group), _on_stream(stream, dev))
        if rc != WG_OK:
            raise WgError(rc, "wg_kv_attend")
