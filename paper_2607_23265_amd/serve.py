"""Python binding of the serving operators (include/wavezip_serve.h): argument marshalling only, in csrc/serve_py.cpp.

A paged key/value cache held in 8 bits, attention over it, and products in 8-bit integers, for a language model that
reads the tokens wavezip.condense() keeps.  Tensors are torch GPU tensors; every call goes to the current HIP stream
of their device.  Where a tensor has rows of heads ([tokens, heads, head_dim]) its rows may lie apart, so parts of one
fused projection are passed as they are; everything else is contiguous.
"""
import ctypes
import operator
import struct

import torch

from . import wavezip as wz

EXPORTS = ("wz_cache_append", "wz_cache_attention", "wz_attention_workspace_bytes", "wz_quantize_rows",
           "wz_matmul_int")
E4M3 = torch.float8_e4m3fn
_P, _I, _L, _S = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t

# For calls of the C entry points by ctypes (lib()): the header's structs as bytes, and below as ctypes.Structure.  The
# functions at the end of this module go through the native half, which packs structs of its own.
_CACHE = struct.Struct("@4P4i").pack      # wz_cache
_RAGGED = struct.Struct("@3P5i4x").pack   # wz_ragged
_ROTATION = struct.Struct("@2P7i4x").pack  # wz_rotation
_ATTENTION = struct.Struct("@3if").pack   # wz_attention


class _Cache(ctypes.Structure):
    """Mirror of wz_cache."""
    _fields_ = [("k", _P), ("v", _P), ("k_scale", _P), ("v_scale", _P), ("pages", _I), ("kv_heads", _I),
                ("page_size", _I), ("head_dim", _I)]


class _Ragged(ctypes.Structure):
    """Mirror of wz_ragged."""
    _fields_ = [("start", _P), ("kv_len", _P), ("table", _P), ("batch", _I), ("tokens", _I), ("max_tokens", _I),
                ("max_kv", _I), ("table_stride", _I)]


class _Rotation(ctypes.Structure):
    """Mirror of wz_rotation."""
    _fields_ = [("table", _P), ("positions", _P), ("max_pos", _I), ("rot_dim", _I), ("axes", _I),
                ("interleaved", _I), ("sections", _I * 3)]


class _Attention(ctypes.Structure):
    """Mirror of wz_attention."""
    _fields_ = [("q_heads", _I), ("causal", _I), ("window", _I), ("scale", ctypes.c_float)]


_lib = None


def lib():
    """libwavezip.so with the serving entry points declared."""
    global _lib
    if _lib is None:
        L = wz.lib()
        L.wz_cache_append.argtypes = [_P, _P, _P, _P, _L, _P, _L, _P, _L, _I, _P, _L,
                                      _I, _P]
        L.wz_attention_workspace_bytes.argtypes = [_P, _P, _P]
        L.wz_attention_workspace_bytes.restype = _S
        L.wz_cache_attention.argtypes = [_P, _P, _P, _P, _L, _P, _L, _P, _P, _S, _P]
        L.wz_quantize_rows.argtypes = [_P, _L, _I, _I, _I, _P, _L, _P, _P]
        L.wz_matmul_int.argtypes = [_P, _L, _P, _P, _L, _P, _P, _I, _I, _I, _P, _L, _I, _P]
        for f in EXPORTS:
            if f != "wz_attention_workspace_bytes":
                getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


class _NotLoaded:
    """Loads the native half of this module at its first use."""

    def __getattr__(self, name):
        global _native
        try:
            from . import _serve
        except ImportError as e:
            raise ImportError("paper_2607_23265_amd/_serve.so cannot be loaded; build it with "
                              "`python -m paper_2607_23265_amd.csrc.build`") from e
        _serve.raise_as(wz.WZError)
        _native = _serve
        return getattr(_serve, name)


_native = _NotLoaded()


def _fixed(*slots):
    """Properties that read the slots and cannot be assigned: the packed struct beside them holds their addresses and
    values, and an assignment would leave it with the old ones."""
    return [property(operator.attrgetter(s)) for s in slots]


class PagedCache:
    """The cache of one layer: k [pages, kv_heads, page_size, head_dim] and v [pages, kv_heads, head_dim, page_size]
    (float8_e4m3fn), k_scale and v_scale [pages, kv_heads] (float32 powers of two).  The fields cannot be assigned."""
    __slots__ = ("_k", "_v", "_k_scale", "_v_scale", "_c")
    k, v, k_scale, v_scale, c = _fixed(*__slots__)

    def __init__(self, k, v, k_scale, v_scale):
        self._c = _native.cache(k, v, k_scale, v_scale)
        self._k, self._v, self._k_scale, self._v_scale = k, v, k_scale, v_scale

    def __reduce__(self):  # (a copy packs its own tensors)
        return type(self), (self._k, self._v, self._k_scale, self._v_scale)

    device = property(lambda self: self._k.device)
    kv_heads = property(lambda self: self._k.shape[1])
    page_size = property(lambda self: self._k.shape[2])
    head_dim = property(lambda self: self._k.shape[3])

    @classmethod
    def new(cls, pages, kv_heads, head_dim, page_size=64, device="cuda:0"):
        """An empty cache (nothing in it needs initialising)."""
        def make(*shape, dtype=E4M3):
            return torch.empty(shape, dtype=dtype, device=device)
        return cls(make(pages, kv_heads, page_size, head_dim), make(pages, kv_heads, head_dim, page_size),
                   make(pages, kv_heads, dtype=torch.float32), make(pages, kv_heads, dtype=torch.float32))


class Ragged:
    """A ragged batch: sequence b brings rows start[b] .. start[b + 1] - 1 of the call and has kv_len[b] tokens in the
    cache, these counted, in the pages table[b] (all int32).  max_tokens and max_kv bound the new tokens and the
    tokens of one sequence.  The fields cannot be assigned; the tensors' contents may change between calls, within the
    bounds."""
    __slots__ = ("_start", "_kv_len", "_table", "_max_tokens", "_max_kv", "_c")
    start, kv_len, table, max_tokens, max_kv, c = _fixed(*__slots__)

    def __init__(self, start, kv_len, table, max_tokens, max_kv):
        self._c = _native.ragged(start, kv_len, table, max_tokens, max_kv)
        self._start, self._kv_len, self._table = start, kv_len, table
        self._max_tokens, self._max_kv = max_tokens, max_kv

    def __reduce__(self):
        return type(self), (self._start, self._kv_len, self._table, self._max_tokens, self._max_kv)

    device = property(lambda self: self._start.device)


class Rotation:
    """Rotation by position: table [max_pos, rot_dim] float32 holds cosines, then sines; sections are the numbers of
    frequencies that go by each row of positions (one section: all by positions[0]).  The fields cannot be assigned."""
    __slots__ = ("_table", "_sections", "_interleaved", "_c")
    table, sections, interleaved, c = _fixed(*__slots__)

    def __init__(self, table, sections=(), interleaved=False):
        self._table, self._sections, self._interleaved = table, tuple(sections), bool(interleaved)
        self._c = _native.rotation(table, self._sections, self._interleaved)

    def __reduce__(self):
        return type(self), (self._table, self._sections, self._interleaved)


def cache_append(cache, batch, k, v, rotation=None, positions=None, q=None, q_out=None):
    """wz_cache_append: store the batch's new keys and values (k, v [tokens, kv_heads, head_dim] float32 or bfloat16),
    rotated by positions [axes, tokens] int32; returns the rotated queries [tokens, q_heads, head_dim] bfloat16 if q
    is given (into q_out if that is)."""
    return _native.append(cache._c, batch._c, k, v, None if rotation is None else rotation._c, positions, q, q_out)


def attention_workspace_bytes(cache, batch, q_heads, tokens, window=0):
    """Bytes of workspace cache_attention() needs for `tokens` rows of q_heads heads (and that window)."""
    return _native.workspace(cache._c, batch._c, q_heads, tokens, window)


def cache_attention(cache, batch, q, scale=None, causal=True, window=0, out=None, lse=None, ws=None):
    """wz_cache_attention: q [tokens, q_heads, head_dim] bfloat16 over the cache -> out of the same shape.  scale
    defaults to head_dim ** -0.5; lse [tokens, q_heads] float32 receives the rows' log-sum-exp; ws is a uint8 workspace
    (allocated if not given and needed)."""
    return _native.attention(cache._c, batch._c, q, scale, causal, window, out, lse, ws)


def quantize_rows(x, out=None, scale=None):
    """wz_quantize_rows: x [rows, cols] float32 or bfloat16 -> (int8 [rows, cols], scale [rows] float32)."""
    return _native.quantize_rows(x, out, scale)


def matmul_int(a, a_scale, w, w_scale, bias=None, out=None, out_dtype=torch.bfloat16):
    """wz_matmul_int: a [M, K] and w [N, K] int8 with scales [M] and [N] -> a w^T, scaled, + bias [N], as out_dtype
    [M, N] (or the type of out)."""
    return _native.matmul_int(a, a_scale, w, w_scale, bias, out, out_dtype)
