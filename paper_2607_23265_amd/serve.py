"""Python binding of the serving operators (include/wavezip_serve.h): argument marshalling only.

A paged key/value cache held in 8 bits, attention over it, and products in 8-bit integers, for a language model that
reads the tokens wavezip.condense() keeps.  Tensors are torch GPU tensors; every call goes to the current HIP stream
of their device.  Where a tensor has rows of heads ([tokens, heads, head_dim]) its rows may lie apart, so parts of one
fused projection are passed as they are; everything else is contiguous.
"""
import ctypes
import struct

import torch

from . import wavezip as wz

EXPORTS = ("wz_cache_append", "wz_cache_attention", "wz_attention_workspace_bytes", "wz_quantize_rows",
           "wz_matmul_int")
E4M3 = torch.float8_e4m3fn
_DTYPE = {torch.float32: wz.WZ_F32, torch.bfloat16: wz.WZ_BF16}
_FLOATS, _INT8 = tuple(_DTYPE), (torch.int8,)
_P, _I, _L, _S = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t

# The header's structs as bytes: packing one costs a third of making a ctypes.Structure, and a step of small calls waits
# for the host.
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


def _dense(name, t, dtype, device=None):
    if not t.is_cuda or not t.is_contiguous() or t.dtype is not dtype or (device is not None and t.device != device):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor" + (f" on {device}" if device else " on a GPU"))
    return t


def _rows(name, t, tokens, heads, dim, device, dtype):
    """Row stride of t [tokens, heads, dim], whose heads must lie together (tokens, heads: None for any)."""
    shape, stride = t.shape, t.stride()
    if (len(shape) != 3 or shape[2] != dim or (heads is not None and shape[1] != heads) or
            (tokens is not None and shape[0] != tokens) or t.dtype is not dtype or t.device != device):
        raise ValueError(f"{name} must be [{'tokens' if tokens is None else tokens}, "
                         f"{'heads' if heads is None else heads}, {dim}] on {device}, of type {dtype}")
    if stride[2] != 1 or (stride[1] != dim and shape[1] > 1):
        raise ValueError(f"{name}: the heads of a row must lie together")
    return stride[0] if shape[0] > 1 else shape[1] * dim  # (a single row has no stride)


# The current stream's handle without a torch.cuda.Stream made for it (0.1 us instead of 2, of a call's 8).
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(device, where, f, *args):
    """f(*args, stream) on `device`'s current stream, with that device current."""
    index = device.index
    if _device() == index:
        st = f(*args, _stream(index))
    else:
        with torch.cuda.device(device):
            st = f(*args, _stream(index))
    if st != 0:
        raise wz.WZError(st, where)


class PagedCache:
    """The cache of one layer: k [pages, kv_heads, page_size, head_dim] and v [pages, kv_heads, head_dim, page_size]
    (float8_e4m3fn), k_scale and v_scale [pages, kv_heads] (float32 powers of two)."""
    __slots__ = ("k", "v", "k_scale", "v_scale", "device", "kv_heads", "head_dim", "page_size", "c")

    def __init__(self, k, v, k_scale, v_scale):
        dev = self.device = k.device
        if k.dim() != 4:
            raise ValueError("k must be [pages, kv_heads, page_size, head_dim]")
        pages, heads, page, dim = k.shape
        if v.shape != (pages, heads, dim, page):
            raise ValueError("v must be [pages, kv_heads, head_dim, page_size]")
        if k_scale.shape != (pages, heads) or v_scale.shape != (pages, heads):
            raise ValueError("k_scale and v_scale must be [pages, kv_heads]")
        _dense("k", k, E4M3), _dense("v", v, E4M3, dev)
        _dense("k_scale", k_scale, torch.float32, dev), _dense("v_scale", v_scale, torch.float32, dev)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.kv_heads, self.head_dim, self.page_size = heads, dim, page
        self.c = _CACHE(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), pages, heads, page, dim)

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
    tokens of one sequence."""
    __slots__ = ("start", "kv_len", "table", "device", "max_tokens", "max_kv", "at")

    def __init__(self, start, kv_len, table, max_tokens, max_kv):
        dev = self.device = _dense("start", start, torch.int32).device
        _dense("kv_len", kv_len, torch.int32, dev)
        _dense("table", table, torch.int32, dev)
        batch = kv_len.numel()
        if kv_len.dim() != 1 or start.shape != (batch + 1,) or table.dim() != 2 or table.shape[0] != batch:
            raise ValueError("start must be [batch + 1], kv_len [batch] and table [batch, pages]")
        self.start, self.kv_len, self.table = start, kv_len, table
        self.max_tokens, self.max_kv = max_tokens, max_kv
        self.at = start.data_ptr(), kv_len.data_ptr(), table.data_ptr(), batch

    def of(self, tokens):
        """wz_ragged of a call with so many rows."""
        return _RAGGED(*self.at, tokens, self.max_tokens, self.max_kv, self.table.shape[1])


class Rotation:
    """Rotation by position: table [max_pos, rot_dim] float32 holds cosines, then sines; sections are the numbers of
    frequencies that go by each row of positions (one section: all by positions[0])."""
    __slots__ = ("table", "sections", "interleaved", "of")

    def __init__(self, table, sections=(), interleaved=False):
        _dense("table", table, torch.float32)
        if table.dim() != 2 or len(sections) > 3:
            raise ValueError("table must be [max_pos, rot_dim], with at most three sections")
        self.table, self.sections, self.interleaved = table, tuple(sections), bool(interleaved)
        if len(sections) == 1 and 2 * sections[0] != table.shape[1]:
            raise ValueError("the sections must sum to rot_dim / 2")
        # what follows the positions in wz_rotation
        self.of = (*table.shape, max(1, len(sections)), int(self.interleaved), *(*self.sections, 0, 0, 0)[:3])


def cache_append(cache, batch, k, v, rotation=None, positions=None, q=None, q_out=None):
    """wz_cache_append: store the batch's new keys and values (k, v [tokens, kv_heads, head_dim] float32 or bfloat16),
    rotated by positions [axes, tokens] int32; returns the rotated queries [tokens, q_heads, head_dim] bfloat16 if q
    is given (into q_out if that is)."""
    dev, dim, tokens, dtype = cache.device, cache.head_dim, k.shape[0], k.dtype
    if dtype not in _DTYPE or batch.device != dev:
        raise ValueError("k must be float32 or bfloat16, and the batch on the cache's device")
    ks = _rows("k", k, None, cache.kv_heads, dim, dev, dtype)
    vs = _rows("v", v, tokens, cache.kv_heads, dim, dev, dtype)
    q_at = out_at = None
    qs = qos = heads = 0
    if q is not None:
        qs, heads = _rows("q", q, tokens, None, dim, dev, dtype), q.shape[1]
        if q_out is None:
            q_out = q.new_empty((tokens, heads, dim), dtype=torch.bfloat16)
        qos = _rows("q_out", q_out, tokens, heads, dim, dev, torch.bfloat16)
        q_at, out_at = q.data_ptr(), q_out.data_ptr()
    turn = None
    if rotation is not None:
        if positions is None:
            raise ValueError("a rotation needs positions")
        _dense("positions", positions, torch.int32, dev)
        if positions.numel() != rotation.of[2] * tokens or rotation.table.device != dev:
            raise ValueError("positions must be [axes, tokens], on the device of the table")
        turn = _ROTATION(rotation.table.data_ptr(), positions.data_ptr(), *rotation.of)
    _call(dev, "wz_cache_append", lib().wz_cache_append, cache.c, batch.of(tokens), turn, k.data_ptr(),
          ks, v.data_ptr(), vs, q_at, qs, heads, out_at, qos, _DTYPE[dtype])
    return q_out if q is not None else None


def attention_workspace_bytes(cache, batch, q_heads, tokens):
    """Bytes of workspace cache_attention() needs for `tokens` rows of q_heads heads."""
    return int(lib().wz_attention_workspace_bytes(cache.c, batch.of(tokens), _ATTENTION(q_heads, 0, 0, 1.0)))


def cache_attention(cache, batch, q, scale=None, causal=True, window=0, out=None, lse=None, ws=None):
    """wz_cache_attention: q [tokens, q_heads, head_dim] bfloat16 over the cache -> out of the same shape.  scale
    defaults to head_dim ** -0.5; lse [tokens, q_heads] float32 receives the rows' log-sum-exp; ws is a uint8 workspace
    (allocated if not given and needed)."""
    dev, dim = cache.device, cache.head_dim
    if batch.device != dev:
        raise ValueError("the batch must be on the cache's device")
    qs = _rows("q", q, None, None, dim, dev, torch.bfloat16)
    tokens, heads = q.shape[0], q.shape[1]
    if out is None:
        out, os_ = q.new_empty((tokens, heads, dim)), heads * dim
    else:
        os_ = _rows("out", out, tokens, heads, dim, dev, torch.bfloat16)
    if lse is not None and _dense("lse", lse, torch.float32, dev).shape != (tokens, heads):
        raise ValueError("lse must be [tokens, q_heads]")
    cfg = _ATTENTION(heads, int(causal), window, dim ** -0.5 if scale is None else scale)
    c, r = cache.c, batch.of(tokens)
    if ws is None:
        need = lib().wz_attention_workspace_bytes(c, r, cfg)
        ws = q.new_empty(need, dtype=torch.uint8) if need else None
    else:
        _dense("ws", ws, torch.uint8, dev)
    _call(dev, "wz_cache_attention", lib().wz_cache_attention, c, r, cfg, q.data_ptr(), qs, out.data_ptr(), os_,
          None if lse is None else lse.data_ptr(), None if ws is None else ws.data_ptr(),
          0 if ws is None else ws.numel())
    return out


def _matrix(name, t, dtypes, device=None):
    if t.dim() != 2 or t.dtype not in dtypes or not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must be a matrix on the GPU of type " + " or ".join(map(str, dtypes)))
    s = t.stride()
    if s[1] != 1 and t.shape[1] > 1:
        raise ValueError(f"{name}: the elements of a row must lie together")
    return s[0] if t.shape[0] > 1 else t.shape[1]  # (a single row has no stride)


def quantize_rows(x, out=None, scale=None):
    """wz_quantize_rows: x [rows, cols] float32 or bfloat16 -> (int8 [rows, cols], scale [rows] float32)."""
    xs, dev = _matrix("x", x, _FLOATS), x.device
    rows, cols = x.shape
    if out is None:
        out, qs = x.new_empty((rows, cols), dtype=torch.int8), cols
    else:
        qs = _matrix("out", out, _INT8, dev)
    if scale is None:
        scale = x.new_empty(rows, dtype=torch.float32)
    else:
        _dense("scale", scale, torch.float32, dev)
    if out.shape != x.shape or scale.shape != (rows,):
        raise ValueError("out must have the shape of x, and scale [rows]")
    _call(dev, "wz_quantize_rows", lib().wz_quantize_rows, x.data_ptr(), xs, rows, cols, _DTYPE[x.dtype],
          out.data_ptr(), qs, scale.data_ptr())
    return out, scale


def matmul_int(a, a_scale, w, w_scale, bias=None, out=None, out_dtype=torch.bfloat16):
    """wz_matmul_int: a [M, K] and w [N, K] int8 with scales [M] and [N] -> a w^T, scaled, + bias [N], as out_dtype
    [M, N] (or the type of out)."""
    as_, dev = _matrix("a", a, _INT8), a.device
    ws = _matrix("w", w, _INT8, dev)
    M, K = a.shape
    N = w.shape[0]
    if w.shape[1] != K:
        raise ValueError("a and w must have the same columns")
    if (_dense("a_scale", a_scale, torch.float32, dev).numel() != M or
            _dense("w_scale", w_scale, torch.float32, dev).numel() != N or
            (bias is not None and _dense("bias", bias, torch.float32, dev).numel() != N)):
        raise ValueError("a_scale must be [M], w_scale and bias [N]")
    if out is None:
        out, os_ = a.new_empty((M, N), dtype=out_dtype), N
    else:
        os_ = _matrix("out", out, _FLOATS, dev)
    if out.shape != (M, N) or out.dtype not in _DTYPE:
        raise ValueError("out must be [M, N] float32 or bfloat16")
    _call(dev, "wz_matmul_int", lib().wz_matmul_int, a.data_ptr(), as_, a_scale.data_ptr(), w.data_ptr(), ws,
          w_scale.data_ptr(), None if bias is None else bias.data_ptr(), M, N, K, out.data_ptr(), os_,
          _DTYPE[out.dtype])
    return out
