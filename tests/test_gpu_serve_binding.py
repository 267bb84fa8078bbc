"""The serving operators' binding on the GPU: what it refuses, streams, given and made outputs, and rows that overlap
against the contract.  Marked gpu.
"""
import numpy as np
import pytest
import torch

import libutil
from paper_2607_23265_amd import serve
from paper_2607_23265_amd import wavezip as wz
from serve_util import DEV, Case

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


def _new(*shape, dtype=BF):
    return torch.randn(*shape, device=DEV).to(dtype)


def _ints(*values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _refused(error, f, *args, **kw):
    with pytest.raises(error):
        f(*args, **kw)


def test_structs():
    k, v = (torch.zeros(2, 3, *s, dtype=torch.uint8, device=DEV).view(serve.E4M3) for s in ((16, 64), (64, 16)))
    s = torch.ones(2, 3, device=DEV)
    serve.PagedCache(k, v, s, s)
    for bad in ((k, k, s, s), (k[0], v, s, s), (k.view(torch.uint8), v, s, s), (k, v, s[:1], s), (k, v, s, s.double()),
                (k.transpose(0, 1), v, s, s), (k.cpu(), v, s, s), (k, v.cpu(), s, s), (None, v, s, s), (k, v, s, 3)):
        _refused(ValueError, serve.PagedCache, *bad)
    start, kv, table = _ints(0, 1, 2), _ints(1, 1), _ints(0, 1).view(2, 1)
    serve.Ragged(start, kv, table, 1, 1)
    for bad in ((start[:2], kv, table), (start, kv[:1], table), (start, kv, table[0]), (start.long(), kv, table),
                (start, kv.cpu(), table), (start, kv, table.expand(2, 4))):
        _refused(ValueError, serve.Ragged, *bad, 1, 1)
    _refused(ValueError, serve.Ragged, start, kv, table, 1 << 40, 1)
    _refused(TypeError, serve.Ragged, start, kv, table, "1", 1)
    turns = torch.zeros(8, 64, device=DEV)
    serve.Rotation(turns, [16, 8, 8], True)
    for bad in ((turns[0],), (turns.half(),), (turns, (8, 8, 8, 8)), (turns, (30,))):
        _refused(ValueError, serve.Rotation, *bad)


def test_cache_calls():
    c = Case([2, 1], [20, 5], 2, 64, 16, seed=1).fill()
    cache, batch = c.device_cache(), c.batch()
    k, v, q = _new(3, 2, 64), _new(3, 2, 64), _new(3, 4, 64)
    turn, at = serve.Rotation(torch.zeros(40, 64, device=DEV)), _ints(0, 1, 2)
    f = serve.cache_append
    for bad in ((k.half(), v), (k, v[:2]), (k, v.float()), (k[:, :1], v), (k, v.cpu()), (_new(3, 64, 2).transpose(1, 2), v),
                (k[..., :32], v)):
        _refused(ValueError, f, cache, batch, *bad)
    _refused(ValueError, f, cache, batch, k, v, turn)
    _refused(ValueError, f, cache, batch, k, v, turn, at[:2])
    _refused(ValueError, f, cache, batch, k, v, turn, at.long())
    _refused(ValueError, f, cache, batch, k, v, q=q[:2])
    _refused(ValueError, f, cache, batch, k, v, q=q, q_out=q.float())
    _refused(wz.WZError, f, cache, batch, k, v, q=q, q_out=q)
    _refused(wz.WZError, f, cache, batch, k, v, serve.Rotation(torch.zeros(40, 40, device=DEV)), at)
    f = serve.cache_attention
    for bad in (q.float(), q[..., :32], q[0], q.cpu(), _new(3, 64, 4).transpose(1, 2)):
        _refused(ValueError, f, cache, batch, bad)
    _refused(wz.WZError, f, cache, batch, _new(3, 3, 64))
    _refused(wz.WZError, f, cache, batch, q, scale=float("inf"))
    _refused(wz.WZError, f, cache, batch, q, causal=False, window=4)
    _refused(TypeError, f, cache, batch, q, scale="1")
    _refused(ValueError, f, cache, batch, q, out=q.float())
    _refused(ValueError, f, cache, batch, q, lse=torch.zeros(3, 5, device=DEV))
    _refused(ValueError, f, cache, batch, q, ws=torch.zeros(8, device=DEV))
    long = c.batch()
    wide = torch.full((2, 300), -1, dtype=torch.int32, device=DEV)
    wide[:, :long.table.shape[1]] = long.table
    long = serve.Ragged(long.start, long.kv_len, wide, 2, 4800)
    need = serve.attention_workspace_bytes(cache, long, 4, 3)
    assert need > 0
    with pytest.raises(wz.WZError) as e:
        f(cache, long, q, ws=torch.zeros(need - 256, dtype=torch.uint8, device=DEV))
    assert e.value.status == 7 and "wz_cache_attention" in str(e.value)


def test_int8_calls():
    x = _new(5, 64)
    q, s = serve.quantize_rows(x)
    f = serve.quantize_rows
    for bad in (x[0], x.t(), x.half(), x.cpu()):
        _refused(ValueError, f, bad)
    _refused(wz.WZError, f, x[:, :24])
    _refused(ValueError, f, x, out=q[:4])
    _refused(ValueError, f, x, scale=s[:4])
    _refused(ValueError, f, x, out=x)
    w, ws = f(_new(7, 64))
    g = serve.matmul_int
    for bad in ((q, s, w[:, :32], ws), (q, s[:4], w, ws), (q, s, w, ws[:3]), (q.t(), s, w, ws), (x, s, w, ws),
                (q, s, w.cpu(), ws)):
        _refused(ValueError, g, *bad)
    _refused(ValueError, g, q, s, w, ws, bias=ws[:2])
    _refused(ValueError, g, q, s, w, ws, out_dtype=torch.float16)
    _refused(ValueError, g, q, s, w, ws, out=_new(5, 8))
    _refused(ValueError, g, q, s, w, ws, out=_new(5, 7).half())
    _refused(wz.WZError, g, q, s, w, ws, out=torch.zeros(1, 7, device=DEV).expand(5, 7))


def test_given_outputs_are_returned():
    x = _new(5, 64, dtype=torch.float32).requires_grad_()
    q0, s0 = serve.quantize_rows(x)
    q, s = torch.zeros_like(q0), torch.zeros_like(s0)
    got = serve.quantize_rows(x, q, s)
    assert got[0] is q and got[1] is s and torch.equal(q, q0) and torch.equal(s, s0)
    y = torch.zeros(5, 5, device=DEV)
    assert serve.matmul_int(q, s, q, s, out=y) is y
    assert torch.equal(y, serve.matmul_int(q, s, q, s, out_dtype=torch.float32))


def test_the_current_stream():
    """Work goes to the current stream: behind what that stream holds, and seen by what follows on it."""
    x = torch.zeros(512, 4096, device=DEV)
    big = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(8):
            big = big @ big * 0.01
        x.fill_(2.0)
        q, scale = serve.quantize_rows(x)
        total = q.int().sum()
    s.synchronize()
    assert int(total) == 127 * 512 * 4096 and torch.equal(scale, torch.full_like(scale, 2 / 127))


def test_rows_that_overlap_stay_in_the_workspace():
    """Decreasing starts make more blocks than the batch can have: nothing behind the workspace is written."""
    n = 64
    c = Case([1] * n, [2000] * n, 1, 64, 128, seed=2, garbage=False).fill()
    cache, b = c.device_cache(), c.batch()
    start = torch.arange(n + 1, device=DEV, dtype=torch.int32) % 2
    for max_tokens in (1, 70):
        batch = serve.Ragged(start, b.kv_len, b.table, max_tokens, 2000)
        q = _new(1, 1, 64)
        need = serve.attention_workspace_bytes(cache, batch, 1, 1)
        assert need > 0
        space = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device=DEV)
        serve.cache_attention(cache, batch, q, ws=space[:need])
        torch.cuda.synchronize()
        assert bool((space[need:] == 0x5A).all())
    k = _new(1, 1, 64)
    bits = {x: getattr(cache, x).view(torch.int32) for x in ("k_scale", "v_scale")}  # (NaN in pages without a token)
    before = {x: t.clone() for x, t in bits.items()}
    serve.cache_append(cache, serve.Ragged(start, b.kv_len, b.table, 1, 2000), k, k)
    torch.cuda.synchronize()
    pages = np.unique(c.table[::2, (2000 - 1) // 128])
    same = torch.ones(c.pages, dtype=torch.bool, device=DEV)
    same[torch.from_numpy(pages).to(DEV).long()] = False
    for x, was in before.items():
        assert torch.equal(bits[x][same], was[same])
