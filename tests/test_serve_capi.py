"""The serving operators' C ABI and binding: exports, struct layouts and refusals (no GPU needed).

Every call here fails validation or has nothing to do, which returns before any HIP call is made.
"""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve
from paper_2607_23265_amd import wavezip as wz

OK, NULL, ALIGN, SHAPE, DTYPE, PARAM, BUDGET, WORKSPACE = range(8)
AT = 0x10000


@pytest.fixture(scope="module")
def L():
    libutil.ensure_built()
    return serve.lib()


def cache(**kw):
    d = dict(k=AT, v=AT, k_scale=AT, v_scale=AT, pages=100, kv_heads=4, page_size=64, head_dim=128)
    return serve._Cache(**{**d, **kw})


def ragged(**kw):
    d = dict(start=AT, kv_len=AT, table=AT, batch=2, tokens=5, max_tokens=3, max_kv=640, table_stride=10)
    return serve._Ragged(**{**d, **kw})


def turn(**kw):
    d = dict(table=AT, positions=AT, max_pos=1000, rot_dim=128, axes=3, interleaved=0,
             sections=(ctypes.c_int32 * 3)(16, 24, 24))
    return serve._Rotation(**{**d, **kw})


def append(L, c=None, r=None, t=None, **kw):
    a = dict(k=AT, ks=512, v=AT, vs=512, q=AT, qs=3584, heads=28, out=2 * AT, os=3584, dtype=wz.WZ_BF16)
    a.update(kw)
    return L.wz_cache_append(ctypes.byref(c or cache()), ctypes.byref(r or ragged()),
                             ctypes.byref(t) if t else None, a["k"], a["ks"], a["v"], a["vs"], a["q"], a["qs"],
                             a["heads"], a["out"], a["os"], a["dtype"], None)


def attend(L, c=None, r=None, cfg=None, **kw):
    a = dict(q=AT, qs=3584, out=AT, os=3584, lse=None, ws=AT, bytes=1 << 30)
    a.update(kw)
    f = dict(q_heads=28, causal=1, window=0, scale=0.1)
    f.update(cfg or {})
    return L.wz_cache_attention(ctypes.byref(c or cache()), ctypes.byref(r or ragged()),
                                ctypes.byref(serve._Attention(**f)), a["q"], a["qs"], a["out"], a["os"], a["lse"],
                                a["ws"], a["bytes"], None)


def test_every_declared_symbol_is_exported(L):
    header = os.path.join(libutil.ROOT, "include", "wavezip_serve.h")
    text = re.sub(r"/\*.*?\*/", "", open(header).read(), flags=re.S)
    assert set(re.findall(r"\b(wz_[a-z_]+)\s*\(", text)) == set(serve.EXPORTS)
    dyn = subprocess.run(["nm", "-D", "--defined-only", wz.LIB_PATH], capture_output=True, text=True).stdout
    exported = {line.split()[-1] for line in dyn.splitlines() if line.strip()}
    assert set(serve.EXPORTS) <= exported


def test_header_is_c_and_structs_match(tmp_path):
    """The header compiles as C, and the binding's structs have its sizes and offsets."""
    structs = {"wz_cache": serve._Cache, "wz_ragged": serve._Ragged, "wz_rotation": serve._Rotation,
               "wz_attention": serve._Attention}
    checks = "".join(
        f'  printf("%zu\\n", sizeof({n}));\n' + "".join(f'  printf("%zu\\n", offsetof({n}, {f[0]}));\n'
                                                        for f in s._fields_) for n, s in structs.items())
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "wavezip_serve.h"\nint main(void) {\n' + checks + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(libutil.ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = list(map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()))
    want = []
    for s in structs.values():
        want += [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]
    assert got == want
    # what the binding passes: the same structs, packed
    a = serve._Cache(1 << 40, 2, 3, 4, 5, 6, 7, 8)
    assert bytes(a) == serve._CACHE(1 << 40, 2, 3, 4, 5, 6, 7, 8)
    b = serve._Ragged(1 << 40, 2, 3, 4, 5, 6, 7, 8)
    assert bytes(b) == serve._RAGGED(1 << 40, 2, 3, 4, 5, 6, 7, 8)
    c = serve._Rotation(1 << 40, 2, 3, 4, 5, 6, (ctypes.c_int32 * 3)(7, 8, 9))
    assert bytes(c) == serve._ROTATION(1 << 40, 2, 3, 4, 5, 6, 7, 8, 9)
    assert bytes(serve._Attention(1, 2, 3, 0.5)) == serve._ATTENTION(1, 2, 3, 0.5)


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(page_size=8), dict(page_size=48), dict(page_size=256),
                                dict(kv_heads=0), dict(kv_heads=257), dict(pages=0)])
def test_cache_shapes(L, kw):
    assert append(L, c=cache(**kw)) == SHAPE
    assert attend(L, c=cache(**kw)) == SHAPE
    f = serve._Attention(28, 1, 0, 0.1)
    assert L.wz_attention_workspace_bytes(ctypes.byref(cache(**kw)), ctypes.byref(ragged()), ctypes.byref(f)) == 0


@pytest.mark.parametrize("kw", [dict(batch=0), dict(batch=65537), dict(tokens=-1), dict(tokens=1 << 24),
                                dict(max_tokens=-1), dict(max_kv=1 << 24, table_stride=1 << 20), dict(max_kv=-1),
                                dict(max_kv=641), dict(table_stride=9), dict(table_stride=-1)])
def test_batch_shapes(L, kw):
    assert append(L, r=ragged(**kw)) == SHAPE
    assert attend(L, r=ragged(**kw)) == SHAPE


@pytest.mark.parametrize("kw,code", [(dict(rot_dim=8), SHAPE), (dict(rot_dim=144), SHAPE), (dict(rot_dim=40), SHAPE),
                                     (dict(max_pos=0), SHAPE), (dict(axes=0), SHAPE), (dict(axes=4), SHAPE),
                                     (dict(axes=2), SHAPE), (dict(rot_dim=64), SHAPE), (dict(interleaved=2), PARAM),
                                     (dict(sections=(ctypes.c_int32 * 3)(-16, 56, 24)), SHAPE),
                                     (dict(table=None), NULL), (dict(table=AT + 8), ALIGN),
                                     (dict(positions=None), NULL), (dict(positions=AT + 2), ALIGN)])
def test_rotations(L, kw, code):
    assert append(L, t=turn(**kw)) == code


@pytest.mark.parametrize("kw,code", [(dict(dtype=2), DTYPE), (dict(k=None), NULL), (dict(v=None), NULL),
                                     (dict(k=AT + 8), ALIGN), (dict(v=AT + 4), ALIGN), (dict(ks=504), SHAPE),
                                     (dict(vs=516), SHAPE), (dict(heads=0), SHAPE), (dict(out=None), NULL),
                                     (dict(out=AT), PARAM), (dict(qs=3576), SHAPE), (dict(os=3580), SHAPE),
                                     (dict(out=2 * AT + 8), ALIGN)])
def test_append_arguments(L, kw, code):
    assert append(L, t=turn(), **kw) == code


def test_append_arrays(L):
    assert L.wz_cache_append(None, None, None, AT, 512, AT, 512, None, 0, 0, None, 0, 1, None) == NULL
    for name in ("k", "v", "k_scale", "v_scale"):
        assert append(L, c=cache(**{name: None})) == NULL
        assert append(L, c=cache(**{name: AT + 2})) == ALIGN
        assert attend(L, c=cache(**{name: None})) == NULL
    for name in ("start", "kv_len", "table"):
        assert append(L, r=ragged(**{name: None})) == NULL
        assert attend(L, r=ragged(**{name: AT + 2})) == ALIGN


@pytest.mark.parametrize("cfg,code", [(dict(q_heads=0), SHAPE), (dict(q_heads=30), SHAPE), (dict(q_heads=260), SHAPE),
                                      (dict(causal=2), PARAM), (dict(window=-1), PARAM),
                                      (dict(window=5, causal=0), PARAM), (dict(scale=float("nan")), PARAM),
                                      (dict(scale=float("inf")), PARAM)])
def test_attention_config(L, cfg, code):
    assert attend(L, cfg=cfg) == code


def test_attention_arguments(L):
    assert attend(L, q=None) == NULL and attend(L, q=AT + 8) == ALIGN and attend(L, qs=3576) == SHAPE
    assert attend(L, out=None) == NULL and attend(L, out=AT + 2) == ALIGN and attend(L, os=3590) == SHAPE
    assert attend(L, lse=AT + 2) == ALIGN
    long = ragged(max_kv=64000, table_stride=1000)
    need = L.wz_attention_workspace_bytes(ctypes.byref(cache()), ctypes.byref(long),
                                          ctypes.byref(serve._Attention(28, 1, 0, 0.1)))
    assert 0 < need <= 128 << 20 and need % 256 == 0
    assert attend(L, r=long, ws=None) == NULL and attend(L, r=long, bytes=need - 1) == WORKSPACE
    assert attend(L, r=long, ws=AT + 16) == WORKSPACE


def test_too_many_workgroups(L):
    many = ragged(batch=65536, tokens=65536, max_tokens=1)
    assert attend(L, c=cache(kv_heads=256), r=many, cfg=dict(q_heads=256), qs=256 * 128, os=256 * 128) == SHAPE
    assert append(L, c=cache(kv_heads=256), r=many, ks=256 * 128, vs=256 * 128, q=None) == SHAPE
    f = serve._Attention(256, 1, 0, 0.1)
    assert L.wz_attention_workspace_bytes(ctypes.byref(cache(kv_heads=256)), ctypes.byref(many), ctypes.byref(f)) == 0


def test_nothing_to_do(L):
    assert append(L, r=ragged(tokens=0), k=None, v=None) == OK
    assert attend(L, r=ragged(tokens=0), q=None) == OK
    assert L.wz_quantize_rows(None, 64, 0, 64, 1, None, 64, None, None) == OK
    assert L.wz_matmul_int(None, 64, None, None, 64, None, None, 0, 5, 64, None, 5, 1, None) == OK


def test_workspace_is_bounded(L):
    r = np.random.default_rng(1)
    for _ in range(2000):
        heads = int(r.choice([1, 2, 3, 4, 8, 16, 40, 256]))
        c = cache(kv_heads=heads, head_dim=int(r.choice([64, 128])))
        n = int(r.integers(1, 1 << int(r.integers(1, 15))))
        b = int(r.integers(1, 1 << int(r.integers(1, 12))))
        kv = int(r.integers(1, 1 << int(r.integers(1, 21))))
        q = ragged(batch=b, max_tokens=n, tokens=min(b * n, (1 << 24) - 1), max_kv=kv, table_stride=kv)
        f = serve._Attention(heads * int(r.choice([1, 2, 7, 8, 64])), 1, 0, 0.1)
        assert L.wz_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(q), ctypes.byref(f)) <= 128 << 20


def test_int8_arguments(L):
    def quant(x=AT, xs=64, rows=3, cols=64, dtype=1, q=AT, qs=64, s=AT):
        return L.wz_quantize_rows(x, xs, rows, cols, dtype, q, qs, s, None)
    assert quant(dtype=3) == DTYPE and quant(rows=-1) == SHAPE and quant(cols=24) == SHAPE and quant(cols=0) == SHAPE
    assert quant(cols=65552, xs=70000) == SHAPE and quant(xs=56) == SHAPE and quant(qs=72) == SHAPE
    assert quant(x=None) == NULL and quant(q=AT + 8) == ALIGN and quant(s=None) == NULL and quant(s=AT + 1) == ALIGN

    def mul(a=AT, as_=64, sa=AT, w=AT, ws=64, sw=AT, b=None, M=3, N=5, K=64, o=AT, os_=5, dtype=1):
        return L.wz_matmul_int(a, as_, sa, w, ws, sw, b, M, N, K, o, os_, dtype, None)
    assert mul(dtype=5) == DTYPE and mul(M=-1) == SHAPE and mul(N=0) == SHAPE and mul(K=20) == SHAPE
    assert mul(as_=48) == SHAPE and mul(ws=72) == SHAPE and mul(os_=4) == SHAPE and mul(K=65552, as_=70000) == SHAPE
    assert mul(M=1 << 20, N=1 << 19, os_=1 << 19) == SHAPE
    assert mul(as_=(1 << 22) + 16) == SHAPE and mul(ws=(1 << 22) + 16) == SHAPE
    assert mul(a=None) == NULL and mul(w=AT + 8) == ALIGN and mul(sa=None) == NULL and mul(sw=AT + 2) == ALIGN
    assert mul(b=AT + 2) == ALIGN and mul(o=None) == NULL and mul(o=AT + 1) == ALIGN


def test_binding_refuses_cpu_tensors():
    z = torch.zeros
    with pytest.raises(ValueError):
        serve.PagedCache(z(2, 1, 16, 64, dtype=serve.E4M3), z(2, 1, 64, 16, dtype=serve.E4M3), z(2, 1), z(2, 1))
    with pytest.raises(ValueError):
        serve.Ragged(z(2, dtype=torch.int32), z(1, dtype=torch.int32), z(1, 1, dtype=torch.int32), 1, 1)
    with pytest.raises(ValueError):
        serve.Rotation(z(4, 64))
    with pytest.raises(ValueError):
        serve.quantize_rows(z(2, 16))
    with pytest.raises(ValueError):
        serve.matmul_int(z(2, 16, dtype=torch.int8), z(2), z(2, 16, dtype=torch.int8), z(2))


# --- the oracle itself ------------------------------------------------------

def test_oracle_codes_are_torchs():
    """Every code's value, and the rounding, against torch's float8_e4m3fn."""
    every = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(so.decode(every.numpy()), every.view(torch.float8_e4m3fn).double().numpy())
    x = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.1, 0.1, 20001), so.E4M3[:126] + np.diff(so.E4M3[:127]) / 2])
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(so.encode(x), want)


def test_oracle_scales():
    for amax, e in ((448.0, 0), (448.0001, 1), (1.0, -8), (1.75, -8), (1.7501, -7), (0.0, -100), (3e38, 119)):
        assert so.scale_of(amax) == np.float32(2.0 ** e), amax


def test_oracle_attention_is_softmax():
    """Against torch's float64 softmax on one dense sequence."""
    r = np.random.default_rng(0)
    P, D, n = 16, 64, 40
    c = dict(k=np.zeros((3, 1, P, D), np.uint8), v=np.zeros((3, 1, D, P), np.uint8),
             k_scale=np.ones((3, 1), np.float32), v_scale=np.ones((3, 1), np.float32))
    k, v = (r.normal(size=(n, 1, D)).astype(np.float32) for _ in range(2))
    table = np.array([[2, 0, 1]])
    so.append(c, [0, n], [n], table, k, v)
    q = r.normal(size=(5, 2, D)).astype(np.float32)
    out, _, lse, _ = so.attention(c, [0, 5], [n], table, q, 0.3)
    K = (so.decode(c["k"]) * c["k_scale"][..., None, None])[table[0], 0].reshape(-1, D)[:n]
    V = (so.decode(c["v"]) * c["v_scale"][..., None, None])[table[0], 0].transpose(0, 2, 1).reshape(-1, D)[:n]
    assert np.abs(K - k[:, 0]).max() < 0.3 and np.abs(V - v[:, 0]).max() < 0.3
    s = torch.from_numpy(np.einsum("nhd,kd->nhk", q.astype(np.float64), K) * 0.3)
    s[torch.arange(n)[None, None] > torch.arange(n - 5, n)[:, None, None].expand(5, 2, 1)] = -np.inf
    np.testing.assert_allclose(out, torch.softmax(s, -1).numpy() @ V, rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(lse, torch.logsumexp(s, -1).numpy(), rtol=1e-12)
