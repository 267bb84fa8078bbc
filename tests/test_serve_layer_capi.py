"""The C ABI of what a served layer has beside softmax attention: layouts, refusals, and the oracle (no GPU needed).

Every call here fails validation or has nothing to do, which returns before any HIP call is made.
"""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve
from test_serve_capi import ALIGN, AT, DTYPE, NULL, OK, PARAM, SHAPE, WORKSPACE, ragged


@pytest.fixture(scope="module")
def L():
    libutil.ensure_built()
    return serve.lib()


def test_states_struct_matches(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "wavezip_serve.h"\nint main(void) {\n  printf("%zu\\n", sizeof(wz_states));\n'
                   + "".join(f'  printf("%zu\\n", offsetof(wz_states, {f[0]}));\n' for f in serve._States._fields_)
                   + '  printf("%d %d %d %d\\n", WZ_ACT_RELU, WZ_ACT_SILU, WZ_ACT_GELU, WZ_ACT_GELU_TANH);\n  return 0;\n}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(libutil.ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = list(map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()))
    want = [ctypes.sizeof(serve._States)] + [getattr(serve._States, f[0]).offset for f in serve._States._fields_]
    assert got == want + [1, 2, 3, 4]


def epilogue(L, **kw):
    d = dict(a=AT, as_=64, sa=AT, w=AT, ws=64, sw=AT, b=None, act=2, r=AT, rs=5, M=3, N=5, K=64, o=2 * AT, os_=5, dtype=1)
    d.update(kw)
    return L.wz_matmul_int_epilogue(d["a"], d["as_"], d["sa"], d["w"], d["ws"], d["sw"], d["b"], d["act"], d["r"], d["rs"],
                                    d["M"], d["N"], d["K"], d["o"], d["os_"], d["dtype"], None)


def gated(L, **kw):
    d = dict(a=AT, as_=64, sa=AT, g=AT, gs=64, sg=AT, bg=None, u=AT, us=64, su=AT, bu=None, act=2, M=3, N=5, K=64,
             o=2 * AT, os_=5, dtype=1)
    d.update(kw)
    return L.wz_gated_int(d["a"], d["as_"], d["sa"], d["g"], d["gs"], d["sg"], d["bg"], d["u"], d["us"], d["su"], d["bu"],
                          d["act"], d["M"], d["N"], d["K"], d["o"], d["os_"], d["dtype"], None)


PRODUCT = [(dict(dtype=5), DTYPE), (dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=20), SHAPE), (dict(as_=48), SHAPE),
           (dict(os_=4), SHAPE), (dict(K=65552, as_=70000), SHAPE), (dict(as_=(1 << 22) + 16), SHAPE), (dict(a=None), NULL),
           (dict(a=AT + 8), ALIGN), (dict(sa=None), NULL), (dict(o=None), NULL), (dict(o=AT + 1), ALIGN),
           (dict(act=5), PARAM), (dict(act=-1), PARAM), (dict(M=1 << 24), SHAPE)]


@pytest.mark.parametrize("kw,code", PRODUCT + [
    (dict(ws=72), SHAPE), (dict(ws=(1 << 22) + 16), SHAPE), (dict(w=None), NULL), (dict(w=AT + 8), ALIGN),
    (dict(sw=AT + 2), ALIGN), (dict(b=AT + 2), ALIGN), (dict(rs=4), SHAPE), (dict(r=AT + 1), ALIGN),
    (dict(r=2 * AT, rs=6), PARAM), (dict(N=1 << 24), SHAPE), (dict(M=1 << 20, N=1 << 19, os_=1 << 19, rs=1 << 19), SHAPE)])
def test_epilogue_arguments(L, kw, code):
    assert epilogue(L, **kw) == code


@pytest.mark.parametrize("kw,code", PRODUCT + [
    (dict(gs=72), SHAPE), (dict(us=48), SHAPE), (dict(g=None), NULL), (dict(u=None), NULL), (dict(u=AT + 8), ALIGN),
    (dict(sg=None), NULL), (dict(su=AT + 2), ALIGN), (dict(bg=AT + 1), ALIGN), (dict(bu=AT + 2), ALIGN),
    (dict(N=1 << 23, os_=1 << 23), SHAPE), (dict(M=1 << 19, N=1 << 19, os_=1 << 19), SHAPE)])
def test_gated_arguments(L, kw, code):
    assert gated(L, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), DTYPE), (dict(rows=-1), SHAPE), (dict(rows=1 << 24), SHAPE), (dict(cols=24), SHAPE),
    (dict(cols=0), SHAPE), (dict(cols=65552, xs=70000), SHAPE), (dict(xs=56), SHAPE), (dict(xs=68), SHAPE),
    (dict(qs=72), SHAPE), (dict(x=None), NULL), (dict(x=AT + 8), ALIGN), (dict(w=None), NULL), (dict(w=AT + 4), ALIGN),
    (dict(q=AT + 8), ALIGN), (dict(s=None), NULL), (dict(s=AT + 2), ALIGN), (dict(eps=0.0), PARAM), (dict(eps=-1.0), PARAM),
    (dict(eps=float("nan")), PARAM), (dict(eps=float("inf")), PARAM), (dict(r=AT + 4), ALIGN), (dict(rs=56), SHAPE),
    (dict(t=None), NULL), (dict(t=AT + 2), ALIGN), (dict(ts=60), SHAPE), (dict(t=AT, ts=72), PARAM),
    (dict(r=3 * AT, t=3 * AT, ts=72), PARAM)])
def test_norm_arguments(L, kw, code):
    d = dict(x=AT, xs=64, r=2 * AT, rs=64, w=AT, eps=1e-6, rows=3, cols=64, dtype=1, t=4 * AT, ts=64, q=AT, qs=64, s=AT)
    d.update(kw)
    assert L.wz_norm_quantize(d["x"], d["xs"], d["r"], d["rs"], d["w"], d["eps"], d["rows"], d["cols"], d["dtype"], d["t"],
                              d["ts"], d["q"], d["qs"], d["s"], None) == code


def states(**kw):
    return serve._States(**{**dict(state=AT, slots=9, heads=28, head_dim=128), **kw})


def decay(L, z=None, r=None, **kw):
    d = dict(slot=AT, ld=AT, q=AT, qs=3584, k=AT, ks=512, v=AT, vs=512, kv=4, scale=0.1, o=2 * AT, os_=3584, ws=AT,
             bytes=1 << 28)
    d.update(kw)
    return L.wz_decay_attention(ctypes.byref(z or states()), ctypes.byref(r or ragged()), d["slot"], d["ld"], d["q"],
                                d["qs"], d["k"], d["ks"], d["v"], d["vs"], d["kv"], d["scale"], d["o"], d["os_"], d["ws"],
                                d["bytes"], None)


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(head_dim=32), dict(heads=0), dict(heads=257), dict(slots=0)])
def test_state_shapes(L, kw):
    assert decay(L, z=states(**kw)) == SHAPE
    assert L.wz_decay_workspace_bytes(ctypes.byref(states(**kw)), ctypes.byref(ragged())) == 0


@pytest.mark.parametrize("kw", [dict(batch=0), dict(batch=65537), dict(tokens=-1), dict(tokens=1 << 24),
                                dict(max_tokens=-1), dict(max_tokens=1 << 24), dict(max_kv=1 << 24), dict(max_kv=-1)])
def test_batch_shapes(L, kw):
    assert decay(L, r=ragged(**kw)) == SHAPE


@pytest.mark.parametrize("kw,code", [
    (dict(kv=0), SHAPE), (dict(kv=3), SHAPE), (dict(kv=56), SHAPE), (dict(scale=float("nan")), PARAM),
    (dict(scale=float("inf")), PARAM), (dict(slot=None), NULL), (dict(slot=AT + 2), ALIGN), (dict(ld=None), NULL),
    (dict(ld=AT + 1), ALIGN), (dict(q=None), NULL), (dict(q=AT + 8), ALIGN), (dict(qs=3576), SHAPE), (dict(qs=3588), SHAPE),
    (dict(k=None), NULL), (dict(ks=504), SHAPE), (dict(v=AT + 2), ALIGN), (dict(vs=516), SHAPE), (dict(o=None), NULL),
    (dict(o=AT), PARAM), (dict(os_=3580), SHAPE), (dict(qs=(1 << 22) + 8), SHAPE), (dict(ks=1 << 23), SHAPE), (dict(vs=1 << 30), SHAPE)])
def test_decay_arguments(L, kw, code):
    assert decay(L, **kw) == code


def test_decay_arrays(L):
    assert decay(L, z=states(state=None)) == NULL and decay(L, z=states(state=AT + 8)) == ALIGN
    for name in ("start", "kv_len"):
        assert decay(L, r=ragged(**{name: None})) == NULL and decay(L, r=ragged(**{name: AT + 2})) == ALIGN
    assert L.wz_decay_workspace_bytes(None, ctypes.byref(ragged())) == 0
    assert L.wz_decay_workspace_bytes(ctypes.byref(states()), None) == 0
    # the batch's table is not looked at
    assert decay(L, r=ragged(table=None, table_stride=0, tokens=0)) == OK
    assert decay(L, z=states(heads=256), r=ragged(batch=65536, tokens=65536, max_tokens=1), qs=32768, os_=32768) == SHAPE


def test_nothing_to_do(L):
    assert decay(L, r=ragged(tokens=0), q=None) == OK and decay(L, r=ragged(max_tokens=0), q=None) == OK
    assert epilogue(L, M=0, a=None, w=None, o=None) == OK and gated(L, M=0, a=None, g=None, o=None) == OK
    assert L.wz_norm_quantize(None, 64, None, 0, None, 1e-6, 0, 64, 1, None, 0, None, 64, None, None) == OK


def test_workspace_is_bounded_and_asked_for(L):
    r = np.random.default_rng(1)
    some = 0
    for _ in range(2000):
        z = states(heads=int(r.choice([1, 2, 3, 4, 8, 16, 28, 40, 256])), head_dim=int(r.choice([64, 128])))
        n = int(r.integers(1, 1 << int(r.integers(1, 24))))
        b = int(r.integers(1, 1 << int(r.integers(1, 12))))
        x = ragged(batch=b, max_tokens=n, tokens=min(b * n, (1 << 24) - 1), max_kv=0, table_stride=0)
        need = L.wz_decay_workspace_bytes(ctypes.byref(z), ctypes.byref(x))
        assert need <= 65 << 20 and need % 256 == 0
        if need:
            some += 1
            kw = dict(z=z, r=x, qs=32768, os_=32768, ks=512, vs=512, kv=1)
            assert decay(L, ws=None, **kw) == NULL and decay(L, ws=AT + 16, **kw) == WORKSPACE
            assert decay(L, bytes=need - 1, **kw) == WORKSPACE


def test_binding_refuses_cpu_tensors():
    z = torch.zeros
    q, s = z(2, 16, dtype=torch.int8), z(2)
    for f, a in ((serve.States, (z(2, 1, 64, 64),)), (serve.norm_quantize, (z(2, 16), z(16))),
                 (serve.gated_int, (q, s, q, s, q, s)), (serve.matmul_int, (q, s, q, s, None, None, torch.float32, "silu"))):
        with pytest.raises(ValueError):
            f(*a)


# --- the oracle itself ------------------------------------------------------

def test_oracle_activations():
    x = np.linspace(-12, 12, 2001)
    t, f = torch.from_numpy(x), torch.nn.functional
    for name, want in (("relu", f.relu(t)), ("silu", f.silu(t)), ("gelu", f.gelu(t)),
                       ("gelu_tanh", f.gelu(t, approximate="tanh")), (None, t)):
        y, slope = so.activation(x, name)
        np.testing.assert_allclose(y, want.numpy(), rtol=1e-9, atol=1e-15)
        assert np.abs(np.diff(y)).max() <= slope * np.diff(x).max() * (1 + 1e-9)


def test_oracle_norm():
    r = np.random.default_rng(0)
    h, w = r.normal(size=(7, 48)).astype(np.float32), r.normal(size=48).astype(np.float32)
    q, s = so.norm_quantize(h, w, 1e-5)
    want = torch.nn.functional.rms_norm(torch.from_numpy(h).double(), (48,), torch.from_numpy(w).double(), 1e-5).numpy()
    assert np.abs(q * s[:, None] - want).max() <= 0.51 * s.max()
    assert (np.abs(q).max(1) == 127).all()


def test_oracle_decay_is_the_unrolled_sum():
    r = np.random.default_rng(3)
    q, k, v = (r.normal(size=(9, h, 4)) for h in (2, 1, 1))
    state = r.normal(size=(3, 2, 4, 4))
    ld = np.array([-0.3, 0.2])  # (above 0: counts as 0)
    out, mag, new, _ = so.decay_attention(state, [0, 3, 3, 9], [True, True, False], [2, 1, -1], q, k, v, ld, 0.5)
    for h, l in enumerate((np.exp(-0.3), 1.0)):
        for i in range(3):
            want = q[i, h] @ state[2, h] * l ** (i + 1) + sum(l ** (i - j) * (q[i, h] @ k[j, 0]) * v[j, 0] for j in range(i + 1))
            np.testing.assert_allclose(out[i, h], 0.5 * want, rtol=1e-12)
        want = sum(l ** (5 - j) * (q[8, h] @ k[3 + j, 0]) * v[3 + j, 0] for j in range(6))
        np.testing.assert_allclose(out[8, h], 0.5 * want, rtol=1e-12)
        np.testing.assert_allclose(new[2, h], l ** 3 * state[2, h] + sum(l ** (2 - j) * np.outer(k[j, 0], v[j, 0]) for j in range(3)))
    assert (new[:2] == state[:2]).all() and (np.abs(out) <= mag * (1 + 1e-12)).all()
