"""wz_matmul_int_epilogue and wz_gated_int in every tile they choose from, with ragged edges, and cut into two launches,
with the residual in another tensor and in place.  Marked gpu.

Tolerances, with u = 2^-24: the sum x of a product with its bias is off by 4 u of the size of its terms (an exact integer
and three fp32 operations), and an activation passes that on by at most 1.13.  silu's own steps: at most 8 u of its result
and 2 u (tests/test_gpu_serve_layer.py); gelu's: u (21 + 1.5 a^2) of a erfc(a / sqrt 2) / 2, a = |x|, and a rounding
(tests/test_gpu_serve_gelu.py).  A residual adds one rounding; a product of two factors adds their errors times the other,
and a rounding; bf16 half a step of 2^-8.  The reference is torch's float64 products, whose sums of whole numbers are exact.
"""
import math

import pytest
import torch

import libutil
import tile_cases as tc
from paper_2607_23265_amd import serve
from serve_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


def codes(g, rows, cols, pad):
    """Codes as a view of wider rows, and scales that make a product's elements of ordinary size."""
    wide = torch.full((rows, cols + pad), 77, dtype=torch.int8, device=DEV)
    wide[:, 16:16 + cols] = torch.randint(-127, 128, (rows, cols), generator=g, device=DEV, dtype=torch.int8)
    scale = torch.exp(0.5 * torch.randn(rows, generator=g, device=DEV)) / (70 * cols ** 0.25)
    return wide[:, 16:16 + cols], scale


def product(a, sa, w, sw, bias):
    """In float64, with the size of its terms."""
    y = (a.double() @ w.double().t()).mul_(sa.double()[:, None]).mul_(sw.double())
    size = y.abs()
    return (y, size) if bias is None else (y.add_(bias.double()), size.add_(bias.double().abs()))


def activation(x, size, name):
    """And how far the kernel's may be off."""
    tol = 1.13 * 4 * U * size if name else 4 * U * size
    if name is None:
        return x, tol
    if name == "silu":
        y = x / (1 + torch.exp(-x))
        return y, tol.add_(U * (8 * y.abs() + 2))
    a = x.abs()
    part = 0.5 * a * torch.special.erfc(a * math.sqrt(0.5))
    y = x.clamp_min(0) - part
    return y, tol.add_(U * ((21 + 1.5 * a.clamp_max(16).square()) * part + y.abs()) + 2.0 ** -126)


def check(got, want, tol, what):
    if got.dtype == BF:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    worst = float(((got.double() - want).abs() / tol.clamp_min(1e-30)).max())
    print(f"[err] {what} {got.dtype}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0


@pytest.mark.parametrize("act,M,N,K,tiles", tc.RICH)
def test_epilogue(act, M, N, K, tiles):
    print(f"[case] epilogue {M}x{N}x{K} {act} {tiles}", flush=True)
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    a, sa = codes(g, M, K, 48)
    w, sw = codes(g, N, K, 32)
    bias = torch.randn(N, generator=g, device=DEV) if M % 2 else None
    y, tol = activation(*product(a, sa, w, sw, bias), act)
    for dtype in (BF, F32):
        res = (4 * torch.randn(M, N, generator=g, device=DEV)).to(dtype)
        far = torch.full((M, N + 5), float("nan"), dtype=dtype, device=DEV)  # (rows and elements that are not the residual's)
        far[:, 3:3 + N] = res
        both = y + res.double()
        more = tol + U * (both.abs() + tol)
        out = torch.full((M + 1, N + 3), 5.0, dtype=dtype, device=DEV)
        got = out[:M, 1:1 + N]
        calls = [("residual", far[:, 3:3 + N], both, more), ("in place", got, both, more)]
        if act:
            calls.append(("alone", None, y, tol))
        for how, residual, want, off in calls:
            if how == "in place":
                got.copy_(res)
            serve.matmul_int(a, sa, w, sw, bias, out=got, activation=act, residual=residual)
            torch.cuda.synchronize()
            check(got, want, off, f"epilogue {M}x{N}x{K} {act} {how}")
            assert (out[:, 0] == 5).all() and (out[:, N + 1:] == 5).all() and (out[M] == 5).all()


@pytest.mark.parametrize("act,M,N,K,tiles", tc.GATED)
def test_gated(act, M, N, K, tiles):
    print(f"[case] gated {M}x{N}x{K} {act} {tiles}", flush=True)
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    a, sa = codes(g, M, K, 48)
    gate, sg = codes(g, N, K, 32)
    up, su = codes(g, N, K, 64)  # (the two lie apart, with other strides)
    bg, bu = (torch.randn(N, generator=g, device=DEV) if z else None for z in (M % 2, M % 3))
    x, tx = activation(*product(a, sa, gate, sg, bg), act)
    z, size = product(a, sa, up, su, bu)
    tz = 4 * U * size
    tol = z.abs() * tx + x.abs() * tz + tx * tz + U * (x * z).abs()
    for dtype in (BF, F32):
        out = torch.full((M + 1, N + 3), 5.0, dtype=dtype, device=DEV)
        got = out[:M, 1:1 + N]
        serve.gated_int(a, sa, gate, sg, up, su, activation=act, gate_bias=bg, up_bias=bu, out=got)
        torch.cuda.synchronize()
        check(got, x * z, tol, f"gated {M}x{N}x{K} {act}")
        assert (out[:, 0] == 5).all() and (out[:, N + 1:] == 5).all() and (out[M] == 5).all()
