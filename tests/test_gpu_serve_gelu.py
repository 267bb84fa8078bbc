"""The gelu of products with an epilogue, over all of its range.  Marked gpu.

With u = 2^-24, a = |x| and g = erfc(a / sqrt 2) / 2, the result is max(x, 0) - a g.  g is a polynomial of degree 9 in t =
1 / (1 + c a) times exp(-a^2 / 2): the polynomial with its rounded coefficients is within 1.2 u of the function, its nine
sums are worth at most 7 u (their terms' magnitudes sum to 2.3 of it), t is off by 3 u and the polynomial by 2.4 times that,
the power by 2 u and by its exponent's three roundings, 1.5 u a^2, and three products and roundings add 3 u: together
u (21 + 1.5 a^2).  The difference adds a rounding of the result.  What is below fp32's normal numbers may be zero.
"""
import math

import numpy as np
import pytest
import torch

import libutil
from paper_2607_23265_amd import serve
from serve_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


def gelu(x, call, dtype):
    """Of exactly x: a product of zeros with the bias x."""
    a, one = torch.zeros(2, 16, dtype=torch.int8, device=DEV), torch.ones(2, device=DEV)
    w, ones = torch.zeros(len(x), 16, dtype=torch.int8, device=DEV), torch.ones(len(x), device=DEV)
    bias = torch.from_numpy(x).to(DEV)
    if call == "matmul_int":
        y = serve.matmul_int(a, one, w, ones, bias, activation="gelu", out_dtype=dtype)
    else:
        y = serve.gated_int(a, one, w, ones, w, ones, activation="gelu", gate_bias=bias, up_bias=ones, out_dtype=dtype)
    torch.cuda.synchronize()
    assert torch.equal(y[0], y[1])
    return y[0].double().cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("call", ["matmul_int", "gated_int"])
def test_gelu(call, dtype):
    r = np.random.default_rng(1)
    x = np.concatenate([np.linspace(-15, 15, 60001), r.normal(size=20000), r.normal(size=2000) * 1e-3,
                        [0.0, 16, -16, 16.5, -16.5, 100, -100, 1e30, -1e30, 1e-30, -1e-30]]).astype(np.float32)
    got, z = gelu(x, call, dtype), x.astype(np.float64)
    a = np.abs(z)
    part = a * 0.5 * np.array([math.erfc(v / math.sqrt(2)) for v in a])
    want = np.maximum(z, 0) - part
    tol = U * (21 + 1.5 * np.minimum(a, 16) ** 2) * part + U * np.abs(want) + 2.0 ** -126
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    worst = np.abs(got - want) / tol
    print(f"[err] gelu {call} {dtype}: {worst.max():.3f} of the bound, at {x[worst.argmax()]:.4f}", flush=True)
    assert worst.max() <= 1
