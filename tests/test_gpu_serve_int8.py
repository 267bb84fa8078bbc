"""wz_quantize_rows and wz_matmul_int.  Marked gpu.

Integers are those of the oracle bit for bit (each fp32 operation is the header's); the product's sums are exact, so what
is left are three fp32 roundings of the scaled sum (the int's, two scales) and one of the bias, and the output's own.
"""
import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve
from serve_util import DEV, bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 16), (3, 48), (70, 3584), (5, 2064), (2, 65536), (4, 18944), (9, 8192)])
def test_quantize(rows, cols, dtype):
    r = np.random.default_rng(rows * cols)
    x = (r.normal(size=(rows, cols)) * np.exp(2 * r.normal(size=(rows, 1)))).astype(np.float32)
    if rows > 4:
        x[1], x[2], x[3, 5], x[4, 0] = 0, 1e-37, np.nan, -np.inf
        x[0, :16] = np.arange(16) + 0.5  # ties, if the row's largest is 127
        x[0, 16:] = np.clip(x[0, 16:], -127, 127)
        x[0, 15] = 127
    x = bf16(x) if dtype == torch.bfloat16 else x
    wide = torch.zeros(rows, cols + 24, dtype=dtype, device=DEV)
    wide[:, 8:8 + cols] = torch.from_numpy(x).to(DEV)
    q = torch.full((rows, cols + 32), 99, dtype=torch.int8, device=DEV)
    # (the first element of a row of the view is 16-byte aligned in both types)
    got, scale = serve.quantize_rows(wide[:, 8:8 + cols], out=q[:, 16:16 + cols])
    want, want_scale = so.quantize_rows(x)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(scale.cpu().numpy(), want_scale)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    edge = q.cpu().numpy()
    assert (edge[:, :16] == 99).all() and (edge[:, 16 + cols:] == 99).all()


SHAPES = [(1, 1, 16), (1, 100, 48), (2, 17, 3584), (16, 64, 64), (31, 33, 80), (64, 4608, 3584), (65, 130, 1040),
          (17, 1000, 8192), (128, 128, 128), (130, 257, 3600), (200, 515, 272), (300, 640, 16), (1286, 384, 1152),
          (513, 769, 2064), (256, 256, 65536), (1, 16384, 256), (90, 2048, 4096), (700, 3584, 560),
          # one for each tile the product is done in, with ragged edges
          (31, 4600, 1104), (63, 4601, 1168), (33, 9000, 144), (391, 2040, 528), (1286, 4600, 48), (2499, 4601, 144)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_matmul(M, N, K, out_dtype):
    r = np.random.default_rng(M + N + K)
    a = r.integers(-127, 128, (M, K), dtype=np.int8)
    w = r.integers(-127, 128, (N, K), dtype=np.int8)
    if M > 16:
        a[3], w[0] = 127, -128  # the largest sums
    a_scale, w_scale = (np.exp(r.normal(size=n)).astype(np.float32) for n in (M, N))
    bias = r.normal(size=N).astype(np.float32) * 100 if M % 2 else None
    d = {n: torch.from_numpy(x).to(DEV) for n, x in (("a_scale", a_scale), ("w_scale", w_scale))}
    # rows that lie apart, with numbers between them that must not be read into the sums
    wa, ww = (torch.full((n, K + 48), 77, dtype=torch.int8, device=DEV) for n in (M, N))
    wa[:, 16:16 + K], ww[:, 32:32 + K] = torch.from_numpy(a).to(DEV), torch.from_numpy(w).to(DEV)
    big = torch.full((M, N + 3), 5.0, dtype=out_dtype, device=DEV)
    serve.matmul_int(wa[:, 16:16 + K], d["a_scale"], ww[:, 32:32 + K], d["w_scale"],
                     None if bias is None else torch.from_numpy(bias).to(DEV), out=big[:, 1:1 + N])
    torch.cuda.synchronize()
    want, size = so.matmul_int(a, a_scale, w, w_scale, bias)
    got = big[:, 1:1 + N].float().cpu().numpy().astype(np.float64)
    tol = 2.0 ** -24 * 4 * size + (2.0 ** -8 * np.abs(want) if out_dtype == torch.bfloat16 else 0)
    worst = np.max(np.abs(got - want) / np.maximum(tol, 1e-30))
    print(f"[err] matmul {M}x{N}x{K}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0
    assert (big[:, 0] == 5).all() and (big[:, N + 1:] == 5).all()


def test_no_rows():
    x = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    q, s = serve.quantize_rows(x)
    w = torch.zeros(5, 64, dtype=torch.int8, device=DEV)
    y = serve.matmul_int(q, s, w, torch.ones(5, device=DEV))
    torch.cuda.synchronize()
    assert y.shape == (0, 5) and q.shape == (0, 64)


def test_one_row_of_a_matrix_of_any_stride():
    x = torch.randn(3, 67, device=DEV)
    q, s = serve.quantize_rows(x[:1, :64])
    want, scale = so.quantize_rows(x[:1, :64].cpu().numpy())
    w = torch.randint(-9, 9, (5, 67), dtype=torch.int8, device=DEV)[:1, :64]
    y = serve.matmul_int(q, s, w, torch.ones(1, device=DEV), out=torch.empty(3, 7, device=DEV)[:1, :1])
    torch.cuda.synchronize()
    np.testing.assert_array_equal(q.cpu().numpy(), want)
    ref = so.matmul_int(want, scale, w.cpu().numpy(), np.ones(1, np.float32))[0]
    np.testing.assert_allclose(y.cpu().numpy(), ref, rtol=2.0 ** -21)


def test_not_a_number_row():
    x = torch.ones(3, 64, device=DEV)
    x[1, 7] = float("nan")
    q, s = serve.quantize_rows(x)
    w = torch.ones(4, 64, dtype=torch.int8, device=DEV)
    y = serve.matmul_int(q, s, w, torch.ones(4, device=DEV), out_dtype=torch.float32)
    torch.cuda.synchronize()
    assert torch.isnan(y[1]).all() and torch.isfinite(y[[0, 2]]).all()


def test_far_rows():
    """Rows whose bytes lie past 2^32."""
    K, stride = 64, 1 << 20
    rows = (1 << 32) // stride + 3
    a = torch.zeros(rows * stride, dtype=torch.int8, device=DEV).view(rows, stride)
    a[-1, :K], a[-2, :K] = 3, -2
    y = serve.matmul_int(a[:, :K], torch.ones(rows, device=DEV), a[-2:, :K], torch.ones(2, device=DEV),
                         out_dtype=torch.float32)
    torch.cuda.synchronize()
    assert y[-1].tolist() == [-6 * K, 9 * K] and y[-2].tolist() == [4 * K, -6 * K] and not y[:-2].any()
