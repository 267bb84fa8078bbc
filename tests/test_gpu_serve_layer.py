"""wz_matmul_int_epilogue, wz_gated_int and wz_norm_quantize.  Marked gpu.

Products.  With u = 2^-24: the scaled sum x with its bias is off by 4 u of the size of its terms (as wz_matmul_int's
tests have it).  An activation passes that on by at most its slope, 1.13.  Its own steps:
  silu, gelu_tanh  x s(z), s(z) = 1 / (1 + exp2(-z log2 e)): the exponent is off by at most 5 u of itself, which moves s by
                   (1 - s) |z| 5 u of itself; |x| s (1 - s) |z| is below 0.3 of 1 for every x < 0 and below 0.3 |y| above,
                   so 1.5 u + 1.5 u |y|; exp2 and the reciprocal are good to 2 u each, the sum and the product to u
  gelu             the error function is good to 16 steps of 2 u and 1 where |x| > 6, so 16 u |x| up to 6; three products
together at most u (6 size + 8 |y| + 18 min(|x|, 6) + 2).  A residual adds one rounding of the result, bf16 a half step of
2^-8, and a product of two such factors adds their errors times the other, and a rounding.

Norms.  Codes and the sum of the stream are those of the oracle bit for bit (each operation is the header's).  A thread adds
at most cols / 64 squares one after the other, and its sum meets at most 9 others: u (cols / 64 + 9) of the mean, half of that
of its root, and six roundings.
"""
import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve
from paper_2607_23265_amd import wavezip as wz
from serve_util import DEV, bf16

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def codes(r, rows, cols, pad, at):
    """Codes and scales, on the host and as a view of wider rows on the GPU."""
    x = r.integers(-127, 128, (rows, cols), dtype=np.int8)
    wide = torch.full((rows, cols + pad), 77, dtype=torch.int8, device=DEV)
    wide[:, at:at + cols] = dev(x)
    scale = (np.exp(0.5 * r.normal(size=rows)) / np.sqrt(cols) / 70).astype(np.float32)
    return x, scale, wide[:, at:at + cols], dev(scale)


def act_error(x, size, y):
    return U * (6 * size + 8 * np.abs(y) + 18 * np.minimum(np.abs(x), 6) + 2)


def check(got, want, tol, dtype, what):
    tol = tol + (2.0 ** -8 * (np.abs(want) + tol) if dtype == BF else 0)
    worst = np.max(np.abs(got - want) / np.maximum(tol, 1e-30))
    print(f"[err] {what}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0


# one for each tile that a product is done in, with ragged edges, and the smallest
SHAPES = [(1, 1, 16), (1, 100, 48), (2, 17, 3584), (31, 33, 80), (64, 4608, 1152), (65, 130, 1040), (130, 257, 3600),
          (300, 640, 16), (1286, 384, 1152), (513, 769, 2064), (33, 9000, 144), (391, 2040, 528), (1286, 4600, 48),
          (2499, 4601, 144), (100, 15, 8192), (3, 2300, 65536), (4100, 3000, 272)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("act,residual,dtype", [(None, True, BF), ("silu", True, BF), ("gelu", False, BF), ("relu", True, F32),
                                                ("gelu_tanh", True, F32), ("gelu", True, F32), ("silu", False, F32)])
def test_epilogue(M, N, K, act, residual, dtype):
    r = np.random.default_rng(M + N + K)
    a, sa, da, dsa = codes(r, M, K, 48, 16)
    w, sw, dw, dsw = codes(r, N, K, 32, 32)
    sw *= 40
    bias = r.normal(size=N).astype(np.float32) if M % 2 else None
    big = torch.full((M, N + 3), 5.0, dtype=dtype, device=DEV)
    res = r.normal(size=(M, N)).astype(np.float32) * 4
    res = bf16(res) if dtype == BF else res
    far = torch.full((M, N + 5), float("nan"), dtype=dtype, device=DEV)  # (rows and elements that are not the residual's)
    far[:, 3:3 + N] = dev(res).to(dtype)
    got = serve.matmul_int(da, dsa, dw, dev(sw), None if bias is None else dev(bias), out=big[:, 1:1 + N], activation=act,
                           residual=far[:, 3:3 + N] if residual else None)
    torch.cuda.synchronize()
    x, size = so.matmul_int(a, sa, w, sw, bias)
    y, _ = so.activation(x, act)
    tol = act_error(x, size, y)
    if residual:
        tol, y = tol + U * (np.abs(y + res) + tol), y + res
    check(got.double().cpu().numpy(), y, tol, dtype, f"epilogue {M}x{N}x{K} {act} {dtype}")
    assert (big[:, 0] == 5).all() and (big[:, N + 1:] == 5).all()


@pytest.mark.parametrize("M,N,K", [(65, 130, 1040), (1286, 4600, 48), (1, 7, 64), (2499, 4601, 144)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_residual_in_place(M, N, K, dtype):
    """The residual may be the result itself: the same numbers as onto another tensor."""
    r = np.random.default_rng(1)
    _, _, a, sa = codes(r, M, K, 16, 16)
    _, _, w, sw = codes(r, N, K, 16, 0)
    x = torch.randn(M, N + 1, device=DEV).to(dtype)[:, 1:]
    want = serve.matmul_int(a, sa, w, sw, out_dtype=dtype, residual=x)
    assert serve.matmul_int(a, sa, w, sw, out=x, residual=x) is x
    torch.cuda.synchronize()
    assert torch.equal(x, want)


def test_no_epilogue_is_the_product():
    """Without an activation and a residual the two entry points agree bit for bit."""
    r = np.random.default_rng(2)
    for M, N, K in ((65, 130, 1040), (1286, 4600, 48)):
        _, _, a, sa = codes(r, M, K, 16, 16)
        _, _, w, sw = codes(r, N, K, 16, 0)
        for dtype, code in ((BF, wz.WZ_BF16), (F32, wz.WZ_F32)):
            want, got = serve.matmul_int(a, sa, w, sw, out_dtype=dtype), torch.zeros(M, N, dtype=dtype, device=DEV)
            st = serve.lib().wz_matmul_int_epilogue(a.data_ptr(), a.stride(0), sa.data_ptr(), w.data_ptr(), w.stride(0),
                                                    sw.data_ptr(), None, 0, None, 0, M, N, K, got.data_ptr(), N, code,
                                                    torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            assert st == 0 and torch.equal(got, want)


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("act,biases,dtype", [("silu", "", BF), ("silu", "gu", F32), ("gelu", "g", BF), ("gelu_tanh", "u", F32),
                                              ("relu", "", F32), (None, "gu", BF)])
def test_gated(M, N, K, act, biases, dtype):
    r = np.random.default_rng(M + N + K)
    a, sa, da, dsa = codes(r, M, K, 48, 16)
    g, sg, dg, _ = codes(r, N, K, 32, 32)
    p, sp, dp, _ = codes(r, N, K, 64, 16)  # (the two lie apart, with other strides)
    sg, sp = sg * 40, sp * 40
    bg, bp = (r.normal(size=N).astype(np.float32) if z in biases else None for z in "gu")
    big = torch.full((M, N + 3), 5.0, dtype=dtype, device=DEV)
    got = serve.gated_int(da, dsa, dg, dev(sg), dp, dev(sp), activation=act, gate_bias=None if bg is None else dev(bg),
                          up_bias=None if bp is None else dev(bp), out=big[:, 1:1 + N])
    torch.cuda.synchronize()
    x, size = so.matmul_int(a, sa, g, sg, bg)
    up, up_size = so.matmul_int(a, sa, p, sp, bp)
    y, _ = so.activation(x, act)
    ty, tu = act_error(x, size, y), 4 * U * up_size
    tol = np.abs(up) * ty + np.abs(y) * tu + ty * tu + U * np.abs(y * up)
    check(got.double().cpu().numpy(), y * up, tol, dtype, f"gated {M}x{N}x{K} {act} {dtype}")
    assert (big[:, 0] == 5).all() and (big[:, N + 1:] == 5).all()


def test_gated_halves_of_one_tensor():
    """Gate and up as the halves of one fused projection, and the composition of the two products it stands for."""
    r = np.random.default_rng(4)
    _, _, a, sa = codes(r, 200, 512, 0, 0)
    _, _, w, sw = codes(r, 2 * 300, 512, 0, 0)
    got = serve.gated_int(a, sa, w[:300], sw[:300], w[300:], sw[300:], activation=None, out_dtype=F32)
    both = serve.matmul_int(a, sa, w, sw, out_dtype=F32)
    torch.cuda.synchronize()
    assert torch.equal(got, both[:, :300] * both[:, 300:])
    assert serve.gated_int(a, sa, w, sw, w, sw).dtype == BF


def test_numbers_at_the_ends():
    """Activations of large and infinite sums are their limits; a row without a scale is NaN, and no other."""
    a = torch.full((6, 16), 100, dtype=torch.int8, device=DEV)
    a_scale = torch.tensor([1e30, -1e30, 1e9, -1e9, float("nan"), 0.0], device=DEV)
    w, w_scale = torch.full((40, 16), 100, dtype=torch.int8, device=DEV), torch.ones(40, device=DEV)
    for act in ("relu", "silu", "gelu", "gelu_tanh"):
        y = serve.matmul_int(a, a_scale, w, w_scale, out_dtype=F32, activation=act)
        x = serve.matmul_int(a, a_scale, w, w_scale, out_dtype=F32)
        torch.cuda.synchronize()
        assert torch.equal(y[[0, 2]], x[[0, 2]]) and not y[[1, 3, 5]].any() and torch.isnan(y[4]).all(), act


def test_infinite_sums():
    """Infinities go through an activation as through its formula: the upper one stays."""
    inf = float("inf")
    a, w = torch.ones(2, 16, dtype=torch.int8, device=DEV), torch.ones(40, 16, dtype=torch.int8, device=DEV)
    one, bias = torch.ones(2, device=DEV), torch.zeros(40, device=DEV)
    bias[3] = inf
    for act in (None, "relu", "silu", "gelu", "gelu_tanh"):
        y = serve.matmul_int(a, one, w, torch.ones(40, device=DEV), bias, out_dtype=F32, activation=act)
        torch.cuda.synchronize()
        assert (y[:, 3] == inf).all() and torch.isfinite(y[:, :3]).all() and torch.isfinite(y[:, 4:]).all(), act


def test_no_rows():
    a, s = torch.empty(0, 64, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV)
    w, sw = torch.zeros(5, 64, dtype=torch.int8, device=DEV), torch.ones(5, device=DEV)
    assert serve.gated_int(a, s, w, sw, w, sw).shape == (0, 5)
    assert serve.matmul_int(a, s, w, sw, activation="silu").shape == (0, 5)
    q, z = serve.norm_quantize(torch.empty(0, 64, device=DEV), torch.ones(64, device=DEV))
    assert q.shape == (0, 64) and z.shape == (0,)


def test_far_weights():
    """Weights whose bytes lie past 2^32 from the first."""
    K, stride = 64, 1 << 20
    rows = (1 << 32) // stride + 3
    w = torch.zeros(rows * stride, dtype=torch.int8, device=DEV).view(rows, stride)[:, :K]
    w[-1], w[-2] = 3, -2
    a, one, ones = torch.full((2, K), 5, dtype=torch.int8, device=DEV), torch.ones(2, device=DEV), torch.ones(rows, device=DEV)
    y = serve.gated_int(a, one, w, ones, w, ones, activation=None, out_dtype=F32)
    z = serve.matmul_int(a, one, w, ones, out_dtype=F32, activation="relu")
    torch.cuda.synchronize()
    assert y[0, -2:].tolist() == [(10 * K) ** 2, (15 * K) ** 2] and not y[:, :-2].any()
    assert z[1, -2:].tolist() == [0, 15 * K] and not z[:, :-2].any()


# --- norms ------------------------------------------------------------------

ROWS = [(1, 16), (3, 48), (70, 3584), (5, 2064), (2, 65536), (4, 18944), (9, 8192), (7, 1024), (129, 1040), (6, 4096), (5, 4112),
        (3, 16400)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols", ROWS)
@pytest.mark.parametrize("residual", [False, True])
def test_norm(rows, cols, dtype, residual):
    r = np.random.default_rng(rows * cols)
    x = (r.normal(size=(rows, cols)) * np.exp(2 * r.normal(size=(rows, 1)))).astype(np.float32)
    y = (3 * r.normal(size=(rows, cols))).astype(np.float32)
    weight = (1 + 0.4 * r.normal(size=cols)).astype(np.float32)
    weight[3] = 0
    if rows > 4:
        x[1], x[2], x[3, 5], x[4, 3], y[1], y[2], y[4, 0] = 0, 1e-37, np.nan, -np.inf, 0, 0, np.inf
        x[4, 0] = -np.inf  # (and with the residual: no number; x[4, 3] has no weight)
    if dtype == BF:
        x, y = bf16(x), bf16(y)
    pad = 24
    wide, other, total = (torch.zeros(rows, cols + pad, dtype=dtype, device=DEV) for _ in range(3))
    wide[:, 8:8 + cols], other[:, 16:16 + cols] = dev(x), dev(y)
    q = torch.full((rows, cols + 32), 99, dtype=torch.int8, device=DEV)
    got = serve.norm_quantize(wide[:, 8:8 + cols], dev(weight), 1e-5, other[:, 16:16 + cols] if residual else None,
                              total[:, 8:8 + cols] if residual else None, q[:, 16:16 + cols])
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        h = torch.from_numpy(x + y).to(dtype).float().numpy() if residual else x
    if residual:
        np.testing.assert_array_equal(got[2].float().cpu().numpy(), h)
        assert not total[:, :8].any() and not total[:, 8 + cols:].any()
    want, scale = so.norm_quantize(h, weight, np.float32(1e-5))
    np.testing.assert_array_equal(got[0].cpu().numpy(), want)
    np.testing.assert_allclose(got[1].cpu().numpy(), scale, rtol=U * ((cols / 64 + 9) / 2 + 6))
    edge = q.cpu().numpy()
    assert (edge[:, :16] == 99).all() and (edge[:, 16 + cols:] == 99).all()


@pytest.mark.parametrize("cols", [64, 3584, 20000])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_in_place(cols, dtype):
    """The sum may go to where x or the residual lies."""
    x, y = (torch.randn(5, cols, device=DEV).to(dtype) for _ in range(2))
    w = torch.rand(cols, device=DEV)
    want = serve.norm_quantize(x, w, residual=y)
    for a, b, into in ((x.clone(), y, 0), (x, y.clone(), 1)):
        got = serve.norm_quantize(a, w, residual=b, total=(a, b)[into])
        torch.cuda.synchronize()
        assert got[2] is (a, b)[into] and all(torch.equal(u, v) for u, v in zip(got, want))


@pytest.mark.parametrize("cols", [64, 2048, 8192, 40000])
def test_norm_of_large_numbers(cols):
    """Squares past fp32: the norm is still the norm."""
    x = torch.randn(3, cols, device=DEV) * torch.tensor([[1e25], [1e37], [1.0]], device=DEV)
    w = torch.ones(cols, device=DEV)
    q, s = serve.norm_quantize(x, w)
    torch.cuda.synchronize()
    want, scale = so.norm_quantize(x.cpu().numpy(), w.cpu().numpy(), np.float32(1e-6))
    np.testing.assert_array_equal(q.cpu().numpy(), want)
    np.testing.assert_allclose(s.cpu().numpy(), scale, rtol=U * ((cols / 64 + 9) / 2 + 8))


def test_refusals():
    x, w = torch.randn(5, 64, device=DEV), torch.ones(64, device=DEV)
    q, s = serve.norm_quantize(x, w)
    f = serve.norm_quantize
    for bad in ((x[0], w), (x.half(), w), (x, w[:32]), (x, w.to(BF)), (x, w.cpu()), (x.t(), w)):
        with pytest.raises(ValueError):
            f(*bad)
    for kw in (dict(residual=x.to(BF)), dict(residual=x[:4]), dict(total=x), dict(residual=x, total=x[:, :32]),
               dict(out=q[:4]), dict(scale=s[:4]), dict(residual=x, total=x.to(BF))):
        with pytest.raises(ValueError):
            f(x, w, **kw)
    for kw in (dict(eps=0.0), dict(eps=float("nan"))):
        with pytest.raises(wz.WZError):
            f(x, w, **kw)
    g = serve.gated_int
    for bad in ((q, s, q, s, q[:4], s[:4]), (q, s, q[:, :32], s, q, s), (q, s[:4], q, s, q, s), (q, s, q, s, q, s[:4]),
                (x, s, q, s, q, s), (q, s, q.cpu(), s, q, s)):
        with pytest.raises(ValueError):
            g(*bad)
    for kw in (dict(activation="tanh"), dict(activation=2), dict(gate_bias=s[:2]), dict(up_bias=s.double()),
               dict(out=torch.zeros(5, 6, device=DEV)), dict(out_dtype=torch.float16)):
        with pytest.raises(ValueError):
            g(q, s, q, s, q, s, **kw)
    m = serve.matmul_int
    for kw in (dict(activation="swish"), dict(residual=torch.zeros(5, 5, device=DEV)),
               dict(residual=torch.zeros(5, 4, device=DEV, dtype=BF)), dict(residual=s)):
        with pytest.raises(ValueError):
            m(q, s, q, s, **kw)


def block(s, x, out):
    """A feed-forward block onto the residual stream, as a layer runs it."""
    h, hs, total = serve.norm_quantize(x, s["norm"], residual=s["res"])
    act = serve.gated_int(h, hs, s["w"][:s["n"]], s["ws"][:s["n"]], s["w"][s["n"]:], s["ws"][s["n"]:])
    a, asc = serve.quantize_rows(act)
    y = serve.matmul_int(a, asc, s["down"], s["downs"], residual=total)
    serve.matmul_int(h, hs, s["down2"], s["ws"][:s["down2"].shape[0]], bias=s["norm"][:s["down2"].shape[0]], out=out,
                     activation="gelu")
    return y


@pytest.mark.parametrize("M", [1, 64, 1300])
def test_captured_and_beside_another_stream(M):
    """A block captured and replayed with other rows, and two at once on streams of their own: the eager results."""
    C, N = 512, 1152
    r = np.random.default_rng(M)
    _, _, w, ws = codes(r, 2 * N, C, 0, 0)
    _, _, down, downs = codes(r, C, N, 0, 0)
    _, _, down2, _ = codes(r, 300, C, 0, 0)
    s = dict(norm=1 + 0.1 * torch.randn(C, device=DEV), res=torch.randn(M, C, device=DEV).to(BF), w=w, ws=ws, n=N, down=down,
             downs=downs, down2=down2)
    xs = [torch.randn(M, C, device=DEV).to(BF) for _ in range(4)]
    want = []
    for x in xs:
        out = torch.zeros(M, 300, dtype=BF, device=DEV)
        want.append((block(s, x, out), out))
    x, out = xs[0].clone(), torch.zeros(M, 300, dtype=BF, device=DEV)
    block(s, x, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = block(s, x, out)
    for k in (1, 2, 3, 0, 2):
        x.copy_(xs[k])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[k][0]) and torch.equal(out, want[k][1]), k
        block(s, xs[k], torch.empty_like(out))  # (work of the program's own between replays)
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    torch.cuda.synchronize()
    for k in range(4):
        with torch.cuda.stream(streams[k % 2]):
            out = torch.zeros(M, 300, dtype=BF, device=DEV)
            got[k % 2].append((block(s, xs[k], out), out))
    torch.cuda.synchronize()
    for k in range(4):
        a, b = got[k % 2][k // 2]
        assert torch.equal(a, want[k][0]) and torch.equal(b, want[k][1]), k
