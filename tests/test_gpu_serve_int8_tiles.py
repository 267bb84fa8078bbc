"""wz_matmul_int in every tile it chooses from, with ragged edges, and cut into two launches.  Marked gpu.

Tolerance: the integer sum is exact; three fp32 operations and the rounding to bfloat16 follow.
"""
import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

SHAPES = [(70, 510, 8192),      # 32 x 32, four groups of waves
          (500, 1020, 2064),    # 64 x 32, two
          (190, 4990, 528),     # 64 x 64
          (300, 3600, 1040),    # 128 x 64
          (128, 14330, 3600),
          (690, 4590, 3600),    # 128 x 128, one to a CU
          (1500, 4100, 1040),   # 128 x 128, two
          (700, 4500, 1040),    # 192 x 128
          (1290, 4604, 1040),
          (3900, 4090, 2064),   # 256 x 256
          (2318, 14330, 2064)]  # 2304 rows in tiles of 256 x 256, 14 in small ones


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_tiles(M, N, K):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()
    print(f"[case] matmul {M}x{N}x{K}", flush=True)
    r = np.random.default_rng(M + N + K)
    a, w = (r.integers(-127, 128, (n, K), dtype=np.int8) for n in (M, N))
    a[-1], w[-1] = 127, -128  # the largest sums, in the last row and column
    sa, sw = (np.exp(r.normal(size=n)).astype(np.float32) for n in (M, N))
    bias = r.normal(size=N).astype(np.float32) * 100
    d = [torch.from_numpy(x).to(DEV) for x in (a, sa, w, sw, bias)]
    want, size = (torch.from_numpy(x).to(DEV) for x in so.matmul_int(a, sa, w, sw, bias))
    for out_dtype in (torch.bfloat16, torch.float32):
        out = torch.full((M + 1, N + 5), 5.0, dtype=out_dtype, device=DEV)
        serve.matmul_int(*d[:4], bias=d[4], out=out[:M, 3:3 + N])
        tol = 2.0 ** -24 * 4 * size + (2.0 ** -8 * want.abs() if out_dtype == torch.bfloat16 else 0)
        worst = float(((out[:M, 3:3 + N].double() - want).abs() / tol.clamp_min(1e-30)).max())
        print(f"[err] matmul {M}x{N}x{K} {out_dtype}: {worst:.3f} of the bound", flush=True)
        assert worst <= 1.0
        assert bool((out[:, :3] == 5).all()) and bool((out[:, 3 + N:] == 5).all()) and bool((out[M] == 5).all())
