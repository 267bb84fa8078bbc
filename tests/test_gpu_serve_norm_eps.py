"""wz_norm_quantize with an eps of the size of the squares, where those pass fp32.  Marked gpu.

Tolerance: tests/test_gpu_serve_layer.py's of norms of large numbers, and a rounding of eps.
"""
import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve
from serve_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("cols", [16, 3584, 20000])
@pytest.mark.parametrize("eps", [1e-6, 1e33, 1e38, 3.3e38])
def test_eps_beside_large_squares(cols, eps):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()
    r = np.random.default_rng(cols)
    size = np.array([[1e16], [4e18], [1e19], [1e21], [1.0]])
    x = (r.choice([-1.0, 1.0], (5, cols)) * r.uniform(0.9, 1.0, (5, cols)) * size).astype(np.float32)
    w = r.uniform(0.5, 1.0, cols).astype(np.float32)
    q, s = serve.norm_quantize(torch.from_numpy(x).to(DEV), torch.from_numpy(w).to(DEV), eps=eps)
    torch.cuda.synchronize()
    want, scale = so.norm_quantize(x, w, np.float64(np.float32(eps)))
    np.testing.assert_array_equal(q.cpu().numpy(), want)
    np.testing.assert_allclose(s.cpu().numpy(), scale, rtol=U * ((cols / 64 + 9) / 2 + 9))
