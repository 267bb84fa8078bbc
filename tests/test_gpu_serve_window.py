"""Windows longer than any sequence: the rows of a batch whose first tokens stand before the cache see what they see
without a window (tolerance: as in test_gpu_serve_attention).  Marked gpu.
"""
import numpy as np
import pytest
import torch

import libutil
from serve_util import Case, bf16
from test_gpu_serve_attention import _run

pytestmark = pytest.mark.gpu

CASES = [
    # new, kv, q heads (of one), dim; where n > kv, some rows of the first block stand at negative places, others do not
    ([12], [7], 1, 64),        # a block of 16 rows
    ([20], [15], 1, 64),       # of 32
    ([9], [5], 7, 128),        # two of 32
    ([30], [21], 2, 64),       # of 64
    ([200], [130], 1, 64),     # of 128
    ([90, 3], [70, 700], 2, 128),
    ([8], [1700], 1, 64),      # shared by several workgroups
    ([200], [2100], 1, 128),
]


@pytest.mark.parametrize("i", range(len(CASES)))
@pytest.mark.parametrize("window", [1 << 24, 2 ** 31 - 60, 2 ** 31 - 1])
def test_longest_windows(i, window):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()
    new, kv, q_heads, dim = CASES[i]
    print(f"[case] window {window} {CASES[i]}", flush=True)
    c = Case(new, kv, 1, dim, 64, seed=400 + i).fill()
    q = bf16(c.rng.normal(size=(c.tokens, q_heads, dim)) * 1.5)
    out, lse = _run(c, q_heads, window=window, q=q)
    plain, plain_lse = _run(c, q_heads, q=q)
    assert torch.equal(out, plain) and torch.equal(lse, plain_lse)
    seen = np.concatenate([np.arange(m - n, m) >= 0 for n, m in zip(new, kv)])
    assert np.array_equal(np.isfinite(lse.cpu().numpy()).all(1), seen)
