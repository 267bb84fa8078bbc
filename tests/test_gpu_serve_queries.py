"""wz_cache_append's queries: every row of the call is rotated, whichever of them a sequence has, and where no token is
stored.  Against the oracle, bit for bit.  Marked gpu.
"""
import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve
from serve_util import DEV, Case, bf16, same_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_tokens", [0, 2, 4])  # (two sequences of three and of four new tokens)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_row_is_rotated(max_tokens, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()
    print(f"[case] queries max_tokens={max_tokens} {dtype}", flush=True)
    c = Case([3, 4], [40, 4], 2, 64, 16, seed=500 + max_tokens)
    c.put([37, 0], [37, 0], *(bf16(c.rng.normal(size=(37, 2, 64))) for _ in range(2)))
    rows = c.tokens + 5  # five more than the sequences have
    k, v, q = (bf16(c.rng.normal(size=(rows, h, 64))) for h in (2, 2, 10))
    angle = np.arange(50)[:, None] * 10000.0 ** (-np.arange(16) / 16)
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    pos = c.rng.integers(0, 50, (1, rows)).astype(np.int32)
    cache = c.device_cache()
    d = [torch.from_numpy(x).to(DEV).to(dtype) for x in (k, v, q)]
    out = torch.full((rows, 10, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    got = serve.cache_append(cache, c.batch(max_tokens=max_tokens), d[0], d[1],
                             serve.Rotation(torch.from_numpy(table).to(DEV)), torch.from_numpy(pos).to(DEV), q=d[2],
                             q_out=out)
    torch.cuda.synchronize()
    assert got is out
    args = (pos, table, (16,), False)
    np.testing.assert_array_equal(out.float().cpu().numpy(), bf16(so.rotate(q, *args)))
    if max_tokens == 0:  # nothing is stored
        same_cache(cache, c.cache)
    if max_tokens == 4:
        c.put(c.new, c.kv, so.rotate(k, *args), v)
        same_cache(cache, c.cache)
