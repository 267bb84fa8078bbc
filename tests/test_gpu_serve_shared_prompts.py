"""Prompts whose blocks several workgroups share, against the float64 oracle (tolerance: as in
test_gpu_serve_attention).  The bounds, above the lengths, are what has the blocks shared.  Marked gpu.
"""
import numpy as np
import pytest
import torch

import libutil
from paper_2607_23265_amd import serve
from serve_util import Case
from test_gpu_serve_attention import _run

pytestmark = pytest.mark.gpu

CASES = [
    # new, kv, heads, q heads, dim, page, causal, window, max_kv
    ([96], [1700], 64, 512, 64, 64, True, 0, 9000),       # one group of four waves: 384 blocks
    ([400], [700], 16, 112, 128, 16, True, 0, 6000),      # 352
    ([70, 5], [1100, 600], 2, 4, 128, 64, True, 0, 3000),  # two groups
    ([300], [300], 4, 28, 128, 128, True, 0, 6000),
    ([90, 0, 200], [90, 40, 150], 1, 3, 64, 32, True, 0, 6000),
    ([150], [1600], 1, 7, 64, 16, False, 0, 6000),
    ([200], [2900], 1, 2, 128, 32, True, 2500, 6000),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_shared_prompts(i):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()
    new, kv, heads, q_heads, dim, page, causal, window, max_kv = CASES[i]
    print(f"[case] shared prompts {CASES[i]}", flush=True)
    c = Case(new, kv, heads, dim, page, seed=600 + i).fill(loud=1.0 + i % 3)
    c.table = np.concatenate([c.table, np.full((len(kv), max_kv // page + 1), -1, np.int32)], 1)
    cache, batch = c.device_cache(), c.batch(max_kv=max_kv)
    assert serve.attention_workspace_bytes(cache, batch, q_heads, c.tokens, window) > 0
    _run(c, q_heads, causal=causal, window=window, max_kv=max_kv)
