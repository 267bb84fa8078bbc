"""Attention of few rows whose blocks are cut into pieces by themselves, against the float64 oracle (tolerance: as in
test_gpu_serve_attention).  Marked gpu.
"""
import pytest
import torch

import libutil
from paper_2607_23265_amd import serve
from serve_util import Case
from test_gpu_serve_attention import _run

pytestmark = pytest.mark.gpu

CASES = [
    # new, kv, heads, q heads, dim, page, causal, window, max_kv
    ([1], [1286], 4, 28, 128, 64, True, 0, None),         # 21 tiles, pieces of 4 or fewer
    ([1], [1025], 1, 3, 64, 16, True, 0, None),
    ([1, 1], [1700, 1601], 2, 4, 128, 32, True, 0, None),
    ([1, 1, 1], [2600, 64, 0], 1, 7, 128, 16, True, 0, None),  # one piece, and none
    ([1, 0, 1], [5000, 9, 257], 4, 8, 64, 128, True, 0, None),
    ([1], [1], 1, 1, 64, 16, True, 0, 9000),              # a bound far above the lengths
    ([1, 1], [0, 129], 2, 2, 128, 64, True, 0, 9000),
    ([5], [2300], 1, 5, 128, 64, True, 0, None),          # 25 rows
    ([9, 2], [1900, 1100], 1, 7, 64, 32, True, 0, None),  # 63 rows
    ([16], [2100], 1, 4, 128, 16, False, 0, None),
    ([2, 1], [4000, 3000], 2, 4, 64, 64, True, 1500, None),
    ([9, 5], [1900, 1100], 1, 7, 128, 32, True, 0, None),  # 63 and 35 rows: two blocks of 32 each
    ([5] * 12, [900 + 60 * i for i in range(12)], 2, 14, 128, 16, True, 0, None),
    ([5] * 3, [2600, 3000, 90], 2, 14, 128, 64, True, 300, None),
    ([90], [4000], 2, 8, 128, 64, True, 211, None),       # a prompt whose window is short: not shared
    ([16], [2100], 1, 4, 64, 16, False, 0, None),
    ([1] * 31, [1600 + 13 * i for i in range(31)], 4, 8, 64, 16, True, 0, None),
    ([1] * 33, [1600 + 13 * i for i in range(33)], 4, 8, 64, 16, True, 0, None),  # a block too many for it
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_pieces(i):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()
    new, kv, heads, q_heads, dim, page, causal, window, max_kv = CASES[i]
    print(f"[case] pieces {CASES[i]}", flush=True)
    c = Case(new, kv, heads, dim, page, seed=300 + i).fill(loud=1.0 + i % 3)
    if max_kv:
        import numpy as np
        c.table = np.concatenate([c.table, np.full((len(kv), max_kv // page + 1), -1, np.int32)], 1)
    _run(c, q_heads, causal=causal, window=window, max_kv=max_kv)


def test_pieces_of_a_block_give_the_bits_again():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()
    c = Case([1], [1286], 4, 128, 64, seed=320).fill()
    cache, batch = c.device_cache(), c.batch()
    q = torch.randn(1, 28, 128, device="cuda:0").to(torch.bfloat16)
    assert serve.attention_workspace_bytes(cache, batch, 28, 1) > 0
    want = serve.cache_attention(cache, batch, q)
    for _ in range(5):
        assert torch.equal(serve.cache_attention(cache, batch, q), want)
