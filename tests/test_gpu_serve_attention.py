"""wz_cache_attention against the float64 oracle.  Marked gpu.

Tolerance, from the kernel's roundings (u = 2^-8, bfloat16's unit): each probability is rounded to bfloat16 once (u
times the sum of p |v|), the result once (u times its magnitude); scores are fp32 sums of exact products, off by at
most (head_dim + 4) 2^-24 of the sum of |q k| |scale|, which moves a probability by that share, twice with the sum's; the
sums over tokens and the exponentials add less than 2^-12 of p |v|.
"""
import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve
from serve_util import DEV, Case, bf16

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


def _check(got, lse, want):
    out, mag, ref_lse, reach = want
    got = got.float().cpu().numpy().astype(np.float64)
    score = (got.shape[2] + 4) * 2.0 ** -24 * reach
    tol = U * np.abs(out) * (1 + U) + (U + 2.0 ** -12 + 2 * score[..., None]) * mag
    assert np.array_equal(np.isnan(got), np.isnan(out))
    worst = np.nanmax(np.abs(got - out) / np.maximum(tol, 1e-30), initial=0.0)
    print(f"[err] attention: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0
    if lse is not None:
        lse = lse.cpu().numpy().astype(np.float64)
        empty = np.isneginf(ref_lse)
        assert np.array_equal(np.isneginf(lse), empty)
        off = np.abs(lse - ref_lse)[~empty] - score[~empty]
        assert np.all(np.isnan(ref_lse[~empty]) == np.isnan(lse[~empty]))
        # the sum of up to 2^13 fp32 exponentials, its logarithm, and the rounding of lse itself
        assert np.nanmax(off - 2.0 ** -22 * np.abs(ref_lse[~empty]), initial=0.0) <= 2.0 ** -14


def _run(c, q_heads, scale=None, causal=True, window=0, pad=0, loud=1.5, max_tokens=None, max_kv=None, q=None):
    if q is None:
        q = bf16(c.rng.normal(size=(c.tokens, q_heads, c.dim)) * loud)
    x = torch.from_numpy(q).to(DEV).to(torch.bfloat16)
    if pad:
        wide = torch.zeros(c.tokens, q_heads + pad, c.dim, dtype=torch.bfloat16, device=DEV)
        wide[:, pad:] = x
        x = wide[:, pad:]
    out = torch.full((c.tokens, q_heads + pad, c.dim), 7.0, dtype=torch.bfloat16, device=DEV)[:, :q_heads]
    lse = torch.full((c.tokens, q_heads), 7.0, device=DEV)
    serve.cache_attention(c.device_cache(), c.batch(max_tokens, max_kv), x, scale=scale, causal=causal, window=window,
                          out=out, lse=lse)
    torch.cuda.synchronize()
    scale = c.dim ** -0.5 if scale is None else scale
    want = so.attention(c.cache, c.start, c.kv, c.table, q, scale, causal, window)
    _check(out, lse, want)
    return out, lse


CASES = [
    # new, kv, heads, q heads, dim, page, causal, window
    ([1], [1], 1, 1, 64, 16, True, 0),
    ([1], [64], 1, 7, 128, 64, True, 0),
    ([1], [65], 4, 28, 128, 64, True, 0),
    ([1, 1, 1], [700, 3, 1500], 2, 16, 128, 16, True, 0),
    ([1] * 5, [0, 1, 15, 16, 17], 1, 4, 64, 16, True, 0),
    ([1] * 67, [9 * i for i in range(67)], 1, 2, 64, 32, True, 0),
    ([3, 0, 5], [300, 20, 5], 2, 2, 64, 32, True, 0),
    ([5, 2], [900, 1200], 1, 5, 128, 128, True, 0),      # 25 rows
    ([9, 1], [40, 1300], 2, 14, 128, 64, True, 0),       # 63 rows
    ([16], [700], 1, 4, 64, 64, False, 0),               # 64 rows, no order
    ([4, 4], [600, 90], 1, 3, 64, 16, True, 50),
    ([1, 1], [2000, 31], 2, 8, 128, 32, True, 100),
    ([65], [65], 1, 1, 64, 64, True, 0),                 # the prompt kernel from here
    ([100, 3], [163, 700], 2, 4, 128, 16, True, 0),
    ([128], [128], 1, 1, 128, 64, False, 0),
    ([150, 0, 7], [150, 40, 64], 1, 7, 128, 128, True, 0),
    ([90, 33], [500, 33], 2, 2, 64, 32, True, 70),
    ([200], [130], 1, 1, 64, 16, True, 0),               # 70 rows stand before the cache and see nothing
    ([70], [0], 1, 1, 128, 16, True, 0),
    ([70, 70], [1000, 70], 1, 1, 64, 64, False, 0),
    ([300], [1300], 1, 1, 64, 64, True, 1),              # each token sees itself
    # long: several workgroups to a block, for each number of rows
    ([1, 1, 1], [5000, 64, 1700], 2, 14, 128, 16, True, 0),
    ([1] * 80, [1600 + 7 * i for i in range(80)], 1, 4, 64, 128, True, 0),
    ([3, 1], [2500, 1601], 1, 8, 64, 64, True, 0),
    ([12, 2], [1700, 3000], 1, 5, 128, 32, True, 900),
    ([70, 5], [2100, 1600], 2, 4, 128, 64, True, 0),
    ([96], [1700], 64, 512, 64, 64, True, 0),            # 384 blocks of a prompt
    ([200, 70], [1800, 1900], 1, 3, 64, 16, False, 0),
    ([90], [3000], 1, 2, 64, 32, True, 2000),
    ([350, 200], [350, 201], 32, 128, 64, 64, True, 0),  # more blocks than workgroups run at once
    ([1300], [1300], 1, 1, 64, 64, True, 0),             # blocks of 1 to 21 tiles
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_attention(i):
    new, kv, heads, q_heads, dim, page, causal, window = CASES[i]
    print(f"[case] attention {CASES[i]}", flush=True)
    c = Case(new, kv, heads, dim, page, seed=100 + i).fill(loud=1.0 + i % 3)
    _run(c, q_heads, causal=causal, window=window, pad=i % 2)


def test_scales_of_the_scores():
    for scale in (0.0, -0.2, 3.0):
        for new in (1, 80):
            c = Case([new], [150], 1, 64, 16, seed=20).fill()
            _run(c, 2, scale=scale)


def test_loud_and_quiet_pages():
    """Pages of very different scales."""
    for new in (1, 66):
        c = Case([new], [400], 1, 64, 16, seed=21)
        n = 400
        loud = np.exp2(np.repeat(c.rng.integers(-20, 3, 25), 16))[:, None, None]
        k, v = (c.rng.normal(size=(n, 1, 64)).astype(np.float32) * loud.astype(np.float32) for _ in range(2))
        c.put([n], [n], k, v)
        _run(c, 1)


def test_entries_without_a_page():
    for new, kv in ((2, 333), (90, 333), (2, 2000), (90, 2000)):
        c = Case([new, new], [kv, 200], 2, 64, 16, seed=22).fill()
        c.table[0, 3], c.table[0, 20], c.table[1, :13] = -1, c.pages + 5, -3  # the second sequence has nothing at all
        _run(c, 4)


def test_not_numbers_stay_with_the_rows_that_see_them():
    for new in (3, 100):
        c = Case([new], [200], 1, 64, 32, seed=23)
        k, v = (c.rng.normal(size=(200, 1, 64)).astype(np.float32) for _ in range(2))
        k[150, 0, 3] = np.nan
        v[198, 0, 9] = np.inf
        c.put([200], [200], k, v)
        out, _ = _run(c, 2)
        bad = torch.isnan(out.float()).any(-1).cpu().numpy()
        place = 200 - new + np.arange(new)
        assert np.array_equal(bad.all(1), place >= 150) and np.array_equal(bad.any(1), place >= 150)
        _run(c, 2, window=40)


def test_every_score_not_a_number():
    """Sequences whose every key is NaN, alone and shared by several workgroups."""
    for new, kv in ((1, 40), (1, 3000), (70, 1000), (70, 3000)):
        c = Case([new], [kv], 1, 64, 64, seed=24).fill()
        c.cache["k"][:] = 127
        out, lse = _run(c, 1)
        assert torch.isnan(out.float()).all() and torch.isnan(lse).all()


def test_bounds_larger_than_the_batch():
    """max_tokens and max_kv are bounds: the same rows come out, of another plan."""
    c = Case([1, 2], [500, 90], 2, 64, 16, seed=25).fill()
    c.table = np.concatenate([c.table, np.full((2, 400), -1, np.int32)], 1)
    _run(c, 4)
    _run(c, 4, max_kv=6000)
    _run(c, 4, max_tokens=100, max_kv=6000)


def test_same_bits_again():
    c = Case([1, 1], [5000, 777], 1, 128, 64, seed=26).fill()
    q = bf16(c.rng.normal(size=(2, 7, 128)))
    a, la = _run(c, 7, q=q)
    b, lb = _run(c, 7, q=q)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_workspace_contents_do_not_matter():
    c = Case([1], [4000], 1, 64, 16, seed=27).fill()
    cache, batch = c.device_cache(), c.batch()
    q = torch.from_numpy(bf16(c.rng.normal(size=(1, 4, 64)))).to(DEV).to(torch.bfloat16)
    need = serve.attention_workspace_bytes(cache, batch, 4, 1)
    assert need > 0
    first = None
    for byte in (0, 0xFF, 0x7F):
        ws = torch.full((need,), byte, dtype=torch.uint8, device=DEV)
        out = serve.cache_attention(cache, batch, q, ws=ws)
        first = out if first is None else first
        assert torch.equal(first, out)


def test_far_pages():
    """Pages whose bytes lie past 2^32, with few rows and with many."""
    heads, dim, page = 8, 128, 128
    pages = (1 << 32) // (heads * dim * page) + 40
    big = serve.PagedCache.new(pages, heads, dim, page)
    for new in (1, 80):
        c = Case([new], [300], heads, dim, page, seed=28, spare=0).fill()
        far = np.array([pages - 1, pages - 20, 3])
        for name in ("k", "v", "k_scale", "v_scale"):
            x = torch.from_numpy(np.ascontiguousarray(c.cache[name][c.table[0, :3]])).to(DEV)
            t = getattr(big, name)
            (t.view(torch.uint8) if name in ("k", "v") else t)[torch.from_numpy(far).to(DEV)] = x
        q = bf16(c.rng.normal(size=(new, heads, dim)))
        want = so.attention(c.cache, c.start, c.kv, c.table, q, dim ** -0.5)
        c.table[0, :3] = far
        got = serve.cache_attention(big, c.batch(), torch.from_numpy(q).to(DEV).to(torch.bfloat16))
        torch.cuda.synchronize()
        _check(got, None, want)


def test_graph_replays():
    """Captured and replayed with other work between: the same bits as the eager call."""
    c = Case([1, 1], [3000, 500], 2, 64, 16, seed=29).fill()
    cache, batch = c.device_cache(), c.batch()
    q = torch.from_numpy(bf16(c.rng.normal(size=(2, 4, 64)))).to(DEV).to(torch.bfloat16)
    ws = torch.empty(serve.attention_workspace_bytes(cache, batch, 4, 2), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    want = serve.cache_attention(cache, batch, q, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serve.cache_attention(cache, batch, q, out=out, ws=ws)
    for _ in range(4):
        out.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
