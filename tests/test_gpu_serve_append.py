"""wz_cache_append against the oracle, codes and scales bit for bit.  Marked gpu.

The oracle rotates in float32 products and sums, as the header defines it, so every rounding that follows is of the
same number; no tolerance is needed.  Rotated queries are the oracle's rounded to bfloat16.
"""
import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve
from serve_util import DEV, Case, bf16, same_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


def _table(max_pos, rot):
    f = np.arange(max_pos)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
    return np.concatenate([np.cos(f), np.sin(f)], 1).astype(np.float32)


def _rows(c, heads, dtype, tokens, loud=1.0):
    x = c.rng.normal(size=(tokens, heads, c.dim)) * np.exp(c.rng.normal(size=(tokens, heads, 1))) * loud
    return bf16(x) if dtype == torch.bfloat16 else x.astype(np.float32)


def _dev(x, dtype, pad=0):
    """On the device; pad > 0: as part of wider rows."""
    t = torch.from_numpy(x).to(DEV).to(dtype)
    if pad:
        wide = torch.full((t.shape[0], t.shape[1] + pad, t.shape[2]), float("nan"), dtype=dtype, device=DEV)
        wide[:, 1:1 + t.shape[1]] = t
        return wide[:, 1:1 + t.shape[1]]
    return t


CASES = [
    # new, kv, heads, q heads, dim, page, rot, sections, interleaved, dtype
    ([1], [1], 1, 1, 64, 16, 64, (), False, torch.bfloat16),
    ([5, 0, 1, 33], [5, 0, 17, 40], 2, 4, 128, 16, 128, (), False, torch.bfloat16),
    ([70, 1, 64], [75, 129, 64], 4, 28, 128, 64, 128, (16, 24, 24), False, torch.bfloat16),
    ([3, 130], [35, 191], 3, 3, 64, 32, 32, (5, 11), True, torch.float32),
    ([200, 1], [201, 128], 2, 2, 128, 128, 64, (10, 11, 11), False, torch.float32),
    ([129], [257], 1, 8, 64, 128, 16, (), True, torch.bfloat16),
    ([17] * 70, [20 + i for i in range(70)], 1, 2, 64, 16, 48, (24,), False, torch.bfloat16),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_append(i):
    new, kv, heads, q_heads, dim, page, rot, sections, inter, dtype = CASES[i]
    print(f"[case] append {CASES[i]}", flush=True)
    c = Case(new, kv, heads, dim, page, seed=i)
    held = [b - a for a, b in zip(new, kv)]
    n = sum(held)
    if n:  # what the sequences held before, quieter than most of what comes
        c.put(held, held, _rows(c, heads, dtype, n, 0.3), _rows(c, heads, dtype, n, 0.3))
    cache = c.device_cache()
    k, v, q = (_rows(c, h, dtype, c.tokens) for h in (heads, heads, q_heads))
    table = _table(max(kv) + 3, rot)
    axes = max(1, len(sections))
    pos = c.rng.integers(-2, max(kv) + 6, (axes, c.tokens)).astype(np.int32)  # some outside the table
    turn = serve.Rotation(torch.from_numpy(table).to(DEV), sections, inter)
    got = serve.cache_append(cache, c.batch(), _dev(k, dtype, 2), _dev(v, dtype, i % 2), turn,
                             torch.from_numpy(pos).to(DEV), q=_dev(q, dtype, 3))
    args = (pos, table, sections or (rot // 2,), inter)
    c.put(new, kv, so.rotate(k, *args), v)
    same_cache(cache, c.cache)
    np.testing.assert_array_equal(got.float().cpu().numpy(), bf16(so.rotate(q, *args)))


def test_one_by_one():
    """A prompt, then token after token, some louder: the page's scale grows and what it holds moves with it."""
    c = Case([21, 5], [21, 5], 2, 64, 32, seed=9)
    cache = c.device_cache()
    new, kv = [21, 5], [21, 5]
    c.table = np.concatenate([c.table, c.table * 0 - 1], 1)
    c.table[:, :3] = [[0, 1, 2], [3, 4, -1]]
    c.pages, pool = 5, {}
    for name, x in c.cache.items():
        pool[name] = np.concatenate([x, x, x])[:5].copy()
    c.cache = pool
    cache = c.device_cache()
    for step in range(30):
        c.new, c.kv = new, kv
        c.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        c.tokens = sum(new)
        loud = 2.0 ** (step % 7 - 3)
        k, v = _rows(c, 2, torch.bfloat16, c.tokens, loud), _rows(c, 2, torch.bfloat16, c.tokens, 1 / loud)
        serve.cache_append(cache, c.batch(), _dev(k, torch.bfloat16), _dev(v, torch.bfloat16))
        c.put(new, kv, k, v)
        same_cache(cache, c.cache)
        new, kv = [1, 1], [kv[0] + 1, kv[1] + 1]


def test_extremes():
    """The least and the largest scale, zeros, subnormal codes, numbers beyond the largest code."""
    c = Case([6], [6], 1, 64, 16, seed=3)
    k = np.zeros((6, 1, 64), np.float32)
    v = np.zeros((6, 1, 64), np.float32)
    k[0] = 3.3e38
    k[1] = np.linspace(-3e38, 3e38, 64)
    k[2, 0, ::2] = 1e-38
    v[3] = 448.0
    v[4] = np.linspace(0, 4, 64) * 2.0 ** -9
    v[5, 0, 7] = -449.0
    cache = c.device_cache()
    serve.cache_append(cache, c.batch(), _dev(k, torch.float32), _dev(v, torch.float32))
    c.put([6], [6], k, v)
    same_cache(cache, c.cache)
    c2 = Case([3], [3], 1, 128, 16, seed=4)  # nothing but zeros: the least scale
    z = np.zeros((3, 1, 128), np.float32)
    cache = c2.device_cache()
    serve.cache_append(cache, c2.batch(), _dev(z, torch.float32), _dev(z, torch.float32))
    c2.put([3], [3], z, z)
    same_cache(cache, c2.cache)


def test_not_numbers():
    """NaN and infinities: a NaN key for exactly those tokens and heads, finite values, scales untouched."""
    c = Case([40], [44], 2, 64, 32, seed=5)
    c.put([4], [4], *(_rows(c, 2, torch.float32, 4) for _ in range(2)))
    cache = c.device_cache()
    k, v = _rows(c, 2, torch.float32, 40), _rows(c, 2, torch.float32, 40)
    k[3, 0, 5], k[9, 1, 60], v[3, 1, 2], v[30, 0, 0], v[31, 1] = np.nan, np.inf, -np.inf, np.nan, np.inf
    serve.cache_append(cache, c.batch(), _dev(k, torch.float32), _dev(v, torch.float32))
    c.put([40], [44], k, v)
    same_cache(cache, c.cache)


def test_no_page_and_negative_places():
    """Tokens of entries that hold no page, and of places before the sequence, are dropped; nothing else moves."""
    c = Case([50, 9], [50, 5], 1, 64, 16, seed=6)
    c.table[0, 1], c.table[0, 2] = -1, c.pages  # neither is a page
    cache = c.device_cache()
    k, v = _rows(c, 1, torch.bfloat16, 59), _rows(c, 1, torch.bfloat16, 59)
    serve.cache_append(cache, c.batch(), _dev(k, torch.bfloat16), _dev(v, torch.bfloat16))
    c.put([50, 9], [50, 5], k, v)
    same_cache(cache, c.cache)


def test_no_tokens():
    c = Case([0, 0], [3, 0], 1, 64, 16, seed=7)
    cache = c.device_cache()
    empty = torch.empty(0, 1, 64, dtype=torch.bfloat16, device=DEV)
    serve.cache_append(cache, c.batch(), empty, empty)
    same_cache(cache, c.cache)


def test_far_pages():
    """Pages whose bytes lie past 2^32."""
    heads, dim, page = 8, 128, 128
    pages = (1 << 32) // (heads * dim * page) + 40
    cache = serve.PagedCache.new(pages, heads, dim, page)
    c = Case([300], [300], heads, dim, page, seed=8, spare=0)
    far = np.array([pages - 1, pages - 20, 3], np.int32)
    small = c.table[0, :3].copy()
    c.put([300], [300], *(x := [_rows(c, heads, torch.bfloat16, 300) for _ in range(2)]))
    c.table[0, :3] = far
    serve.cache_append(cache, c.batch(), *(_dev(y, torch.bfloat16) for y in x))
    torch.cuda.synchronize()
    at = torch.from_numpy(far.astype(np.int64)).to(DEV)
    for name in ("k", "v"):
        got = getattr(cache, name).view(torch.uint8)[at].cpu().numpy()
        want = c.cache[name][small]
        for i, m in enumerate((128, 128, 44)):  # slots behind the last token are not defined here
            assert np.array_equal(got[i][:, :m] if name == "k" else got[i][..., :m],
                                  want[i][:, :m] if name == "k" else want[i][..., :m]), (name, i)
    assert np.array_equal(cache.k_scale[at].cpu().numpy(), c.cache["k_scale"][small])


def test_other_stream():
    c = Case([64], [64], 2, 64, 16, seed=11)
    cache = c.device_cache()
    k, v = _rows(c, 2, torch.bfloat16, 64), _rows(c, 2, torch.bfloat16, 64)
    args = c.batch(), _dev(k, torch.bfloat16), _dev(v, torch.bfloat16)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        serve.cache_append(cache, *args)
    side.synchronize()
    c.put([64], [64], k, v)
    same_cache(cache, c.cache)
