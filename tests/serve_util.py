"""Shared by the serving operators' tests: ragged batches over shuffled pages, kept in NumPy for the oracle."""
import numpy as np
import torch

from oracle import serve_oracle as so
from paper_2607_23265_amd import serve

DEV = "cuda:0"


def bf16(x):
    """float32 rounded to bfloat16, as float32."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


class Case:
    """Lengths (new tokens and tokens in the cache, these counted), a shuffled page table and a pool of garbage."""

    def __init__(self, new, kv, heads, dim, page, seed=0, spare=2, garbage=True):
        r = self.rng = np.random.default_rng(seed)
        self.new, self.kv, self.heads, self.dim, self.page = list(new), list(kv), heads, dim, page
        need = [-(-x // page) for x in kv]
        self.pages = sum(need) + spare
        ids = r.permutation(self.pages)
        width = max(need) + 1
        self.table = np.full((len(kv), width), -7, np.int32)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = ids[at:at + m]
            at += m
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.tokens = int(self.start[-1])
        # whatever lies in a fresh pool: NaN codes among it, and scales that are not numbers
        fill = r.integers(0, 256, (self.pages, heads, page, dim), dtype=np.uint8) if garbage else np.zeros(
            (self.pages, heads, page, dim), np.uint8)
        self.cache = dict(k=fill, v=np.ascontiguousarray(np.roll(fill, 3, 0).transpose(0, 1, 3, 2)),
                          k_scale=np.full((self.pages, heads), np.nan, np.float32),
                          v_scale=np.full((self.pages, heads), np.nan, np.float32))

    def put(self, new, kv, k, v):
        """The oracle's append of rows to this case's cache."""
        start = np.concatenate([[0], np.cumsum(new)])
        so.append(self.cache, start, kv, self.table, k, v)

    def fill(self, loud=1.0):
        """The whole of every sequence appended by the oracle at once."""
        n = sum(self.kv)
        k = self.rng.normal(size=(n, self.heads, self.dim)).astype(np.float32)
        v = self.rng.normal(size=(n, self.heads, self.dim)).astype(np.float32) + np.float32(0.3)
        self.put(self.kv, self.kv, loud * k, v)
        return self

    def device_cache(self):
        c = self.cache
        t = {n: torch.from_numpy(np.ascontiguousarray(c[n])).to(DEV) for n in c}
        return serve.PagedCache(t["k"].view(serve.E4M3), t["v"].view(serve.E4M3), t["k_scale"], t["v_scale"])

    def batch(self, max_tokens=None, max_kv=None):
        def dev(x):
            return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)
        return serve.Ragged(dev(self.start), dev(self.kv), dev(self.table),
                            max(self.new) if max_tokens is None else max_tokens,
                            max(self.kv) if max_kv is None else max_kv)


def codes(t):
    return t.view(torch.uint8).cpu().numpy()


def same_cache(got, want):
    """Codes and scales bit for bit (NaN scales of pages that nothing wrote among them)."""
    torch.cuda.synchronize()
    for name in ("k_scale", "v_scale"):
        np.testing.assert_array_equal(getattr(got, name).cpu().numpy(), want[name], err_msg=name)
    for name in ("k", "v"):
        np.testing.assert_array_equal(codes(getattr(got, name)), want[name], err_msg=name)
