"""Outputs and workspaces that the serving binding makes are tensors as torch makes them: filled beforehand where the
program asks for that, and seen by dispatch modes.  Marked gpu.
"""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

import libutil
from paper_2607_23265_amd import serve
from serve_util import DEV

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


@pytest.fixture
def deterministic():
    was, warn = torch.are_deterministic_algorithms_enabled(), torch.is_deterministic_algorithms_warn_only_enabled()
    fill = torch.utils.deterministic.fill_uninitialized_memory
    torch.use_deterministic_algorithms(True)
    torch.utils.deterministic.fill_uninitialized_memory = True
    yield
    torch.use_deterministic_algorithms(was, warn_only=warn)
    torch.utils.deterministic.fill_uninitialized_memory = fill


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def rows(tokens, heads, dim=64):
    return torch.randn(tokens, heads, dim, device=DEV).to(BF)


def attention(tokens, new):
    """Softmax attention of `new` rows of `tokens` over a cache of their own."""
    cache = serve.PagedCache.new(4, 2, 64, page_size=32)
    batch = serve.Ragged(ints(0, new), ints(new), ints(0, 1, 2, 3)[None], new, new)
    k, v, q = rows(tokens, 2), rows(tokens, 2), rows(tokens, 4)
    serve.cache_append(cache, batch, k, v)
    return serve.cache_attention(cache, batch, q)


def decay(tokens, new):
    """Linear attention of the same rows."""
    states = serve.States.new(2, 4, 64)
    batch = serve.Ragged(ints(0, new), ints(new), torch.zeros(1, 0, dtype=torch.int32, device=DEV), new, new)
    return serve.decay_attention(states, batch, ints(1), rows(tokens, 4), rows(tokens, 2), rows(tokens, 2),
                                 torch.full((4,), -0.1, device=DEV))


@pytest.mark.parametrize("new", [5, 100])
@pytest.mark.parametrize("call", [attention, decay])
def test_rows_of_no_sequence_are_filled(call, new, deterministic):
    """Such rows are not written: where torch fills memory that is not initialised they hold its NaN."""
    junk = [torch.full((1 << 16,), 3.0, dtype=BF, device=DEV) for _ in range(8)]  # (what the allocator hands out next)
    del junk
    out = call(new + 7, new)
    torch.cuda.synchronize()
    assert torch.isnan(out[new:]).all() and torch.isfinite(out[:new]).all()


class Made(TorchDispatchMode):
    """Shapes and types of the tensors that torch makes."""

    def __init__(self):
        super().__init__()
        self.made = []

    def __torch_dispatch__(self, f, types, args=(), kwargs=None):
        out = f(*args, **(kwargs or {}))
        if f is torch.ops.aten.empty.memory_format:
            self.made.append((tuple(out.shape), out.dtype))
        return out


def test_dispatch_modes_see_the_outputs():
    x, w = torch.randn(6, 64, device=DEV), torch.ones(64, device=DEV)
    q, s = serve.quantize_rows(x)
    cache = serve.PagedCache.new(4, 2, 64, page_size=32)
    batch = serve.Ragged(ints(0, 6), ints(6), ints(0, 1, 2, 3)[None], 6, 6)
    states, one = serve.States.new(2, 4, 64), ints(1)
    k, h, ld = rows(6, 2), rows(6, 4), torch.full((4,), -0.1, device=DEV)
    int8, row, mat = ((6, 64), torch.int8), ((6,), F32), ((6, 6), BF)
    for f, want in ((lambda: serve.quantize_rows(x), [int8, row]),
                    (lambda: serve.norm_quantize(x, w, residual=x), [int8, row, ((6, 64), F32)]),
                    (lambda: serve.matmul_int(q, s, q, s), [mat]),
                    (lambda: serve.matmul_int(q, s, q, s, activation="gelu"), [mat]),
                    (lambda: serve.gated_int(q, s, q, s, q, s, out_dtype=F32), [((6, 6), F32)]),
                    (lambda: serve.cache_append(cache, batch, k, k, q=h), [((6, 4, 64), BF)]),
                    (lambda: serve.cache_attention(cache, batch, h), [((6, 4, 64), BF)]),
                    (lambda: serve.decay_attention(states, batch, one, h, k, k, ld), [((6, 4, 64), BF)])):
        with Made() as mode:
            f()
        torch.cuda.synchronize()
        assert all(x in mode.made for x in want), (want, mode.made)
