"""Arguments of the serving operators' binding that have the right size but not the right meaning.  Marked gpu."""
import copy

import pytest
import torch

import libutil
from paper_2607_23265_amd import serve
from serve_util import DEV, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


def _new(*shape):
    return torch.randn(*shape, device=DEV).to(torch.bfloat16)


def test_positions_go_by_axis():
    """[tokens, axes] has as many positions as [axes, tokens], of other tokens."""
    c = Case([4], [20], 2, 64, 16, seed=1).fill()
    cache, batch = c.device_cache(), c.batch()
    k, v = _new(4, 2, 64), _new(4, 2, 64)
    at = torch.arange(12, dtype=torch.int32, device=DEV).view(3, 4)
    table = torch.zeros(40, 64, device=DEV)
    three, one = serve.Rotation(table, (16, 8, 8)), serve.Rotation(table)
    for good in (at, at.flatten(), at[:, None]):  # axis by axis, however it is shaped
        serve.cache_append(cache, batch, k, v, three, good)
    for bad in (at.t().contiguous(), at.view(2, 6), at.view(4, 3), at[:2], at[:, :3].contiguous()):
        with pytest.raises(ValueError):
            serve.cache_append(cache, batch, k, v, three, bad)
    for good in (at[:1], at[0], at[0].view(4, 1)):
        serve.cache_append(cache, batch, k, v, one, good)
    with pytest.raises(ValueError):
        serve.cache_append(cache, batch, k, v, one, at)
    torch.cuda.synchronize()


def test_arguments_in_the_wrong_order():
    """A cache, a batch and a rotation are refused in each other's place; what is packed of them is the header's structs."""
    c = Case([3], [20], 2, 64, 16, seed=2).fill()
    cache, batch = c.device_cache(), c.batch()
    turn = serve.Rotation(torch.zeros(40, 64, device=DEV), (16, 8, 8), True)
    k, q, at = _new(3, 2, 64), _new(3, 4, 64), torch.zeros(3, 3, dtype=torch.int32, device=DEV)
    for a, b in ((batch, cache), (cache, cache), (batch, batch), (turn, batch), (cache, turn)):
        with pytest.raises(ValueError):
            serve.cache_append(a, b, k, k)
        with pytest.raises(ValueError):
            serve.cache_attention(a, b, q)
        with pytest.raises(ValueError):
            serve.attention_workspace_bytes(a, b, 4, 3)
    for bad in (cache, batch):
        with pytest.raises(ValueError):
            serve.cache_append(cache, batch, k, k, bad, at)
    mirrors = (
        (cache, serve._Cache(*(t.data_ptr() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)), *cache.k.shape)),
        (batch, serve._Ragged(batch.start.data_ptr(), batch.kv_len.data_ptr(), batch.table.data_ptr(), 1, 0, 3, 20,
                              batch.table.shape[1])),
        (turn, serve._Rotation(turn.table.data_ptr(), None, 40, 64, 3, 1, (16, 8, 8))))
    for x, m in mirrors:
        used = type(m)
        last = used._fields_[-1][0]  # (what follows it is padding)
        size = getattr(used, last).offset + getattr(used, last).size
        assert x.c[:size] == bytes(m)[:size], used


def test_fields_stay_and_copies_have_their_own():
    c = Case([1], [20], 2, 64, 16, seed=3).fill()
    cache, batch, q = c.device_cache(), c.batch(), _new(1, 4, 64)
    want = serve.cache_attention(cache, batch, q)
    with pytest.raises(AttributeError):
        batch.kv_len = batch.kv_len - 5
    with pytest.raises(AttributeError):
        batch.max_kv = 5
    assert torch.equal(serve.cache_attention(cache, batch, q), want)
    batch.kv_len.sub_(5)  # contents may change
    shorter = serve.cache_attention(cache, batch, q)
    assert not torch.equal(shorter, want)
    batch.kv_len.add_(5)
    twin, alike = copy.deepcopy((cache, batch))
    cache.k.view(torch.uint8).zero_(), batch.kv_len.zero_()
    assert torch.equal(serve.cache_attention(twin, alike, q), want)
    assert twin.k.data_ptr() != cache.k.data_ptr() and (alike.max_tokens, alike.max_kv) == (1, 20)
    turn = copy.deepcopy(serve.Rotation(torch.zeros(40, 64, device=DEV), (16, 8, 8), True))
    assert (turn.sections, turn.interleaved) == ((16, 8, 8), True) and turn.c[:8] == turn.table.data_ptr().to_bytes(8, "little")
