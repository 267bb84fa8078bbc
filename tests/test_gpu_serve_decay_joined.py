"""wz_decay_attention: prompts whose runs' sums are added up by a launch of their own, and the precision of states and
outputs as a whole.  Marked gpu.

With u = 2^-24, a state meets, for each chunk of 64 tokens, a rounding for each of 12 products (four of 16 tokens, of three
parts each) and one where it is faded or raised, and two for each run that is added to it.  Element by element they add up
at worst: u (13 chunks + 2 runs) of the sum of the terms' magnitudes, and 160 u for the weights (tests/test_gpu_serve_decay.py).
As a whole (2-norms over all states of a call, of terms of either sign) roundings of sums are independent of one another: the
root of their number, each at most u of a sum no larger than the last one's by more than the decay that it still meets; and the
weights, each off by at most u (3 x + 3) with x = the decay's exponent, of which the terms that count have 1 to 2: 10 u.
An output as a whole is off by its rounding to bf16, at most half a step of 2^-7 of a number's power of two, evenly spread:
2^-8 / sqrt 3 of it, and the 2^-14 of its two products (for thousands of outputs, of which a mean square is that of a random
one to within some per cent).
"""
import math

import numpy as np
import pytest
import torch

import decay_cases as dc
import libutil
import test_gpu_serve_decay as td
from paper_2607_23265_amd import serve
from serve_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


def sums_of(new, runs):
    """Chunks of the longest sequence, and runs at most."""
    chunks = -(-max(new) // 64)
    return chunks, min(chunks, runs)


def state_norm_bound(new, runs):
    c, r = sums_of(new, runs)
    return U * (math.sqrt(13 * c + 2 * r) + 10)


def off(a, b):
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


def check(c, got, states, what):
    """Layer.check, and the bounds above."""
    c.check(got, states, what)
    z = serve.States(torch.from_numpy(c.state).to(DEV))
    runs = serve.decay_workspace_bytes(z, c.batch(), c.q.shape[0]) // (2 * c.state.shape[1] * c.dim ** 2 * 4)
    out, _, state, size = c.want()
    rows = int(c.start[-1])
    touched = [int(s) for s, n in zip(c.slot, c.new) if n]
    g, s = got[:rows].double().cpu().numpy(), states.state.double().cpu().numpy()
    chunks, r = sums_of(c.new, runs)
    worst = np.max(np.abs(s - state) / (U * (13 * chunks + 2 * r + 160) * size))
    norms = (off(s[touched], state[touched]) / state_norm_bound(c.new, runs),
             off(g, out[:rows]) / (2.0 ** -8 / 3 ** 0.5 + 2.0 ** -14))
    print(f"[err] {what}: state {worst:.3f} of the bound, as a whole {norms[0]:.3f}, outputs {norms[1]:.3f}", flush=True)
    assert worst <= 1 and norms[0] <= 1 and norms[1] <= 1


@pytest.mark.parametrize("new,held,heads,kv,dim,behind", dc.JOINED + dc.PADDED)
def test_joined_runs(new, held, heads, kv, dim, behind):
    c = td.Layer(new, held, heads, kv, dim, seed=sum(new) + dim, behind=behind)
    batch = c.batch(sum(new) + behind) if behind > 1000 else c.batch()
    z = serve.States(torch.from_numpy(c.state).to(DEV))
    ws = torch.full((serve.decay_workspace_bytes(z, batch, c.q.shape[0]),), 0xFF, dtype=torch.uint8, device=DEV)
    check(c, *c.run(batch=batch, ws=ws), f"joined {new[-2:]} {heads}/{kv} x {dim}")


@pytest.mark.parametrize("new,dim", dc.AGREE)
def test_joined_runs_agree_bit_for_bit(new, dim):
    """Again, with whatever lies in the workspace, on a stream of its own, captured and replayed."""
    td.test_runs_agree_bit_for_bit(new, dim)


@pytest.mark.parametrize("new,held", [([1] * 5, [1, 0, 1, 1, 1]), ([8, 3, 5], [1, 1, 0]), ([20], [1]), ([64, 129], [1, 1]),
                                      ([200], [0]), ([1286], [1]), ([700, 31, 1000], [0, 1, 1])])
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 128), (6, 2, 64)])
def test_precision(new, held, heads, kv, dim):
    c = td.Layer(new, held, heads, kv, dim, seed=sum(new))
    check(c, *c.run(), f"precision {new} {heads}/{kv} x {dim}")


@pytest.mark.parametrize("each", [1, 7])
def test_precision_over_many_calls(each):
    """A long answer, token by token: a state meets three roundings for each token, and the decay no drift."""
    steps, heads, dim = 420, 3, 64
    c = td.Layer([steps, steps], [1, 0], heads, 1, dim, seed=each)
    z = serve.States(torch.from_numpy(c.state).to(DEV))
    slot, ld = td.ints(c.slot), torch.from_numpy(c.log_decay).to(DEV)
    table = torch.zeros(2, 0, dtype=torch.int32, device=DEV)
    for i in range(0, steps, each):
        at = torch.cat([torch.arange(b * steps + i, b * steps + i + each, device=DEV) for b in range(2)])
        batch = serve.Ragged(td.ints([0, each, 2 * each]), td.ints([7 + i + each, i + each]), table, each, 7 + steps)
        serve.decay_attention(z, batch, slot, c.q[at], c.k[at], c.v[at], ld, scale=c.scale)
    torch.cuda.synchronize()
    state = c.want()[2]
    got = z.state.double().cpu().numpy()
    rel = off(got[c.slot], state[c.slot])
    print(f"[err] {steps} tokens, {each} at a time: {rel:.2e}", flush=True)
    assert rel <= U * (math.sqrt(3 * steps) + 10)
