"""wz_decay_attention against its recurrence in float64.  Marked gpu.

With u = 2^-24 and n tokens of a sequence: each term of a state passes at most 2 n roundings of sums (4 n with those of a
chunk's and a segment's partial sums), and its weight exp(-x) is off by at most 1.5 x u of itself, x below 104 where fp32 has
a weight at all: a state is within u (4 n + 160) of the sum of its terms' magnitudes.  An output adds the two products that
take a factor in two parts of bf16, each off by at most 2^-15 of its terms, and its rounding to bf16, half a step of 2^-8.
"""
import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import serve
from paper_2607_23265_amd import wavezip as wz
from serve_util import DEV, bf16

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


class Layer:
    """A ragged batch's rows as parts of one projection, states full of what was there before, and the oracle's results."""

    def __init__(self, new, held, heads, kv, dim, seed=0, spare=2, slots=None, log_decay=None, behind=3):
        r = self.rng = np.random.default_rng(seed)
        self.new, self.held, self.dim, self.scale = list(new), list(held), dim, 0.37
        B, T = len(self.new), sum(self.new)
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        x = bf16(r.normal(size=(T + behind, heads + 2 * kv, dim)))
        self.x = dev = torch.from_numpy(x).to(DEV).to(BF)
        self.q, self.k, self.v = dev[:, :heads], dev[:, heads:heads + kv], dev[:, heads + kv:]
        self.state = r.normal(size=(B + spare, heads, dim, dim)).astype(np.float32)
        self.slot = r.permutation(B + spare)[:B].astype(np.int32) if slots is None else np.array(slots, np.int32)
        self.log_decay = (-np.exp(np.linspace(-8, -1, heads)) if log_decay is None else np.array(log_decay)).astype(np.float32)
        self.kv_len = [n + 7 * bool(h) for n, h in zip(self.new, self.held)]

    def batch(self, max_tokens=None):
        table = torch.zeros(len(self.new), 0, dtype=torch.int32, device=DEV)
        return serve.Ragged(ints(self.start), ints(self.kv_len), table, max(self.new) if max_tokens is None else max_tokens,
                            max(self.kv_len))

    def want(self):
        f = lambda t: t.float().cpu().numpy()  # noqa: E731
        return so.decay_attention(self.state, self.start, self.held, self.slot, f(self.q), f(self.k), f(self.v),
                                  self.log_decay, self.scale)

    def run(self, states=None, out=None, ws=None, batch=None, **kw):
        states = states or serve.States(torch.from_numpy(self.state).to(DEV))
        if out is None:
            out = torch.full(self.q.shape, 9.0, dtype=BF, device=DEV)
        got = serve.decay_attention(states, batch or self.batch(), ints(self.slot), self.q, self.k, self.v,
                                    torch.from_numpy(self.log_decay).to(DEV), scale=self.scale, out=out, ws=ws)
        torch.cuda.synchronize()
        return got, states

    def check(self, got, states, what):
        out, mag, state, size = self.want()
        rows = int(self.start[-1])
        n = max(self.new) + 1
        g = got.float().cpu().numpy().astype(np.float64)
        assert (g[rows:] == 9).all()  # rows of no sequence
        s = states.state.cpu().numpy().astype(np.float64)
        touched = {int(z) for z, m in zip(self.slot, self.new) if m and 0 <= z < len(s)}
        for z in set(range(len(s))) - touched:
            np.testing.assert_array_equal(s[z], self.state[z])
        worst = []
        sums = U * (4 * n + 160)
        for a, b, m, rel in ((g[:rows], out[:rows], mag[:rows], 2.0 ** -14 + sums), (s, state, size, sums)):
            fine = np.isfinite(b)
            np.testing.assert_array_equal(np.isfinite(a), fine)
            tol = rel * m[fine]
            if a is not s:
                tol = tol + 2.0 ** -8 * (np.abs(b[fine]) + tol)
            off = np.abs(a[fine] - b[fine])
            worst.append(float(np.max(off / np.maximum(tol, 1e-30), initial=0)))
            worst.append(float(np.linalg.norm(off) / max(np.linalg.norm(b[fine]), 1e-30)))
        print(f"[err] decay {what}: out {worst[0]:.3f} of the bound (norm {worst[1]:.2e}), state {worst[2]:.3f} ({worst[3]:.2e})",
              flush=True)
        assert worst[0] <= 1 and worst[2] <= 1


LENGTHS = [([1], [1]), ([1], [0]), ([2, 1, 5], [1, 0, 1]), ([63], [0]), ([64], [1]), ([65, 1, 0, 3], [1, 1, 1, 0]),
           ([0, 130, 17], [0, 1, 0]), ([31, 33, 32, 16, 15, 128], [1, 0, 1, 1, 0, 1]), ([700], [1]), ([0, 0], [1, 0]),
           ([1000, 3, 257], [0, 1, 1])]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv", [(2, 2), (6, 2)])
@pytest.mark.parametrize("new,held", LENGTHS)
def test_lengths(new, held, heads, kv, dim):
    c = Layer(new, held, heads, kv, dim, seed=sum(new) + heads)
    c.check(*c.run(), f"{new} {heads}/{kv} x {dim}")


@pytest.mark.parametrize("new,held,heads,kv,dim", [
    # runs of chunks that begin and end inside sequences, at their ends, and over several of them
    ([300, 0, 64, 1000, 9, 129, 640], [1, 1, 0, 1, 0, 0, 1], 3, 1, 64), ([128] * 9, [0, 1] * 4 + [1], 2, 2, 128),
    ([1500], [1], 1, 1, 64), ([4000], [1], 1, 1, 64), ([3000, 9, 2500], [1, 0, 1], 2, 1, 128),
    ([64, 1200, 64], [1, 1, 1], 2, 2, 64), ([700, 1] * 3, [0] * 6, 40, 20, 64),
    # the most heads
    ([3, 1], [1, 0], 256, 64, 64), ([70], [1], 256, 256, 64)])
def test_runs(new, held, heads, kv, dim):
    c = Layer(new, held, heads, kv, dim, seed=sum(new) + dim)
    c.check(*c.run(), f"runs {new} {heads}/{kv} x {dim}")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 3, 300])
def test_decays_at_the_ends(n, dim):
    """Nothing forgotten, all forgotten, hardly anything left of the last token, factors above 1 (which count as 1)."""
    ld = [0.0, -np.inf, -90.0, -3e38, 5.0, -1e-7, -0.69314718]
    c = Layer([n, n], [1, 0], len(ld), 1, dim, seed=n, log_decay=ld)
    c.check(*c.run(), f"decays at the ends, {n}")


@pytest.mark.parametrize("n", [1, 5, 200])
def test_a_decay_that_is_no_number(n):
    c = Layer([n], [1], 3, 3, 64, seed=n, log_decay=[-0.1, np.nan, -0.2])
    got, states = c.run()
    assert torch.isnan(got[:n, 1]).all() and torch.isnan(states.state[c.slot[0], 1]).all()
    assert torch.isfinite(got[:n, [0, 2]]).all() and torch.isfinite(states.state[c.slot[0]][[0, 2]]).all()


@pytest.mark.parametrize("n", [2, 90, 400])
def test_slots_outside(n):
    """A slot that is none of the states': from zeros, and nothing is stored."""
    for slots in ([-1, 1, 99], [3, -(1 << 31), 2]):
        c = Layer([n, n, 3], [1, 1, 1], 2, 1, 64, seed=n, slots=slots)
        c.check(*c.run(), f"slots {slots}")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("where", [0, 5, 63, 64, 100, 189])
@pytest.mark.parametrize("part", ["q", "k", "v"])
def test_numbers_that_are_none(where, part, dim):
    """A NaN or an infinity reaches what depends on its token by the formula, and nothing else: no row before it, no element
    of the state that it does not meet."""
    c = Layer([190, 40], [1, 1], 2, 1, dim, seed=where)
    x = dict(q=c.q, k=c.k, v=c.v)[part]
    x[where, 0, 3], x[min(where + 30, 189), 0, 7] = float("nan"), float("inf")
    x[191, 0, 9] = -float("inf")
    x[230:] = float("nan")  # rows of no sequence
    c.check(*c.run(), f"{part} at {where}")


def test_states_of_infinities():
    c = Layer([1, 5, 100], [1, 1, 1], 2, 2, 64, seed=1)
    for b in range(3):
        c.state[c.slot[b], 0, 3, 4 + b], c.state[c.slot[b], 1, 2, 1] = np.inf, np.nan
    c.check(*c.run(), "states of infinities")


@pytest.mark.parametrize("n", [1, 150])
def test_large_and_small_numbers(n):
    c = Layer([n], [1], 2, 2, 64, seed=n)
    c.k.mul_(2.0 ** 60), c.v.mul_(2.0 ** 30), c.q.mul_(2.0 ** -60)
    c.state *= np.float32(2.0 ** 90)
    c.check(*c.run(), "large keys")


@pytest.mark.parametrize("n", [20, 400])
def test_the_largest_states(n):
    """A state's elements of 2^110 keep their precision where they are kept raised for some chunks, and fade."""
    c = Layer([n], [1], 3, 1, 64, seed=n, log_decay=[-0.003, -0.05, -0.6])
    c.state = np.sign(c.state) * np.float32(2.0 ** 109)
    c.q.mul_(2.0 ** -60)
    c.check(*c.run(), f"the largest states, {n}")


@pytest.mark.parametrize("new", [[1, 1, 1], [5, 70, 300]])
def test_strides(new):
    """Rows that lie apart in every tensor, and a batch whose start is not the first row."""
    c = Layer(new, [1, 0, 1], 4, 2, 64, seed=9)
    want, states = c.run()
    T = c.q.shape[0]
    wide = torch.full((T, 4 * 64 + 40), 7.0, dtype=BF, device=DEV)
    parts = {}
    for name, t in (("q", c.q), ("k", c.k), ("v", c.v)):
        w = torch.full((T, t.shape[1] * 64 + 16), float("nan"), dtype=BF, device=DEV)
        w[:, 8:8 + t.shape[1] * 64] = t.reshape(T, -1)
        parts[name] = w[:, 8:8 + t.shape[1] * 64].unflatten(1, (-1, 64))
    c.q, c.k, c.v = parts["q"], parts["k"], parts["v"]
    got, again = c.run(out=wide[:, 16:16 + 256].unflatten(1, (4, 64)))
    rows = int(c.start[-1])
    assert torch.equal(got[:rows], want[:rows]) and torch.equal(again.state, states.state)
    assert (wide[:, :16] == 7).all() and (wide[:, 272:] == 7).all() and (wide[rows:] == 7).all()


@pytest.mark.parametrize("new", [[3, 1], [100, 129], [1200, 60]])
def test_in_parts(new):
    """A prompt in one call, and the same tokens in two and token by token: the state carries all there is."""
    c = Layer(new, [0, 0], 2, 2, 64, seed=3)
    whole, states = c.run()
    z = serve.States.new(4, 2, 64)
    z.state.fill_(float("nan"))  # (nothing in it needs initialising)
    got = torch.zeros_like(whole)
    cuts = [[0, n // 2, n - 1, n] for n in new]
    for i in range(3):
        rows = [torch.arange(c.start[b] + cuts[b][i], c.start[b] + cuts[b][i + 1], device=DEV) for b in range(2)]
        at = torch.cat(rows)
        start = np.concatenate([[0], np.cumsum([len(x) for x in rows])])
        batch = serve.Ragged(ints(start), ints([cuts[b][i + 1] for b in range(2)]), torch.zeros(2, 0, dtype=torch.int32, device=DEV),
                             max(len(x) for x in rows), max(new))
        got[at] = serve.decay_attention(z, batch, ints(c.slot), c.q[at], c.k[at], c.v[at],
                                        torch.from_numpy(c.log_decay).to(DEV), scale=c.scale)
    torch.cuda.synchronize()
    c.check(torch.cat([got[:c.start[-1]], whole[c.start[-1]:]]), type("S", (), dict(state=torch.where(
        torch.isnan(z.state), torch.from_numpy(c.state).to(DEV), z.state))), f"in parts {new}")


def test_bounds_above_the_lengths_and_below():
    """max_tokens above the lengths changes nothing but the plan; below, a sequence is cut to it."""
    c = Layer([5, 20], [1, 1], 2, 2, 64, seed=4)
    for most in (20, 64, 700, 5000):
        c.check(*c.run(batch=c.batch(most)), f"max_tokens {most}")
    got, _ = c.run(batch=c.batch(3))  # (another plan: the same rows to within the bounds of both)
    out, mag, _, _ = c.want()
    g = got.float().cpu().numpy().astype(np.float64)
    for rows in (slice(0, 3), slice(5, 8)):
        tol = (2.0 ** -14 + U * (4 * 21 + 160)) * mag[rows]
        assert (np.abs(g[rows] - out[rows]) <= tol + 2.0 ** -8 * (np.abs(out[rows]) + tol)).all()
    assert (got[3:5] == 9).all() and (got[8:25] == 9).all()


@pytest.mark.parametrize("new", [[200], [129, 0, 65], [63], [0, 0, 0], [64, 320] + [0] * 70 + [130]])
@pytest.mark.parametrize("dim", [64, 128])
def test_fewer_tokens_than_rows(new, dim):
    """A padded batch: rows, and max_tokens, far above what the sequences bring, so that the plan has more runs than
    there are chunks."""
    c = Layer(new, [1, 0, 1] if len(new) == 3 else [1] * len(new), 4, 2, dim, seed=sum(new), behind=6000)
    z = serve.States(torch.from_numpy(c.state).to(DEV))
    for most in (6000, 330):
        batch = c.batch(most)
        ws = torch.full((serve.decay_workspace_bytes(z, batch, c.q.shape[0]) + 256,), 0xFF, dtype=torch.uint8, device=DEV)
        c.check(*c.run(batch=batch, ws=ws), f"{new} of 6000, {most} at most")


@pytest.mark.parametrize("new,dim", [([1] * 5, 128), ([900, 40], 64), ([2000], 128), ([5000], 64)])
def test_runs_agree_bit_for_bit(new, dim):
    """The same call again, with whatever lies in its workspace, on a stream of its own, and captured and replayed."""
    c = Layer(new, [1] * len(new), 3, 1, dim, seed=5)
    want, states = c.run()
    batch = c.batch()
    z = serve.States(torch.from_numpy(c.state).to(DEV))
    need = serve.decay_workspace_bytes(z, batch, c.q.shape[0])
    ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device=DEV)
    got, again = c.run(ws=ws)
    assert torch.equal(got, want) and torch.equal(again.state, states.state)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got, again = c.run(ws=ws)
    assert torch.equal(got, want) and torch.equal(again.state, states.state)
    # a graph: its replays go on from the state, as calls do
    slot, ld, out = ints(c.slot), torch.from_numpy(c.log_decay).to(DEV), torch.zeros_like(want)
    first = z.state.clone()
    serve.decay_attention(z, batch, slot, c.q, c.k, c.v, ld, scale=c.scale, out=out, ws=ws)
    torch.cuda.synchronize()
    z.state.copy_(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        serve.decay_attention(z, batch, slot, c.q, c.k, c.v, ld, scale=c.scale, out=out, ws=ws)
    z.state.copy_(first)
    eager = serve.States(first.clone())
    for i in range(4):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = serve.decay_attention(eager, batch, slot, c.q, c.k, c.v, ld, scale=c.scale)
        torch.cuda.synchronize()
        rows = int(c.start[-1])
        assert torch.equal(out[:rows], want[:rows]) and torch.equal(z.state, eager.state), i


def test_two_calls_at_once():
    """Two calls on streams of their own, each with a workspace and states of its own."""
    cs = [Layer([2100, 30], [1, 1], 8, 2, 128, seed=11), Layer([900, 1, 1300], [0, 1, 1], 8, 2, 64, seed=12)]
    want = [c.run() for c in cs]
    streams, states = [torch.cuda.Stream() for _ in cs], [serve.States(torch.from_numpy(c.state).to(DEV)) for c in cs]
    args = [(ints(c.slot), torch.from_numpy(c.log_decay).to(DEV), c.batch(), torch.full(c.q.shape, 9.0, dtype=BF, device=DEV))
            for c in cs]
    for _ in range(3):
        for c, z in zip(cs, states):
            z.state.copy_(torch.from_numpy(c.state))
        torch.cuda.synchronize()
        for c, z, s, (slot, ld, batch, out) in zip(cs, states, streams, args):
            with torch.cuda.stream(s):
                serve.decay_attention(z, batch, slot, c.q, c.k, c.v, ld, scale=c.scale, out=out)
        torch.cuda.synchronize()
        for (rows, z0), z, (_, _, _, out) in zip(want, states, args):
            assert torch.equal(out, rows) and torch.equal(z.state, z0.state)


def test_nothing_behind_the_workspace_is_written():
    c = Layer([1500, 900], [1, 0], 4, 2, 64, seed=6)
    z, batch = serve.States(torch.from_numpy(c.state).to(DEV)), c.batch()
    need = serve.decay_workspace_bytes(z, batch, c.q.shape[0])
    space = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device=DEV)
    got, _ = c.run(ws=space[:need] if need else None)
    assert bool((space[need:] == 0x5A).all())


def test_overlapping_rows_stay_in_the_workspace():
    """Starts that decrease or pass the rows, against the contract: cut on the device, nothing outside is touched."""
    c = Layer([400, 400], [1, 1], 2, 2, 64, seed=7)
    batch = serve.Ragged(ints([700, -5, 900]), ints([400, 1 << 20]), torch.zeros(2, 0, dtype=torch.int32, device=DEV), 400, 500)
    z = serve.States(torch.from_numpy(c.state).to(DEV))
    need = serve.decay_workspace_bytes(z, batch, c.q.shape[0])
    space = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device=DEV)
    c.run(states=z, batch=batch, ws=space[:need] if need else None)
    assert bool((space[need:] == 0x5A).all())
    for i in set(range(4)) - set(c.slot.tolist()):
        assert torch.equal(z.state[i].cpu(), torch.from_numpy(c.state[i]))


def test_far_slots():
    """States past 2^32 elements."""
    slots = (1 << 32) // (8 * 128 * 128) + 4
    z = serve.States.new(slots, 8, 128)
    z.state[-1], z.state[-2] = 0.5, 0.25
    q, k, v = (torch.randn(2, 8, 128, device=DEV).to(BF) for _ in range(3))
    batch = serve.Ragged(ints([0, 1, 2]), ints([5, 5]), torch.zeros(2, 0, dtype=torch.int32, device=DEV), 1, 5)
    small = serve.States(z.state[-2:].clone())
    ld = torch.full((8,), -0.1, device=DEV)
    got = serve.decay_attention(z, batch, ints([slots - 1, slots - 2]), q, k, v, ld)
    want = serve.decay_attention(small, batch, ints([1, 0]), q, k, v, ld)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(z.state[-2:], small.state)


def test_binding():
    c = Layer([3, 40], [1, 0], 4, 2, 64, seed=8)
    z, b = serve.States(torch.from_numpy(c.state).to(DEV)), c.batch()
    slot, ld = ints(c.slot), torch.from_numpy(c.log_decay).to(DEV)
    f = serve.decay_attention
    ok = (z, b, slot, c.q, c.k, c.v, ld)
    f(*ok)
    for i, bad in ((0, b), (1, z), (2, slot[:1]), (2, slot.long()), (2, slot.cpu()), (3, c.q.float()), (3, c.q[:, :2]),
                   (3, c.q[..., :32]), (4, c.k[:3]), (4, c.k.float()), (5, c.v[:, :1]), (6, ld[:2]), (6, ld.to(BF)), (6, None)):
        with pytest.raises(ValueError):
            f(*ok[:i], bad, *ok[i + 1:])
    for kw in (dict(out=torch.zeros(c.q.shape, device=DEV)), dict(ws=torch.zeros(8, device=DEV))):
        with pytest.raises(ValueError):
            f(*ok, **kw)
    with pytest.raises(wz.WZError):
        f(*ok, scale=float("nan"))
    with pytest.raises(wz.WZError):
        f(*ok, out=c.q)
    three = torch.zeros(c.q.shape[0], 3, 64, dtype=BF, device=DEV)
    with pytest.raises(wz.WZError):
        f(*ok[:4], three, three, ld)
    for bad in (torch.zeros(2, 3, 64, 32, device=DEV), torch.zeros(3, 64, 64, device=DEV),
                torch.zeros(2, 3, 64, 64, device=DEV, dtype=BF), torch.zeros(2, 3, 64, 64)):
        with pytest.raises(ValueError):
            serve.States(bad)
    with pytest.raises(wz.WZError):
        f(serve.States.new(4, 4, 32), b, slot, *(torch.zeros(43, n, 32, dtype=BF, device=DEV) for n in (4, 2, 2)), ld)
    with pytest.raises(AttributeError):
        z.state = z.state
    import copy
    twin = copy.deepcopy(z)
    assert twin.state.data_ptr() != z.state.data_ptr() and (twin.slots, twin.heads, twin.head_dim) == (4, 4, 64)
