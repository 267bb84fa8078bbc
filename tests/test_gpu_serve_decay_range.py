"""wz_decay_attention at the ends of the range that its header states.  Marked gpu.

Tolerances: those of tests/test_gpu_serve_decay.py.
"""
import numpy as np
import pytest
import torch

import libutil
from test_gpu_serve_decay import Layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("decay", [-0.003, -0.02, -0.05, -0.17, -0.6])
@pytest.mark.parametrize("n", [5, 300, 900])
def test_values_that_keep_the_state_at_its_limit(n, decay, dim):
    """States of up to 2^110 throughout, of one sign, under queries of ordinary size: outputs are far below fp32's end,
    and finite."""
    c = Layer([n, n], [1, 0], 1, 1, dim, seed=n, log_decay=[decay])
    for x in (c.q, c.k, c.v):
        x.abs_()
    c.state = np.abs(c.state)
    top = np.max(c.want()[2][c.slot])  # (states of positive terms: their limit, or what they began with)
    up = 110 - np.ceil(np.log2(max(top, np.max(c.state) + 1)))
    c.v.mul_(2.0 ** up)
    c.state *= np.float32(2.0 ** up)
    assert 2.0 ** 108 < max(np.max(c.want()[2]), np.max(c.state)) <= 2.0 ** 110
    out = c.want()[0]
    assert np.nanmax(out) < 2.0 ** 120
    got, states = c.run()
    assert torch.isfinite(got[:2 * n]).all()
    c.check(got, states, f"states at their limit, {n} x {dim}, {decay}")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [5, 300, 900])
def test_small_states(n, dim):
    """States of 2^-80, far above what counts as zero, keep their precision."""
    c = Layer([n, n], [1, 0], 3, 3, dim, seed=n, log_decay=[-0.003, -0.05, -0.6])
    c.v.mul_(2.0 ** -80), c.q.mul_(2.0 ** 70)
    c.state *= np.float32(2.0 ** -80)
    c.check(*c.run(), f"small states, {n} x {dim}")
