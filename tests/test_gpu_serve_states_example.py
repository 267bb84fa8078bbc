"""A layer of linear attention and a gated feed-forward block, from condensation to the next tokens, against the oracle's
chain of the same steps.  Marked gpu.

Each step's result is the oracle's of the step's own inputs up to its rounding to bfloat16, so the layer's output, six such
roundings deep (projection, attention, output, residual, gated block, residual), is held to 6 x 2^-8 of the outputs' 2-norm.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import synth
from serve_util import DEV, bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(repo_root):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()
    spec = importlib.util.spec_from_file_location("answer_video_states",
                                                  os.path.join(repo_root, "examples", "answer_video_states.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _np(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def test_layer_from_video_to_answer(example):
    wl = synth.small("t64_14x14_c3584", T=8, C=256, Q=16, B=157)
    g = torch.Generator(device=DEV).manual_seed(3)
    H, D = 4, 64
    layer = example.StateLayer(256, H, D, 704, g)
    system = torch.randn(5, 256, generator=g, device=DEV).to(torch.bfloat16)
    steps = 20
    got = example.answer(wl, layer, steps, system)
    torch.cuda.synchronize()
    x, W = _np(got["x"]), {k: _np(v) for k, v in vars(layer).items() if torch.is_tensor(v)}
    assert x.shape[0] == 5 + 157 + 16
    eps, scale = np.float32(1e-6), np.float32(D ** -0.5)
    state = np.zeros((1, H, D, D))
    for step in range(steps + 1):
        rows = x if step == 0 else _np(got["rows"][step - 1])[-1:]  # each step from the layer's own input
        n = len(rows)
        a, s = so.norm_quantize(rows, W["norm"], eps)
        qkv = bf16(so.matmul_int(a, s, W["qkv"], W["qkv_scale"], W["bias"])[0]).reshape(n, 3 * H, D)
        o, _, state, _ = so.decay_attention(state, [0, n], [step > 0], [0], qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:],
                                            W["log_decay"], scale)
        a, s = so.quantize_rows(bf16(o).reshape(n, -1))
        y = bf16(rows + bf16(so.matmul_int(a, s, W["out"], W["out_scale"])[0]))
        a, s = so.norm_quantize(y, W["norm2"], eps)
        h = so.activation(so.matmul_int(a, s, W["gate"], W["gate_scale"])[0], "silu")[0] * so.matmul_int(
            a, s, W["up"], W["up_scale"])[0]
        a, s = so.quantize_rows(bf16(h))
        want = y + so.matmul_int(a, s, W["down"], W["down_scale"])[0]
        off = np.linalg.norm(_np(got["rows"][step]) - want) / np.linalg.norm(want)
        print(f"[err] step {step}: {off:.2e}", flush=True)
        assert off <= 6 * 2.0 ** -8, (step, off)
    # the state itself: 21 calls' projections, each rounded to bfloat16 once
    off = np.linalg.norm(_np(got["states"].state)[2] - state[0]) / np.linalg.norm(state)
    assert off <= 2 * 2.0 ** -8, off


def test_example_runs(example, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["answer_video_states.py", "--frames", "8", "--steps", "3"])
    example.main()
    assert "8 frames of 14x14" in capsys.readouterr().out
