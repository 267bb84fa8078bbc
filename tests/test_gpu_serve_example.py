"""The example's layer, from condensation to the next tokens, against the oracles' chain of the same steps.  Marked gpu.

Each step's result is the oracle's of the step's own inputs up to its rounding to bfloat16, so the layer's output, four
such roundings deep (projection, rotated query, attention, output), is held to 4 x 2^-8 of the outputs' 2-norm.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

import libutil
from oracle import serve_oracle as so
from paper_2607_23265_amd import synth
from serve_util import DEV, bf16, codes

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(repo_root):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    libutil.ensure_built()
    spec = importlib.util.spec_from_file_location("answer_video", os.path.join(repo_root, "examples", "answer_video.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _np(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def test_layer_from_video_to_answer(example):
    wl = synth.small("t64_14x14_c3584", T=8, C=256, Q=16, B=157)
    g = torch.Generator(device=DEV).manual_seed(3)
    layer = example.AttentionLayer(256, 4, 2, 64, g)
    system = torch.randn(5, 256, generator=g, device=DEV).to(torch.bfloat16)
    steps, page = 20, 16
    got = example.answer(wl, layer, steps, system, page_size=page)
    torch.cuda.synchronize()
    x, positions, table = _np(got["x"]), _np(got["positions"]), _np(got["table"])
    n = x.shape[0]
    assert n == 5 + 157 + 16 and positions.shape == (3, n)
    assert (positions[:, :5] == np.arange(5)).all() and (np.diff(positions[:, 5 + 157:]) == 1).all()
    pages = got["cache"].k.shape[0]
    cache = dict(k=np.zeros((pages, 2, page, 64), np.uint8), v=np.zeros((pages, 2, 64, page), np.uint8),
                 k_scale=np.zeros((pages, 2), np.float32), v_scale=np.zeros((pages, 2), np.float32))
    W = {k: _np(getattr(layer, k)) for k in ("qkv", "qkv_scale", "bias", "out", "out_scale")}
    turn = (_np(got["rotation"].table), got["rotation"].sections, False)
    held = 0
    for step in range(steps + 1):
        rows = x if step == 0 else _np(got["rows"][step - 1])[-1:]  # each step from the layer's own input
        at = positions if step == 0 else positions[:, -1:] + step
        a, s = so.quantize_rows(rows)
        heads = bf16(so.matmul_int(a, s, W["qkv"], W["qkv_scale"], W["bias"])[0]).reshape(len(rows), 8, 64)
        q = bf16(so.rotate(heads[:, :4], at, *turn))
        held += len(rows)
        so.append(cache, [0, len(rows)], [held], table, so.rotate(heads[:, 4:6], at, *turn), heads[:, 6:])
        o = bf16(so.attention(cache, [0, len(rows)], [held], table, q, 64 ** -0.5)[0])
        a, s = so.quantize_rows(o.reshape(len(rows), -1))
        want = rows + so.matmul_int(a, s, W["out"], W["out_scale"])[0]
        off = np.linalg.norm(_np(got["rows"][step]) - want) / np.linalg.norm(want)
        assert off <= 4 * 2.0 ** -8, (step, off)
    # the cache itself: the same codes but where a projection was rounded to the other side
    used = [int(p) for p in table[0][:-(-held // page)]]
    last = held - (len(used) - 1) * page
    for name in ("k", "v"):
        a, b = codes(getattr(got["cache"], name)), cache[name]
        for i, p in enumerate(used):
            m = page if i + 1 < len(used) else last
            u, v = (a[p][:, :m], b[p][:, :m]) if name == "k" else (a[p][..., :m], b[p][..., :m])
            assert np.mean(u != v) < 0.02, (name, i)


def test_example_runs(example, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["answer_video.py", "--frames", "8", "--steps", "3"])
    example.main()
    assert "8 frames of 14x14" in capsys.readouterr().out
