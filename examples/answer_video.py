"""From a video's tokens to the next tokens of an answer, in one attention layer held in 8 bits.

    python examples/answer_video.py [--frames 64] [--steps 16]

What a video-LLM server does with one layer, on random weights: condense the video for a question, put the kept tokens
and the question behind a system prompt, project them with 8-bit integer weights, append keys and values to a paged
8-bit cache with the kept tokens' positions in time, row and column, attend over the cache, and go on token by token.
(There is no vocabulary here: a step's input is the last step's output row.)
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_23265_amd import serve, synth  # noqa: E402
from paper_2607_23265_amd import wavezip as wz  # noqa: E402


class AttentionLayer:
    """Query, key and value projection, attention over a paged cache, output projection and residual."""

    def __init__(self, channels, q_heads, kv_heads, head_dim, generator):
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim

        def weights(rows, cols):
            w = torch.randn(rows, cols, generator=generator, device=generator.device) / cols ** 0.5
            return serve.quantize_rows(w)  # int8 with a scale for each output channel

        self.qkv, self.qkv_scale = weights((q_heads + 2 * kv_heads) * head_dim, channels)
        self.bias = 0.1 * torch.randn(self.qkv.shape[0], generator=generator, device=generator.device)
        self.out, self.out_scale = weights(channels, q_heads * head_dim)

    def __call__(self, x, cache, batch, rotation, positions):
        rows, Hq, Hkv = x.shape[0], self.q_heads, self.kv_heads
        a, scale = serve.quantize_rows(x)
        heads = serve.matmul_int(a, scale, self.qkv, self.qkv_scale, bias=self.bias).view(rows, -1, self.head_dim)
        q, k, v = heads[:, :Hq], heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:]
        q = serve.cache_append(cache, batch, k, v, rotation, positions, q=q)
        a, scale = serve.quantize_rows(serve.cache_attention(cache, batch, q).view(rows, -1))
        return x + serve.matmul_int(a, scale, self.out, self.out_scale)


def rotation_table(max_pos, dim, device, base=10000.0):
    """Cosines and sines [max_pos, dim] of dim / 2 frequencies."""
    half = dim // 2
    angle = torch.arange(max_pos, dtype=torch.float64, device=device)[:, None] * base ** (
        -torch.arange(half, dtype=torch.float64, device=device) / half)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prompt_positions(before, index, H, W, after):
    """Positions [3, tokens] of `before` text tokens, the kept tokens of a video and `after` text tokens.  Text goes on
    by one in all three axes; a kept token has its frame, row and column, whatever was dropped around it."""
    text = torch.arange(before, device=index.device, dtype=torch.int32).expand(3, -1)
    video = torch.stack([index // (H * W), index // W % H, index % W]) + before
    end = int(video.max()) + 1 if index.numel() else before
    return torch.cat([text, video, torch.arange(end, end + after, device=index.device, dtype=torch.int32).expand(3, -1)],
                     1).int().contiguous()


def answer(wl, layer, steps, system, video=None, seed=0, page_size=64, device="cuda:0"):
    """Outputs of the prompt's rows and of `steps` further tokens, with the cache and everything they came from.
    video: frames and question on the GPU (made from the seed if not given)."""
    X, query = video or wz.to_device(synth.generate(wl, seed), device)
    p = wz.problem_of(wl, out_dtype=wz.WZ_BF16)
    tokens, index, _, offset = wz.condense(p, X, query)
    kept = int(offset[-1])
    x = torch.cat([system, tokens[:kept], query.to(torch.bfloat16)])
    positions = prompt_positions(system.shape[0], index[:kept], wl.H, wl.W, query.shape[0])
    total = x.shape[0] + steps
    half = layer.head_dim // 2
    side = 3 * half // 8
    rotation = serve.Rotation(rotation_table(int(positions.max()) + steps + 1, layer.head_dim, device),
                              (half - 2 * side, side, side))
    pages = -(-total // page_size)
    cache = serve.PagedCache.new(pages, layer.kv_heads, layer.head_dim, page_size, device)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))  # a pool hands pages out in any order
    table = order.to(device=device, dtype=torch.int32)[None].contiguous()

    def batch(new, held):
        def on(*v):
            return torch.tensor(v, dtype=torch.int32, device=device)
        return serve.Ragged(on(0, new), on(held), table, new, held)

    rows = [layer(x, cache, batch(x.shape[0], x.shape[0]), rotation, positions)]
    for step in range(steps):
        at = positions[:, -1:] + 1 + step
        rows.append(layer(rows[-1][-1:], cache, batch(1, x.shape[0] + step + 1), rotation, at.contiguous()))
    return dict(x=x, positions=positions, rotation=rotation, cache=cache, table=table, rows=rows)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--frames", type=int, default=64)
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    base = synth.WORKLOADS["t64_14x14_c3584"]
    wl = synth.small("t64_14x14_c3584", T=a.frames, B=base.B * a.frames // base.T)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    layer = AttentionLayer(wl.C, wl.C // 128, 4, 128, g)
    system = torch.randn(37, wl.C, generator=g, device="cuda:0").to(torch.bfloat16)
    video = wz.to_device(synth.generate(wl, 0))
    answer(wl, layer, 2, system, video)
    took = []
    for steps in (0, a.steps):
        torch.cuda.synchronize()
        t = time.perf_counter()
        got = answer(wl, layer, steps, system, video)
        torch.cuda.synchronize()
        took.append(1e3 * (time.perf_counter() - t))
    rows = got["x"].shape[0]
    print(f"{wl.T} frames of {wl.H}x{wl.W} -> {rows} prompt rows (37 system, {rows - 37 - wl.Q} kept, {wl.Q} question): "
          f"{took[0]:.2f} ms from the frames to the layer's output, {a.steps} further tokens {took[1] - took[0]:.2f} ms")


if __name__ == "__main__":
    main()
