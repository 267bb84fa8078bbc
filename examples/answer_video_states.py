"""From a video's tokens to the next tokens of an answer, in a layer whose memory does not grow with the video.

    python examples/answer_video_states.py [--frames 64] [--steps 16]

The layer of answer_video.py with linear attention in the place of softmax attention and the rest of a transformer's
layer around it, on random weights in 8 bits: the kept tokens and the question behind a system prompt go through a norm, the
projections, linear attention with a decay for each head from a state that stays with the conversation, the projection
back onto the residual stream, and a gated feed-forward block; then token by token.  (There is no vocabulary here: a
step's input is the last step's output row.)
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_23265_amd import serve, synth  # noqa: E402
from paper_2607_23265_amd import wavezip as wz  # noqa: E402


class StateLayer:
    """Norm, linear attention over a state of a fixed size, norm, gated feed-forward block; both onto the residual
    stream."""

    def __init__(self, channels, heads, head_dim, width, generator):
        self.heads, self.head_dim = heads, head_dim
        g, dev = generator, generator.device

        def weights(rows, cols):
            return serve.quantize_rows(torch.randn(rows, cols, generator=g, device=dev) / cols ** 0.5)

        self.norm, self.norm2 = (1 + 0.1 * torch.randn(channels, generator=g, device=dev) for _ in range(2))
        self.qkv, self.qkv_scale = weights(3 * heads * head_dim, channels)
        self.bias = 0.1 * torch.randn(self.qkv.shape[0], generator=g, device=dev)
        self.out, self.out_scale = weights(channels, heads * head_dim)
        self.gate, self.gate_scale = weights(width, channels)
        self.up, self.up_scale = weights(width, channels)
        self.down, self.down_scale = weights(channels, width)
        # heads forget within some tokens to some thousand
        self.log_decay = -torch.exp(torch.linspace(-8, -1, heads, device=dev))

    def __call__(self, x, states, batch, slot):
        rows, H = x.shape[0], self.heads
        a, scale = serve.norm_quantize(x, self.norm)
        heads = serve.matmul_int(a, scale, self.qkv, self.qkv_scale, bias=self.bias).view(rows, 3 * H, self.head_dim)
        y = serve.decay_attention(states, batch, slot, heads[:, :H], heads[:, H:2 * H], heads[:, 2 * H:], self.log_decay)
        a, scale = serve.quantize_rows(y.view(rows, -1))
        y = serve.matmul_int(a, scale, self.out, self.out_scale)
        a, scale, x = serve.norm_quantize(y, self.norm2, residual=x, total=y)  # (the sum goes where y lies)
        y = serve.gated_int(a, scale, self.gate, self.gate_scale, self.up, self.up_scale)
        a, scale = serve.quantize_rows(y)
        return serve.matmul_int(a, scale, self.down, self.down_scale, residual=x, out=x)


def answer(wl, layer, steps, system, video=None, seed=0, device="cuda:0"):
    """Outputs of the prompt's rows and of `steps` further tokens, with the states and the prompt.  video: frames and
    question on the GPU (made from the seed if not given)."""
    X, query = video or wz.to_device(synth.generate(wl, seed), device)
    tokens, _, _, offset = wz.condense(wz.problem_of(wl, out_dtype=wz.WZ_BF16), X, query)
    x = torch.cat([system, tokens[:int(offset[-1])], query.to(torch.bfloat16)])
    states = serve.States.new(4, layer.heads, layer.head_dim, device)  # a server's pool; this conversation has one slot
    slot = torch.tensor([2], dtype=torch.int32, device=device)
    no_pages = torch.zeros(1, 0, dtype=torch.int32, device=device)

    def batch(new, held):
        def on(*v):
            return torch.tensor(v, dtype=torch.int32, device=device)
        return serve.Ragged(on(0, new), on(held), no_pages, new, held)

    rows = [layer(x, states, batch(x.shape[0], x.shape[0]), slot)]
    for step in range(steps):
        rows.append(layer(rows[-1][-1:], states, batch(1, x.shape[0] + step + 1), slot))
    return dict(x=x, states=states, slot=slot, rows=rows)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--frames", type=int, default=64)
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    base = synth.WORKLOADS["t64_14x14_c3584"]
    wl = synth.small("t64_14x14_c3584", T=a.frames, B=base.B * a.frames // base.T)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    layer = StateLayer(wl.C, wl.C // 128, 128, 4 * wl.C, g)
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
    state = got["states"].state
    print(f"{wl.T} frames of {wl.H}x{wl.W} -> {got['x'].shape[0]} prompt rows, {state[0].numel() * 4 >> 10} KiB of state: "
          f"{took[0]:.2f} ms from the frames to the layer's output, {a.steps} further tokens {took[1] - took[0]:.2f} ms")


if __name__ == "__main__":
    main()
