"""Performance cases of what a served layer has beside softmax attention.

Four kinds of case, each a call of paper_2607_23265_amd.serve:

  decay    linear attention with a decay for each head, on a state [head_dim, head_dim] for each sequence and head:
           single tokens, and whole prompts of a ragged batch
  gated    both projections of a gated feed-forward block in 8-bit integers, the activation and the product
  project  a product in 8-bit integers with bias, activation and residual
  norm     residual sum, root-mean-square norm and rounding of the rows to 8 bits

Sizes are those of the condensation pass's workloads (1254, 3499 and 9331 kept tokens, questions of 32 and 128 tokens,
the 3584 channels of the language model as 28 heads of 128, 1152 channels of a vision encoder, 64 frames of 196 tokens)
and of the other serving cases (a feed-forward width of 14336, batches of 64).  Lengths inside a ragged batch are drawn
from the case alone; the seed draws the values.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"

DECAY = dict(kind="decay", B=1, n_lo=1, n_hi=1, held=1, H=28, Hkv=28, D=128, shape=1)
GATED = dict(kind="gated", M=1, K=3584, N=14336, act="silu", bias=False, out="bf16")
PROJECT = dict(kind="project", M=1, K=14336, N=3584, act="none", bias=False, residual=True, out="bf16")
NORM = dict(kind="norm", M=1, N=3584, residual=True, dtype="bf16")


def listed():
    return [
        # the next token of one conversation: all latency
        {"name": "decay_step", **DECAY},
        # the next token of 64 conversations: their states, read and written
        {"name": "decay_step_b64", **DECAY, "B": 64},
        # a clip's prompt (1254 kept tokens and a 32-token question) behind a 37-token system prompt; few key heads
        {"name": "decay_clip", **DECAY, "n_lo": 1286, "n_hi": 1286, "Hkv": 4},
        # eight long videos' prompts at once, of different lengths, from empty states
        {"name": "decay_videos", **DECAY, "B": 8, "n_lo": 3531, "n_hi": 9459, "held": 0, "shape": 2},
        # the feed-forward block's first half: a decoding step's batch, a clip's prompt, a long video's
        {"name": "gated_step_b64", **GATED, "M": 64},
        {"name": "gated_clip", **GATED, "M": 1286},
        {"name": "gated_video", **GATED, "M": 9459},
        # its second half, onto the residual stream
        {"name": "down_step_b64", **PROJECT, "M": 64},
        {"name": "down_video", **PROJECT, "M": 9459},
        # a vision encoder's 64 frames of 196 tokens into the language model's width: bias and activation
        {"name": "vision_in", **PROJECT, "M": 12544, "K": 1152, "act": "gelu", "bias": True, "residual": False},
        # what comes before either block: a decoding step's batch, a long video's prompt
        {"name": "norm_step_b64", **NORM, "M": 64},
        {"name": "norm_video", **NORM, "M": 9459},
    ]


MAX_TOKENS = 8 * 6000 * 28 * 128   # tokens times heads times elements of one call
MAX_STATE = 64 * 28 * 128 * 128    # elements of one call's states
MAX_MACS = 9459 * 3584 * 14336
MAX_ROWS = 9459 * 14336            # elements of one norm


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choices(["decay", "gated", "project", "norm"], [6, 3, 4, 2])[0]
    if kind == "norm":
        c = dict(NORM, M=log_int(1, 9459), N=16 * log_int(4, 1024), residual=rng.random() < 0.7,
                 dtype=rng.choice(["bf16", "bf16", "f32"]))
        c["M"] = max(1, min(c["M"], MAX_ROWS // c["N"]))
        return c
    if kind != "decay":
        c = dict(GATED if kind == "gated" else PROJECT, M=log_int(1, 12544), K=16 * log_int(16, 896),
                 N=log_int(100, 14336), bias=rng.random() < 0.5, out=rng.choice(["bf16", "bf16", "f32"]))
        c["act"] = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"] if kind == "gated" else
                              ["none", "none", "silu", "gelu", "gelu_tanh", "relu"])
        if kind == "project":
            c["residual"] = rng.random() < 0.6
        c["M"] = max(1, min(c["M"], (MAX_MACS if kind == "gated" else 2 * MAX_MACS) // (c["K"] * c["N"])))
        return c
    c = dict(DECAY, D=rng.choice([64, 128, 128]), Hkv=rng.choice([1, 2, 4, 8, 16, 28]), shape=rng.randrange(1 << 20))
    c["H"] = c["Hkv"] * rng.choice([1, 1, 2, 4, 7] if c["Hkv"] < 16 else [1, 1, 2])
    long = rng.random() < 0.6  # prompts; else single tokens or a few
    c["B"] = log_int(1, 16) if long else log_int(1, 128)
    c["B"] = max(1, min(c["B"], MAX_STATE // (c["H"] * c["D"] ** 2)))
    c["n_hi"] = log_int(20, 16384) if long else rng.choice([1, 1, 1, 2, 5, 16])
    c["n_hi"] = max(1, min(c["n_hi"], MAX_TOKENS // (c["B"] * c["H"] * c["D"])))
    c["n_lo"] = rng.choice([c["n_hi"], max(1, c["n_hi"] // 3)])
    c["held"] = rng.choice([0, 1, 1])
    return c


def _lengths(c):
    """New tokens of each sequence, from the case alone."""
    r = random.Random(c["shape"])
    lo, hi = c["n_lo"], c["n_hi"]
    return [lo if lo >= hi else max(1, int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))) for _ in range(c["B"])]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _codes(rows, cols, g, loud=1.0):
    """Rows held in 8-bit integers, with their scales: rows of different size, as a prompt's are."""
    x = torch.randn(rows, cols, generator=g, device=DEV) * torch.exp(0.3 * torch.randn(rows, 1, generator=g, device=DEV))
    scale = x.abs().amax(1) * (loud / 127)
    return torch.round(x * (loud / scale)[:, None]).to(torch.int8), scale.contiguous()


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = SimpleNamespace(kind=c["kind"])
    if c["kind"] == "norm":
        dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        loud = torch.exp(0.5 * torch.randn(c["N"], generator=g, device=DEV))  # a few channels are louder, as in a stream
        s.x = (torch.randn(c["M"], c["N"], generator=g, device=DEV) * loud).to(dt)
        s.residual = (3 * torch.randn(c["M"], c["N"], generator=g, device=DEV) * loud).to(dt) if c["residual"] else None
        s.weight = 1 + 0.3 * torch.randn(c["N"], generator=g, device=DEV)
        s.eps = 1e-6
        return s
    if c["kind"] != "decay":
        M, N, K = c["M"], c["N"], c["K"]
        s.act, s.out_dtype = c["act"], torch.bfloat16 if c["out"] == "bf16" else torch.float32
        s.a, s.a_scale = _codes(M, K, g)
        s.w, s.w_scale = _codes(N, K, g, K ** -0.5)
        s.bias = 0.3 * torch.randn(N, generator=g, device=DEV) if c["bias"] else None
        if c["kind"] == "gated":
            s.up, s.up_scale = _codes(N, K, g, K ** -0.5)
            s.up_bias = 0.3 * torch.randn(N, generator=g, device=DEV) if c["bias"] else None
        else:
            s.residual = 3 * torch.randn(M, N, generator=g, device=DEV) if c["residual"] else None
            s.residual = s.residual.to(s.out_dtype) if c["residual"] else None
        return s
    new, B, H, Hkv, D = _lengths(c), c["B"], c["H"], c["Hkv"], c["D"]
    T = sum(new)
    s.max_tokens, s.held = max(new), c["held"]
    s.start = torch.tensor([0] + new, dtype=torch.int32, device=DEV).cumsum(0, dtype=torch.int32)
    before = 37 if c["held"] else 0
    s.kv_len = s.start.diff() + before
    s.max_kv = s.max_tokens + before
    s.table = torch.zeros(B, 0, dtype=torch.int32, device=DEV)  # no pages: this layer has states alone
    # the rows of one fused projection: queries, keys and values side by side
    x = torch.randn(T, H + 2 * Hkv, D, generator=g, device=DEV).to(torch.bfloat16)
    s.q, s.k, s.v = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
    # heads forget within 3 tokens to 3000
    s.log_decay = -torch.exp(torch.linspace(-8.0, -1.0, H, device=DEV)) if H > 1 else torch.tensor([-0.02], device=DEV)
    s.state = torch.randn(B + 2, H, D, D, generator=g, device=DEV)
    s.slot = torch.randperm(B + 2, generator=g, device=DEV)[:B].int()
    s.scale = D ** -0.5
    # a server keeps the scratch of its attention; its plain form takes what it needs
    s.ws = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------
# The operators
# ---------------------------------------------------------------------------

def run(s):
    if own:
        from paper_2607_23265_amd import serve
        if s.kind == "norm":
            return serve.norm_quantize(s.x, s.weight, eps=s.eps, residual=s.residual)
        if s.kind == "gated":
            return serve.gated_int(s.a, s.a_scale, s.w, s.w_scale, s.up, s.up_scale, activation=s.act,
                                   gate_bias=s.bias, up_bias=s.up_bias, out_dtype=s.out_dtype)
        if s.kind == "project":
            return serve.matmul_int(s.a, s.a_scale, s.w, s.w_scale, bias=s.bias, out_dtype=s.out_dtype,
                                    activation=None if s.act == "none" else s.act, residual=s.residual)
        states = serve.States(s.state)
        batch = serve.Ragged(s.start, s.kv_len, s.table, s.max_tokens, s.max_kv)
        out = serve.decay_attention(states, batch, s.slot, s.q, s.k, s.v, s.log_decay, scale=s.scale, ws=s.ws)
        return out, s.state
    return {"norm": _norm, "gated": _gated, "project": _project, "decay": _decay}[s.kind](s)


def _norm(s):
    h = s.x if s.residual is None else (s.x.float() + s.residual.float()).to(s.x.dtype)
    x = h.float()
    y = x * s.weight  # the norm's factor is the row's: it cancels in the codes
    top = y.abs().amax(1, keepdim=True).clamp_min(2.0 ** -100)
    full = torch.full_like(top, 127.0)
    q = torch.round(y * torch.div(full, top)).to(torch.int8)
    scale = (torch.div(top, full) / torch.sqrt((x * x).mean(1, keepdim=True) + s.eps))[:, 0]
    return (q, scale) if s.residual is None else (q, scale, h)


def _act(x, name):
    if name == "silu":
        return x / (1 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return x.clamp_min(0) if name == "relu" else x


def _linear(a, a_scale, w, w_scale, bias):
    y = (a.float() @ w.float().t()) * a_scale[:, None] * w_scale
    return y if bias is None else y + bias


def _gated(s):
    g = _linear(s.a, s.a_scale, s.w, s.w_scale, s.bias)
    return (_act(g, s.act) * _linear(s.a, s.a_scale, s.up, s.up_scale, s.up_bias)).to(s.out_dtype)


def _project(s):
    y = _act(_linear(s.a, s.a_scale, s.w, s.w_scale, s.bias), s.act)
    return (y if s.residual is None else y + s.residual.float()).to(s.out_dtype)


CHUNK = 64


def _decay(s):
    """Chunks of 64 tokens: what a token has from its own chunk, and from the state that the chunk begins with."""
    T, H, D = s.q.shape
    B, G = s.kv_len.numel(), H // s.k.shape[1]
    count = s.start.diff()
    seq = torch.searchsorted(s.start, torch.arange(T, device=DEV, dtype=torch.int32), right=True) - 1
    row = torch.arange(T, device=DEV) - s.start[seq]
    chunks = -(-s.max_tokens // CHUNK)

    def split(x, heads):  # [B * H, chunks, 64, D], zeros behind a sequence's end
        y = torch.zeros(B, chunks * CHUNK, heads, D, device=DEV)
        y[seq, row] = x.float()
        y = y.view(B, chunks, CHUNK, heads, D).permute(0, 3, 1, 2, 4)
        return y.repeat_interleave(H // heads, 1).reshape(B * H, chunks, CHUNK, D)

    q, k, v = split(s.q, H), split(s.k, H // G), split(s.v, H // G)
    rate = s.log_decay.double()[:, None, None]  # far tokens: angles in 64 bits, weights in 32

    def weights(gap):  # [H, *gap.shape]: exp(rate * gap), zero where the gap is negative
        w = torch.exp(rate * gap.clamp_min(0)) * (gap >= 0)
        return w.float().repeat(B, 1, 1)

    i = torch.arange(CHUNK, device=DEV)
    inside = weights(i[:, None] - i[None])
    out = torch.matmul(torch.matmul(q, k.transpose(2, 3).contiguous()) * inside[:, None], v)
    # what each chunk adds to the state, as of the chunk's end
    grown = torch.matmul((k * weights((CHUNK - 1 - i)[:, None])[:, None]).transpose(2, 3).contiguous(), v)
    first = s.state[s.slot.long()].reshape(B * H, 1, D, D) if s.held else torch.zeros(B * H, 1, D, D, device=DEV)
    grown = torch.cat([first, grown], 1)  # (the state held before counts as a chunk of its own)
    c = torch.arange(chunks + 1, device=DEV)
    begins = torch.matmul(weights((c[:chunks, None] - c[None]) * CHUNK), grown.view(B * H, chunks + 1, -1))
    q = q * weights((i + 1)[:, None])[:, None]
    out = (out + torch.matmul(q, begins.view(B * H, chunks, D, D))) * s.scale
    out = out.view(B, H, chunks * CHUNK, D).permute(0, 2, 1, 3)[seq, row].to(torch.bfloat16)
    # the last state of each sequence: its chunk's beginning, and the chunk's tokens up to its end
    last = (count - 1) // CHUNK
    part = count - last * CHUNK  # tokens of the last chunk
    at = torch.arange(B * H, device=DEV)
    pick = last.repeat_interleave(H).long()
    part = part.repeat_interleave(H)
    rates = s.log_decay.double().repeat(B)
    gap = part[:, None] - 1 - i
    w = (torch.exp(rates[:, None] * gap.clamp_min(0)) * (gap >= 0)).float()[:, :, None]
    ends = torch.matmul((k[at, pick] * w).transpose(1, 2).contiguous(), v[at, pick])
    ends = ends + begins.view(B * H, chunks, D, D)[at, pick] * torch.exp(rates * part).float()[:, None, None]
    s.state[s.slot.long()] = ends.view(B, H, D, D)
    return out, s.state


# ---------------------------------------------------------------------------
# What a pass cannot do without, and its value in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "norm":
        size = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": c["M"] * c["N"] * (size * (3 if c["residual"] else 1) + 1) + 4 * c["N"] + 4 * c["M"],
                "flops": 5 * c["M"] * c["N"]}
    if c["kind"] != "decay":
        M, N, K = c["M"], c["N"], c["K"]
        two, size = (2 if c["kind"] == "gated" else 1), 2 if c["out"] == "bf16" else 4
        return {"bytes": M * K + 4 * M + two * (N * K + 4 * N * (2 if c["bias"] else 1)) + M * N * size *
                (2 if c.get("residual") else 1), "flops": 2 * two * M * N * K}
    T, D = sum(_lengths(c)), c["D"]
    return {"bytes": 2 * T * D * (2 * c["H"] + 2 * c["Hkv"]) + 4 * c["B"] * c["H"] * D * D * (2 if c["held"] else 1),
            "flops": 4 * T * c["H"] * D * D}


def exact(case, seed):
    s = prepare(case, seed)
    if s.kind == "norm":
        h = s.x.double() if s.residual is None else s.x.double() + s.residual.double()
        stream = h
        if s.residual is not None:  # (the norm is of the stream as it is stored)
            h = h.to(s.x.dtype).double()
        y = h * s.weight.double() * torch.rsqrt(h.square().mean(1, keepdim=True) + s.eps)
        scale = y.abs().amax(1) / 127
        return (None, scale) if s.residual is None else (None, scale, stream)
    if s.kind != "decay":
        def linear(w, scale, bias):
            y = torch.matmul(s.a.double(), w.double().t())
            y.mul_(s.a_scale.double()[:, None]).mul_(scale.double())
            return y if bias is None else y.add_(bias.double())

        act = {"none": lambda x: x, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
               "gelu_tanh": lambda x: torch.nn.functional.gelu(x, approximate="tanh")}[s.act]
        y = act(linear(s.w, s.w_scale, s.bias))
        if s.kind == "gated":
            return y.mul_(linear(s.up, s.up_scale, s.up_bias))
        return y if s.residual is None else y.add_(s.residual.double())
    # the recurrence unrolled: token i has what token j <= i brought, times the decay to the power i - j
    start, slot = s.start.tolist(), s.slot.tolist()
    H, G = s.q.shape[1], s.q.shape[1] // s.k.shape[1]
    out = torch.empty(s.q.shape, dtype=torch.float64, device=DEV)
    state = s.state.double()
    for b, z in enumerate(slot):
        rows = slice(start[b], start[b + 1])
        n = start[b + 1] - start[b]
        at = torch.arange(n, device=DEV, dtype=torch.float64)
        for h in range(H):
            q, k, v = s.q[rows, h].double(), s.k[rows, h // G].double(), s.v[rows, h // G].double()
            r = s.log_decay[h].double()
            x = (at[:, None] - at[None]).mul_(r).exp_().tril_() if n < 4096 else None
            old = state[z, h] if s.held else torch.zeros_like(state[z, h])
            y = torch.exp((at + 1) * r)[:, None] * (q @ old)
            if x is not None:
                y += (x * (q @ k.t())) @ v
            else:  # (a block of rows at a time)
                for i in range(0, n, 2048):
                    j = min(n, i + 2048)
                    x = (at[i:j, None] - at[None, :j]).clamp_min_(0).mul_(r).exp_().tril_(i)
                    y[i:j] += (x * (q[i:j] @ k[:j].t())) @ v[:j]
            out[rows, h] = y * s.scale
            state[z, h] = torch.exp(r * n) * old + (k * torch.exp(r * (n - 1 - at))[:, None]).t() @ v
    return out, state
