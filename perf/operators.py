"""Performance cases of the serving operators: what a video-LLM server does with the condensed tokens in one layer.

Three kinds of case, each a call of paper_2607_23265_amd.serve:

  append     new keys and values, rotated by their positions, go into a paged cache held in 8 bits (e4m3 with one
             power-of-two scale for each page and head); queries are rotated on the way
  attention  queries of a ragged batch over that cache: single tokens, a few tokens, whole prompts
  linear     a matrix product in 8-bit integers, activations quantized row by row in the same call

Sizes are those of the condensation pass's workloads (1254, 3499 and 9331 kept tokens, questions of 32 and 128 tokens,
the 3584 channels of the language model as 28 query heads of 128) and generic ones around them.  Lengths inside a
ragged batch are drawn from the case alone; the seed draws the values, the pages' order and the positions.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"
F8 = torch.float8_e4m3fn
F8_MAX = 448.0

APPEND = dict(kind="append", B=1, n_lo=1, n_hi=1, held_lo=0, held_hi=0, Hq=28, Hkv=4, D=128, P=64, rot=128, axes=1,
              interleaved=False, dtype="bf16", shape=1)
ATTENTION = dict(kind="attention", B=1, n_lo=1, n_hi=1, held_lo=0, held_hi=0, Hq=28, Hkv=4, D=128, P=64, causal=True,
                 window=0, shape=1)
LINEAR = dict(kind="linear", M=1, K=3584, N=3584, bias=False, out="bf16")


def listed():
    return [
        # one decoding step of a server's batch: a token for each of 64 conversations, small pages
        {"name": "append_step_b64", **APPEND, "B": 64, "held_lo": 900, "held_hi": 4100, "P": 16},
        # a clip's prompt: 1254 kept tokens and a 32-token question behind a 37-token system prompt; positions in
        # time, row and column
        {"name": "append_clip", **APPEND, "n_lo": 1286, "n_hi": 1286, "held_lo": 37, "held_hi": 37, "axes": 3},
        # eight long videos' prompts at once, of different lengths
        {"name": "append_videos", **APPEND, "B": 8, "n_lo": 3531, "n_hi": 9459, "held_lo": 11, "held_hi": 90,
         "axes": 3},
        # the next token of one short conversation: all latency
        {"name": "answer_clip", **ATTENTION, "held_lo": 1286, "held_hi": 1286},
        # the next token of 64 conversations of different lengths, small pages
        {"name": "answer_b64", **ATTENTION, "B": 64, "held_lo": 500, "held_hi": 8200, "P": 16, "shape": 2},
        # the next token of a few very long videos
        {"name": "answer_long", **ATTENTION, "B": 4, "held_lo": 60000, "held_hi": 131071, "shape": 3},
        # a few proposed tokens verified together, one key head for each query head
        {"name": "verify_b16", **ATTENTION, "B": 16, "n_lo": 3, "n_hi": 6, "held_lo": 1000, "held_hi": 6000, "Hq": 16,
         "Hkv": 16, "D": 64, "P": 32, "shape": 4},
        # a clip's prompt
        {"name": "prompt_clip", **ATTENTION, "n_lo": 1286, "n_hi": 1286, "held_lo": 37, "held_hi": 37},
        # the prompts of two long videos
        {"name": "prompt_videos", **ATTENTION, "B": 2, "n_lo": 8300, "n_hi": 9459, "held_lo": 37, "held_hi": 37,
         "shape": 5},
        # the query, key and value rows of a decoding step's batch (28 + 2 * 4 heads of 128)
        {"name": "qkv_step_b64", **LINEAR, "M": 64, "N": 4608, "bias": True},
        # the same of a clip's prompt
        {"name": "qkv_clip", **LINEAR, "M": 1286, "N": 4608, "bias": True},
        # the wide product of the feed-forward block, for a long video's prompt
        {"name": "wide_video", **LINEAR, "M": 9459, "N": 14336},
    ]


MAX_TOKENS = 8 * 9459          # of one append
MAX_CACHE = 4 * 131072 * 4     # tokens times key heads of one attention, and of one append's cache
MAX_PAIRS = 2 * 9000 ** 2 / 2 * 28  # query-key pairs times heads, of heads of 128
MAX_MACS = 9459 * 3584 * 14336


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choices(["append", "attention", "linear"], [4, 6, 3])[0]
    if kind == "linear":
        c = dict(LINEAR, M=log_int(1, 9459), K=16 * log_int(16, 512), N=log_int(100, 16384),
                 bias=rng.random() < 0.5, out=rng.choice(["bf16", "bf16", "f32"]))
        c["M"] = max(1, min(c["M"], MAX_MACS // (c["K"] * c["N"])))
        return c
    c = dict(APPEND if kind == "append" else ATTENTION)
    c["D"] = rng.choice([64, 128, 128])
    c["Hkv"] = rng.choice([1, 2, 4, 8, 16])
    c["Hq"] = c["Hkv"] * rng.choice([1, 2, 4, 7, 8] if c["Hkv"] < 16 else [1, 2])
    c["P"] = rng.choice([16, 32, 64, 128])
    c["shape"] = rng.randrange(1 << 20)
    long = rng.random() < 0.5  # prompts; else single tokens or a few
    if kind == "append":
        c["B"] = log_int(1, 16) if long else log_int(1, 256)
        c["n_hi"] = log_int(16, 9459) if long else rng.choice([1, 1, 1, 4])
        c["n_hi"] = max(1, min(c["n_hi"], MAX_TOKENS // c["B"]))
        c["n_lo"] = rng.choice([c["n_hi"], max(1, c["n_hi"] // 3)])
        c["held_hi"] = min(log_int(1, 8192), MAX_CACHE // (c["Hkv"] * c["B"]))
        c["held_lo"] = rng.choice([c["held_hi"], c["held_hi"] // 4])
        c["axes"] = rng.choice([1, 3])
        c["rot"] = rng.choice([c["D"], c["D"], c["D"] // 2])
        c["interleaved"] = rng.random() < 0.25
        c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
        return c
    c["B"] = log_int(1, 8) if long else log_int(1, 128)
    c["n_hi"] = log_int(32, 9459) if long else rng.choice([1, 1, 1, 2, 5, 16])
    c["held_hi"] = log_int(1, 16384) if long else log_int(16, 131072)
    c["held_hi"] = max(1, min(c["held_hi"], MAX_CACHE // (c["Hkv"] * c["B"])))
    pairs = MAX_PAIRS * 128 / (c["D"] * c["Hq"] * c["B"])
    while c["n_hi"] > 1 and c["n_hi"] * (c["held_hi"] + c["n_hi"] / 2) > pairs:
        c["n_hi"] = max(1, c["n_hi"] * 7 // 8)
        c["held_hi"] = max(1, c["held_hi"] * 7 // 8)
    c["n_lo"] = rng.choice([c["n_hi"], max(1, c["n_hi"] // 3)])
    c["held_lo"] = rng.choice([c["held_hi"], max(1, c["held_hi"] // 8)])
    c["causal"] = rng.random() < 0.85
    if c["causal"] and rng.random() < 0.25:
        c["window"] = log_int(16, 4096)
    return c


def _lengths(c):
    """(new tokens, tokens held before) of each sequence, from the case alone."""
    r = random.Random(c["shape"])

    def spread(lo, hi):
        return lo if lo >= hi else int(round(math.exp(r.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1

    got = [(spread(c["n_lo"], c["n_hi"]), spread(c["held_lo"], c["held_hi"])) for _ in range(c["B"])]
    return [max(1, n) for n, _ in got], [max(0, h) for _, h in got]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _paged(c, g):
    """The ragged batch and a filled cache: pages in random order, contents as an append of N(0, 1) rows leaves them."""
    new, held = _lengths(c)
    kv = [n + h for n, h in zip(new, held)]
    P, Hkv, D = c["P"], c["Hkv"], c["D"]
    per = [-(-x // P) for x in kv]
    pages = sum(per) + 3
    order = torch.randperm(pages, generator=g, device=DEV, dtype=torch.int32)
    table = torch.full((c["B"], max(per)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, m in enumerate(per):
        table[b, :m] = order[at:at + m]
        at += m
    s = SimpleNamespace(kind=c["kind"], max_tokens=max(new), max_kv=max(kv), table=table, P=P)
    s.start = torch.tensor([0] + new, dtype=torch.int32, device=DEV).cumsum(0, dtype=torch.int32)
    s.kv_len = torch.tensor(kv, dtype=torch.int32, device=DEV)
    s.tokens = sum(new)

    def fill(shape, loud, values):
        # channels of different size, as keys have; pages of different size, so that scales differ
        x = torch.empty(shape, dtype=F8, device=DEV)
        scale = torch.empty(shape[:2], device=DEV)
        step = max(1, (1 << 26) // (shape[1] * shape[2] * shape[3]))
        channel = torch.exp(0.4 * torch.randn(Hkv, D, generator=g, device=DEV)) * loud
        channel = channel[:, :, None] if values else channel[:, None, :]
        for i in range(0, shape[0], step):
            y = torch.randn((min(step, shape[0] - i), *shape[1:]), generator=g, device=DEV) * channel
            y = y * torch.exp(0.3 * torch.randn((y.shape[0], Hkv, 1, 1), generator=g, device=DEV))
            z = _pow2_scale(y.abs().amax((2, 3)))
            x[i:i + step] = (y / z[:, :, None, None]).to(F8)
            scale[i:i + step] = z
        return x, scale

    s.k, s.k_scale = fill((pages, Hkv, P, D), 1.0, False)
    s.v, s.v_scale = fill((pages, Hkv, D, P), 0.7, True)  # values lie channel by channel
    return s, new, held


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    if c["kind"] == "linear":
        s = SimpleNamespace(kind="linear")
        x = torch.randn(c["M"], c["K"], generator=g, device=DEV) * torch.exp(
            0.5 * torch.randn(c["K"], generator=g, device=DEV))
        s.x = x.to(torch.bfloat16)
        w = torch.randn(c["N"], c["K"], generator=g, device=DEV) / math.sqrt(c["K"])
        s.w_scale = (w.abs().amax(1) / 127).contiguous()
        s.w = torch.round(w / s.w_scale[:, None]).to(torch.int8)
        s.bias = torch.randn(c["N"], generator=g, device=DEV) if c["bias"] else None
        s.out_dtype = torch.bfloat16 if c["out"] == "bf16" else torch.float32
        return s
    s, new, held = _paged(c, g)
    T, Hq, Hkv, D = s.tokens, c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "attention":
        s.q = (1.5 * torch.randn(T, Hq, D, generator=g, device=DEV)).to(torch.bfloat16)
        s.causal, s.window, s.scale = c["causal"], c["window"], 1 / math.sqrt(D)
        # a server keeps the scratch of its attention; its plain form takes what it needs
        s.ws = torch.empty(128 << 20, dtype=torch.uint8, device=DEV)
        return s
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    # the rows of one fused projection: queries, keys and values side by side
    x = torch.randn(T, Hq + 2 * Hkv, D, generator=g, device=DEV)
    x *= torch.exp(0.4 * torch.randn(T, 1, 1, generator=g, device=DEV))
    x = x.to(dt)
    s.q, s.new_k, s.new_v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    s.q_out = torch.empty(T, Hq, D, dtype=torch.bfloat16, device=DEV)
    max_pos = s.max_kv + 1
    half = c["rot"] // 2
    angle = torch.arange(max_pos, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(half, device=DEV, dtype=torch.float64) / half)
    s.table_cs = torch.cat([angle.cos(), angle.sin()], 1).float()
    s.rot, s.interleaved = c["rot"], c["interleaved"]
    s.sections = (half,) if c["axes"] == 1 else (half - 2 * (3 * half // 8), 3 * half // 8, 3 * half // 8)
    seq = torch.repeat_interleave(torch.arange(c["B"], device=DEV), s.start.diff().long())
    at = torch.arange(T, device=DEV) - s.start[seq] + (s.kv_len - s.start.diff())[seq]
    if c["axes"] == 1:
        s.positions = at[None].int()
    else:  # time runs with the token, rows and columns inside a frame
        s.positions = torch.stack([at.int(), *(torch.randint(0, min(28, max_pos), (T,), generator=g, device=DEV,
                                                            dtype=torch.int32) for _ in range(2))])
    return s


# ---------------------------------------------------------------------------
# The operators
# ---------------------------------------------------------------------------

def run(s):
    if own:
        from paper_2607_23265_amd import serve
        if s.kind == "linear":
            a, a_scale = serve.quantize_rows(s.x)
            return serve.matmul_int(a, a_scale, s.w, s.w_scale, bias=s.bias, out_dtype=s.out_dtype)
        cache = serve.PagedCache(s.k, s.v, s.k_scale, s.v_scale)
        batch = serve.Ragged(s.start, s.kv_len, s.table, s.max_tokens, s.max_kv)
        if s.kind == "append":
            turn = serve.Rotation(s.table_cs, s.sections, s.interleaved)
            serve.cache_append(cache, batch, s.new_k, s.new_v, turn, s.positions, q=s.q, q_out=s.q_out)
            return s.q_out, s.k, s.v, s.k_scale, s.v_scale
        return serve.cache_attention(cache, batch, s.q, scale=s.scale, causal=s.causal, window=s.window, ws=s.ws)
    return {"linear": _linear, "append": _append, "attention": _attention}[s.kind](s)


def _linear(s):
    x = s.x.float()
    amax = x.abs().amax(1, keepdim=True).clamp_min(2.0 ** -100)
    full = torch.full_like(amax, 127.0)
    q = torch.round(x * torch.div(full, amax))
    y = (q @ s.w.float().t()) * torch.div(amax, full) * s.w_scale
    if s.bias is not None:
        y = y + s.bias
    return y.to(s.out_dtype)


def _pow2_scale(amax):
    """The least power of two z, of 2^-100 to 2^119, with amax <= 448 z."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-100, 119)
    return torch.ldexp(torch.ones_like(amax), torch.where(amax > 0, e, torch.full_like(e, -100)))


def _rotate(x, s, cos, sin):
    """x [T, heads, D] in 32 bits with its first `rot` elements turned by the angles [T, rot / 2]."""
    half = s.rot // 2
    cos, sin = cos[:, None], sin[:, None]
    if s.interleaved:
        a, b = x[..., 0:s.rot:2], x[..., 1:s.rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:s.rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., s.rot:]], -1)


def _angles(s):
    """cos and sin [T, rot / 2] of each token: section a of the frequencies goes by positions[a]."""
    half = s.rot // 2
    cs = [s.table_cs[p.long()] for p in s.positions]
    at = [sum(s.sections[:a]) for a in range(len(s.sections) + 1)]
    cos = torch.cat([x[:, i:j] for x, i, j in zip(cs, at, at[1:])], 1)
    sin = torch.cat([x[:, half + i:half + j] for x, i, j in zip(cs, at, at[1:])], 1)
    return cos, sin


def _placed(s):
    """Page, slot and sequence of every new token; the tokens that each sequence held before."""
    n = s.start.diff()
    seq = torch.searchsorted(s.start, torch.arange(s.tokens, device=DEV, dtype=torch.int32), right=True) - 1
    held = s.kv_len - n
    at = torch.arange(s.tokens, device=DEV) - s.start[seq] + held[seq]
    return s.table[seq, at // s.P].long(), at % s.P, seq, held.long()


def _append(s):
    cos, sin = _angles(s)
    s.q_out.copy_(_rotate(s.q.float(), s, cos, sin))
    k, v = _rotate(s.new_k.float(), s, cos, sin), s.new_v.float()
    page, slot, seq, held = _placed(s)
    touched = torch.zeros(s.k.shape[0], dtype=torch.bool, device=DEV)
    touched[page] = True
    first = s.table[torch.arange(held.numel(), device=DEV), held // s.P].long()  # the page each sequence goes on in
    prior = held % s.P
    kept = torch.arange(s.P, device=DEV) < prior[:, None]  # [B, P]: the slots it already holds there
    for x, cache, scale, values in ((k, s.k, s.k_scale, False), (v, s.v, s.v_scale, True)):
        pages = cache.view(torch.uint8)
        amax = torch.zeros_like(scale)
        amax.scatter_reduce_(0, page[:, None].expand(-1, amax.shape[1]), x.abs().amax(-1), "amax")
        new = _pow2_scale(amax)
        before = scale[first]
        after = torch.where(prior[:, None] > 0, torch.maximum(new[first], before), new[first])
        new[first] = after
        # what the page holds already moves to its new scale
        old = cache[first].float() * torch.div(before, after)[:, :, None, None]
        keep = kept[:, None, None, :] if values else kept[:, None, :, None]
        pages[first] = torch.where(keep, old.to(F8).view(torch.uint8), pages[first])
        stored = (x / new[page][:, :, None]).to(F8).view(torch.uint8)
        if values:
            pages[page, :, :, slot] = stored
        else:
            pages[page, :, slot] = stored
        scale.copy_(torch.where(touched[:, None], new, scale))
    return s.q_out, s.k, s.v, s.k_scale, s.v_scale


def _attention(s):
    B, n, kv = s.kv_len.numel(), s.max_tokens, s.max_kv
    T, Hq, D = s.q.shape
    Hkv = s.k.shape[1]
    table = s.table[:, :-(-kv // s.P)].clamp_min(0).long()
    k = (s.k[table].float() * s.k_scale[table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    v = (s.v[table].float() * s.v_scale[table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(B, Hkv, -1, D)
    count = s.start.diff()
    seq = torch.searchsorted(s.start, torch.arange(T, device=DEV, dtype=torch.int32), right=True) - 1
    row = torch.arange(T, device=DEV) - s.start[seq]
    q = torch.zeros(B, n, Hq, D, device=DEV)
    q[seq, row] = s.q.float()
    q = q.view(B, n, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s.scale).view(B, Hkv, Hq // Hkv, n, -1)
    j = torch.arange(x.shape[-1], device=DEV)
    seen = (j < s.kv_len[:, None])[:, None]  # [B, n, kv]
    if s.causal:
        at = (s.kv_len - count)[:, None] + torch.arange(n, device=DEV)
        seen = seen & (j <= at[..., None])
        if s.window:
            seen = seen & (j > at[..., None] - s.window)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True).clamp_min(-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    y = torch.matmul(x.view(B, Hkv, -1, x.shape[-1]), v).view(B, Hkv, -1, n, D)
    y = y / torch.where(total > 0, total, torch.ones_like(total))
    return y.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)[seq, row].to(torch.bfloat16)


# ---------------------------------------------------------------------------
# What a pass cannot do without, and its value in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": 2 * M * K + N * K + 4 * N * (2 if c["bias"] else 1) + M * N * (2 if c["out"] == "bf16" else 4),
                "flops": 2 * M * N * K}
    new, held = _lengths(c)
    T, Hq, Hkv, D, P = sum(new), c["Hq"], c["Hkv"], c["D"], c["P"]
    if c["kind"] == "append":
        size = 2 if c["dtype"] == "bf16" else 4
        rows = T * (Hq + 2 * Hkv) * D * size + T * c["axes"] * 4
        written = T * Hq * D * 2 + T * 2 * Hkv * D
        pages = sum(-(-(n + h) // P) - h // P for n, h in zip(new, held))
        return {"bytes": rows + written + pages * (4 + 16 * Hkv), "flops": 3 * T * (Hq + Hkv) * c["rot"]}
    pairs = cells = 0
    for n, h in zip(new, held):
        w = c["window"] or n + h
        # tokens that some row sees, and row-token pairs
        first = max(0, h + 1 - w) if c["causal"] else 0
        cells += n + h - first
        if not c["causal"]:
            pairs += n * (n + h)
        elif w >= n + h:
            pairs += n * h + n * (n + 1) // 2
        else:
            pairs += sum(min(h + i + 1, w) for i in range(n))
    pages = -(-cells // P) + len(new)
    return {"bytes": 2 * T * Hq * D * 2 + cells * Hkv * D * 2 + pages * (4 + 8 * Hkv), "flops": 4 * pairs * Hq * D}


def _grid_e4m3(x):
    """x rounded to the e4m3 grid: four significant bits, steps of 2^-9 below 2^-6; ties to even."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 4).clamp_min(-9))
    return torch.round(x / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if s.kind == "linear":
        x = s.x.double()
        unit = x.abs().amax(1, keepdim=True).clamp_min(2.0 ** -100) / 127
        y = torch.matmul(torch.round(x / unit), s.w.double().t()) * unit * s.w_scale.double()
        return y if s.bias is None else y + s.bias.double()
    start, kv_len, table = s.start.tolist(), s.kv_len.tolist(), s.table.tolist()
    Hkv, D, P = s.k.shape[1], s.q.shape[2], s.P
    if s.kind == "append":
        def turned(x):
            y = x.double().clone()
            half, lo = s.rot // 2, 0
            for section, p in zip(s.sections, s.positions):
                for j in range(lo, lo + section):
                    a, b = (2 * j, 2 * j + 1) if s.interleaved else (j, j + half)
                    cos, sin = s.table_cs[p.long(), j].double()[:, None], s.table_cs[p.long(), half + j].double()[:, None]
                    u, v = x[..., a].double(), x[..., b].double()
                    y[..., a], y[..., b] = u * cos - v * sin, u * sin + v * cos
                lo += section
            return y
        k, v = turned(s.new_k), s.new_v.double()
        kc, vc = s.k.double(), s.v.double()
        ks, vs = s.k_scale.double(), s.v_scale.double()
        for b, total in enumerate(kv_len):
            n = start[b + 1] - start[b]
            at, i = total - n, start[b]
            while at < total:
                page, slot = table[b][at // P], at % P
                m = min(P - slot, total - at)
                for x, c, z, axis in ((k, kc, ks, 1), (v, vc, vs, 2)):
                    rows = x[i:i + m].transpose(0, 1)  # [Hkv, m, D]
                    unit = torch.exp2(torch.ceil(torch.log2(rows.abs().amax((1, 2)).clamp_min(2.0 ** -90) / F8_MAX)))
                    if slot:
                        unit = torch.maximum(unit, z[page])
                        moved = c[page].narrow(axis, 0, slot)
                        moved.copy_(_grid_e4m3(moved * (z[page] / unit)[:, None, None]))
                    rows = _grid_e4m3(rows / unit[:, None, None])
                    c[page].narrow(axis, slot, m).copy_(rows if axis == 1 else rows.transpose(1, 2))
                    z[page] = unit
                at, i = at + m, i + m
        return turned(s.q), kc, vc, ks, vs
    out = torch.zeros(s.q.shape, dtype=torch.float64, device=DEV)
    G = s.q.shape[1] // Hkv
    for b, total in enumerate(kv_len):
        n = start[b + 1] - start[b]
        ids = s.table[b, :-(-total // P)].long()
        at = torch.arange(total - n, total, device=DEV)[:, None]
        j = torch.arange(total, device=DEV)[None]
        hide = torch.zeros(n, total, dtype=torch.bool, device=DEV)
        if s.causal:
            hide = (j > at) | (j <= at - s.window) if s.window else j > at
        for h in range(Hkv):
            k = (s.k[ids, h].double() * s.k_scale[ids, h].double()[:, None, None]).reshape(-1, D)[:total]
            v = (s.v[ids, h].double() * s.v_scale[ids, h].double()[:, None, None]).transpose(1, 2).reshape(-1, D)[:total]
            for i in range(h * G, (h + 1) * G):
                x = s.q[start[b]:start[b + 1], i].double() @ k.t() * s.scale
                p = torch.softmax(x.masked_fill_(hide, -math.inf), -1)
                out[start[b]:start[b + 1], i] = p @ v
    return out
