"""Plain CPU oracle of the serving operators (include/wavezip_serve.h): codes bit for bit, sums in float64.

Written from the header's definitions with loops over sequences, pages and heads; it shares no code with the library.
"""
import math

import numpy as np


def _e4m3_table():
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = np.nan if (c & 127) == 127 else m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = -x if c & 128 else x
    return v


E4M3 = _e4m3_table()


def decode(codes):
    return E4M3[np.asarray(codes, dtype=np.uint8)]


def encode(x):
    """Nearest e4m3 code, ties to the even one, beyond the range the largest (x finite)."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.minimum(np.abs(x), 448.0)
    grid = E4M3[:127]
    hi = np.clip(np.searchsorted(grid, mag), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = mag - grid[lo], grid[hi] - mag
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_of(amax):
    """The least 2^e, -100 <= e <= 119, with amax <= 448 2^e."""
    e = -100
    while e < 119 and amax > 448.0 * 2.0 ** e:
        e += 1
    return np.float32(2.0 ** e)


def rotate(x, positions, table, sections, interleaved):
    """x [tokens, heads, dim] float32, turned in float32 products and sums."""
    y = np.array(x, dtype=np.float32)
    half = table.shape[1] // 2
    axis = np.zeros(half, int)
    if len(sections) > 1:
        axis = np.repeat(np.arange(len(sections)), sections)
    pos = np.clip(positions, 0, table.shape[0] - 1)
    with np.errstate(all="ignore"):
        for j in range(half):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
            cos, sin = table[pos[axis[j]], j][:, None], table[pos[axis[j]], half + j][:, None]
            u, v = x[..., a].astype(np.float32), x[..., b].astype(np.float32)
            y[..., a], y[..., b] = u * cos - v * sin, v * cos + u * sin
    return y


def append(cache, start, kv_len, table, k, v):
    """cache: dict of k [pages, heads, P, D], v [pages, heads, D, P] (uint8 codes), k_scale, v_scale [pages, heads];
    changed in place.  k, v [tokens, heads, D] float32 (keys rotated already)."""
    pages, heads, P, _ = cache["k"].shape
    for b in range(len(kv_len)):
        n = start[b + 1] - start[b]
        place0 = kv_len[b] - n
        at = max(place0, 0)
        while at < kv_len[b]:
            entry, slot = at // P, at % P
            m = min(P - slot, kv_len[b] - at)
            page = table[b][entry]
            rows = slice(start[b] + at - place0, start[b] + at - place0 + m)
            at += m
            if not 0 <= page < pages:
                continue
            for h in range(heads):
                kk, vv = k[rows, h].astype(np.float64), v[rows, h].astype(np.float64)
                bad = ~(np.isfinite(kk).all(1) & np.isfinite(vv).all(1))
                for x, codes, scale, values in ((kk, cache["k"], cache["k_scale"], False),
                                                (vv, cache["v"], cache["v_scale"], True)):
                    fine = np.isfinite(x)
                    z = scale_of(np.abs(x[fine]).max() if fine.any() else 0.0)
                    block = codes[page, h].T if values else codes[page, h]  # [P, D]
                    if slot:
                        old = scale[page, h]
                        if old < z:
                            moved = block[:slot]
                            block[:slot] = np.where((moved & 127) == 127, moved,
                                                    encode(np.nan_to_num(decode(moved)) * (float(old) / float(z))))
                        else:
                            z = old
                    scale[page, h] = z
                    new = encode(np.where(fine, x, 0.0) / float(z))
                    if not values:
                        new[bad] = 127
                    block[slot:slot + m] = new


def attention(cache, start, kv_len, table, q, scale, causal=True, window=0):
    """q [tokens, q_heads, D] -> (out, sum of p |v|, log-sum-exp [tokens, q_heads], sum of |q||k| * |scale| at most),
    float64."""
    pages, heads, P, D = cache["k"].shape
    T, Hq, _ = q.shape
    G = Hq // heads
    out, mag = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, reach = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    K = decode(cache["k"]) * cache["k_scale"].astype(np.float64)[..., None, None]
    V = decode(cache["v"]) * cache["v_scale"].astype(np.float64)[..., None, None]
    for b in range(len(kv_len)):
        n, total = start[b + 1] - start[b], kv_len[b]
        place0 = total - n
        there = np.array([0 <= table[b][j // P] < pages for j in range(total)], bool)
        for h in range(heads):
            k, v = np.zeros((total, D)), np.zeros((total, D))
            for j in np.flatnonzero(there):
                p = table[b][j // P]
                k[j], v[j] = K[p, h, j % P], V[p, h, :, j % P]
            j = np.arange(total)[None]
            seen = np.broadcast_to(there[None], (n, total))
            if causal:
                place = place0 + np.arange(n)[:, None]
                seen = seen & (j <= place)
                if window:
                    seen = seen & (j > place - window)
            some = seen.any(1)
            if not some.any():
                continue
            rows = start[b] + np.flatnonzero(some)
            for g in range(h * G, (h + 1) * G):
                x = q[rows, g].astype(np.float64)
                with np.errstate(invalid="ignore"):
                    s = np.where(seen[some], x @ k.T * scale, -np.inf)
                    m = s.max(1, keepdims=True)
                    p = np.where(seen[some], np.exp(s - m), 0.0)
                    total_p = p.sum(1, keepdims=True)
                    out[rows, g], mag[rows, g] = p @ v / total_p, p @ np.abs(v) / total_p
                    lse[rows, g] = (m + np.log(total_p))[:, 0]
                    reach[rows, g] = np.where(seen[some], np.abs(x) @ np.abs(k).T, 0.0).max(1) * abs(scale)
    return out, mag, lse, reach


def quantize_rows(x):
    """x [rows, cols] float32 -> (int8, scale float32), each operation in float32."""
    x = np.asarray(x, dtype=np.float32)
    fine = np.isfinite(x).all(1)
    amax = np.maximum(np.where(fine, np.abs(np.nan_to_num(x)).max(1), 1).astype(np.float32), np.float32(2.0 ** -100))
    up = np.float32(127) / amax
    with np.errstate(all="ignore"):
        q = np.where(fine[:, None], np.rint(np.nan_to_num(x) * up[:, None]), 0).astype(np.int8)
    return q, np.where(fine, amax / np.float32(127), np.float32(np.nan)).astype(np.float32)


def matmul_int(a, a_scale, w, w_scale, bias=None):
    """(product, magnitude of its terms) in float64."""
    acc = a.astype(np.float64) @ w.astype(np.float64).T  # whole numbers below 2^53: exact
    y = acc * a_scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)
    return (y, np.abs(y)) if bias is None else (y + bias.astype(np.float64), np.abs(y) + np.abs(bias))


def norm_quantize(h, weight, eps):
    """h [rows, cols] float32 (the stream as it is stored) -> (int8, scale float64): codes from h * weight, each operation
    in float32; the norm in float64."""
    h, weight = np.asarray(h, dtype=np.float32), np.asarray(weight, dtype=np.float32)
    with np.errstate(all="ignore"):
        t = h * weight
    q, scale = quantize_rows(t)
    top = np.maximum(np.abs(np.nan_to_num(t)).max(1), np.float32(2.0 ** -100)).astype(np.float64)
    with np.errstate(all="ignore"):
        norm = np.sqrt(np.square(h.astype(np.float64)).mean(1) + eps)
        return q, np.where(np.isfinite(scale), top / 127 / norm, np.nan)


def activation(x, name):
    """(activation of x, a bound of its slope) in float64."""
    x = np.asarray(x, dtype=np.float64)
    if name in (None, "none"):
        return x, 1.0
    if name == "relu":
        return np.maximum(x, 0), 1.0
    with np.errstate(over="ignore"):
        if name == "silu":
            return x / (1 + np.exp(-x)), 1.1
        if name == "gelu":
            return 0.5 * x * np.vectorize(math.erfc)(-x / math.sqrt(2)), 1.13
        return x / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))), 1.13  # (1 + tanh(z)) / 2


def decay_attention(state, start, held, slot, q, k, v, log_decay, scale):
    """The recurrence token by token in float64.  state [slots, heads, D, D] (not changed), held[b]: whether the sequence
    goes on from its slot; q [tokens, heads, D], k and v [tokens, kv_heads, D].  Returns (out, the sum of its terms'
    magnitudes, states, theirs); rows of no sequence are NaN."""
    T, H, D = q.shape
    G = H // k.shape[1]
    out, mag = np.full((T, H, D), np.nan), np.full((T, H, D), np.nan)
    state = state.astype(np.float64)
    size = np.abs(state)
    with np.errstate(all="ignore"):
        decay = np.exp(np.minimum(np.asarray(log_decay, dtype=np.float64), 0.0))
        for b in range(len(slot)):
            kept = 0 <= slot[b] < state.shape[0]
            if start[b + 1] <= start[b]:
                continue
            for h in range(H):
                S, M = np.zeros((D, D)), np.zeros((D, D))
                if kept and held[b]:
                    S, M = state[slot[b], h].copy(), size[slot[b], h].copy()
                for t in range(start[b], start[b + 1]):
                    x = np.outer(k[t, h // G].astype(np.float64), v[t, h // G].astype(np.float64))
                    S, M = decay[h] * S + x, decay[h] * M + np.abs(x)
                    y = q[t, h].astype(np.float64)
                    out[t, h], mag[t, h] = scale * (y @ S), abs(scale) * (np.abs(y) @ M)
                if kept:
                    state[slot[b], h], size[slot[b], h] = S, M
    return out, mag, state, size
