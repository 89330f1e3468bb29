"""Float64 oracle of the operators around the attention: the definitions executed literally in numpy.

Test infrastructure only; nothing here is imported by the product path.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128


def rms_norm(x, residual, weight, eps):
    """(h, y) with h = x + residual and y = h / sqrt(mean(h^2) + eps) * weight, row by row."""
    h = x.astype(np.float64) + (0.0 if residual is None else residual.astype(np.float64))
    return h, h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps) * weight.astype(np.float64)


def gated(x, gate):
    x, g = x.astype(np.float64), gate.astype(np.float64)
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-g)) * x


# Every value an e4m3 byte stands for: sign, four bits of exponent (bias 7), three bits behind the point; all ones is NaN.
E4M3 = np.array([math.nan if b & 0x7F == 0x7F else
                 (-1.0 if b & 0x80 else 1.0) * ((b & 7) / 8 * 2.0 ** -6 if (b >> 3) & 15 == 0 else
                                                (1 + (b & 7) / 8) * 2.0 ** (((b >> 3) & 15) - 7)) for b in range(256)])


def scale_byte(block):
    """The byte of the smallest scale 2^(b - 127), 0 <= b, that brings the block's largest magnitude to 448 or below."""
    if not np.isfinite(block).all():
        return 255
    top = float(np.abs(block).max()) if block.size else 0.0
    b = 0
    while top > 448.0 * 2.0 ** (b - 127):
        b += 1
    return b


def to_e4m3(v):
    """The bytes of the nearest e4m3 values (|v| <= 448); of two equally near ones that with the even last bit."""
    pos = E4M3[:0x7F]  # ascending
    a = np.abs(v)
    hi = np.clip(np.searchsorted(pos, a), 0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    up, down = pos[hi] - a, a - pos[lo]
    at = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return (at | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def quantize(y, rows_per_scale=1):
    """(bytes, scale bytes) of rows [rows, n]."""
    rows, n = y.shape
    rb, nb = -(-rows // rows_per_scale), -(-n // BLOCK)
    q, s = np.zeros((rows, n), np.uint8), np.zeros((rb, nb), np.uint8)
    for i in range(rb):
        for j in range(nb):
            at = slice(i * rows_per_scale, (i + 1) * rows_per_scale), slice(j * BLOCK, (j + 1) * BLOCK)
            b = scale_byte(y[at])
            s[i, j] = b
            q[at] = 0x7F if b == 255 else to_e4m3(y[at] * 2.0 ** (127 - b))
    return q, s


def values(q, scales, rows_per_scale=1):
    """What 8-bit rows stand for."""
    s = np.where(scales == 255, math.nan, 2.0 ** (scales.astype(np.float64) - 127))
    s = np.repeat(np.repeat(s, rows_per_scale, 0)[: q.shape[0]], BLOCK, 1)[:, : q.shape[1]]
    return E4M3[q] * s


def frequencies(rot, base, factor=1.0, original_length=0, low=0.0, high=0.0):
    f = []
    for i in range(rot // 2):
        v = base ** (-2.0 * i / rot)
        if factor != 1.0:
            g = 0.0
            if original_length:
                turns = original_length * v / (2 * math.pi)
                g = (min(1.0, max(0.0, (turns - low) / (high - low))) if high > low else float(turns >= low))
            v *= g + (1 - g) / factor
        f.append(v)
    return np.array(f)


def rotate(x, cos, sin, rot, neighbours, inverse):
    """x [..., d] with cos, sin [..., rot / 2]: pair by pair."""
    y = x.astype(np.float64).copy()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)
        c, s = cos[..., i], -sin[..., i] if inverse else sin[..., i]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def sample(logits, noise, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probability) of one row."""
    l = np.where(np.isnan(logits), -math.inf, logits.astype(np.float64))
    n = len(l)
    order = sorted(range(n), key=lambda i: (-l[i], i))
    if l[order[0]] == -math.inf:
        return -1, 0.0
    if not temperature > 0:
        return order[0], 1.0
    top = l[order[0]]
    if top == math.inf:
        w = np.where(l == math.inf, 1.0, 0.0)
    else:
        with np.errstate(over="ignore"):
            w = np.exp((l - top) / temperature)
    w = w[order]
    live = int((l[order] > -math.inf).sum())
    kept = live if top_k <= 0 or top_k >= n else min(top_k, live)
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[:kept])])[:-1]
        kept = max(1, int((before < top_p * w[:kept].sum()).sum()))
    keep = [i for i in range(kept) if i == 0 or w[i] >= min_p]
    best = None
    for i in keep:
        if w[i] == 0:
            continue
        key = math.log(w[i]) - (math.log(noise[order[i]]) if noise is not None else 0.0)
        if best is None or key > best[0] or (key == best[0] and order[i] < order[best[1]]):
            best = (key, i)
    return order[best[1]], w[best[1]] / sum(w[i] for i in keep)


# ---- keys and values in pages, log probabilities ----

def seen(past, new, window, sinks):
    """[new, past + new]: whether the i-th new token, at position past + i, sees token j."""
    m = np.zeros((new, past + new), bool)
    for i in range(new):
        p = past + i
        for j in range(p + 1):
            m[i, j] = j < sinks or p - j < window
    return m


def gather(pages, row, n):
    """pages [pages, heads, page_size, d] -> the sequence's [heads, n, d]; row: its entries of the table."""
    size = pages.shape[2]
    return np.stack([pages[row[j // size], :, j % size] for j in range(n)], 1)


def attend(q, k, v, mask):
    """q [new, heads, d], k, v [kv_heads, n, d], mask [new, n]: (o, sum of p |v|, largest sum of |q k| / sqrt(d) that a row sees)."""
    new, heads, d = q.shape
    group = heads // k.shape[0]
    o, size, reach = (np.zeros((new, heads, d)), np.zeros((new, heads, d)), np.zeros((new, heads, 1)))
    for h in range(heads):
        kh, vh = k[h // group], v[h // group]
        for i in range(new):
            at = mask[i]
            s = kh[at] @ q[i, h] / math.sqrt(d)
            with np.errstate(invalid="ignore"):
                p = np.exp(s - s.max())
                p /= p.sum()
            o[i, h], size[i, h] = p @ vh[at], p @ np.abs(vh[at])
            reach[i, h] = (np.abs(kh[at]) @ np.abs(q[i, h])).max() / math.sqrt(d)
    return o, size, reach


def log_probs(logits):
    """(log p of every token, entropy, tokens by falling logit, equal ones by index) of one row."""
    x = logits.astype(np.float64)
    order = sorted(range(len(x)), key=lambda i: (math.inf if np.isnan(x[i]) else -x[i], i))
    if np.isnan(x).any() or x.max() in (math.inf, -math.inf):
        return np.full(len(x), math.nan), math.nan, order
    y = x - x.max()
    w = np.exp(y)
    z = w.sum()
    with np.errstate(invalid="ignore"):
        return y - math.log(z), math.log(z) - np.where(w > 0, w * y, 0.0).sum() / z, order
