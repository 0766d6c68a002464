"""Plain references in 64 bits for the operators on a paged cache and on trees of drafted tokens (test infrastructure)."""
import math

import numpy as np


TWO_PI = np.longdouble("6.283185307179586476925286766559")


def bf16_round(x):
    """float array -> the nearest bf16 numbers, as float64 (x finite and within bf16's normal range)"""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32).astype(np.float64)


def frequencies(rot_dim, base, scaling=None, stretch=1.0, original=None):
    """Radians per position of every pair, and the magnitude, in extended precision."""
    ld = np.longdouble
    R, s = rot_dim, ld(stretch)
    b = ld(base) * s ** (ld(R) / ld(R - 2)) if scaling == "base" else ld(base)
    w = b ** (-2 * np.arange(R // 2).astype(ld) / R)
    if scaling == "linear":
        w = w / s
    magnitude = 1.0
    if scaling == "parts":
        g = np.clip((ld(original) * w / TWO_PI - 1) / 31, 0, 1)
        w = g * w + (1 - g) * w / s
        magnitude = 0.1 * math.log(stretch) + 1.0
    return w, magnitude


def rotate(x, positions, w, magnitude, interleaved, inverse=False):
    """x [..,heads,D] float64, positions [..]: rotated, in float64."""
    R = 2 * len(w)
    a = (np.asarray(positions).astype(np.longdouble)[..., None, None] * w) % TWO_PI
    c, s = np.cos(a).astype(np.float64) * magnitude, np.sin(a).astype(np.float64) * magnitude
    if inverse:
        s = -s
    y = x.astype(np.float64).copy()
    if interleaved:
        u, v = x[..., 0:R:2], x[..., 1:R:2]
        y[..., 0:R:2], y[..., 1:R:2] = u * c - v * s, v * c + u * s
    else:
        u, v = x[..., :R // 2], x[..., R // 2:R]
        y[..., :R // 2], y[..., R // 2:R] = u * c - v * s, v * c + u * s
    return y


def rotate_bound(x, w, magnitude, interleaved, bf16, y):
    """How far rounding may take a rotated value.  Sine and cosine are within 2^-23 of theirs; with the magnitude's rounding and the
    product by it they are off by 2^-23 + 2 * 2^-24, two products and a sum by 2^-24 each: 2^-21 (|u| + |v|) covers it.  bf16: half a step more."""
    R = 2 * len(w)
    b = np.zeros_like(y)
    if interleaved:
        both = (np.abs(x[..., 0:R:2]) + np.abs(x[..., 1:R:2])) * magnitude
        b[..., 0:R:2] = b[..., 1:R:2] = both
    else:
        both = (np.abs(x[..., :R // 2]) + np.abs(x[..., R // 2:R])) * magnitude
        b[..., :R // 2] = b[..., R // 2:R] = both
    b *= 2.0 ** -21
    return b + (np.abs(y) + b) * 2.0 ** -8 if bf16 else b


def ancestors(parents, count):
    """[count, count] truth values: what the tokens of one tree see."""
    see = np.zeros((count, count), dtype=bool)
    for i in range(count):
        a = i
        while a >= 0:
            see[i, a] = True
            p = parents[a] if a > 0 else -1
            a = p if 0 <= p < a else -1
    return see


def pack_bits(see, B):
    """[n, m] truth values -> int64 words [n, ceil(B / 64)]"""
    n = see.shape[0]
    wide = np.zeros((n, (B + 63) // 64 * 64), dtype=bool)
    wide[:, :see.shape[1]] = see
    return np.packbits(wide, axis=1, bitorder="little").view(np.int64)


def attention(q, k, v, see, scale):
    """q [n,D], k, v [m,D], see [n,m]: (average [n,D], average of |v| [n,D]); rows that see nothing are 0."""
    s = q @ k.T * scale
    s = np.where(see, s, -np.inf)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    l = p.sum(-1, keepdims=True)
    p = p / np.where(l > 0, l, 1.0)
    return p @ v, p @ np.abs(v)


def attention_bound(q, k, scale, average, absolute, bf16):
    """A probability is off by what its score is off by, twice (in the sum below it too): products are summed in fp32 in some order, D + 2
    roundings of partial sums no larger than sum |q k|, and the exponent's product and difference add 2^-22 of the scores' size.  bf16
    probabilities are rounded to 2^-8, and averages of pieces of the keys to 2^-11 (fp16, with a factor of the row's: 2^-39 of its largest
    element at least); sums over m keys add m 2^-24 at most; the result is rounded to half a step."""
    size = (np.abs(q) @ np.abs(k).T).max() * scale if k.size else 0.0
    D, m = q.shape[-1], k.shape[0]
    eps = 2 * size * ((D + 2) * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -20 + m * 2.0 ** -24
    if bf16:
        return absolute * (2.0 ** -8 + 2.0 ** -11 + eps) * (1 + 2.0 ** -8) + absolute.max(-1, keepdims=True) * 2.0 ** -39 + np.abs(average) * 2.0 ** -8
    return absolute * eps + np.abs(average) * 2.0 ** -24


def softmax(z, temperature):
    y = z.astype(np.float64) / temperature
    e = np.exp(y - y.max())
    return e / e.sum()


def verify(logits, tokens, uniforms, parents, count, temperature, draft=None, draft_temperature=1.0):
    """One request, from the definition: (path, emitted, chances)."""
    B, V = logits.shape
    chances = np.zeros(B)
    if count == 0:
        return [], [], chances
    chances[0] = 1.0
    of = [-1] + [int(parents[j]) if 0 <= parents[j] < j else -1 for j in range(1, B)]
    inside = lambda x: 0 <= x < V
    for j in range(1, count):
        i, x = of[j], int(tokens[j])
        if i < 0 or not inside(x):
            continue
        if temperature == 0.0:
            chances[j] = float(int(np.argmax(logits[i])) == x)
        else:
            p = softmax(logits[i], temperature)[x]
            q = 1.0 if draft is None else softmax(draft[i], draft_temperature)[x]
            chances[j] = min(1.0, p / q) if q > 0 else float(p > 0)
    path, emitted = [0], []
    while True:
        i = path[-1]
        children = [j for j in range(i + 1, count) if of[j] == i]
        go = None
        if temperature == 0.0:
            token = int(np.argmax(logits[i]))
            go = next((j for j in children if int(tokens[j]) == token), None)
        else:
            p = softmax(logits[i], temperature)
            w, W = p.copy(), 1.0
            for j in children:
                x = int(tokens[j])
                if draft is not None:
                    q = softmax(draft[i], draft_temperature)
                    q_x = q[x] if inside(x) else 0.0
                else:
                    q_x = 1.0
                if inside(x) and float(uniforms[j, 0]) * q_x * W < w[x]:
                    go = j
                    break
                if draft is not None:
                    w = np.maximum(p - q, 0.0)
                elif inside(x):
                    w[x] = 0.0
                W = w.sum()
            if go is None:
                if W < 2.0 ** -40:
                    w = p
                cum = np.cumsum(w)
                token = int(np.searchsorted(cum, float(uniforms[i, 1]) * cum[-1], side="right"))
                token = min(token, int(np.flatnonzero(w)[-1]))
        if go is None:
            emitted.append(token)
            return path, emitted, chances
        path.append(go)
        emitted.append(int(tokens[go]))
