"""Plain 64-bit forms of the 8-bit experts' operators (numpy), with how far 32-bit sums
may lie from them."""
from __future__ import annotations

import numpy as np

from tests.paged_ref import decode, encode

B = 128
TOP = 448.0
U32 = 2.0 ** -23  # a 32-bit sum's term may be cut instead of rounded: a whole step


def blocks(n: int) -> int:
    return -(-n // B)


def scale_of(amax):
    """The smallest power of two that holds amax, at least 2^-100; NaN where it is not
    finite."""
    amax = np.asarray(amax, np.float64)
    m, e = np.frexp(np.maximum(np.where(np.isfinite(amax), amax, 1.0) / TOP, 2.0 ** -101))
    s = np.ldexp(1.0, np.maximum(np.where(m == 0.5, e - 1, e), -100))
    return np.where(np.isfinite(amax), s, np.nan)


def spread(scale, rows, cols, by_rows=False):
    """Scales of blocks as an array of the numbers' shape."""
    s = np.repeat(scale, B, axis=-1)[..., :cols]
    return np.repeat(s, B, axis=-2)[..., :rows, :] if by_rows else s


def _encode(x, s):
    return np.where(np.isnan(s), np.uint8(0x7f), encode(np.where(np.isnan(s), 0.0, x / s)))


def quantize_rows(x):
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    p = np.pad(np.abs(x), ((0, 0), (0, blocks(cols) * B - cols))).reshape(rows, -1, B)
    bad = ~np.isfinite(p).all(-1)
    s = scale_of(np.where(bad, np.inf, np.where(np.isfinite(p), p, 0).max(-1)))
    return _encode(x, spread(s, rows, cols)), s


def quantize_blocks(w):
    w = np.asarray(w, np.float64)
    n, rows, cols = w.shape
    p = np.pad(np.abs(w), ((0, 0), (0, blocks(rows) * B - rows), (0, blocks(cols) * B - cols)))
    p = p.reshape(n, blocks(rows), B, blocks(cols), B)
    bad = ~np.isfinite(p).all((2, 4))
    s = scale_of(np.where(bad, np.inf, np.where(np.isfinite(p), p, 0).max((2, 4))))
    return _encode(w, spread(s, rows, cols, True)), s


def rows64(q, scale):
    return decode(q) * spread(np.asarray(scale, np.float64), *q.shape)


def matrix64(q, scale):
    return decode(q) * spread(np.asarray(scale, np.float64), *q.shape[-2:], True)


def product(x, w):
    """x . w^T and what its 32-bit form may be off by: every one of the n products and
    their sums at most a step of 2^-23 of the terms' magnitudes, beside the two scales'
    product and its multiplication."""
    n = x.shape[1]
    return x @ w.T, (n + 8) * U32 * (np.abs(x) @ np.abs(w).T)


def silu(a):
    return a / (1.0 + np.exp(-a))


def ffn(x, w1, v1, w2):
    """One expert on rows x (their 8-bit values): y and its allowance.  What h may be off
    by can put a number of it on the other side of a border between two 8-bit numbers, or
    the block's largest one under another scale: the distance of the outermost of these
    values is allowed, times the weight it meets."""
    a, ea = product(x, w1)
    b, eb = product(x, v1)
    h = silu(a) * b
    # |silu'| < 1.1; of its own, the argument of 2^x is a log2(e) rounded, off by half a step of
    # |a| 1.45 2^-24, so the exponential by |a| 2^-24 of itself, and it, the quotient and the
    # products by 8 steps together
    eh = 1.1 * ea * (np.abs(b) + eb) + np.abs(silu(a)) * eb + (8 + np.abs(a)) * U32 * np.abs(h)
    rows, cols = h.shape
    pad = lambda v: np.pad(v, ((0, 0), (0, blocks(cols) * B - cols))).reshape(rows, -1, B)
    lo = scale_of(np.maximum(pad(np.abs(h) - eh), 0).max(-1))
    hi = scale_of(pad(np.abs(h) + eh).max(-1))
    held = []
    for s in (lo, hi):
        s = spread(s, rows, cols)
        held += [decode(encode(np.clip(v / s, -TOP, TOP))) * s for v in (h, h - eh, h + eh)]
    top, low = np.max(held, 0), np.min(held, 0)
    h8 = rows64(*quantize_rows(h))
    room = np.maximum(top - h8, h8 - low)
    y, ey = product(h8, w2)
    return y, ey + room @ np.abs(w2).T


def experts(x, idx, gate, w1, v1, w2, residual=None):
    """The experts' part of the layer, and its allowance before the output's rounding.
    x: 8-bit values [T, D]; weights [E, ., .] as their values; slots outside [0, E) left
    out."""
    T, K = idx.shape
    out = np.zeros((T, x.shape[1])) if residual is None else np.array(residual, np.float64)
    room = (K + 2) * U32 * np.abs(out)
    for e in range(w1.shape[0]):
        t, k = np.nonzero(idx == e)
        if len(t) == 0:
            continue
        y, ey = ffn(x[t], w1[e], v1[e], w2[e])
        g = gate[t, k][:, None].astype(np.float64)
        np.add.at(out, t, g * y)
        np.add.at(room, t, np.abs(g) * (ey + (K + 2) * U32 * np.abs(y)))
    return out, room


def order(v):
    """Keys with NaN below every number, for comparisons."""
    return [(-np.inf, 0) if np.isnan(k) else (k, 1) for k in v]


def select(logits, bias, K, score, n_groups=1, top_groups=1, group_top=1, renormalise=True, scale=1.0):
    """idx, gate and the smallest distance between keys (or groups' values) that decided,
    relative to their magnitude, one token at a time."""
    l = np.asarray(logits, np.float64)
    T, E = l.shape
    idx, gate = np.zeros((T, K), np.int32), np.zeros((T, K))
    gs = E // n_groups
    with np.errstate(all="ignore"):
        for t in range(T):
            if score == "softmax":
                z = np.exp(l[t] - (np.nan if np.isnan(l[t]).any() else l[t].max()))
                s = z / z.sum()
            else:
                s = 1.0 / (1.0 + np.exp(-l[t]))
            key = l[t] if bias is None else s + np.asarray(bias, np.float64)
            if n_groups > 1:
                of = s if bias is None and group_top == 2 else key
                of = np.where(np.isnan(of), -np.inf, of).reshape(n_groups, gs)
                value = np.sort(of, 1)[:, ::-1][:, :group_top].sum(1)
                ranks = order(value)
                kept = sorted(range(n_groups), key=lambda g: (-ranks[g][0], -ranks[g][1], g))[:top_groups]
            else:
                kept = [0]
            ranks = order(key)
            left = [e for e in range(E) if e // gs in kept]
            idx[t] = sorted(left, key=lambda e: (-ranks[e][0], -ranks[e][1], e))[:K]
            g = s[idx[t]]
            gate[t] = (g / g.sum() if renormalise else g) * scale
    return idx, gate
