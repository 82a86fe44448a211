"""Plain 64-bit forms of the paged cache's operators (numpy, one token and one
page at a time), and calls to try them on."""
from __future__ import annotations

import numpy as np

DH = 128
TOP = 448.0


def e4m3_values() -> np.ndarray:
    """The 256 values: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and
    0xff are NaN, there is no infinity."""
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[b] = np.nan if (b & 127) == 127 else (-x if b & 128 else x)
    return v


E4M3 = e4m3_values()


def decode(b) -> np.ndarray:
    return E4M3[np.asarray(b, np.uint8)]


def encode(x) -> np.ndarray:
    """Nearest e4m3, ties to even, at most 448 in magnitude; NaN and infinities
    as NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0)), TOP)
    pos = E4M3[:127]
    hi = np.minimum(np.searchsorted(pos, a), 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    pick = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    b = pick.astype(np.uint8) | np.where(np.signbit(x), 128, 0).astype(np.uint8)
    return np.where(np.isfinite(x), b, 0x7f).astype(np.uint8)


def scale_for(a: float) -> float:
    """The smallest power of two >= a / 448, at least 2^-100."""
    e = -100
    while 448.0 * 2.0 ** e < a:
        e += 1
    return 2.0 ** e


def inside(c, t) -> bool:
    return 0 <= c["seq"][t] < c["table"].shape[0] and \
        0 <= c["pos"][t] < c["table"].shape[1] * c["page"]


def page_of(c, s, p) -> int:
    pg = int(c["table"][s, p // c["page"]])
    return pg if 0 <= pg < c["n_pages"] else -1


def rope(x, pos, base):
    """x [heads, 128] turned to position pos."""
    w = float(base) ** (-2.0 * np.arange(DH // 2) / DH) * float(pos)
    a, b = x[:, :DH // 2], x[:, DH // 2:]
    return np.concatenate([a * np.cos(w) - b * np.sin(w), b * np.cos(w) + a * np.sin(w)], 1)


def append(c, qkv, k, v, ks, vs):
    """The call's queries and, by (page, head), what is stored: `rows` of
    (value, bound on the terms that made it), the scale, and what becomes of the
    page's other rows (their multiplier)."""
    hq, hkv, ps = c["hq"], c["hkv"], c["page"]
    T = len(c["seq"])
    q = np.zeros((T, hq, DH))
    room = np.zeros((T, hq, DH))
    pages = {}
    for t in range(T):
        if not inside(c, t):
            continue
        s, p = int(c["seq"][t]), int(c["pos"][t])
        x = np.asarray(qkv[t], np.float64).reshape(-1, DH)
        turned = rope(x[:hq + hkv], p, c["base"])
        mag = np.abs(x)[:, :DH // 2] + np.abs(x)[:, DH // 2:]
        mag = np.concatenate([mag, mag], 1)
        q[t], room[t] = turned[:hq], mag[:hq]
        pg = page_of(c, s, p)
        if pg < 0:
            continue
        for h in range(hkv):
            pages.setdefault(("k", pg, h), {})[p % ps] = (turned[hq + h], mag[hq + h])
            pages.setdefault(("v", pg, h), {})[p % ps] = (x[hq + hkv + h], 0 * mag[0])
    out = {}
    for (w, pg, h), rows in pages.items():
        old = float((ks if w == "k" else vs)[pg, h])
        finite = [np.abs(r[np.isfinite(r)]) for r, _ in rows.values()]
        a = max([f.max() for f in finite if f.size], default=0.0)
        need = scale_for(a)
        out[(w, pg, h)] = {"rows": rows, "old": old, "fresh": 0 in rows, "amax": a,
                           "scale": need if 0 in rows else max(old, need)}
    return q, room, out


def attend(c, q, k, v, ks, vs):
    """ctx [T, Hq, 128] and, for the tolerance, sum_j p_j |v_j|."""
    hq, hkv, ps = c["hq"], c["hkv"], c["page"]
    T, G = len(c["seq"]), hq // hkv
    ctx, room = np.zeros((T, hq, DH)), np.zeros((T, hq, DH))
    kept = {}
    for t in range(T):
        if not inside(c, t):
            continue
        s, p = int(c["seq"][t]), int(c["pos"][t])
        pgs = np.array([page_of(c, s, j) for j in range(0, p + 1, ps)])
        j = np.arange(p + 1)
        j = j[pgs[j // ps] >= 0]
        if j.size == 0:
            continue
        pg, off = pgs[j // ps], j % ps
        for g in range(hkv):
            key = (s, p, g)
            if key not in kept:
                kept[key] = (decode(k[pg, g, off]) * ks[pg, g][:, None].astype(np.float64),
                             decode(v[pg, g, off]) * vs[pg, g][:, None].astype(np.float64))
            kk, vv = kept[key]
            z = np.asarray(q[t, g * G:(g + 1) * G], np.float64) @ kk.T / np.sqrt(DH)
            z = np.exp(z - z.max(1, keepdims=True))
            z /= z.sum(1, keepdims=True)
            ctx[t, g * G:(g + 1) * G] = z @ vv
            room[t, g * G:(g + 1) * G] = z @ np.abs(vv)
        kept = {x: y for x, y in kept.items() if x[0] == s and x[1] == p}
    return ctx, room


def call(hq, hkv, page, runs, seed=0, pad=0, order="given", extra_pages=2, max_pages=None,
         spread=1.5):
    """A call: `runs` are (sequence, first position, tokens); the sequences'
    tables hold just the pages that those need, -1 elsewhere."""
    rng = np.random.default_rng(seed)
    n_seq = max([r[0] for r in runs], default=0) + 1
    need = [0] * n_seq
    for s, p, n in runs:
        need[s] = max(need[s], -(-(p + n) // page))
    n_pages = sum(need) + extra_pages
    perm = rng.permutation(n_pages).astype(np.int32)
    table = np.full((n_seq, max_pages or max(max(need), 1)), -1, np.int32)
    at = 0
    for s in range(n_seq):
        table[s, :need[s]] = perm[at:at + need[s]]
        at += need[s]
    seq = np.concatenate([np.full(n, s, np.int32) for s, _, n in runs] +
                         [np.full(pad, -1, np.int32)])
    pos = np.concatenate([np.arange(p, p + n, dtype=np.int32) for _, p, n in runs] +
                         [np.zeros(pad, np.int32)])
    if order == "shuffled":
        mix = rng.permutation(len(seq))
        seq, pos = seq[mix], pos[mix]
    shape = (n_pages, hkv, page, DH)
    bytes_ = [rng.integers(0, 256, shape, dtype=np.uint8) for _ in range(2)]
    scales = [(2.0 ** rng.integers(-9, -6, shape[:2])).astype(np.float32) for _ in range(2)]
    # earlier entries: ordinary numbers (a NaN only where no position lies)
    for b in bytes_:
        b[...] = encode(rng.normal(size=shape) * 100.0)
    return {"hq": hq, "hkv": hkv, "page": page, "base": 10000.0, "seq": seq, "pos": pos,
            "table": table, "n_pages": n_pages, "k": bytes_[0], "v": bytes_[1], "ks": scales[0],
            "vs": scales[1], "rng": rng, "spread": spread}
