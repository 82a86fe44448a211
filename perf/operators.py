"""The measured work of the paged 8-bit key/value cache: appending to it and attending over it.

The cache holds keys and values as e4m3 numbers in pages of 16 to 128 positions, one scale for each page and
key/value head, and a table of each sequence's pages.  Head layouts are this repository's own (48 query and 8
key/value heads of 128, and smaller ones of its tests), queries, keys and values have the spread that a
projection with weights N(0, 0.02^2) gives them.  Every case says in plain numbers which tokens a call brings:
`dec` sequences with one token each, their lengths spread over a quarter to all of `ctx`, then `chunks` of
consecutive tokens that start at position `before` of sequences of their own, then `pad` padding tokens.

With `own` false every operator is computed in elementary torch operations.
"""
import math

import torch

own = False

DEV = "cuda"
DH = 128
ROPE = 500000.0
STD = 1.5677  # 0.02 sqrt(6144)
TOP = 448.0  # the largest e4m3 number


def listed():
    return [
        # a token of one user's generation: launch latency and nothing else
        {"name": "append_1", "kind": "append", "hq": 48, "hkv": 8, "page": 64, "dtype": "bf16", "dec": 1,
         "ctx": 1000, "chunks": "", "before": 0, "pad": 0},
        # a decode step of 61 users in a batch padded to 64, straight from an fp32 projection, small pages
        {"name": "append_decode_61", "kind": "append", "hq": 48, "hkv": 8, "page": 16, "dtype": "f32", "dec": 61,
         "ctx": 2048, "chunks": "", "before": 0, "pad": 3},
        # a step of continuous batching: 24 users decode, chunks of two prompts start inside a page
        {"name": "append_mixed", "kind": "append", "hq": 48, "hkv": 8, "page": 32, "dtype": "f32", "dec": 24,
         "ctx": 2048, "chunks": "300,205", "before": 500, "pad": 0},
        # a whole prompt
        {"name": "append_prompt_2048", "kind": "append", "hq": 48, "hkv": 8, "page": 64, "dtype": "bf16",
         "dec": 0, "ctx": 64, "chunks": "2048", "before": 0, "pad": 0},
        # the largest call of a prefill server: several prompts at once, large pages
        {"name": "append_prompts_12000", "kind": "append", "hq": 48, "hkv": 8, "page": 128, "dtype": "bf16",
         "dec": 0, "ctx": 128, "chunks": "8000,2001,1999", "before": 0, "pad": 0},
        # a token of one user's generation over 2048 positions: latency
        {"name": "attend_1", "kind": "attend", "hq": 48, "hkv": 8, "page": 64, "dec": 1, "ctx": 2048,
         "chunks": "", "before": 0, "pad": 0},
        # a decode step of 11 users of different lengths in a batch padded to 16, small pages
        {"name": "attend_decode_11", "kind": "attend", "hq": 48, "hkv": 8, "page": 16, "dec": 11, "ctx": 4096,
         "chunks": "", "before": 0, "pad": 5},
        # a full serving batch with long contexts: the cache is the traffic
        {"name": "attend_decode_64", "kind": "attend", "hq": 48, "hkv": 8, "page": 64, "dec": 64, "ctx": 16384,
         "chunks": "", "before": 0, "pad": 0},
        # one user's very long document, 8 query heads on one key/value head: the work split along the positions
        {"name": "attend_long_1", "kind": "attend", "hq": 8, "hkv": 1, "page": 128, "dec": 1, "ctx": 200001,
         "chunks": "", "before": 0, "pad": 0},
        # a whole prompt whose length is no multiple of anything
        {"name": "attend_prompt_1000", "kind": "attend", "hq": 48, "hkv": 8, "page": 64, "dec": 0, "ctx": 64,
         "chunks": "1000", "before": 0, "pad": 0},
        # the next chunk of a long prompt beside 24 users that decode
        {"name": "attend_mixed", "kind": "attend", "hq": 48, "hkv": 8, "page": 32, "dec": 24, "ctx": 2048,
         "chunks": "512", "before": 5000, "pad": 0},
        # a prompt with as many key/value heads as query heads
        {"name": "attend_prompt_2000_mha", "kind": "attend", "hq": 16, "hkv": 16, "page": 16, "dec": 0,
         "ctx": 64, "chunks": "2000", "before": 0, "pad": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hq, hkv = rng.choice([(48, 8), (48, 8), (48, 8), (8, 1), (16, 16), (6, 2), (32, 8), (28, 4)])
    c = {"hq": hq, "hkv": hkv, "page": rng.choice([16, 32, 64, 128]), "dec": 0, "ctx": 64, "chunks": "",
         "before": 0, "pad": rng.choice([0, 0, rng.randint(1, 9)])}
    what = rng.choice(["decode", "decode", "prompt", "mixed"])
    if rng.random() < 0.4:
        c = {"kind": "append", "dtype": rng.choice(["bf16", "f32"]), **c}
        if what == "decode":
            c.update(dec=_log(rng, 1, 128), ctx=_log(rng, 16, 2048))
        elif what == "prompt":
            c.update(chunks=str(_log(rng, 1, 8000)), before=rng.choice([0, rng.randint(1, 5000)]))
        else:
            c.update(dec=rng.randint(1, 48), ctx=_log(rng, 64, 2048), before=rng.choice([0, rng.randint(1, 2048)]),
                     chunks=",".join(str(_log(rng, 2, 1500)) for _ in range(rng.randint(1, 3))))
        return c
    c = {"kind": "attend", **c}
    if what == "decode":
        n = _log(rng, 1, 64)
        c.update(dec=n, ctx=_log(rng, 64, min(100000, 8000000 // (n * hkv))))
    elif what == "prompt":
        c.update(chunks=str(_log(rng, 2, 2048)), before=rng.choice([0, _log(rng, 1, 8000)]))
    else:
        c.update(dec=rng.randint(1, 32), ctx=_log(rng, 64, 4096), before=rng.choice([0, _log(rng, 1, 4000)]),
                 chunks=",".join(str(_log(rng, 2, 600)) for _ in range(rng.randint(1, 2))))
    return c


def _tokens(case):
    """What the call brings: (first position, tokens) of each sequence; sequence i is row i of the table."""
    n, ctx = case["dec"], case["ctx"]
    runs = [(max(0, math.ceil(ctx * (128 - (i * 41) % 97) / 128) - 1), 1) for i in range(n)]
    return runs + [(case["before"], int(c)) for c in case["chunks"].split(",") if c]


def _page_counts(case):
    return [-(-(p + n) // case["page"]) for p, n in _tokens(case)]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    hq, hkv, ps = case["hq"], case["hkv"], case["page"]
    runs, counts = _tokens(case), _page_counts(case)
    n_pages = sum(counts) + 3  # a few pages belong to nobody
    seq, pos = [], []
    for i, (p, n) in enumerate(runs):
        seq += [i] * n
        pos += range(p, p + n)
    seq += [-1] * case["pad"]
    pos += [0] * case["pad"]
    order = torch.randperm(n_pages, device=DEV, generator=g, dtype=torch.int32)
    table = torch.full((len(runs), max(counts)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, c in enumerate(counts):
        table[i, :c] = order[at:at + c]
        at += c
    pages, scales = [], []
    for _ in range(2):
        # earlier entries of spread STD under scales of a few powers of two around 2^-6
        x = torch.randn((n_pages, hkv, ps, DH), device=DEV, generator=g, dtype=torch.bfloat16)
        e = torch.randint(-7, -5, (n_pages, hkv), device=DEV, generator=g).float()
        x = (x * STD) * torch.exp2(-e)[:, :, None, None].bfloat16()
        pages.append(x.clamp_(-TOP, TOP).to(torch.float8_e4m3fn))
        scales.append(torch.exp2(e))
        del x
    T = len(seq)
    s = {"case": case, "T": T, "n_real": T - case["pad"], "tmax": max(n for _, n in runs),
         "seq": torch.tensor(seq, dtype=torch.int32, device=DEV), "pos": torch.tensor(pos, dtype=torch.int32, device=DEV),
         "table": table, "k": pages[0], "v": pages[1], "ks": scales[0], "vs": scales[1]}
    if case["kind"] == "append":
        x = torch.randn((T, (hq + 2 * hkv) * DH), device=DEV, generator=g) * STD
        s["qkv"] = x.bfloat16() if case["dtype"] == "bf16" else x
    else:
        s["q"] = (torch.randn((T, hq, DH), device=DEV, generator=g) * STD).bfloat16()
    if own:
        from paper_2506_23635_gb300 import moe

        s["dims"] = moe.sa_dims(6144, hq, hkv, DH, ROPE)
        s["cache"] = moe.PagedCache(s["k"], s["v"], s["ks"], s["vs"], table)
        if case["kind"] == "attend":
            s["ws"] = moe.paged_alloc_workspace(s["dims"], T)
    return s


# ---- the operators in elementary operations -------------------------------------------------------------


def _firsts(s):
    """The first token of each sequence."""
    n, real = s["table"].shape[0], s["n_real"]
    at = torch.arange(real, device=DEV)
    return torch.full((n,), real, device=DEV).scatter_reduce_(0, s["seq"][:real].long(), at, "amin")


def _store(s, x, pages, scale):
    """Rows x [tokens, heads, 128] into their pages: the page's scale is the smallest power of two that holds
    the call's rows, or the page's own where that is larger and the page was not started by this call; its
    earlier rows follow a larger scale."""
    ps, real = s["case"]["page"], s["n_real"]
    seq, pos = s["seq"][:real].long(), s["pos"][:real].long()
    page, off = s["table"].long()[seq, pos // ps], pos % ps
    bits = (x.abs().amax(-1) / TOP).view(torch.int64)  # (a logarithm may miss a power of two by a rounding)
    up = (bits >> 52) - 1023 + ((bits & ((1 << 52) - 1)) != 0)
    need = torch.exp2(up.clamp(min=-100).double())
    most = torch.zeros(scale.shape, dtype=torch.float64, device=DEV).index_reduce_(0, page, need, "amax")
    fresh = torch.zeros(scale.shape[0], device=DEV).index_reduce_(0, page, (off == 0).float(), "amax")[:, None] > 0
    new = torch.where(most > 0, torch.where(fresh, most, torch.maximum(scale.double(), most)), scale.double())
    part = page[_firsts(s)]  # the pages that may hold earlier rows
    ratio = torch.where(fresh, 1.0, scale.double() / new)[part]
    raw = pages.view(torch.uint8)
    kept = (raw[part].view(torch.float8_e4m3fn).float() * ratio.float()[:, :, None, None]).to(torch.float8_e4m3fn)
    raw[part] = kept.view(torch.uint8)
    raw[page, :, off] = (x / new[page][:, :, None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
    scale.copy_(new)


def _append(s):
    hq, hkv, T, real = s["case"]["hq"], s["case"]["hkv"], s["T"], s["n_real"]
    x = s["qkv"].double().view(T, hq + 2 * hkv, DH)
    rate = ROPE ** (-2.0 * torch.arange(DH // 2, device=DEV, dtype=torch.float64) / DH)
    angle = s["pos"].double()[:, None, None] * rate
    a, b = x[:, :hq + hkv, :DH // 2], x[:, :hq + hkv, DH // 2:]
    turned = torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)
    q = torch.where(s["seq"][:, None, None] >= 0, turned[:, :hq], 0.0).float().bfloat16()
    _store(s, turned[:real, hq:], s["k"], s["ks"])
    _store(s, x[:real, hq + hkv:], s["v"], s["vs"])
    return {"q": q, "k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _cached(s, pages, scale):
    """[sequences, heads, positions, 128] in 32 bits."""
    at = s["table"].clamp(min=0).long()
    x = pages.view(torch.uint8)[at].view(torch.float8_e4m3fn).float() * scale[at][:, :, :, None, None]
    n, m, h, p, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, h, m * p, d)


def _attend(s):
    hq, hkv, T, real, most = s["case"]["hq"], s["case"]["hkv"], s["T"], s["n_real"], s["tmax"]
    n, group = s["table"].shape[0], hq // hkv
    seq = s["seq"][:real].long()
    first = _firsts(s)
    at = (first[:, None] + torch.arange(most, device=DEV)).clamp(max=real - 1)
    pos = torch.where(seq[at] == torch.arange(n, device=DEV)[:, None], s["pos"][:real].long()[at], 0)
    q = s["q"].float()[at].view(n, most, hkv, group, DH).permute(0, 2, 1, 3, 4).reshape(n, hkv, most * group, DH)
    k, v = _cached(s, s["k"], s["ks"]), _cached(s, s["v"], s["vs"])
    score = (q @ k.transpose(2, 3) / math.sqrt(DH)).view(n, hkv, most, group, -1)
    seen = torch.arange(k.shape[2], device=DEV) <= pos[:, None, :, None, None]
    score = torch.where(seen, score, -math.inf)
    e = torch.exp(score - score.amax(-1, keepdim=True))
    e = (e / e.sum(-1, keepdim=True)).view(n, hkv, most * group, -1)
    out = (e @ v).view(n, hkv, most, group, DH).permute(0, 2, 1, 3, 4).reshape(n, most, hq * DH)
    ctx = torch.zeros((T, hq * DH), device=DEV)
    ctx[:real] = out[seq, torch.arange(real, device=DEV) - first[seq]]
    return {"ctx": ctx.bfloat16()}


def run(s):
    if own:
        from paper_2506_23635_gb300 import moe

        if s["case"]["kind"] == "append":
            q = moe.paged_append(s["dims"], s["cache"], s["qkv"], s["seq"], s["pos"])
            return {"q": q, "k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}
        return {"ctx": moe.paged_attend(s["dims"], s["cache"], s["q"], s["seq"], s["pos"], ws=s["ws"])}
    return _append(s) if s["case"]["kind"] == "append" else _attend(s)


def work(case):
    hq, hkv = case["hq"], case["hkv"]
    runs = _tokens(case)
    T = sum(n for _, n in runs)
    if case["kind"] == "append":
        size = 2 if case["dtype"] == "bf16" else 4
        scales = sum((p + n - 1) // case["page"] - p // case["page"] + 1 for p, n in runs) * hkv * 2 * 4
        return {"bytes": T * DH * ((hq + 2 * hkv) * size + hq * 2 + 2 * hkv) + scales, "flops": 6 * T * DH * (hq + hkv)}
    seen = sum(n * p + n * (n + 1) // 2 for p, n in runs)
    rows = sum(p + n for p, n in runs)
    return {"bytes": rows * hkv * DH * 2 + sum(_page_counts(case)) * (hkv * 2 * 4 + 4) + 2 * T * hq * DH * 2,
            "flops": 4 * seen * hq * DH}


# ---- the same in 64 bits, one sequence and one page at a time -------------------------------------------


def exact(case, seed):
    if work(case)["flops"] > 2e12:
        return None
    s = prepare(case, seed)
    hq, hkv, ps = case["hq"], case["hkv"], case["page"]
    runs, counts = _tokens(case), _page_counts(case)
    table = s["table"].tolist()
    T = s["T"]
    if case["kind"] == "attend":
        ctx = torch.zeros((T, hq, DH), dtype=torch.float64, device=DEV)
        t0 = 0
        for i, (p, n) in enumerate(runs):
            own_pages = table[i][:counts[i]]
            for h in range(hkv):
                k = _rows(s["k"], s["ks"], own_pages, h)[:p + n]
                v = _rows(s["v"], s["vs"], own_pages, h)[:p + n]
                hs = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                z = torch.einsum("thd,jd->thj", s["q"][t0:t0 + n, hs].double(), k) / DH ** 0.5
                late = torch.arange(p + n, device=DEV)[None, :] > torch.arange(p, p + n, device=DEV)[:, None]
                z.masked_fill_(late[:, None, :], -math.inf)
                ctx[t0:t0 + n, hs] = torch.einsum("thj,jd->thd", torch.softmax(z, -1), v)
            t0 += n
        return {"ctx": ctx.view(T, hq * DH)}
    w = torch.tensor([ROPE ** (-2.0 * i / DH) for i in range(DH // 2)], dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["pos"].double()[:, None] * w)[:, None, :]
    x = s["qkv"].double().view(T, hq + 2 * hkv, 2, DH // 2)
    z = torch.complex(x[:, :, 0], x[:, :, 1])
    z[:, :hq + hkv] *= turn
    x = torch.cat([z.real, z.imag], -1)
    x[s["n_real"]:] = 0
    out = {"q": x[:, :hq].contiguous()}
    for name, rows in (("k", x[:, hq:hq + hkv]), ("v", x[:, hq + hkv:])):
        pool, scale = s[name].double(), s[name + "s"].double()
        t0 = 0
        for i, (p, n) in enumerate(runs):
            for j in range(p // ps, (p + n - 1) // ps + 1):
                a, lo, hi = table[i][j], max(p, j * ps), min(p + n, (j + 1) * ps)
                new = rows[t0 + lo - p:t0 + hi - p].transpose(0, 1)
                mant, e = torch.frexp(new.abs().amax((1, 2)) / TOP)
                e = torch.where(mant == 0.5, e - 1, e).clamp(min=-100)
                want = torch.ldexp(torch.ones_like(mant), e)
                if lo > j * ps:
                    want = torch.maximum(want, scale[a])
                    pool[a] *= (scale[a] / want)[:, None, None]
                pool[a, :, lo - j * ps:hi - j * ps] = new / want[:, None, None]
                scale[a] = want
            t0 += n
        out[name], out[name + "s"] = pool, scale
    return out


def _rows(pages, scales, which, h):
    at = torch.tensor(which, device=DEV)
    x = pages.view(torch.uint8)[at, h].view(torch.float8_e4m3fn).double() * scales[at, h].double()[:, None, None]
    return x.reshape(-1, DH)
