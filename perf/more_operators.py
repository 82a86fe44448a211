"""The measured work of the 8-bit experts: quantising in blocks of 128, choosing experts, grouped products, whole FFNs.

Numbers of 8 bits are e4m3 with one fp32 scale for each 128 numbers of a row (activations) or each 128 x 128
block of a matrix (weights).  The quantiser's scales are the smallest powers of two that hold the block; the
products take any scales.  Expert sizes are this repository's own layer (6144 x 10752, 16 experts, 4 chosen) and
generic ones.

The experts' outputs are bf16: what lies next to a border between two 8-bit numbers of the hidden vector may fall
on either side of it in 32 bits, which an fp32 output would show.

With `own` false every operator is computed in elementary torch operations.
"""
import math

import torch

own = False

DEV = "cuda"
B = 128
TOP = 448.0  # the largest e4m3 number


def listed():
    return [
        # the rows of a small decode batch, straight from an fp32 residual stream
        {"name": "rows_61", "kind": "rows", "rows": 61, "cols": 6144, "dtype": "f32"},
        # a long prompt's activations, a row count that is no multiple of anything
        {"name": "rows_8190", "kind": "rows", "rows": 8190, "cols": 6144, "dtype": "bf16"},
        # loading: the up projections of four experts turned to 8 bits
        {"name": "blocks_4x10752", "kind": "blocks", "n": 4, "rows": 10752, "cols": 6144, "dtype": "bf16"},
        # one user's token, the layer's own router rule: launch latency and nothing else
        {"name": "select_1", "kind": "select", "T": 1, "E": 16, "K": 4, "score": "softmax", "bias": False,
         "groups": 1, "kept": 1, "best": 1, "renorm": True, "scale": 1.0},
        # a large batch over many experts: sigmoid scores, a balancing bias, half of eight groups kept
        {"name": "select_8191", "kind": "select", "T": 8191, "E": 256, "K": 8, "score": "sigmoid", "bias": True,
         "groups": 8, "kept": 4, "best": 2, "renorm": True, "scale": 2.5},
        # one token through a projection as wide as the attention block's: 50 MB of weights
        {"name": "product_1", "kind": "product", "groups": "1", "out": 8192, "in": 6144, "dtype": "bf16"},
        # uneven groups, empty ones among them, sizes that end inside a block of 128
        {"name": "product_ragged", "kind": "product", "groups": "0,300,1,77,0,129,5,265", "out": 1992, "in": 1488,
         "dtype": "f32"},
        # a prompt through the same projection: the tensor cores
        {"name": "product_2048", "kind": "product", "groups": "2048", "out": 8192, "in": 6144, "dtype": "bf16"},
        # a token of one user's generation through the layer's experts
        {"name": "experts_1", "kind": "experts", "T": 1, "D": 6144, "F": 10752, "E": 16, "K": 4, "dtype": "bf16",
         "residual": False},
        # a decode batch that reaches every expert: all weights are read once
        {"name": "experts_64", "kind": "experts", "T": 64, "D": 6144, "F": 10752, "E": 16, "K": 4, "dtype": "bf16",
         "residual": False},
        # many small experts with odd sizes, fp32 activations, a residual
        {"name": "experts_300_small", "kind": "experts", "T": 300, "D": 2000, "F": 1424, "E": 40, "K": 6,
         "dtype": "f32", "residual": True},
        # a whole prompt
        {"name": "experts_2048", "kind": "experts", "T": 2048, "D": 6144, "F": 10752, "E": 16, "K": 4,
         "dtype": "bf16", "residual": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rows", "blocks", "select", "select", "product", "product", "experts", "experts", "experts"])
    dtype = rng.choice(["bf16", "f32"])
    if kind == "rows":
        cols = 16 * _log(rng, 4, 640)
        return {"kind": kind, "rows": _log(rng, 1, min(16000, 50000000 // cols)), "cols": cols, "dtype": dtype}
    if kind == "blocks":
        return {"kind": kind, "n": rng.randint(1, 4), "rows": 8 * _log(rng, 16, 1300), "cols": 16 * _log(rng, 8, 380),
                "dtype": dtype}
    if kind == "select":
        groups, size = rng.choice([(1, 8), (1, 16), (1, 60), (1, 100), (4, 10), (4, 16), (8, 8), (8, 20), (8, 32)])
        kept = rng.randint(1, groups)
        return {"kind": kind, "T": _log(rng, 1, 8000), "E": groups * size, "K": rng.randint(1, min(8, kept * size)),
                "score": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.6, "groups": groups, "kept": kept,
                "best": rng.randint(1, 2), "renorm": rng.random() < 0.7, "scale": rng.choice([1.0, 2.5])}
    if kind == "product":
        n = rng.choice([1, 1, 3, 8, 20])
        groups = [rng.choice([0, _log(rng, 1, 2000 // n)]) if n > 1 else _log(rng, 1, 2048) for _ in range(n)]
        groups[-1] += 1 - min(1, sum(groups))
        return {"kind": kind, "groups": ",".join(str(g) for g in groups), "out": 8 * _log(rng, 16, 1024),
                "in": 16 * _log(rng, 16, 384), "dtype": dtype}
    D, F, E, K = rng.choice([(6144, 10752, 16, 4), (6144, 10752, 16, 4), (1008, 2512, 8, 2), (2048, 768, 64, 6),
                             (4096, 1536, 128, 8), (720, 400, 10, 3)])
    return {"kind": kind, "T": _log(rng, 1, 2048), "D": D, "F": F, "E": E, "K": K, "dtype": dtype,
            "residual": rng.random() < 0.5}


_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _blocks(n):
    return -(-n // B)


def _matrices(g, n, rows, cols):
    """Weights of spread 0.02 in e4m3, under scales that are no powers of two."""
    q = torch.empty((n, rows, cols), dtype=torch.float8_e4m3fn, device=DEV)
    for i in range(n):
        w = torch.randn((rows, cols), device=DEV, generator=g, dtype=torch.bfloat16)
        q[i].view(torch.uint8).copy_(w.mul_(100.0).clamp_(-TOP, TOP).to(torch.float8_e4m3fn).view(torch.uint8))
    s = torch.rand((n, _blocks(rows), _blocks(cols)), device=DEV, generator=g)
    return q, (s * 0.5 + 0.75) * 0.0002


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if own:
        from paper_2506_23635_gb300 import moe
    if kind in ("rows", "blocks"):
        shape = (case["rows"], case["cols"]) if kind == "rows" else (case["n"], case["rows"], case["cols"])
        x = torch.randn(shape, device=DEV, generator=g, dtype=torch.bfloat16 if kind == "blocks" else torch.float32)
        if kind == "rows":  # rows of different size, a few columns that stand out
            x *= torch.exp2(torch.randint(-3, 4, (shape[0], 1), device=DEV, generator=g).float())
            x[:, ::97] *= 20.0
        s["x"] = (x if kind == "rows" else x.mul_(0.02)).to(_DT[case["dtype"]])
    elif kind == "select":
        T, E = case["T"], case["E"]
        s["logits"] = torch.randn((T, E), device=DEV, generator=g) * 1.57
        s["bias"] = torch.randn((E,), device=DEV, generator=g) * 0.05 if case["bias"] else None
        if own:
            s["dims"] = moe.dims(1024, 1024, E, case["K"], torch.bfloat16)
            s["router"] = moe.router(case["score"], case["groups"], case["kept"], case["best"], case["renorm"],
                                     case["scale"])
    elif kind == "product":
        groups = [int(v) for v in case["groups"].split(",")]
        S, n_in = sum(groups), case["in"]
        s["w"], s["ws"] = _matrices(g, len(groups), case["out"], n_in)
        x = torch.randn((S, n_in), device=DEV, generator=g) * 100.0
        s["x"] = x.clamp_(-TOP, TOP).to(torch.float8_e4m3fn)
        s["xs"] = (torch.rand((S, _blocks(n_in)), device=DEV, generator=g) * 0.5 + 0.75) * 0.01
        ends = [0]
        for n in groups:
            ends.append(ends[-1] + n)
        s["ends"] = ends
        s["offsets"] = torch.tensor(ends, dtype=torch.int32, device=DEV) if len(groups) > 1 else None
        if own:
            s["scratch"] = moe.quant_product_alloc_workspace(len(groups), case["out"], n_in, S)
    else:
        T, D, F, E, K = (case[k] for k in ("T", "D", "F", "E", "K"))
        s["w1"], s["s1"] = _matrices(g, E, F, D)
        s["v1"], s["sv"] = _matrices(g, E, F, D)
        s["w2"], s["s2"] = _matrices(g, E, D, F)
        s["x"] = torch.randn((T, D), device=DEV, generator=g).to(_DT[case["dtype"]])
        # some experts are better liked than others
        score = torch.randn((T, E), device=DEV, generator=g) + 0.3 * torch.randn((E,), device=DEV, generator=g)
        top, idx = torch.topk(score, K, dim=1)
        s["idx"], s["gate"] = idx.int(), torch.softmax(top, 1)
        s["res"] = torch.randn((T, D), device=DEV, generator=g).bfloat16() if case["residual"] else None
        if own:
            s["dims"] = moe.dims(D, F, E, K, _DT[case["dtype"]], out_dtype=torch.bfloat16)
            s["experts"] = moe.QuantExperts(s["w1"], s["s1"], s["v1"], s["sv"], s["w2"], s["s2"])
            s["scratch"] = moe.quant_alloc_workspace(s["dims"], T)
    return s


# ---- the operators in elementary operations -------------------------------------------------------------


def _scale(amax):
    """The smallest power of two that holds amax, not below 2^-100."""
    bits = amax.float().contiguous().view(torch.int32)
    up = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000).int()  # 448 is 1.75 2^8
    return torch.exp2(up.clamp(min=-100).double()).float()


def _quantize(x):
    """e4m3 numbers and scales of each row's blocks."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.float(), (0, _blocks(cols) * B - cols)).view(rows, -1, B)
    scale = _scale(x.abs().amax(-1))
    q = (x / scale[:, :, None]).view(rows, -1)[:, :cols]
    return q.to(torch.float8_e4m3fn), scale


def _quantize_blocks(w):
    n, rows, cols = w.shape
    q = torch.empty((n, rows, cols), dtype=torch.float8_e4m3fn, device=DEV)
    scale = torch.empty((n, _blocks(rows), _blocks(cols)), device=DEV)
    for i in range(n):
        x = torch.nn.functional.pad(w[i].float(), (0, -cols % B, 0, -rows % B))
        x = x.view(_blocks(rows), B, _blocks(cols), B)
        scale[i] = _scale(x.abs().amax((1, 3)))
        x = (x / scale[i][:, None, :, None]).reshape(_blocks(rows) * B, -1)[:rows, :cols]
        q[i].view(torch.uint8).copy_(x.to(torch.float8_e4m3fn).view(torch.uint8))
    return q, scale


def _rows32(q, scale):
    return q.float() * scale.repeat_interleave(B, 1)[:, :q.shape[1]]


def _matrix32(q, scale):
    s = scale.repeat_interleave(B, 0)[:q.shape[0]].repeat_interleave(B, 1)[:, :q.shape[1]]
    return q.float() * s


def _select(s):
    c = s["case"]
    E, K, G = c["E"], c["K"], c["groups"]
    x = s["logits"].double()
    if c["score"] == "softmax":
        e = torch.exp(x - x.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-x))
    key = x if s["bias"] is None else score + s["bias"].double()
    if G > 1:
        if c["best"] == 1:
            group = key.view(-1, G, E // G).amax(2)
        else:
            of = score if s["bias"] is None else key
            group = torch.sort(of.view(-1, G, E // G), dim=2, descending=True)[0][:, :, :2].sum(2)
        order = torch.sort(group, dim=1, descending=True, stable=True)[1]
        out = torch.ones_like(group, dtype=torch.bool).scatter_(1, order[:, :c["kept"]], False)
        key = torch.where(out.repeat_interleave(E // G, 1), -math.inf, key)
    idx = torch.sort(key, dim=1, descending=True, stable=True)[1][:, :K]
    gate = torch.gather(score, 1, idx)
    if c["renorm"]:
        gate = gate / gate.sum(1, keepdim=True)
    return {"idx": idx.int(), "gate": (gate * c["scale"]).float()}


def _product(s):
    x = _rows32(s["x"], s["xs"])
    y = torch.empty((x.shape[0], s["case"]["out"]), device=DEV)
    for e in range(len(s["ends"]) - 1):
        a, b = s["ends"][e:e + 2]
        if b > a:
            y[a:b] = x[a:b] @ _matrix32(s["w"][e], s["ws"][e]).t()
    return {"y": y.to(_DT[s["case"]["dtype"]])}


def _experts(s):
    c = s["case"]
    x = _rows32(*_quantize(s["x"]))
    out = torch.zeros((c["T"], c["D"]), device=DEV) if s["res"] is None else s["res"].float()
    order = torch.sort(s["idx"].flatten(), stable=True)[1]
    counts = torch.bincount(s["idx"].flatten(), minlength=c["E"]).tolist()
    for e, at in enumerate(order.split(counts)):
        if counts[e] == 0:
            continue
        t = at // c["K"]
        a = x[t] @ _matrix32(s["w1"][e], s["s1"][e]).t()
        b = x[t] @ _matrix32(s["v1"][e], s["sv"][e]).t()
        h = _rows32(*_quantize(a / (1 + torch.exp(-a)) * b))
        y = h @ _matrix32(s["w2"][e], s["s2"][e]).t()
        out.index_add_(0, t, y * s["gate"].flatten()[at][:, None])
    return {"out": out.bfloat16()}


def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2506_23635_gb300 import moe

        if kind in ("rows", "blocks"):
            q, scale = (moe.quantize_rows if kind == "rows" else moe.quantize_blocks)(s["x"])
            return {"q": q, "scale": scale}
        if kind == "select":
            idx, gate = moe.route_select(s["dims"], s["router"], s["logits"], s["bias"])
            return {"idx": idx, "gate": gate}
        if kind == "product":
            return {"y": moe.quant_product(s["x"], s["xs"], s["w"], s["ws"], s["offsets"],
                                           _DT[s["case"]["dtype"]], ws=s["scratch"])}
        return {"out": moe.quant_experts_forward(s["dims"], s["experts"], s["x"], s["idx"], s["gate"], s["res"],
                                                 ws=s["scratch"])}
    if kind in ("rows", "blocks"):
        q, scale = (_quantize if kind == "rows" else _quantize_blocks)(s["x"])
        return {"q": q, "scale": scale}
    return {"select": _select, "product": _product, "experts": _experts}[kind](s)


def work(case):
    kind = case["kind"]
    size = 2 if case.get("dtype") == "bf16" else 4
    if kind in ("rows", "blocks"):
        n, rows, cols = case.get("n", 1), case["rows"], case["cols"]
        scales = n * _blocks(cols) * (rows if kind == "rows" else _blocks(rows))
        return {"bytes": n * rows * cols * (size + 1) + 4 * scales, "flops": 2 * n * rows * cols}
    if kind == "select":
        T, E, K = case["T"], case["E"], case["K"]
        return {"bytes": 4 * T * E + 8 * T * K + (4 * E if case["bias"] else 0), "flops": 4 * T * E}
    if kind == "product":
        groups = [int(v) for v in case["groups"].split(",")]
        S, n_out, n_in = sum(groups), case["out"], case["in"]
        used = sum(1 for n in groups if n)
        return {"bytes": used * (n_out * n_in + 4 * _blocks(n_out) * _blocks(n_in))
                + S * (n_in + 4 * _blocks(n_in) + n_out * size), "flops": 2 * S * n_out * n_in}
    T, D, F, E, K = (case[k] for k in ("T", "D", "F", "E", "K"))
    used = E * (1 - (1 - K / E) ** T)  # the experts that T tokens reach, were all liked alike
    matrix = D * F + 4 * _blocks(D) * _blocks(F)
    return {"bytes": int(used * 3 * matrix) + T * D * (size + (4 if case["residual"] else 2)) + 8 * T * K,
            "flops": 6 * T * K * D * F}


# ---- the same in 64 bits, one block of 128 at a time ----------------------------------------------------


def _held(x):
    """x [rows, cols] in 64 bits as blocks of each row hold it: (numbers, scales)."""
    rows, cols = x.shape
    q = torch.empty((rows, cols), dtype=torch.float64, device=DEV)
    scales = []
    for c0 in range(0, cols, B):
        part = x[:, c0:c0 + B]
        one = _power(part.abs().amax(1))
        q[:, c0:c0 + B] = _nearest(part / one[:, None])
        scales.append(one)
    return q, torch.stack(scales, 1)


def _power(amax):
    mant, e = torch.frexp(torch.clamp(amax / TOP, min=2.0 ** -101))
    return _two_to(torch.where(mant == 0.5, e - 1, e).clamp(min=-100))


def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)  # (a power function may be off by a rounding)


def _nearest(v):
    """The nearest e4m3 number: steps of 2^(exponent - 3), not below 2^-9; halves go to the even one."""
    e = torch.frexp(v)[1] - 1
    step = _two_to(e.clamp(min=-6) - 3)
    return torch.round(v / step) * step


def _times(x, xs, w, ws):
    """Rows of 8-bit numbers times one matrix, block by block."""
    y = torch.zeros((x.shape[0], w.shape[0]), dtype=torch.float64, device=DEV)
    rows = torch.arange(w.shape[0], device=DEV) // B
    for b in range(ws.shape[1]):
        k = slice(b * B, (b + 1) * B)
        y += (x[:, k].double() @ w[:, k].double().t()) * xs[:, b, None].double() * ws[rows, b].double()
    return y


def exact(case, seed):
    if work(case)["flops"] > 4e12:
        return None
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rows":
        q, scale = _held(s["x"].double())
        return {"q": q, "scale": scale}
    if kind == "blocks":
        n, rows, cols = s["x"].shape
        q = torch.empty((n, rows, cols), dtype=torch.float64, device=DEV)
        scale = torch.empty((n, _blocks(rows), _blocks(cols)), dtype=torch.float64, device=DEV)
        for i in range(n):
            for r in range(_blocks(rows)):
                band = s["x"][i, r * B:(r + 1) * B].double()
                scale[i, r] = _power(torch.stack([p.abs().amax() for p in band.split(B, 1)]))
                q[i, r * B:(r + 1) * B] = _nearest(band / scale[i, r].repeat_interleave(B)[:cols])
        return {"q": q, "scale": scale}
    if kind == "select":
        return _exact_select(s)
    if kind == "product":
        y = torch.zeros((s["x"].shape[0], case["out"]), dtype=torch.float64, device=DEV)
        for e, (a, b) in enumerate(zip(s["ends"], s["ends"][1:])):
            if b > a:
                y[a:b] = _times(s["x"][a:b], s["xs"][a:b], s["w"][e], s["ws"][e])
        return {"y": y}
    x, xs = _held(s["x"].double())
    out = torch.zeros((case["T"], case["D"]), dtype=torch.float64, device=DEV)
    if s["res"] is not None:
        out += s["res"].double()
    for e in range(case["E"]):
        hit = s["idx"] == e
        t = hit.any(1).nonzero().flatten()
        if len(t) == 0:
            continue
        a = _times(x[t], xs[t], s["w1"][e], s["s1"][e])
        b = _times(x[t], xs[t], s["v1"][e], s["sv"][e])
        h, hs = _held(a * torch.sigmoid(a) * b)
        gate = (s["gate"].double() * hit).sum(1)[t]
        out[t] += gate[:, None] * _times(h, hs, s["w2"][e], s["s2"][e])
    return {"out": out}


def _exact_select(s):
    """Experts taken one at a time, each the best that is left."""
    c = s["case"]
    E, G = c["E"], c["groups"]
    x = s["logits"].double()
    score = torch.softmax(x, 1) if c["score"] == "softmax" else torch.sigmoid(x)
    key = x.clone() if s["bias"] is None else score + s["bias"].double()
    if G > 1:
        each = (score if s["bias"] is None and c["best"] == 2 else key).view(-1, G, E // G)
        value = torch.topk(each, c["best"], dim=2)[0].sum(2)
        keep = torch.zeros_like(value, dtype=torch.bool)
        for _ in range(c["kept"]):
            left = torch.where(keep, -math.inf, value)
            keep.scatter_(1, _first_best(left), True)
        key = torch.where(keep[:, :, None].expand(-1, -1, E // G).reshape(-1, E), key, -math.inf)
    idx = []
    for _ in range(c["K"]):
        idx.append(_first_best(key))
        key.scatter_(1, idx[-1], -math.inf)
    idx = torch.cat(idx, 1)
    gate = torch.gather(score, 1, idx)
    if c["renorm"]:
        gate = gate / gate.sum(1, keepdim=True)
    return {"idx": idx.int(), "gate": gate * c["scale"]}


def _first_best(v):
    best = v == v.amax(1, keepdim=True)
    return best.int().argmax(1, keepdim=True)
