"""8-bit experts on the GPU where their error bounds are at their ends: SiLU of far negative
numbers, choices that near keys of unlike errors decide, shares of the streaming kernel that
hold several tiles."""
import numpy as np
import pytest
import torch

from tests.paged_ref import encode
from tests.test_gpu_quant import check_select, cuda, e4m3, moe, num

pytestmark = pytest.mark.gpu


# ---- SiLU ----------------------------------------------------------------------------


@pytest.mark.parametrize("tens", [[-80.0, -88.0, -96.0], [-88.0, -96.0]], ids=["from80", "from88"])
@pytest.mark.parametrize("T", [1, 20, 60, 200])
def test_silu_of_far_negative_numbers(T, tens):
    """SiLU(a) is a e^a there, not zero (b = 2^100 and more lifts h); a is exact in the products, as
    is y, which is h's 8-bit number.  h: rounded to nearest by at most 2^-4 of itself, or half of the
    smallest step, 2^-10 of its block's scale, which is at most its largest number / 224;
    exponentials down to 2e-42 are numbers of 1450 steps of 2^-149, off by half a step (2^-11) and
    their product with a by less; the rest below 2^-16."""
    m = moe()
    D = F = 128
    x = np.zeros((T, D))
    x[:, :2] = 1.0, 0.25
    x[:, 2] = 2.0 ** (np.arange(T) % 5)
    w1, v1 = np.zeros((1, F, D)), np.zeros((1, F, D))
    w1[0, :, 0] = np.repeat(tens, 64)[:F] if len(tens) == 2 else np.repeat(tens, 43)[:F]
    w1[0, :, 1] = (np.arange(F) % 4) * 2 * (w1[0, :, 0] > -96)
    v1[0, :, 2] = 1.0
    w2 = np.eye(D, F)[None]
    one, big = np.ones((1, 1, 1), np.float32), np.full((1, 1, 1), 2.0 ** 100, np.float32)
    ex = m.QuantExperts(e4m3(encode(w1)), cuda(one), e4m3(encode(v1)), cuda(big), e4m3(encode(w2)), cuda(one))
    d = m.dims(D, F, 1, 1, torch.float32)
    got = num(m.quant_experts_forward(d, ex, cuda(x.astype(np.float32)), cuda(np.zeros((T, 1), np.int32)),
                                      cuda(np.ones((T, 1), np.float32))))
    assert m.get_last_error() == 0
    a = w1[0, :, 0] + 0.25 * w1[0, :, 1]
    want = a * np.exp(a) / (1 + np.exp(a)) * x[:, 2:3] * 2.0 ** 100
    step = np.abs(want).max(1, keepdims=True) / 224 * 2.0 ** -10
    assert (np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), step) + 2.0 ** -10 * np.abs(want)).all()


# ---- the choice of experts -----------------------------------------------------------


@pytest.mark.parametrize("logits,K", [([20, 20, 21], 1), ([8, 8, 8.000001], 1), ([30, 20, 20, 20.5, 40], 2),
                                      ([1, 20, 20, 20, 21, 2], 1), ([-5, 17, 17, 17.000002, 17.000002], 3)], ids=str)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_select_equals_at_the_border(score, logits, K):
    """The last one kept and the first left out are equal, another whose key 32 bits do not tell from
    theirs lies behind."""
    l = np.array([logits] * 5, np.float32)
    l[1:] += np.array([[0], [-0.5], [0.25], [1]], np.float32)
    check_select(moe(), l, np.zeros(l.shape[1]), K, score=score)


def test_select_small_errors_beside_a_large_one():
    """The two at the border are further apart than their own errors; a third, a score near one with a
    bias that takes it to their size, has the largest key."""
    for l, b in (([-6.9995, -6.9995036, 3.3423553], [0, 0, -0.96494204]),
                 ([-7.143973, -7.8893886, 1.6407677], [.00121102, .00162542, -.83563936])):
        l, b = np.array(l, np.float32), np.array(b, np.float32)
        around = np.tile(l, (400, 1))  # (and neighbours of it, so that any exponential meets some)
        around[:, 2] += np.float32(2.0 ** -23) * (np.arange(400) - 200)
        check_select(moe(), around, b, 1, score="sigmoid")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,K,G,kept", [(16, 1, 1, 1), (16, 2, 1, 1), (24, 5, 1, 1), (64, 3, 1, 1), (256, 8, 1, 1),
                                        (24, 2, 4, 2), (256, 4, 8, 4)])
def test_select_wide_biases(score, E, K, G, kept):
    """Biases as wide as the scores, so that small and large scores meet at the same key: keys t + noise
    of 1e-8 to 1e-5 for one t a token."""
    rng = np.random.default_rng(E + K + G)
    T = 2000
    bias = np.where(rng.random(E) < 0.5, 0.0, -rng.random(E) * (0.95 if score == "sigmoid" else 1.6 / E))
    bias = bias.astype(np.float32)
    t = np.exp(rng.uniform(np.log(1e-4), np.log(0.02 if score == "sigmoid" else 0.3 / E), (T, 1)))
    noise = rng.normal(size=(T, E)) * 10.0 ** rng.uniform(-8, -5, (T, 1)) * t ** 0.5
    s = np.clip(t + noise - bias, 1e-7, 0.999)
    if score == "sigmoid":
        logits = np.log(s / (1 - s))
    else:
        s[:, 0] += np.maximum(1.0 - s.sum(1), 1e-3)  # (the rest of the sum: one large score)
        logits = np.log(s / s.sum(1, keepdims=True)) + rng.normal(size=(T, 1))
    check_select(moe(), logits, bias, K, score=score, n_groups=G, top_groups=kept, group_top=2 if G > 1 else 1)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_select_barred_experts(score):
    """Biases of -1e9 bar experts; what rounding does to their keys decides nothing, but among themselves."""
    rng = np.random.default_rng(1)
    logits, bias = rng.normal(size=(500, 64)), rng.normal(size=64) * 0.05
    bias[::3] = -1e9
    check_select(moe(), logits, bias, 6, score=score)
    check_select(moe(), logits, bias, 50, score=score)
    check_select(moe(), logits, bias, 6, score=score, n_groups=8, top_groups=4, group_top=2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("low,best", [(-np.inf, 2), (-np.inf, 1), (-3e38, 2)])
def test_select_groups_barred_by_the_lowest_numbers(score, low, best):
    """Groups whose biases are all the type's lowest rank above those of minus infinity (or by
    how low they are), though the sum of two is no number of 32 bits."""
    rng = np.random.default_rng(3)
    logits, bias = rng.normal(size=(200, 16)), rng.normal(size=16) * 0.05
    bias[:4], bias[4:8] = low, np.finfo(np.float32).min
    if np.isfinite(low):
        bias[:4], bias[4:8] = np.finfo(np.float32).min, low
    check_select(moe(), logits, bias, 11, score=score, n_groups=4, top_groups=3, group_top=best)


def test_select_smallest_scores():
    """Scores about 2^-126, where their 32-bit form may be zero, beside biases of that size."""
    rng = np.random.default_rng(2)
    logits = rng.uniform(-89.5, -86.5, size=(600, 12))
    bias = rng.uniform(0, 2e-38, 12)
    check_select(moe(), logits, bias, 3, score="sigmoid")


def test_select_gates_of_the_smallest_scores():
    """Sigmoids down to the smallest number of 32 bits, lifted by the scale."""
    logits = -80.0 - np.arange(48).reshape(2, 24) * 0.5
    check_select(moe(), logits, None, 24, score="sigmoid", renormalise=False, scale=1e30)


# ---- shares of the streaming kernel ------------------------------------------------------


@pytest.mark.parametrize("n_in", [144, 256, 384, 512])
@pytest.mark.parametrize("S", [1, 20, 33, 64])
def test_product_shares_of_several_tiles(S, n_in):
    """Tiles of few k-blocks: a CTA's share ends one that others began, has whole ones, and begins one that
    others end.  Against 64 bits, and the same bits every time."""
    m, g = moe(), torch.Generator(device="cuda").manual_seed(S + n_in)
    n_out, nb = 40000, -(-n_in // 128)
    f8 = lambda *s: (torch.randn(s, device="cuda", generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    x, w = f8(S, n_in), f8(1, n_out, n_in)
    xs = torch.rand((S, nb), device="cuda", generator=g) + 0.5
    s = torch.rand((1, -(-n_out // 128), nb), device="cuda", generator=g) + 0.5
    x64 = x.double() * xs.double().repeat_interleave(128, 1)[:, :n_in]
    w64 = w[0].double() * s[0].double().repeat_interleave(128, 0)[:n_out].repeat_interleave(128, 1)[:, :n_in]
    want, room = x64 @ w64.t(), (n_in + 8) * 2.0 ** -23 * (x64.abs() @ w64.abs().t())
    ws = m.quant_product_alloc_workspace(1, n_out, n_in, S)
    first = m.quant_product(x, xs, w, s, None, torch.float32, ws=ws)
    assert ((first.double() - want).abs() <= room).all()
    for _ in range(20):
        assert torch.equal(m.quant_product(x, xs, w, s, None, torch.float32, ws=ws), first)
    assert m.get_last_error() == 0


@pytest.mark.parametrize("S", [65, 70, 96, 100, 128])
@pytest.mark.parametrize("n_in", [16, 272, 1024])
def test_product_last_rows_of_a_wide_tile(S, n_in):
    """Tiles of 64 rows with half of them or less: nothing behind the workspace's size is needed, and
    its contents do not matter."""
    m, g = moe(), torch.Generator(device="cuda").manual_seed(S + n_in)
    n_out, nb = 264, -(-n_in // 128)
    f8 = lambda *s: (torch.randn(s, device="cuda", generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    x, w = f8(S, n_in), f8(1, n_out, n_in)
    xs = torch.rand((S, nb), device="cuda", generator=g) + 0.5
    s = torch.rand((1, 3, nb), device="cuda", generator=g) + 0.5
    x64 = x.double() * xs.double().repeat_interleave(128, 1)[:, :n_in]
    w64 = w[0].double() * s[0].double().repeat_interleave(128, 0)[:n_out].repeat_interleave(128, 1)[:, :n_in]
    want, room = x64 @ w64.t(), (n_in + 8) * 2.0 ** -23 * (x64.abs() @ w64.abs().t())
    ws = m.quant_product_alloc_workspace(1, n_out, n_in, S)
    assert ws.numel() == m.quant_product_workspace_size(1, n_out, n_in, S)
    outs = []
    for fill in (0x00, 0xff, 0x7f):
        ws.fill_(fill)
        outs.append(m.quant_product(x, xs, w, s, None, torch.float32, ws=ws))
        assert ((outs[-1].double() - want).abs() <= room).all() and torch.equal(outs[-1], outs[0])
    assert m.get_last_error() == 0


# ---- the largest calls ---------------------------------------------------------------------


def test_largest_rows_and_products():
    """16,777,216 rows: quantised, and times a matrix (whole numbers, so that every sum is exact)."""
    m, rows = moe(), 1 << 24
    x = (torch.arange(rows * 16, device="cuda") % 13 - 6).to(torch.bfloat16).view(rows, 16)
    x[:, 0] = 7.0
    q, s = m.quantize_rows(x)
    assert (s == 2.0 ** -6).all()  # (7 = 448 / 64)
    for part in range(0, rows, 1 << 22):
        assert torch.equal(q[part:part + (1 << 22)].float() * 2.0 ** -6, x[part:part + (1 << 22)].float())
    w = (torch.arange(8 * 16, device="cuda") % 5 - 2).float().view(1, 8, 16)
    off = torch.tensor([5, rows - 3], dtype=torch.int32, device="cuda")
    y = torch.full((rows, 8), 9.0, device="cuda")
    m.quant_product(q, s, w.to(torch.float8_e4m3fn), torch.ones((1, 1, 1), device="cuda"), off, torch.float32, out=y)
    want = x.float() @ w[0].t()  # (numbers of at most 16 * 14: exact in any order)
    want[:5], want[-3:] = 9.0, 9.0
    assert torch.equal(y, want)
    assert m.get_last_error() == 0


@pytest.mark.parametrize("T,E,K", [(20000, 4, 4), (1 << 20, 3, 1), (1 << 17, 200, 128)])
def test_largest_experts(T, E, K):
    """The most tokens and slots: one value a token and an expert, exact all the way."""
    m, D = moe(), 16
    g = torch.Generator(device="cuda").manual_seed(T)
    d = m.dims(D, D, E, K, torch.float32)
    w1, v1, w2 = (torch.zeros((E, D, D), device="cuda") for _ in range(3))
    w1[:, 0, 0], v1[:, 0, 1], w2[:, 0, 0] = 64.0, 0.25, (torch.arange(E, device="cuda") % 7 + 1).float()
    ex = m.QuantExperts.quantize(w1, v1, w2)
    x = torch.zeros((T, D), device="cuda")
    x[:, 0] = 1.0
    x[:, 1] = (torch.randint(0, 8, (T,), device="cuda", generator=g) * 4).float()
    idx = torch.argsort(torch.rand((T, E), device="cuda", generator=g), dim=1)[:, :K].int()
    gate = torch.full((T, K), 0.5, device="cuda")
    got = m.quant_experts_forward(d, ex, x, idx, gate)
    assert m.get_last_error() == 0
    # SiLU(64) is 64 in 32 bits; h = 64 v, v below 8: a number of 8 bits; sums of at most 128 * 7 * 448 halves
    want = 0.5 * 64.0 * 0.25 * x[:, 1] * (idx % 7 + 1).sum(1)
    assert torch.equal(got[:, 0], want) and not got[:, 1:].any()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_largest_select(score):
    """1,048,576 tokens, keys a step of 1/16 apart."""
    m, T, E, K = moe(), 1 << 20, 16, 4
    g = torch.Generator(device="cuda").manual_seed(0)
    order = torch.argsort(torch.rand((T, E), device="cuda", generator=g), dim=1)
    logits = torch.empty((T, E), device="cuda").scatter_(1, order, (-torch.arange(E, device="cuda") / 16.0).expand(T, E))
    for bias in (None, torch.zeros(E, device="cuda")):
        idx, gate = m.route_select(m.dims(1024, 1024, E, K, torch.bfloat16), m.router(score), logits, bias)
        assert torch.equal(idx.long(), order[:, :K])
        p = -torch.arange(E, device="cuda").double() / 16
        s = (torch.softmax(p, 0) if score == "softmax" else torch.sigmoid(p))[:K]
        assert ((gate.double() - s / s.sum()).abs() <= 130 * 2.0 ** -23 * s).all()
    assert m.get_last_error() == 0


def test_calls_of_both_kernels_at_once():
    """Streamed calls and calls in tiles of 128 rows on four streams at once, launched and as graphs, each with
    a workspace of its own."""
    m, g = moe(), torch.Generator(device="cuda").manual_seed(3)
    E, K, D, F = 6, 2, 1024, 1536
    mk = lambda *s: torch.randn(s, device="cuda", generator=g) * 0.05
    ex = m.QuantExperts.quantize(mk(E, F, D), mk(E, F, D), mk(E, D, F))
    d, r = m.dims(D, F, E, K, torch.float32), m.router("sigmoid")
    w_r, sizes = mk(D, E), (1, 40, 300, 1000)
    xs = [mk(T, D) * 20 for T in sizes]
    wss = [m.quant_alloc_workspace(d, T) for T in sizes]
    want = [m.quant_layer_forward(d, ex, x, w_r, r, ws=ws) for x, ws in zip(xs, wss)]
    outs, streams = [torch.zeros_like(x) for x in xs], [torch.cuda.Stream() for _ in sizes]
    torch.cuda.synchronize()
    graphs = []
    for x, o, ws in zip(xs, outs, wss):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            m.quant_layer_forward(d, ex, x, w_r, r, out=o, ws=ws)
    for graphed in (False, True):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for x, o, ws, st, gr in zip(xs, outs, wss, streams, graphs):
                with torch.cuda.stream(st):
                    if graphed:
                        gr.replay()
                    else:
                        m.quant_layer_forward(d, ex, x, w_r, r, out=o, ws=ws)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)
    assert m.get_last_error() == 0
