"""8-bit experts on the GPU against plain 64-bit forms: quantisation bit for bit, the
choice of experts index for index, products and FFNs within the bounds that
tests/quant_ref.py derives."""
import numpy as np
import pytest
import torch

from tests import quant_ref as ref
from tests.gpu_util import need_gpu
from tests.paged_ref import encode

pytestmark = pytest.mark.gpu


def moe():
    need_gpu()
    from paper_2506_23635_gb300 import moe as m
    m.lib()
    return m


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def bits(t):
    return t.view(torch.uint8).cpu().numpy()


def num(t):
    return t.detach().cpu().double().numpy()


DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


# ---- quantisation ----------------------------------------------------------------


def _numbers(rng, shape, dtype):
    x = rng.normal(size=shape) * 2.0 ** rng.integers(-20, 20, shape[:-1] + (1,))
    x = torch.from_numpy(x.astype(np.float32)).to(DT[dtype])
    return x.cuda(), num(x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 128), (3, 144), (61, 6144), (500, 272), (2, 65536), (1500, 1488)])
def test_quantize_rows(rows, cols, dtype):
    m, rng = moe(), np.random.default_rng(rows + cols)
    x, x64 = _numbers(rng, (rows, cols), dtype)
    q, s = m.quantize_rows(x)
    wq, ws = ref.quantize_rows(x64)
    np.testing.assert_array_equal(num(s), ws)
    np.testing.assert_array_equal(bits(q) & np.where(wq == 0x80, 127, 255), wq & np.where(wq == 0x80, 127, 255))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_rows_edges(dtype):
    """Zeros, the scale's smallest and largest, amounts on a power of two's border,
    halves between two numbers, infinities and NaN: one block spoils no other."""
    m = moe()
    x = torch.zeros((12, 384), dtype=torch.float32)
    x[0, 130] = 448.0
    x[1, 130] = 449.0 if dtype == "f32" else 452.0
    x[2, 5] = 2.0 ** -120
    x[3, 5] = 3.3e38
    x[4, 200] = float("inf")
    x[5, 200] = float("-inf")
    x[6, 383] = float("nan")
    x[7, :128] = torch.arange(128) * 3.5
    x[8, :128] = torch.arange(-64, 64) * 0.0625 + 0.03125
    x[8, 0] = 448.0
    x[9, 128:256] = 2.0 ** -126
    x[10] = -448.0 * 2.0 ** -20
    x[11, :16] = torch.tensor([17., 18, 19, 20, 21, 22, 23, 24, 25, 26, 27, 28, 29, 30, 31, 448])
    x[4:7, 0] = 1.5
    x = x.to(DT[dtype])
    q, s = m.quantize_rows(x.cuda())
    with np.errstate(invalid="ignore"):
        wq, ws = ref.quantize_rows(num(x))
    np.testing.assert_array_equal(num(s), ws)
    np.testing.assert_array_equal(q.cpu().double().numpy(), ref.decode(wq))
    w = x.cuda().view(1, 12, 384)[:, :8].contiguous()
    q, s = m.quantize_blocks(w)
    with np.errstate(invalid="ignore"):
        wq, ws = ref.quantize_blocks(num(w))
    np.testing.assert_array_equal(num(s), ws)
    np.testing.assert_array_equal(q.cpu().double().numpy(), ref.decode(wq))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,rows,cols", [(1, 8, 16), (3, 128, 128), (2, 200, 144), (5, 392, 1040), (1, 1000, 2064)])
def test_quantize_blocks(n, rows, cols, dtype):
    m, rng = moe(), np.random.default_rng(rows + cols)
    w, w64 = _numbers(rng, (n, rows, cols), dtype)
    q, s = m.quantize_blocks(w)
    wq, ws = ref.quantize_blocks(w64)
    np.testing.assert_array_equal(num(s), ws)
    np.testing.assert_array_equal(q.cpu().double().numpy(), ref.decode(wq))


# ---- products --------------------------------------------------------------------


def _rows8(rng, S, n):
    q = encode(np.clip(rng.normal(size=(S, n)) * 100, -448, 448))
    return q, (rng.random((S, ref.blocks(n))) * 0.5 + 0.75).astype(np.float32) * np.float32(0.01)


def _matrices8(rng, E, rows, cols, std=0.02):
    q = encode(np.clip(rng.normal(size=(E, rows, cols)) * 100, -448, 448))
    s = rng.random((E, ref.blocks(rows), ref.blocks(cols))) * 0.5 + 0.75
    return q, (s * std / 100).astype(np.float32)


def e4m3(q):
    return torch.from_numpy(q).cuda().view(torch.float8_e4m3fn)


def check_product(m, rng, sizes, n_out, n_in, dtype, extra_rows=0, offsets=True):
    S, E = sum(sizes) + extra_rows, len(sizes)
    xq, xs = _rows8(rng, S, n_in)
    wq, ws = _matrices8(rng, E, n_out, n_in)
    ends = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    out = torch.full((S, n_out), 7.0, dtype=DT[dtype], device="cuda")
    m.quant_product(e4m3(xq), cuda(xs), e4m3(wq), cuda(ws), cuda(ends) if offsets else None,
                    DT[dtype], out=out)
    assert m.get_last_error() == 0
    got = num(out)
    assert (got[ends[-1]:] == 7.0).all()
    x = ref.rows64(xq, xs)
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        want, room = ref.product(x[a:b], ref.matrix64(wq[e], ws[e]))
        err = np.abs(got[a:b] - want)
        assert (err <= room + HALF_STEP[dtype] * (np.abs(want) + room) + 1e-30).all(), \
            (e, float((err - room).max(initial=0)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S", [1, 2, 15, 16, 17, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 300, 513, 700])
def test_product_one_group(S, dtype):
    check_product(moe(), np.random.default_rng(S), [S], 264, 400, dtype, offsets=False)


@pytest.mark.parametrize("n_out,n_in", [(8, 16), (8, 128), (128, 16), (128, 128), (136, 144), (256, 2048),
                                        (1000, 48), (264, 4112), (2048, 256)])
@pytest.mark.parametrize("S", [1, 40, 300])
def test_product_sizes(S, n_out, n_in):
    check_product(moe(), np.random.default_rng(S + n_out), [S], n_out, n_in, "f32", offsets=False)


@pytest.mark.parametrize("sizes", [[0, 300, 1, 77, 0, 129, 5, 265], [0, 0, 0], [1] * 40, [0, 0, 1], [513, 0, 0, 64],
                                   [128, 256, 384, 17]], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_product_groups(sizes, dtype):
    """Groups of all sizes; rows behind the last group stay as they were."""
    check_product(moe(), np.random.default_rng(len(sizes)), sizes, 392, 656, dtype, extra_rows=3)


def test_product_many_groups():
    rng = np.random.default_rng(0)
    sizes = [int(v) for v in rng.integers(0, 6, 256)]
    check_product(moe(), rng, sizes, 72, 160, "f32", extra_rows=1)


@pytest.mark.parametrize("n_out", [8, 264, 520, 776, 1288])
@pytest.mark.parametrize("sizes", [[128, 129, 1, 256, 257, 384, 385, 0, 70, 640], [65, 66, 64], [40] * 48], ids=str)
def test_product_runs(sizes, n_out):
    """Last runs of up to 128 rows, whose weight tiles go two by two, an odd one by itself."""
    check_product(moe(), np.random.default_rng(n_out), sizes, n_out, 272, "f32", extra_rows=2)


def test_product_bad_offsets():
    """Offsets that fall or leave [0, S]: their groups are left out and recorded."""
    m, rng = moe(), np.random.default_rng(5)
    xq, xs = _rows8(rng, 40, 144)
    wq, ws = _matrices8(rng, 4, 136, 144)
    out = torch.full((40, 136), 7.0, device="cuda")
    off = cuda(np.array([0, 10, 5, 20, 100], np.int32))
    m.quant_product(e4m3(xq), cuda(xs), e4m3(wq), cuda(ws), off, torch.float32, out=out)
    assert m.get_last_error() == 6
    got = num(out)
    x = ref.rows64(xq, xs)
    # group 1 falls, group 3 leaves; rows 5..9 are both group 0's and group 2's
    for g, a, b in ((0, 0, 5), (2, 10, 20)):
        want, room = ref.product(x[a:b], ref.matrix64(wq[g], ws[g]))
        assert (np.abs(got[a:b] - want) <= room + 2.0 ** -24 * np.abs(want)).all()
    assert (got[20:] == 7.0).all()


def test_product_nan_and_infinite_scales_stay_in_their_rows():
    m, rng = moe(), np.random.default_rng(6)
    for S in (20, 300):
        xq, xs = _rows8(rng, S, 400)
        wq, ws = _matrices8(rng, 1, 264, 400)
        xq[3, 7] = 0x7f
        xs[5, 1] = np.nan
        xs[9, 2] = np.inf
        ws[0, 1, 2] = 0.0
        y = num(m.quant_product(e4m3(xq), cuda(xs), e4m3(wq), cuda(ws), None, torch.float32))
        assert np.isnan(y[3]).all() and np.isnan(y[5]).all() and not np.isfinite(y[9]).any()
        rest = [i for i in range(S) if i not in (3, 5, 9)]
        want, room = ref.product(ref.rows64(xq, xs)[rest], ref.matrix64(wq[0], ws[0]))
        assert (np.abs(y[rest] - want) <= room + 2.0 ** -24 * np.abs(want)).all()


# ---- the choice of experts ---------------------------------------------------------


def check_select(m, logits, bias, K, atol=2.0 ** -20, **kw):
    T, E = logits.shape
    d = m.dims(1024, 1024, E, K, torch.bfloat16)
    names = dict(renormalise=True, scale=1.0)
    names.update(kw)
    r = m.router(**names)
    idx, gate = m.route_select(d, r, cuda(logits.astype(np.float32)),
                               None if bias is None else cuda(bias.astype(np.float32)))
    assert m.get_last_error() == 0
    wi, wg = ref.select(logits.astype(np.float32), None if bias is None else bias.astype(np.float32), K, **names)
    np.testing.assert_array_equal(idx.cpu().numpy(), wi)
    g = num(gate)
    np.testing.assert_array_equal(np.isnan(g), np.isnan(wg))
    # a score in 32 bits is off by (24 + |d|) 2^-24 of itself at most, d <= 104 where it is
    # not zero, and so is each of the sum; what is below the numbers of 32 bits by their step
    rel = 2 * 130 * 2.0 ** -24
    ok = ~np.isnan(wg)
    assert (np.abs(g - wg)[ok] <= rel * np.abs(wg)[ok] + 2.0 ** -140 * abs(names["scale"])).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("E,K,G,kept,best", [(1, 1, 1, 1, 1), (8, 2, 1, 1, 1), (16, 4, 1, 1, 1), (16, 16, 1, 1, 1),
                                             (33, 7, 1, 1, 1), (60, 6, 4, 2, 2), (64, 8, 8, 4, 1), (100, 40, 10, 5, 2),
                                             (160, 6, 8, 3, 1), (256, 8, 8, 4, 2), (256, 256, 1, 1, 1),
                                             (256, 3, 128, 2, 2), (255, 5, 51, 3, 1), (200, 4, 200, 9, 1)])
@pytest.mark.parametrize("T", [1, 37])
def test_select(T, E, K, G, kept, best, bias, score):
    rng = np.random.default_rng(E + K + T)
    logits = rng.normal(size=(T, E)) * 1.57
    b = rng.normal(size=E) * 0.05 if bias else None
    check_select(moe(), logits, b, K, score=score, n_groups=G, top_groups=kept, group_top=best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,kept,best", [(1, 1, 1), (8, 3, 2), (8, 3, 1)])
def test_select_many_tokens(score, G, kept, best):
    """Enough tokens that keys lie nearer to each other than 32 bits tell."""
    rng = np.random.default_rng(9)
    logits, bias = rng.normal(size=(6000, 64)) * 1.57, rng.normal(size=64) * 0.05
    check_select(moe(), logits, bias, 6, score=score, n_groups=G, top_groups=kept, group_top=best, scale=2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,kept,best", [(1, 1, 1), (4, 2, 2), (4, 2, 1)])
@pytest.mark.parametrize("with_bias", ["none", "zero", "steps"])
def test_select_ties(score, G, kept, best, with_bias):
    """Logits of a few values only, so that most keys have equals: the lower index wins;
    and sums that 32 bits would round together."""
    rng = np.random.default_rng(10)
    logits = rng.integers(-2, 3, size=(300, 48)) * 0.5
    logits[:20] = 0.0
    logits[20:40] += rng.integers(0, 2, size=(20, 48)) * 2.0 ** -22
    bias = {"none": None, "zero": np.zeros(48), "steps": rng.integers(0, 3, 48) * 2.0 ** -24}[with_bias]
    check_select(moe(), logits, bias, 7, score=score, n_groups=G, top_groups=kept, group_top=best)


@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,best", [(1, 1), (4, 2), (4, 1)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_select_not_finite_and_far(score, renormalise, G, best, with_bias):
    """NaN and infinite logits, rows without a finite one, logits so low that 32 bits
    hold no score, biases of minus infinity."""
    rng = np.random.default_rng(11)
    logits = rng.normal(size=(16, 16))
    logits[0, 3] = np.nan
    logits[1, 2:9] = -np.inf
    logits[2, :] = -np.inf
    logits[3, :] = np.nan
    logits[4, 7] = np.inf
    logits[5, :] = -120 - np.arange(16)
    logits[6, :] = 80 + np.arange(16)
    logits[7, :] *= 3e38
    logits[8, 0] = -0.0
    logits[8, 1:] = 0.0
    logits[9, :] = 1e-38 * np.arange(16)
    bias = None
    if with_bias:
        bias = rng.normal(size=16) * 0.1
        bias[5] = -np.inf
        bias[6] = np.nan
    check_select(moe(), logits, bias, 4, score=score, n_groups=G, top_groups=max(1, G // 2), group_top=best,
                 renormalise=renormalise)


# ---- the experts and the layer --------------------------------------------------------


def _experts(m, rng, E, F, D):
    w = [_matrices8(rng, E, F, D), _matrices8(rng, E, F, D), _matrices8(rng, E, D, F, 0.05)]
    dev = [t for q, s in w for t in (e4m3(q), cuda(s))]
    return m.QuantExperts(*dev), [np.stack([ref.matrix64(q[e], s[e]) for e in range(E)]) for q, s in w]


def _routing(rng, T, E, K):
    idx = np.argsort(rng.random((T, E)) + 0.3 * rng.random(E), axis=1)[:, :K].astype(np.int32)
    g = rng.random((T, K)).astype(np.float32)
    return idx, g / g.sum(1, keepdims=True)


def check_experts(got, x64, idx, gate, w, out_dtype, residual=None):
    x8 = ref.rows64(*ref.quantize_rows(x64))
    want, room = ref.experts(x8, idx, gate, *w, residual=residual)
    err = np.abs(got - want)
    lim = room + HALF_STEP[out_dtype] * (np.abs(want) + room) + 1e-30
    assert (err <= lim).all(), float((err - lim).max())
    return want


@pytest.mark.parametrize("x_dtype,out_dtype,res", [("bf16", "bf16", False), ("f32", "f32", True), ("bf16", "f32", True),
                                                   ("f32", "bf16", False)])
@pytest.mark.parametrize("T,E,K,D,F", [(1, 4, 2, 256, 384), (1, 1, 1, 16, 16), (3, 5, 5, 144, 272), (9, 8, 2, 400, 208),
                                       (20, 8, 3, 512, 640), (50, 6, 2, 272, 400), (70, 10, 3, 720, 400),
                                       (300, 12, 4, 336, 464), (700, 3, 2, 272, 528), (2, 200, 9, 128, 128)])
def test_experts(T, E, K, D, F, x_dtype, out_dtype, res):
    m, rng = moe(), np.random.default_rng(T + E + D)
    ex, w = _experts(m, rng, E, F, D)
    d = m.dims(D, F, E, K, DT[x_dtype], out_dtype=DT[out_dtype])
    x = torch.from_numpy(rng.normal(size=(T, D)).astype(np.float32)).to(DT[x_dtype])
    r = torch.from_numpy(rng.normal(size=(T, D)).astype(np.float32)).to(DT[out_dtype]) if res else None
    idx, gate = _routing(rng, T, E, K)
    got = m.quant_experts_forward(d, ex, x.cuda(), cuda(idx), cuda(gate), r.cuda() if res else None)
    assert m.get_last_error() == 0
    check_experts(num(got), num(x), idx, gate, w, out_dtype, num(r) if res else None)


@pytest.mark.parametrize("D,F", [(528, 640), (256, 128), (400, 272)])
@pytest.mark.parametrize("T", [130, 250, 500])
def test_experts_runs(T, D, F):
    m, rng = moe(), np.random.default_rng(T + D)
    d = m.dims(D, F, 3, 2, torch.float32)
    ex, w = _experts(m, rng, 3, F, D)
    idx, gate = _routing(rng, T, 3, 2)
    x = rng.normal(size=(T, D)).astype(np.float32)
    got = m.quant_experts_forward(d, ex, cuda(x), cuda(idx), cuda(gate))
    assert m.get_last_error() == 0
    check_experts(num(got), x.astype(np.float64), idx, gate, w, "f32")


def test_experts_same_expert_twice_and_out_of_range():
    """A token may name an expert twice; an index outside [0, E) is recorded and left out."""
    m, rng = moe(), np.random.default_rng(3)
    ex, w = _experts(m, rng, 4, 272, 144)
    d = m.dims(144, 272, 4, 3, torch.float32)
    x = rng.normal(size=(30, 144)).astype(np.float32)
    idx, gate = _routing(rng, 30, 4, 3)
    idx[:, 1] = idx[:, 0]
    check_experts(num(m.quant_experts_forward(d, ex, cuda(x), cuda(idx), cuda(gate))), x, idx, gate, w, "f32")
    assert m.get_last_error() == 0
    idx[4, 2], idx[7, 0], idx[29] = -1, 4, 1 << 30
    check_experts(num(m.quant_experts_forward(d, ex, cuda(x), cuda(idx), cuda(gate))), x, idx, gate, w, "f32")
    assert m.get_last_error() == 6


def test_experts_one_expert_for_all():
    m, rng = moe(), np.random.default_rng(4)
    ex, w = _experts(m, rng, 8, 272, 256)
    d = m.dims(256, 272, 8, 1, torch.float32)
    for T in (5, 90, 400):
        x = rng.normal(size=(T, 256)).astype(np.float32)
        idx, gate = np.full((T, 1), 5, np.int32), np.ones((T, 1), np.float32)
        check_experts(num(m.quant_experts_forward(d, ex, cuda(x), cuda(idx), cuda(gate))), x, idx, gate, w, "f32")


def test_experts_bad_tokens_stay_to_themselves():
    """Zeros, NaN and infinite tokens: the others' rows are the bits they were."""
    m, rng = moe(), np.random.default_rng(8)
    ex, w = _experts(m, rng, 4, 272, 256)
    d = m.dims(256, 272, 4, 2, torch.float32)
    for T in (12, 200):
        x = rng.normal(size=(T, 256)).astype(np.float32)
        idx, gate = _routing(rng, T, 4, 2)
        before = num(m.quant_experts_forward(d, ex, cuda(x), cuda(idx), cuda(gate)))
        y = x.copy()
        y[2], y[5, 9], y[7, 200], y[9] = 0.0, np.nan, np.inf, -np.inf
        after = num(m.quant_experts_forward(d, ex, cuda(y), cuda(idx), cuda(gate)))
        assert (after[2] == 0).all() and np.isnan(after[[5, 7, 9]]).all()
        rest = [i for i in range(T) if i not in (2, 5, 7, 9)]
        np.testing.assert_array_equal(after[rest], before[rest])


@pytest.mark.parametrize("T,E,K", [(1, 16, 4), (7, 16, 4), (40, 16, 4), (150, 16, 4), (33, 64, 6)])
@pytest.mark.parametrize("kind", ["plain", "sigmoid", "groups"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer(T, E, K, kind, dtype):
    """Routing, experts and residual in one call, against its own steps bit for bit, whose
    results the tests above hold to the plain forms."""
    m, rng = moe(), np.random.default_rng(T + E)
    D, F = 256, 272
    ex, w = _experts(m, rng, E, F, D)
    d = m.dims(D, F, E, K, DT[dtype])
    x = torch.from_numpy(rng.normal(size=(T, D)).astype(np.float32)).to(DT[dtype]).cuda()
    w_r = torch.from_numpy((rng.normal(size=(D, E)) * 0.1).astype(np.float32)).to(DT[dtype]).cuda()
    res = torch.from_numpy(rng.normal(size=(T, D)).astype(np.float32)).to(DT[dtype]).cuda()
    idx, gate, logits = m.route(d, x, w_r, want_logits=True)
    router = bias = None
    if kind != "plain":
        bias = cuda((rng.normal(size=E) * 0.05).astype(np.float32))
        router = m.router("sigmoid", 4 if kind == "groups" else 1, 2 if kind == "groups" else 1, 2, True, 1.5)
        idx, gate = m.route_select(d, router, logits, bias)
    want = m.quant_experts_forward(d, ex, x, idx, gate, res)
    got = m.quant_layer_forward(d, ex, x, w_r, router, bias, res)
    assert m.get_last_error() == 0
    if kind == "plain":  # (the router's one-launch forms may differ in a gate's last bit)
        check_experts(num(got), num(x), idx.cpu().numpy(), num(gate), w, dtype, num(res))
    else:
        np.testing.assert_array_equal(num(got), num(want))
    inplace = res.clone()
    m.quant_layer_forward(d, ex, x, w_r, router, bias, inplace, out=inplace)
    np.testing.assert_array_equal(num(inplace), num(got))


def test_quantized_layer_is_near_the_layer():
    """Weights and activations rounded to 8 bits move the bf16 layer's output by about the
    roundings' size: 2^-4 of a number at most, half of that in the mean square, three
    times in a row (x and w1/v1; h and w2), independent."""
    m, rng = moe(), np.random.default_rng(2)
    D, F, E, K, T = 512, 768, 8, 2, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda *s: (torch.randn(s, device="cuda", generator=g) * 0.05).bfloat16()
    w1, v1, w2, w_r = mk(E, F, D), mk(E, F, D), mk(E, D, F), mk(D, E)
    x = torch.randn((T, D), device="cuda", generator=g).bfloat16()
    d = m.dims(D, F, E, K, torch.bfloat16, out_dtype=torch.float32)
    want = num(m.layer_forward(d, x, w_r, w1, v1, w2))
    got = num(m.quant_layer_forward(d, m.QuantExperts.quantize(w1, v1, w2), x, w_r))
    rel = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert 1e-3 < rel < 6 * 2.0 ** -5


# ---- streams, graphs, workspaces ------------------------------------------------------


@pytest.mark.parametrize("T", [1, 24, 200])
def test_same_bits_again_and_in_graphs(T):
    """The same call twice, on another stream, and captured twice into graphs that share a
    workspace; a workspace of any contents."""
    m, rng = moe(), np.random.default_rng(T)
    D, F, E, K = 512, 656, 8, 2
    ex, _ = _experts(m, rng, E, F, D)
    d = m.dims(D, F, E, K, torch.bfloat16)
    x = torch.from_numpy(rng.normal(size=(T, D)).astype(np.float32)).bfloat16().cuda()
    w_r = torch.from_numpy((rng.normal(size=(D, E)) * 0.1).astype(np.float32)).bfloat16().cuda()
    r = m.router("sigmoid")
    ws = m.quant_alloc_workspace(d, T)
    ws.fill_(0xff)
    first = num(m.quant_layer_forward(d, ex, x, w_r, r, ws=ws))
    ws.random_(0, 256)
    np.testing.assert_array_equal(num(m.quant_layer_forward(d, ex, x, w_r, r, ws=ws)), first)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    out = m.quant_layer_forward(d, ex, x, w_r, r, stream=st)
    st.synchronize()
    np.testing.assert_array_equal(num(out), first)
    outs = [torch.zeros((T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, o in zip(graphs, outs):
        with torch.cuda.graph(g):
            m.quant_layer_forward(d, ex, x, w_r, r, out=o, ws=ws)
    for g in graphs + graphs:
        g.replay()
    torch.cuda.synchronize()
    for o in outs:
        np.testing.assert_array_equal(num(o), first)
    y = x * 2
    x.copy_(y)
    graphs[0].replay()
    torch.cuda.synchronize()
    np.testing.assert_array_equal(num(outs[0]), num(m.quant_layer_forward(d, ex, x, w_r, r, ws=ws)))
    assert m.get_last_error() == 0


def test_product_twice_on_two_streams():
    """Calls at the same time with workspaces of their own."""
    m, rng = moe(), np.random.default_rng(12)
    xq, xs = _rows8(rng, 5, 4096)
    wq, ws = _matrices8(rng, 1, 1024, 4096)
    args = (e4m3(xq), cuda(xs), e4m3(wq), cuda(ws), None, torch.float32)
    want = num(m.quant_product(*args))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [m.quant_product(*args, stream=s) for s in streams for _ in range(4)]
    torch.cuda.synchronize()
    for o in outs:
        np.testing.assert_array_equal(num(o), want)


def test_empty_calls():
    m = moe()
    d = m.dims(256, 272, 4, 2, torch.bfloat16)
    rng = np.random.default_rng(0)
    ex, _ = _experts(m, rng, 4, 272, 256)
    e = lambda *s, t=torch.float32: torch.empty(s, dtype=t, device="cuda")
    bf = torch.bfloat16
    assert m.quant_experts_forward(d, ex, e(0, 256, t=bf), e(0, 2, t=torch.int32), e(0, 2)).shape == (0, 256)
    assert m.quant_layer_forward(d, ex, e(0, 256, t=bf), e(256, 4, t=bf)).shape == (0, 256)
    assert m.route_select(d, m.router(), e(0, 4))[0].shape == (0, 2)
    assert m.quantize_rows(e(0, 128))[1].shape == (0, 1)
    q, s = m.quantize_blocks(e(1, 128, 256))
    assert m.quant_product(e(0, 256, t=torch.float8_e4m3fn), e(0, 2), q, s).shape == (0, 128)
    assert m.get_last_error() == 0


# ---- the launch directly ahead ----------------------------------------------------------


def _behind(m, zero, write, fn):
    """fn() right behind write(), whose kernel lets the next launch start before it has
    written, gives what it gives once everything is there."""
    write()
    torch.cuda.synchronize()
    want = fn().clone()
    for _ in range(8):
        zero.view(torch.uint8).zero_()
        torch.cuda.synchronize()
        write()
        got = fn()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    assert m.get_last_error() == 0


@pytest.mark.parametrize("S", [1, 40, 400])
def test_product_weights_and_rows_written_just_ahead(S):
    m, g = moe(), torch.Generator(device="cuda").manual_seed(S)
    n_out, n_in = 4096, 4096
    src = torch.randn((n_out, n_in), device="cuda", generator=g)
    q, s = m.quantize_rows(src)
    ws = torch.rand((1, 32, 32), device="cuda", generator=g)
    x, xs = m.quantize_rows(torch.randn((S, n_in), device="cuda", generator=g))
    out, sp = torch.empty((S, n_out), device="cuda"), m.quant_product_alloc_workspace(1, n_out, n_in, S)
    run = lambda: m.quant_product(x, xs, q.view(1, n_out, n_in), ws, None, torch.float32, out=out, ws=sp)
    _behind(m, q, lambda: m.quantize_rows(src, q, s), run)
    rows = torch.randn((S, n_in), device="cuda", generator=g)
    _behind(m, x, lambda: m.quantize_rows(rows, x, xs), run)


@pytest.mark.parametrize("T", [1, 40, 300])
def test_experts_inputs_written_just_ahead(T):
    """The choice, the down projection's weights and the tokens."""
    m, g = moe(), torch.Generator(device="cuda").manual_seed(T)
    E, K, D, F = 8, 2, 1024, 2048
    mk = lambda *s: torch.randn(s, device="cuda", generator=g) * 0.05
    ex = m.QuantExperts.quantize(mk(E, F, D), mk(E, F, D), mk(E, D, F))
    d = m.dims(D, F, E, K, torch.float32)
    x, logits, bias = mk(T, D) * 20, mk(T, E) * 20, mk(E)
    idx, gate = m.route_select(d, m.router("sigmoid"), logits, bias)
    out, ws = torch.empty_like(x), m.quant_alloc_workspace(d, T)
    run = lambda: m.quant_experts_forward(d, ex, x, idx, gate, out=out, ws=ws)
    _behind(m, gate, lambda: m.route_select(d, m.router("sigmoid"), logits, bias, idx, gate), run)
    w2, src = ex.tensors[2], mk(E * D, F)
    s = m.quantize_rows(src)[1]
    _behind(m, w2, lambda: m.quantize_rows(src, w2.view(E * D, F), s), run)
    inner = m.dims(D, F, E, K, torch.float32)
    _behind(m, x, lambda: m.quant_experts_forward(inner, ex, logits.new_ones((T, D)), idx, gate, out=x), run)


@pytest.mark.parametrize("T", [1, 16, 65, 300])
def test_calls_back_to_back_share_a_workspace(T):
    """Calls of different sizes behind each other on one stream, over one workspace."""
    m, rng = moe(), np.random.default_rng(T)
    D, F, E, K = 512, 656, 8, 2
    ex, _ = _experts(m, rng, E, F, D)
    d = m.dims(D, F, E, K, torch.bfloat16)
    ws = m.quant_alloc_workspace(d, 400)
    sizes = [T, 1, 400, 7, T, 33, 200, T]
    x = torch.from_numpy(rng.normal(size=(400, D)).astype(np.float32)).bfloat16().cuda()
    idx, gate = (cuda(a) for a in _routing(rng, 400, E, K))
    want = []
    for n in sizes:
        want.append(m.quant_experts_forward(d, ex, x[:n], idx[:n], gate[:n]))
        torch.cuda.synchronize()
    got = [m.quant_experts_forward(d, ex, x[:n], idx[:n], gate[:n], ws=ws) for n in sizes]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert m.get_last_error() == 0


def test_large_offsets():
    """Weights of more than 2^31 bytes, and rows whose outputs lie past 2^31 bytes."""
    m, rng = moe(), np.random.default_rng(1)
    E, n_out, n_in = 9, 16384, 16384
    wq = torch.zeros((E, n_out, n_in), dtype=torch.uint8, device="cuda")
    part, s = _matrices8(rng, 1, 256, n_in)
    wq[E - 1, -256:] = torch.from_numpy(part[0]).cuda()
    ws = torch.ones((E, 128, 128), device="cuda")
    xq, xs = _rows8(rng, 3, n_in)
    off = cuda(np.array([0] * E + [3], np.int32))
    y = num(m.quant_product(e4m3(xq), cuda(xs), wq.view(torch.float8_e4m3fn), ws, off, torch.float32))
    want, room = ref.product(ref.rows64(xq, xs), ref.decode(part[0]))
    assert (np.abs(y[:, -256:] - want) <= room + 2.0 ** -24 * np.abs(want)).all() and (y[:, :-256] == 0).all()
    del wq, ws
    S, n_out, n_in = 40000, 16384, 128
    wq, s = _matrices8(rng, 1, n_out, n_in)
    x = torch.zeros((S, n_in), dtype=torch.uint8, device="cuda")
    xq, xs1 = _rows8(rng, 300, n_in)
    x[-300:] = torch.from_numpy(xq).cuda()
    xs = torch.ones((S, 1), device="cuda")
    xs[-300:] = cuda(xs1)
    y = m.quant_product(x.view(torch.float8_e4m3fn), xs, e4m3(wq), cuda(s), None, torch.float32)
    want, room = ref.product(ref.rows64(xq, xs1), ref.matrix64(wq[0], s[0]))
    got = num(y[-300:])
    assert (np.abs(got - want) <= room + 2.0 ** -24 * np.abs(want)).all()
    assert not y[:-300].any()
    assert m.get_last_error() == 0
