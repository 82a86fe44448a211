"""The attention block and whole decoder layers over the paged 8-bit cache.

The attention is compared over the cache that the call itself has left (its rows
against the projection within e4m3's half step), everything else with the
oracle's formulas and the bounds of the block over the bf16 caches."""
import numpy as np
import pytest
import torch

import oracle
from paper_2506_23635_gb300 import inputs as gen
from tests import paged_ref as ref
from tests.gpu_util import assert_parity, dev, need_gpu, to_numpy

pytestmark = pytest.mark.gpu

EPS = 1e-6


def moe():
    need_gpu()
    from paper_2506_23635_gb300 import moe as m
    return m


def _cache(m, c):
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return m.PagedCache(up(c["k"]).view(torch.float8_e4m3fn), up(c["v"]).view(torch.float8_e4m3fn),
                        up(c["ks"]), up(c["vs"]), up(c["table"]))


def _host(cache):
    return (cache.k_pages.view(torch.uint8).cpu().numpy(), cache.v_pages.view(torch.uint8).cpu().numpy(),
            cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy())


def _block(c, x, w_qkv, w_o, cache):
    """The block on the residual stream x (64 bits), the attention over `cache`
    as it is after the call; the call's keys and values, and where they lie."""
    hq, hkv = c["hq"], c["hkv"]
    T = len(x)
    xn = oracle.round_bf16(oracle.rmsnorm0(np.ascontiguousarray(x), EPS))
    proj = (xn @ gen.to_f64(w_qkv, "bf16").T).reshape(T, hq + 2 * hkv, 128)
    turned = oracle.rope(np.ascontiguousarray(proj[:, :hq + hkv]), np.maximum(c["pos"], 0), c["base"])
    q = oracle.round_bf16(np.ascontiguousarray(turned[:, :hq]))
    ctx, _ = ref.attend(c, q, *cache)
    ctx = oracle.round_bf16(ctx.reshape(T, -1))
    return x + ctx @ gen.to_f64(w_o, "bf16").T, turned[:, hq:], proj[:, hq + hkv:]


def _check_rows(c, keys, values, cache):
    k, v, ks, vs = cache
    for t in range(len(c["seq"])):
        if not ref.inside(c, t):
            continue
        s, p = int(c["seq"][t]), int(c["pos"][t])
        pg, off = ref.page_of(c, s, p), p % c["page"]
        for b, sc, want, what in ((k, ks, keys[t], "key"), (v, vs, values[t], "value")):
            scale = sc[pg].astype(np.float64)[:, None]
            got = ref.decode(b[pg, :, off]) * scale
            # half a step, and 2e-2 of the rows' RMS as the projections' bound
            lim = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * scale) + \
                2e-2 * np.sqrt(np.mean(want * want))
            assert np.all(np.abs(got - want) <= lim), (what, t)


CASES = [
    (256, 4, 2, 16, [(0, 40, 1)], 0),
    (512, 4, 4, 64, [(i, 37 * i, 1) for i in range(7)], 3),
    (768, 6, 1, 32, [(0, 0, 70)], 0),
    (1024, 8, 1, 128, [(0, 100, 200), (1, 3, 1), (2, 900, 1)], 2),
    (384, 3, 1, 16, [(0, 17, 300), (1, 0, 205)] + [(2 + i, 50 * i, 1) for i in range(20)], 5),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"D{c[0]}Hq{c[1]}Hkv{c[2]}page{c[3]}")
def test_block(case):
    m = moe()
    D, hq, hkv, page, runs, pad = case
    c = ref.call(hq, hkv, page, runs, seed=D, pad=pad)
    shape = gen.AttnShape(D, hq, hkv, 128, c["base"], "bf16")
    w_qkv, w_o = gen.host_attn_weights(shape, 5)
    cache = _cache(m, c)
    T = len(c["seq"])
    x = (c["rng"].normal(size=(T, D)) * 2.0).astype(np.float32)
    resid = torch.from_numpy(x).cuda()
    a = m.sa_dims(D, hq, hkv, 128, c["base"])
    seq, pos = torch.from_numpy(c["seq"]).cuda(), torch.from_numpy(c["pos"]).cuda()
    m.paged_sa_forward(a, cache, resid, dev(w_qkv, "bf16"), dev(w_o, "bf16"), seq, pos, eps=EPS)
    assert m.get_last_error() == 0
    want, keys, values = _block(c, x.astype(np.float64), w_qkv, w_o, _host(cache))
    _check_rows(c, keys, values, _host(cache))
    got = to_numpy(resid)
    n = T - pad
    assert_parity(got[:n] - x[:n], want[:n] - x[:n], "bf16", "attention block update")
    np.testing.assert_array_equal(got[n:], x[n:])


def test_block_of_dbrx_shape():
    """600 tokens of DBRX's projections (equal shares of their k-blocks, a row in
    one or two parts), then one decode step."""
    m = moe()
    c = ref.call(48, 8, 64, [(0, 0, 600)], seed=7, max_pages=12)
    c["base"] = 500000.0
    c["table"][0, 10] = (set(range(c["n_pages"])) - set(c["table"][0, :10])).pop()
    shape = gen.AttnShape(6144, 48, 8, 128, 500000.0, "bf16")
    w_qkv, w_o = gen.host_attn_weights(shape, 6)
    cache = _cache(m, c)
    a = m.sa_dims(6144, 48, 8)
    d_qkv, d_o = dev(w_qkv, "bf16"), dev(w_o, "bf16")
    for seq, pos in ((np.zeros(600, np.int32), np.arange(600, dtype=np.int32)),
                     (np.zeros(1, np.int32), np.full(1, 600, np.int32))):
        x = c["rng"].normal(size=(len(seq), 6144)).astype(np.float32)
        resid = torch.from_numpy(x).cuda()
        m.paged_sa_forward(a, cache, resid, d_qkv, d_o, torch.from_numpy(seq).cuda(),
                           torch.from_numpy(pos).cuda(), eps=EPS)
        assert m.get_last_error() == 0
        s = dict(c, seq=seq, pos=pos)
        want, keys, values = _block(s, x.astype(np.float64), w_qkv, w_o, _host(cache))
        _check_rows(s, keys, values, _host(cache))
        assert_parity(to_numpy(resid) - x, want - x, "bf16", "attention block update")


@pytest.mark.parametrize("runs", [[(i, 9 * i, 1) for i in range(5)], [(0, 0, 60), (1, 20, 1)]],
                         ids=["decode", "prompt"])
def test_decoder_layers(runs):
    """Two decoder layers; tokens whose routing is a near tie are left out."""
    m = moe()
    n_layers, page = 2, 16
    c = ref.call(4, 2, page, runs, seed=9, pad=2)
    T = len(c["seq"])
    sa = gen.AttnShape(256, 4, 2, 128, c["base"], "bf16")
    layer = gen.LayerShape(256, 512, 8, 2, "bf16")
    weights, layers = [], []
    for l in range(n_layers):
        w_qkv, w_o = gen.host_attn_weights(sa, 17, l)
        w_r = gen.host_normal((256, 8), gen.W_STD, "bf16", 17, "dec-w_r", l)
        weights.append((w_qkv, w_o, w_r) + tuple(gen.host_expert_weights(layer, 117 + 100 * l)))
        layers.append(tuple(dev(t, "bf16") for t in weights[-1]) + (_cache(m, c),))
    W = m.PagedDecoderWeights(layers)
    a = m.sa_dims(256, 4, 2, 128, c["base"])
    d = m.dims(256, 512, 8, 2, torch.bfloat16, torch.bfloat16, torch.float32)
    seq, pos = torch.from_numpy(c["seq"]).cuda(), torch.from_numpy(c["pos"]).cuda()
    x = c["rng"].normal(size=(T, 256)).astype(np.float32)
    resid = torch.from_numpy(x).cuda()
    ws = torch.empty(m.paged_decoder_workspace_size(a, d, T), dtype=torch.uint8, device="cuda")
    m.paged_decoder_forward(a, d, W, resid, seq, pos, eps=EPS, ws=ws)
    assert m.get_last_error() == 0
    want, gaps = x.astype(np.float64), []
    for l in range(n_layers):
        want, keys, values = _block(c, want, *weights[l][:2], _host(layers[l][6]))
        _check_rows(c, keys, values, _host(layers[l][6]))
        want, g = oracle.moe_block(want, weights[l][2:], "bf16", 2, EPS)
        gaps.append(g)
    ok = np.all(np.array(gaps) >= 0.02, axis=0)
    assert ok.sum() >= (3 * T) // 4
    got = to_numpy(resid)
    rel = np.linalg.norm((got - want)[ok]) / np.linalg.norm((want - x)[ok])
    assert rel <= 5e-3 * np.sqrt(n_layers), f"rel L2 of the update {rel:.3e}"
    # captured and replayed: the same bits (the cache holds the same rows already)
    g = torch.cuda.CUDAGraph()
    again = torch.from_numpy(x).cuda()
    with torch.cuda.graph(g):
        m.paged_decoder_forward(a, d, W, again, seq, pos, eps=EPS, ws=ws)
    for _ in range(2):
        again.copy_(torch.from_numpy(x))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, resid)
    assert m.get_last_error() == 0


def test_refusals_of_the_block():
    m = moe()
    c = ref.call(4, 2, 16, [(0, 0, 3)], seed=10)
    cache = _cache(m, c)
    a = m.sa_dims(256, 4, 2)
    seq, pos = torch.from_numpy(c["seq"]).cuda(), torch.from_numpy(c["pos"]).cuda()
    resid = torch.zeros((3, 256), device="cuda")
    w_qkv = torch.zeros((1024, 256), dtype=torch.bfloat16, device="cuda")
    w_o = torch.zeros((256, 512), dtype=torch.bfloat16, device="cuda")
    f = lambda **kw: m.paged_sa_forward(**{**dict(a=a, cache=cache, resid=resid, w_qkv=w_qkv,
                                                  w_o=w_o, seq=seq, pos=pos), **kw})
    f()
    for kw in (dict(resid=resid.bfloat16()), dict(w_qkv=w_qkv[:512]), dict(w_o=w_qkv),
               dict(seq=seq.long()), dict(pos=pos[:2]), dict(a=m.sa_dims(256, 8, 4))):
        with pytest.raises(ValueError):
            f(**kw)
    with pytest.raises(m.MoeError):
        f(eps=0.0)
    with pytest.raises(m.MoeError):
        f(ws=torch.empty(1024, dtype=torch.uint8, device="cuda"))
    none = seq[:0]
    f(resid=resid[:0], seq=none, pos=none)
    assert m.get_last_error() == 0
