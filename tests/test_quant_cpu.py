"""8-bit experts on the CPU: the plain 64-bit forms against torch and brute force, and what
the entry points refuse before anything is launched."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

from paper_2506_23635_gb300 import build as moe_build
from tests import quant_ref as ref

no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                            reason="placeholder addresses only where no GPU exists")
A = ctypes.c_void_p(0x10000)
MIS = ctypes.c_void_p(0x10004)


@pytest.fixture(scope="module")
def lib():
    moe_build.build()
    from paper_2506_23635_gb300 import moe
    return moe


# ---- the plain forms -------------------------------------------------------------------


def test_rows_are_torchs_roundings():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(7, 300)) * 2.0 ** rng.integers(-30, 30, (7, 1))
    q, s = ref.quantize_rows(x.astype(np.float32))
    for r, b in itertools.product(range(7), range(3)):
        part = torch.from_numpy(x[r, b * 128:(b + 1) * 128].astype(np.float32))
        one = float(s[r, b])
        assert 448 * one >= part.abs().max() > 224 * one and np.log2(one) == round(np.log2(one))
        want = (part.double() / one).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        np.testing.assert_array_equal(q[r, b * 128:(b + 1) * 128], want)


def test_blocks_are_rows_of_blocks():
    rng = np.random.default_rng(1)
    w = rng.normal(size=(2, 136, 144)).astype(np.float32)
    q, s = ref.quantize_blocks(w)
    for n, r, c in itertools.product(range(2), range(2), range(2)):
        part = w[n, r * 128:(r + 1) * 128, c * 128:(c + 1) * 128]
        assert s[n, r, c] == ref.scale_of(np.abs(part).max())
        np.testing.assert_array_equal(q[n, r * 128:(r + 1) * 128, c * 128:(c + 1) * 128],
                                      ref.encode(part.astype(np.float64) / s[n, r, c]))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_select_is_brute_force(score):
    """Every choice of K experts of every choice of groups: the chosen one has the largest
    keys."""
    rng = np.random.default_rng(2)
    l, bias = rng.normal(size=(6, 8)), rng.normal(size=8) * 0.3
    idx, gate = ref.select(l, bias, 3, score, n_groups=4, top_groups=2, group_top=2, scale=1.5)
    s = torch.softmax(torch.from_numpy(l), 1).numpy() if score == "softmax" else torch.sigmoid(torch.from_numpy(l)).numpy()
    key = s + bias
    for t in range(6):
        best = max(itertools.combinations(range(4), 2), key=lambda gs: sum(key[t, 2 * g:2 * g + 2].sum() for g in gs))
        pool = [e for e in range(8) if e // 2 in best]
        chosen = max(itertools.combinations(pool, 3), key=lambda es: key[t, list(es)].sum())
        assert sorted(idx[t]) == sorted(chosen)
        assert (np.diff(key[t, idx[t]]) < 0).all()
        np.testing.assert_allclose(gate[t], 1.5 * s[t, idx[t]] / s[t, idx[t]].sum(), rtol=1e-12)


def test_experts_are_the_oracles_where_nothing_rounds():
    """With numbers that 8 bits hold, also after the GLU, the experts are plain algebra."""
    x = np.array([[1.0, 2.0] + [0.0] * 14])
    w1 = np.zeros((1, 16, 16))
    v1 = np.zeros((1, 16, 16))
    w2 = np.zeros((1, 16, 16))
    w1[0, 0, 0], v1[0, 0, 1], w2[0, 3, 0] = 64.0, 0.25, 2.0
    out, room = ref.experts(x, np.array([[0]]), np.array([[0.5]]), w1, v1, w2)
    want = np.zeros((1, 16))
    want[0, 3] = 0.5 * 2.0 * 64.0 * 0.5  # silu(64) is 64
    np.testing.assert_allclose(out, want)
    assert (room >= 0).all()


# ---- refusals -----------------------------------------------------------------------------


@no_gpu
def test_quantize_refusals(lib):
    L = lib.lib()
    rows = lambda r=4, c=128, x=A, t=0, q=A, s=A: L.moe_quantize_rows(r, c, x, t, q, s, None)
    blocks = lambda n=1, r=128, c=128, w=A, t=0, q=A, s=A: L.moe_quantize_blocks(n, r, c, w, t, q, s, None)
    assert rows(0) == 0 and blocks(0) == 0
    for bad in (dict(r=-1), dict(r=(1 << 24) + 1), dict(c=0), dict(c=8), dict(c=136), dict(c=65552), dict(t=2),
                dict(x=None), dict(x=MIS), dict(q=None), dict(q=MIS), dict(s=None), dict(s=MIS)):
        assert rows(**bad) == 1, bad
    for bad in (dict(n=-1), dict(n=257), dict(r=0), dict(r=12), dict(r=65544), dict(c=24), dict(t=-1),
                dict(w=None), dict(w=MIS), dict(q=MIS), dict(s=None)):
        assert blocks(**bad) == 1, bad


@no_gpu
def test_product_refusals(lib):
    L = lib.lib()

    def call(n=2, out=128, n_in=128, S=8, x=A, xs=A, off=A, w=A, ws=A, y=A, t=0, sp=A, size=1 << 40):
        return L.moe_quant_product(n, out, n_in, S, x, xs, off, w, ws, y, t, sp, size, None)

    assert call(S=0) == 0
    for bad in (dict(n=0), dict(n=257), dict(out=0), dict(out=12), dict(out=65544), dict(n_in=8), dict(n_in=24),
                dict(n_in=65552), dict(S=-1), dict(S=(1 << 24) + 1), dict(t=3), dict(off=None), dict(x=None),
                dict(x=MIS), dict(xs=None), dict(w=MIS), dict(ws=None), dict(y=MIS)):
        assert call(**bad) == 1, bad
    need = lib.quant_product_workspace_size(2, 128, 128, 8)
    for bad in (dict(sp=None), dict(sp=MIS), dict(size=need - 1)):
        assert call(**bad) == 3, bad


@no_gpu
def test_select_refusals(lib):
    L = lib.lib()
    d = lib.dims(256, 256, 16, 4, torch.bfloat16)

    def call(T=4, lg=A, b=None, i=A, g=A, dims=d, **kw):
        r = lib.router()
        for k, v in kw.items():
            setattr(r, k, v)
        return L.moe_route_select(dims, r, T, lg, b, i, g, None)

    assert call(T=0) == 0
    for bad in (dict(T=-1), dict(T=1 << 21), dict(lg=None), dict(lg=MIS), dict(b=MIS), dict(i=None), dict(g=None),
                dict(score=2), dict(score=-1), dict(n_groups=0), dict(n_groups=3), dict(n_groups=17),
                dict(n_groups=4, top_groups=0), dict(n_groups=4, top_groups=5), dict(n_groups=8, top_groups=1),
                dict(n_groups=16, top_groups=8, group_top=2), dict(group_top=0), dict(group_top=3),
                dict(renormalise=2), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(dims=lib.dims(256, 256, 16, 17, torch.bfloat16))):
        assert call(**bad) == 1, bad
    assert L.moe_route_select(d, None, 4, A, None, A, A, None) == 1
    with pytest.raises(ValueError):
        lib.router("tanh")


@no_gpu
@pytest.mark.parametrize("layer", [False, True])
def test_experts_refusals(lib, layer):
    L = lib.lib()
    d = lib.dims(256, 272, 4, 2, torch.bfloat16)
    need = lib.quant_workspace_size(d, 8)

    def call(dims=d, T=8, x=A, a=A, b=A, weights=None, res=None, out=A, ws=A, size=need, bias=None, router=None):
        w = lib._QuantExperts(*[0x10000] * 6)
        for k, v in (weights or {}).items():
            setattr(w, k, v)
        if layer:
            return L.moe_quant_layer_forward(dims, router, T, x, a, bias, w, res, out, ws, size, None)
        return L.moe_quant_experts_forward(dims, T, x, a, b, w, res, out, ws, size, None)

    assert call(T=0) == 0
    bads = [dict(T=-1), dict(x=None), dict(x=MIS), dict(a=None), dict(res=MIS), dict(out=None), dict(out=MIS),
            dict(dims=lib.dims(264, 272, 4, 2, torch.bfloat16)), dict(dims=lib.dims(256, 280, 4, 2, torch.bfloat16)),
            dict(dims=lib.dims(256, 272, 4, 5, torch.bfloat16))]
    bads += [dict(weights={k: v}) for k in ("w1", "v1", "w2", "s1", "sv", "s2") for v in (None, 0x10004)]
    bads += [dict(bias=A), dict(router=lib.router(n_groups=3)), dict(router=lib.router(), bias=MIS)] if layer else [dict(b=None)]
    for bad in bads:
        assert call(**bad) == 1, bad
    assert call(dims=lib.dims(256, 272, 4, 2, torch.bfloat16, torch.float32)) == 2
    for bad in (dict(ws=None), dict(ws=MIS), dict(size=need - 1)):
        assert call(**bad) == 3, bad


def test_binding_refusals(lib):
    """What the binding looks at: types, shapes, contiguity, devices (here: the CPU's)."""
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t)
    f8 = lambda *s: torch.zeros(s, dtype=torch.uint8).view(torch.float8_e4m3fn)
    d = lib.dims(256, 272, 4, 2, torch.bfloat16)
    for call in (lambda: lib.quantize_rows(z(4, 128, t=torch.float16)), lambda: lib.quantize_rows(z(4, 2, 64)),
                 lambda: lib.quantize_rows(z(4, 256)[:, :128]), lambda: lib.quantize_rows(z(4, 128), scale=z(4, 2)),
                 lambda: lib.quantize_rows(z(4, 128)), lambda: lib.quantize_blocks(z(128, 128)),
                 lambda: lib.route_select(d, lib.router(), z(3, 5)), lambda: lib.route_select(d, lib.router(), z(3, 4), z(5)),
                 lambda: lib.quant_product(f8(3, 128), z(3, 1), f8(2, 128, 128), z(2, 1, 1)),
                 lambda: lib.quant_product(f8(3, 128), z(3, 2), f8(1, 128, 128), z(1, 1, 1)),
                 lambda: lib.quant_product(f8(3, 128), z(3, 1), f8(1, 128, 144), z(1, 1, 2)),
                 lambda: lib.quant_product(f8(3, 128), z(3, 1), f8(1, 128, 128), z(1, 1, 1), out_dtype=torch.float16),
                 lambda: lib.QuantExperts(f8(4, 272, 256), z(4, 3, 2), f8(4, 272, 256), z(4, 3, 2), f8(4, 272, 256), z(4, 2, 3)),
                 lambda: lib.QuantExperts(f8(4, 272, 256), z(4, 3, 2), f8(4, 272, 256), z(4, 2, 2), f8(4, 256, 272), z(4, 2, 3))):
        with pytest.raises(ValueError):
            call()
    ex = lib.QuantExperts(f8(4, 272, 256), z(4, 3, 2), f8(4, 272, 256), z(4, 3, 2), f8(4, 256, 272), z(4, 2, 3))
    x, i, g = z(3, 256, t=torch.bfloat16), z(3, 2, t=torch.int32), z(3, 2)
    for call in (lambda: lib.quant_experts_forward(d, ex, x, i, g),  # (not on a GPU)
                 lambda: lib.quant_experts_forward(d, ex, x.float(), i, g),
                 lambda: lib.quant_experts_forward(d, ex, x, i.long(), g),
                 lambda: lib.quant_experts_forward(d, ex, x, i, g, residual=z(3, 256)),
                 lambda: lib.quant_experts_forward(lib.dims(256, 256, 4, 2, torch.bfloat16), ex, x, i, g),
                 lambda: lib.quant_layer_forward(d, ex, x, z(256, 4, t=torch.bfloat16), bias=z(4))):
        with pytest.raises(ValueError):
            call()


def test_workspace_sizes_never_fall(lib):
    L = lib.lib()
    for dims in (lib.dims(6144, 10752, 16, 4, torch.bfloat16), lib.dims(256, 272, 200, 9, torch.float32)):
        most = 0
        for T in list(range(0, 700)) + list(range(700, 20000, 997)):
            n = ctypes.c_size_t(0)
            assert L.moe_quant_workspace_size(dims, T, ctypes.byref(n)) == 0
            assert n.value >= most, T
            most = n.value
    for E in (1, 8, 200):
        most = 0
        for S in list(range(0, 3000)) + list(range(3000, 60000, 997)):
            size = lib.quant_product_workspace_size(E, 1024, 2048, S)
            assert size >= most, (E, S)
            most = size
    d = lib.dims(6144, 10752, 16, 4, torch.bfloat16)
    n = ctypes.c_size_t(0)
    assert L.moe_quant_workspace_size(d, -1, ctypes.byref(n)) == 1
    assert L.moe_quant_workspace_size(d, 1, None) == 1
    assert L.moe_quant_product_workspace_size(1, 100, 128, 1, ctypes.byref(n)) == 1
