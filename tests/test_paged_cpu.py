"""The paged cache on the CPU: its plain 64-bit forms against the oracle and
torch, and what its entry points refuse before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from paper_2506_23635_gb300 import build as moe_build
from tests import paged_ref as ref

no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                            reason="placeholder addresses only where no GPU exists")
A = ctypes.c_void_p(0x10000)
MIS = ctypes.c_void_p(0x10004)


@pytest.fixture(scope="module")
def lib():
    moe_build.build()
    from paper_2506_23635_gb300 import moe
    return moe


def test_e4m3_is_torchs():
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(got, ref.E4M3)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * 2.0 ** rng.integers(-12, 8, 4000),
                        (ref.E4M3[:126] + ref.E4M3[1:127]) / 2, [0.0, -0.0, 448.0, -448.0]])
    x = x[np.abs(x) <= 448.0].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(ref.encode(x), want)


def test_scale_holds_the_largest_and_half_of_it_does_not():
    rng = np.random.default_rng(1)
    for a in list(np.abs(rng.normal(size=50)) * 10.0 ** rng.integers(-6, 6, 50)) + [448.0, 7.0, 7.0001]:
        s = ref.scale_for(a)
        assert 448 * s >= a > 224 * s and np.log2(s) == np.round(np.log2(s))
    assert ref.scale_for(0.0) == 2.0 ** -100


def test_plain_forms_are_the_oracles():
    """The rotation and, over a cache of whole sequences, the attention."""
    c = ref.call(6, 2, 16, [(0, 0, 20), (1, 7, 3), (2, 40, 1)], seed=3)
    T = len(c["seq"])
    x = c["rng"].normal(size=(T, 10, 128))
    q, _, _ = ref.append(c, x, c["k"], c["v"], c["ks"], c["vs"])
    np.testing.assert_allclose(q, oracle.rope(x[:, :6], c["pos"], c["base"]), atol=1e-12)
    L = 48
    kc, vc = np.zeros((3, 2, L, 128)), np.zeros((3, 2, L, 128))
    for s in range(3):
        for p in range(L):
            pg = ref.page_of(c, s, p)
            if pg >= 0:
                kc[s, :, p] = ref.decode(c["k"][pg, :, p % 16]) * c["ks"][pg][:, None]
                vc[s, :, p] = ref.decode(c["v"][pg, :, p % 16]) * c["vs"][pg][:, None]
    want = oracle.attention(q, kc, vc, c["seq"], c["pos"]).reshape(T, 6, 128)
    got, room = ref.attend(c, q, c["k"], c["v"], c["ks"], c["vs"])
    np.testing.assert_allclose(got, want, atol=1e-12)
    assert np.all(np.abs(got) <= room + 1e-12)


@no_gpu
def test_refusals(lib):
    L = lib.lib()
    a = lib.sa_dims(6144, 48, 8)
    n = ctypes.c_size_t(0)
    size = lambda d, T: L.moe_paged_workspace_size(ctypes.byref(d), T, ctypes.byref(n))
    assert size(a, 1) == 0 and n.value > 0
    assert size(a, 65536) == 0
    assert size(a, 65537) == 1
    assert size(a, -1) == 1
    assert size(lib.sa_dims(6144, 48, 8, head_dim=64), 1) == 2
    assert size(lib.sa_dims(6144, 48, 4), 1) == 2
    assert L.moe_paged_workspace_size(ctypes.byref(a), 1, None) == 1
    assert size(a, 8) == 0
    need = n.value
    P = lib.PagedDims

    def app(T=8, d=a, p=P(64, 100, 4, 10), qkv=A, dt=1, seq=A, pos=A, tab=A, q=A, k=A, v=A, ks=A, vs=A):
        return L.moe_paged_append(ctypes.byref(d), ctypes.byref(p), T, qkv, dt, seq, pos, tab, q, k,
                                  v, ks, vs, None)

    def att(T=8, d=a, p=P(64, 100, 4, 10), q=A, seq=A, pos=A, tab=A, k=A, v=A, ks=A, vs=A, ctx=A,
            ws=A, nb=need):
        return L.moe_paged_attend(ctypes.byref(d), ctypes.byref(p), T, q, seq, pos, tab, k, v, ks,
                                  vs, ctx, ws, nb, None)

    for f in (app, att):
        assert f(T=0) == 0
        assert f(T=-1) == 1 and f(T=65537) == 1
        for name in ("seq", "pos", "tab", "k", "v", "ks", "vs", "q"):
            assert f(**{name: None}) == 1, name
            assert f(**{name: MIS}) == 1, name
        for ps in (8, 24, 63, 256):
            assert f(p=P(ps, 100, 4, 10)) == 2, ps
        for bad in (P(0, 100, 4, 10), P(-16, 100, 4, 10), P(64, 0, 4, 10), P(64, 100, 0, 10),
                    P(64, 100, 4, 0), P(128, 1 << 21, 4, 10), P(128, 100, 4, 1 << 24)):
            assert f(p=bad) == 1, bad
        assert f(d=lib.sa_dims(6144, 48, 7)) == 1
        assert f(d=lib.sa_dims(6144, 48, 8, head_dim=64)) == 2
        assert f(T=0, p=P(24, 100, 4, 10)) == 2  # the shape is checked even when there is no token
    assert app(qkv=None) == 1 and app(qkv=MIS) == 1
    assert app(dt=2) == 1 and app(dt=-1) == 1
    assert att(ctx=None) == 1 and att(ctx=MIS) == 1
    assert att(ws=None) == 3 and att(ws=MIS) == 3 and att(nb=need - 1) == 3
    block = ctypes.c_size_t(0)
    assert L.moe_paged_sa_workspace_size(ctypes.byref(a), 8, ctypes.byref(block)) == 0
    assert block.value > need
    assert L.moe_paged_sa_workspace_size(ctypes.byref(a), 65537, ctypes.byref(block)) == 1

    def blk(T=8, d=a, p=P(64, 100, 4, 10), resid=A, w=A, eps=1e-6, ws=A, nb=1 << 40, seq=A, k=A):
        return L.moe_paged_sa_forward(ctypes.byref(d), ctypes.byref(p), T, seq, A, A, resid, w, A, k,
                                      A, A, A, eps, ws, nb, None)

    assert blk(T=0) == 0 and blk(T=0, p=P(24, 100, 4, 10)) == 2
    for kw in (dict(resid=None), dict(resid=MIS), dict(w=None), dict(seq=None), dict(k=MIS),
               dict(eps=0.0), dict(T=-1), dict(p=P(64, 0, 4, 10))):
        assert blk(**kw) == 1, kw
    assert blk(ws=None) == 3 and blk(ws=MIS) == 3 and blk(nb=1024) == 3
    m = lib.dims(6144, 10752, 16, 4, out_dtype=torch.float32)
    assert L.moe_paged_decoder_workspace_size(ctypes.byref(a), ctypes.byref(m), 8,
                                              ctypes.byref(block)) == 0
    arr = (ctypes.c_void_p * 1)(A)

    def dec(T=8, d=a, mo=m, p=P(64, 100, 4, 10), resid=A, seq=A, ks=arr, n=1, ws=A, nb=1 << 40):
        return L.moe_paged_decoder_forward(ctypes.byref(d), ctypes.byref(mo), ctypes.byref(p), n, T,
                                           seq, A, A, resid, arr, arr, arr, arr, arr, arr, arr, arr,
                                           ks, arr, 1e-6, ws, nb, None)

    assert dec(T=0) == 0 and dec(n=0) == 0
    for kw in (dict(mo=lib.dims(6144, 10752, 16, 4)), dict(d=lib.sa_dims(4096, 32, 8)), dict(n=-1),
               dict(T=-1), dict(resid=None), dict(seq=MIS), dict(ks=None), dict(p=P(64, 100, 0, 1))):
        assert dec(**kw) == 1, kw
    assert dec(ws=None) == 3 and dec(nb=4096) == 3
    assert L.moe_paged_append(None, None, 0, *[None, 1] + [None] * 9) == 1
    assert L.moe_paged_append(ctypes.byref(a), None, 0, *[None, 1] + [None] * 9) == 1


def test_injected_failures(lib):
    import os
    import subprocess
    import sys
    code = ("import ctypes\nfrom paper_2506_23635_gb300 import moe\nL = moe.lib()\n"
            "print(L.moe_paged_append(None, None, 1, None, 1, *[None] * 9),\n"
            "      L.moe_paged_attend(None, None, 1, *[None] * 10, 0, None))\n")
    for value, want in (("moe_paged_append:5", [5, 1]), ("moe_paged_attend:4", [1, 4])):
        out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120,
                             env=dict(os.environ, MOE_INJECT_FAILURE=value))
        assert out.returncode == 0, out.stderr
        assert list(map(int, out.stdout.split())) == want


def test_the_binding_refuses(lib):
    """Shapes, types, strides and devices, before the library is called."""
    a = lib.sa_dims(768, 6, 2)
    table = torch.zeros((3, 4), dtype=torch.int32)
    c = lib.PagedCache.alloc(a, 16, 10, table)
    assert c.k_pages.dtype == torch.float8_e4m3fn and c.k_pages.shape == (10, 2, 16, 128)
    parts = lambda **kw: lib.PagedCache(**{**dict(
        k_pages=c.k_pages, v_pages=c.v_pages, k_scale=c.k_scale, v_scale=c.v_scale,
        page_table=table), **kw})
    parts()
    for kw in (dict(k_pages=c.k_pages.view(torch.uint8)), dict(v_pages=c.v_pages[:9]),
               dict(k_scale=c.k_scale.double()), dict(v_scale=c.v_scale[:, :1]),
               dict(page_table=table.long()), dict(page_table=table[0])):
        with pytest.raises(ValueError):
            parts(**kw)
    T = 5
    qkv, q = torch.zeros(T, 1280), torch.zeros(T, 6, 128, dtype=torch.bfloat16)
    seq, pos = torch.zeros(T, dtype=torch.int32), torch.arange(T, dtype=torch.int32)
    for kw in (dict(qkv=qkv[:, :1272]), dict(qkv=qkv.half()), dict(seq=seq[:4]), dict(pos=pos.long()),
               dict(q=q.float()), dict(q=q[:4]), dict(a=lib.sa_dims(768, 6, 3))):
        with pytest.raises(ValueError):
            lib.paged_append(**{**dict(a=a, cache=c, qkv=qkv, seq=seq, pos=pos), **kw})
    for kw in (dict(q=q.float()), dict(q=q[:, :5]), dict(seq=seq[:4]), dict(pos=pos.long()),
               dict(ctx=torch.zeros(T, 768)), dict(a=lib.sa_dims(768, 6, 3))):
        with pytest.raises(ValueError):
            lib.paged_attend(**{**dict(a=a, cache=c, q=q, seq=seq, pos=pos,
                                       ws=torch.empty(4096, dtype=torch.uint8)), **kw})


@no_gpu
def test_limits_of_the_table_and_the_pool(lib):
    L = lib.lib()
    a = lib.sa_dims(6144, 48, 8)

    def app(page, n_pages, max_pages):
        p = lib.PagedDims(page, n_pages, 4, max_pages)
        return L.moe_paged_append(ctypes.byref(a), ctypes.byref(p), 0, A, 1, *[A] * 8, None)

    assert app(128, 10, 1 << 23) == 0 and app(128, 10, (1 << 23) + 1) == 1
    assert app(16, 10, 1 << 26) == 0 and app(16, 10, (1 << 26) + 1) == 1
    assert app(128, (1 << 21) - 1, 10) == 0 and app(128, 1 << 21, 10) == 1
