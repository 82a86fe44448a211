"""Decoder layers: a bad pointer of any layer, and a page table set on a layer that is
not the first, are refused before the first layer is launched."""
import ctypes

import pytest
import torch

from paper_2506_23635_gb300 import build as moe_build

no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                            reason="placeholder addresses only where no GPU exists")
A, MIS = 0x10000, 0x10004


@pytest.fixture(scope="module")
def lib():
    moe_build.build()
    from paper_2506_23635_gb300 import moe
    return moe


def _calls(lib):
    L = lib.lib()
    a = lib.sa_dims(256, 4, 2)
    d = lib.dims(256, 512, 8, 2, torch.bfloat16, torch.bfloat16, torch.float32)
    p = lib.PagedDims(64, 100, 4, 10)
    P = ctypes.c_void_p
    ref = ctypes.byref

    def slab(arrays, resid=P(A), seq=P(A)):
        return L.moe_decoder_forward(ref(a), ref(d), 3, 8, seq, P(A), 4, 64, resid, *arrays, 1e-6, P(A),
                                     1 << 40, None)

    def paged(arrays, resid=P(A), seq=P(A)):
        return L.moe_paged_decoder_forward(ref(a), ref(d), ref(p), 3, 8, seq, P(A), P(A), resid, *arrays,
                                           1e-6, P(A), 1 << 40, None)

    return {"slab": (slab, 8), "paged": (paged, 10)}


@no_gpu
@pytest.mark.parametrize("kind", ["slab", "paged"])
def test_any_layers_pointer_is_looked_at_first(lib, kind):
    call, n = _calls(lib)[kind]
    arrays = lambda: [(ctypes.c_void_p * 3)(A, A, A) for _ in range(n)]
    assert call(arrays()) not in (0, 1)  # (everything in order, but there is no GPU)
    for i in range(n):
        for layer in range(3):
            for bad in (None, MIS):
                w = arrays()
                w[i][layer] = bad
                assert call(w) == 1, (i, layer, bad)


@no_gpu
@pytest.mark.parametrize("kind", ["slab", "paged"])
@pytest.mark.parametrize("name", ["resid", "seq"])
def test_the_calls_own_pointers(lib, kind, name):
    call, n = _calls(lib)[kind]
    w = [(ctypes.c_void_p * 3)(A, A, A) for _ in range(n)]
    for bad in (None, ctypes.c_void_p(MIS)):
        assert call(w, **{name: bad}) == 1


def test_a_page_table_of_another_layer(lib):
    """A call's page table is the first layer's: one that is set on another layer's
    cache alone would not be used, so the call is refused."""
    a = lib.sa_dims(256, 4, 2)
    d = lib.dims(256, 512, 8, 2, torch.bfloat16, torch.bfloat16, torch.float32)
    tables = [torch.full((2, 4), i, dtype=torch.int32) for i in range(4)]
    w = torch.zeros(8)
    caches = [lib.PagedCache.alloc(a, 16, 10, tables[0]) for _ in range(3)]
    W = lib.PagedDecoderWeights([(w,) * 6 + (c,) for c in caches])
    z = torch.zeros(5, dtype=torch.int32)
    call = lambda: lib.paged_decoder_forward(a, d, W, torch.zeros(5, 256), z, z)

    def refused():
        with pytest.raises(ValueError) as e:  # (in the end the tensors' device is)
            call()
        return "page table" in str(e.value)

    assert not refused()
    caches[2].page_table = tables[1]
    assert refused() and refused()
    caches[0].page_table = tables[1]  # the same on the first: this is the call's
    assert not refused()
    caches[0].page_table = tables[2]  # the first's alone
    assert not refused() and not refused()
    for c in reversed(caches):
        c.page_table = tables[3]
    assert not refused()
    caches[1].page_table = tables[0]
    assert refused()
