"""Every *_workspace_size function is for "up to" its number of tokens: what it
returns for T is enough for any smaller call, so it never falls as T grows."""
import ctypes

import pytest
import torch

from paper_2506_23635_gb300 import build as moe_build

ATTN = [(6144, 48, 8), (1024, 8, 1), (256, 4, 4), (6144, 6, 2), (4096, 16, 16), (512, 3, 1)]
FFN = [(512, 8, 2), (10752, 16, 4)]
TOKENS = list(range(0, 2300)) + list(range(2300, 65536, 997)) + [65535, 65536]


@pytest.fixture(scope="module")
def lib():
    moe_build.build()
    from paper_2506_23635_gb300 import moe
    return moe


def _never_falls(size, what):
    most, at = 0, None
    for T in TOKENS:
        n = ctypes.c_size_t(0)
        assert size(T, ctypes.byref(n)) == 0, (what, T)
        assert n.value >= most, f"{what}: {T} tokens {n.value} bytes, {at} tokens {most}"
        most, at = n.value, T


@pytest.mark.parametrize("attn", ATTN, ids=str)
def test_attention_sizes(lib, attn):
    L, a = lib.lib(), lib.sa_dims(*attn)
    for name in ("moe_sa_workspace_size", "moe_paged_workspace_size", "moe_paged_sa_workspace_size"):
        _never_falls(lambda T, n: getattr(L, name)(ctypes.byref(a), T, n), name)


@pytest.mark.parametrize("ffn", FFN, ids=str)
@pytest.mark.parametrize("attn", ATTN, ids=str)
def test_decoder_sizes(lib, attn, ffn):
    L, a = lib.lib(), lib.sa_dims(*attn)
    d = lib.dims(attn[0], *ffn, torch.bfloat16, torch.bfloat16, torch.float32)
    for name in ("moe_decoder_workspace_size", "moe_paged_decoder_workspace_size"):
        _never_falls(lambda T, n: getattr(L, name)(ctypes.byref(a), ctypes.byref(d), T, n), name)


@pytest.mark.parametrize("types", [(torch.bfloat16, torch.bfloat16, torch.float32),
                                   (torch.float32, torch.float32, torch.float32)], ids=["bf16", "fp32"])
@pytest.mark.parametrize("ffn", FFN, ids=str)
@pytest.mark.parametrize("D", sorted({a[0] for a in ATTN}))
def test_layer_sizes(lib, D, ffn, types):
    L, d = lib.lib(), lib.dims(D, *ffn, *types)
    for name in ("moe_workspace_size", "moe_stack_workspace_size", "moe_dense_workspace_size"):
        _never_falls(lambda T, n: getattr(L, name)(ctypes.byref(d), T, n), name)


def test_small_paged_calls_have_no_scratch_for_tiles(lib):
    """The parts of prefill units (20.3 MiB) are for calls that can be sorted into
    tiles: those of 49 tokens or more (48 beyond a table of one row)."""
    a = lib.sa_dims(6144, 48, 8)
    parts = 160 * 2 * 128 * 130 * 4
    assert lib.paged_workspace_size(a, 48) < 4 << 20
    assert lib.paged_workspace_size(a, 49) >= parts
