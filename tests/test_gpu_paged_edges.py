"""The paged 8-bit cache at the edges of what its header allows.  Bounds as in
tests/test_gpu_paged.py unless a test derives its own."""
import numpy as np
import pytest
import torch

from tests import paged_ref as ref
from tests.test_gpu_paged import ATTEND, RUNS, Dev, check_append, moe, queries, rows_for

pytestmark = pytest.mark.gpu


# ---- scales of zero: the page's numbers count as zeros, NaN among them -----------


def _zero_pages(c, share, seed):
    """A share of the (page, head)s gets a scale of zero, and NaN bytes among its
    numbers (a third of them, both signs)."""
    rng = np.random.default_rng(seed)
    for b, s in (("k", "ks"), ("v", "vs")):
        off = rng.random(c[s].shape) < share
        c[s][off] = 0.0
        nan = off[:, :, None, None] & (rng.random(c[b].shape) < 0.33)
        c[b][nan] = np.where(rng.random(c[b].shape) < 0.5, 0x7f, 0xff)[nan]


def _without(c):
    """The host's copies with zeros where the scale is zero."""
    out = []
    for b, s in (("k", "ks"), ("v", "vs")):
        out.append(np.where((c[s] == 0.0)[:, :, None, None], np.uint8(0), c[b]))
    return out + [c["ks"], c["vs"]]


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("runs", ["one", "ends", "mixed", "many", "two_chunks", "far_chunks"])
@pytest.mark.parametrize("share", [0.3, 1.0])
def test_attend_zero_scales_hide_nan(page, runs, share):
    m = moe()
    c = ref.call(6, 2, page, {**RUNS, **ATTEND}[runs], seed=page + 60, pad=1)
    _zero_pages(c, share, page)
    d = Dev(m, c)
    q = queries(c)
    got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos).double().cpu().numpy()
    assert m.get_last_error() == 0
    want, room = ref.attend(c, q.double().cpu().numpy(), *_without(c))
    got = got.reshape(want.shape)
    assert np.all(np.isfinite(got)), "non-finite output"
    assert np.max(np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** -10 * room)) <= 0


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("runs", ["ends", "mixed", "gap"])
def test_append_over_zero_scales(page, runs):
    """Earlier rows under a scale of zero are zeros under the new one."""
    m = moe()
    c = ref.call(6, 2, page, RUNS[runs], seed=page + 61)
    _zero_pages(c, 0.5, page + 1)
    d = Dev(m, c)
    x, xh = rows_for(c, "f32")
    old = d.host()
    q = m.paged_append(d.a, d.cache, x, d.seq, d.pos).double().cpu().numpy()
    assert m.get_last_error() == 0
    after = d.host()
    clean = tuple(a.copy() for a in (*_without(c)[:2], *old[2:]))
    touched = {key: p for key, p in ref.append(c, xh, *old)[2].items()}
    for (w, pg, h), p in touched.items():
        if p["old"] != 0.0 or p["fresh"]:
            continue
        b = after[0 if w == "k" else 1][pg, h]
        rest = [o for o in range(page) if o not in p["rows"]]
        assert not (b[rest] & 0x7f).any(), (w, pg, h)
        b[rest] = 0  # (the sign of a zero is left open)
        clean[0 if w == "k" else 1][pg, h][rest] = 0
    # pages that the call does not write, or starts, keep their other bytes
    for i, w in enumerate("kv"):
        for pg in range(c["n_pages"]):
            for h in range(2):
                p = touched.get((w, pg, h))
                if p is None or p["fresh"]:
                    clean[i][pg, h] = old[i][pg, h]
    with np.errstate(divide="ignore"):  # (the logarithm of an old scale of zero)
        check_append(c, clean, q, after, xh)


@pytest.mark.parametrize("n", [1, 140])
def test_query_not_finite_over_zero_scales(n):
    """NaN times a zero is NaN: the query's row, and no other."""
    m = moe()
    c = ref.call(6, 2, 32, [(0, 300, n)], seed=64)
    c["ks"][...] = 0.0
    d = Dev(m, c)
    q = queries(c)
    q[0, 1, 5], q[n - 1, 4, 0] = float("nan"), float("inf")
    got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos).reshape(n, 6, 128).isnan().cpu().numpy()
    assert m.get_last_error() == 0
    nan = np.zeros((n, 6, 128), bool)
    nan[0, 1] = nan[n - 1, 4] = True
    np.testing.assert_array_equal(got, nan)
