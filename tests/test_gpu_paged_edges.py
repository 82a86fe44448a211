"""The paged 8-bit cache at the edges of what its header allows.  Bounds as in
tests/test_gpu_paged.py unless a test derives its own."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

from tests import paged_ref as ref
from tests.test_gpu_paged import (ATTEND, RUNS, Dev, bf16, check_append, check_attend, moe, queries,
                                  rows_for)

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


# ---- earlier scales that are no powers of two ------------------------------------------


def _near_ties(rng, scale, n):
    """n numbers x whose x / scale lies within 2^-22 of the middle between two e4m3
    numbers, on either side of it and on it (up to 224: need stays below a scale of
    any mantissa)."""
    pos = ref.E4M3[:119]
    mid = ((pos[:-1] + pos[1:]) / 2)[8:]
    assert mid[-1] < 224
    x = (rng.choice(mid, n) * float(scale)).astype(np.float32)
    step = rng.integers(-2, 3, n)
    for _ in range(2):
        x = np.where(step < 0, np.nextafter(x, np.float32(0)), np.where(step > 0, np.nextafter(x, np.float32(np.inf)), x))
        step -= np.sign(step)
    return x * rng.choice([-1.0, 1.0], n).astype(np.float32)


@pytest.mark.parametrize("page,runs", [(16, [(i, 3 + i, 1) for i in range(8)]), (64, [(0, 5, 40), (1, 70, 9)]),
                                       (128, [(0, 1, 127), (1, 130, 1)])], ids=["alone", "chunks", "page"])
def test_append_rounds_the_quotient_once(page, runs):
    """Values next to the middle of two e4m3 numbers under an old scale that stays:
    x / scale, rounded once.  (float64: x / scale of 24-bit numbers is either that
    middle, of five bits, or farther from it than 2^-30 of it, so it lies on its
    right side.)"""
    m = moe()
    c = ref.call(4, 2, page, runs, seed=page + 62)
    rng = np.random.default_rng(page)
    c["vs"] = (rng.uniform(1.0, 2.0, c["vs"].shape) * 2.0 ** rng.integers(-4, 4, c["vs"].shape)).astype(np.float32)
    c["vs"][:, 1] = 1.0  # (and one that is)
    d = Dev(m, c)
    T = len(c["seq"])
    x = np.zeros((T, 8, 128), np.float32)
    for t in range(T):
        pg = ref.page_of(c, c["seq"][t], c["pos"][t])
        for h in range(2):
            x[t, 6 + h] = _near_ties(rng, c["vs"][pg, h], 128)
    before = d.host()
    m.paged_append(d.a, d.cache, torch.from_numpy(x.reshape(T, -1)).cuda(), d.seq, d.pos)
    assert m.get_last_error() == 0
    _, v, _, vs = d.host()
    np.testing.assert_array_equal(vs, before[3])
    for t in range(T):
        pg, off = ref.page_of(c, c["seq"][t], c["pos"][t]), c["pos"][t] % page
        want = ref.encode(x[t, 6:].astype(np.float64) / vs[pg].astype(np.float64)[:, None])
        np.testing.assert_array_equal(v[pg, :, off], want, err_msg=f"token {t}")


@pytest.mark.parametrize("tokens", [1, 5])
def test_append_rounds_the_earlier_rows_once(tokens):
    """A page that grows from a scale that is no power of two: its earlier numbers
    times old / new, rounded once, for multipliers that put products next to the
    middle of two e4m3 numbers."""
    m = moe()
    n = 96
    c = ref.call(2, 1, 64, [(i, 20, tokens) for i in range(n)], seed=63)
    rng = np.random.default_rng(64)
    pos = ref.E4M3[:120]
    mid, num = ((pos[:-1] + pos[1:]) / 2)[40:100], np.arange(9, 16, 2)
    ratio = (rng.choice(mid, c["vs"].shape) / rng.choice(num, c["vs"].shape)).astype(np.float32)
    frac = np.frexp(ratio)[0].astype(np.float32)  # [1/2, 1)
    c["vs"][...] = frac * np.float32(2.0 ** -3)
    d = Dev(m, c)
    T = len(c["seq"])
    x = np.zeros((T, 4, 128), np.float32)
    x[:, 3, 0] = 448.0  # (need = 1)
    before = d.host()
    m.paged_append(d.a, d.cache, torch.from_numpy(x.reshape(T, -1)).cuda(), d.seq, d.pos)
    assert m.get_last_error() == 0
    _, v, _, vs = d.host()
    for s in range(n):
        pg = ref.page_of(c, s, 20)
        assert vs[pg, 0] == 1.0
        rest = [o for o in range(64) if not 20 <= o < 20 + tokens]
        y = ref.decode(before[1][pg, 0, rest]) * float(before[3][pg, 0])  # (28 bits: exact)
        np.testing.assert_array_equal(v[pg, 0, rest] & 0x7f, ref.encode(y) & 0x7f)


# ---- far positions -------------------------------------------------------------------


def _turns(base, pos):
    """[positions, 64]: the angles' fractions of a turn, exact but for the last
    rounding to float64."""
    getcontext().prec = 60
    two_pi = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    rate = [(-(Decimal(2 * i) / 128) * Decimal(base).ln()).exp() / two_pi for i in range(64)]
    return np.array([[float((int(p) * r) % 1) for r in rate] for p in pos])


@pytest.mark.parametrize("base", [10000.0, 500000.0])
@pytest.mark.parametrize("first", [(1 << 20) - 20, (1 << 24) - 7, (1 << 27) + 3, (1 << 30) - 40])
def test_append_at_far_positions(base, first):
    """Queries and keys at positions up to the last one of the largest table.  Their
    angles: 2^-55.5 of a turn a position (64 bits of the rate, of which the 53-bit
    logarithm and division leave that), 2^-26 of a turn where the fraction becomes
    fp32 and 2^-32 where it is cut; at 2^30 2^-25.5 + 2^-26 + 2^-32 of a turn,
    2^-22.0 as an angle; sine and cosine 2^-23, the two products and their sum
    2^-23: 2^-20.9 of the pair's magnitudes, 2^-20 allowed."""
    m = moe()
    page, n = 128, 40
    pos = np.arange(first, first + n, dtype=np.int32)
    table = torch.full((1, (1 << 30) // page), -1, dtype=torch.int32, device="cuda")
    lo, hi = first // page, (first + n - 1) // page
    for i in range(lo, hi + 1):
        table[0, i] = i - lo
    a = m.sa_dims(768, 2, 1, 128, base)
    cache = m.PagedCache.alloc(a, page, 2, table)
    g = torch.Generator().manual_seed(first)
    x = torch.randn((n, 4 * 128), generator=g)
    seq = torch.zeros(n, dtype=torch.int32, device="cuda")
    q = m.paged_append(a, cache, x.cuda(), seq, torch.from_numpy(pos).cuda()).double().cpu().numpy()
    assert m.get_last_error() == 0
    xh = x.double().numpy().reshape(n, 4, 128)
    w = 2 * np.pi * _turns(base, pos)[:, None, :]
    lo_, hi_ = xh[:, :3, :64], xh[:, :3, 64:]
    turned = np.concatenate([lo_ * np.cos(w) - hi_ * np.sin(w), hi_ * np.cos(w) + lo_ * np.sin(w)], -1)
    mag = np.abs(lo_) + np.abs(hi_)
    room = 2.0 ** -20 * np.concatenate([mag, mag], -1)
    err = np.abs(q - turned[:, :2]) - (2.0 ** -8 * np.abs(turned[:, :2]) + room[:, :2])
    assert np.max(err) <= 0, f"queries past their bound by {np.max(err):.3e}"
    k, ks = cache.k_pages.view(torch.uint8).cpu().numpy(), cache.k_scale.cpu().numpy()
    for t in range(n):
        pg, off = pos[t] // page - lo, pos[t] % page
        s = float(ks[pg, 0])
        y = turned[t, 2] / s
        lim = np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10) + room[t, 2] / s
        assert np.all(np.abs(ref.decode(k[pg, 0, off]) - y) <= lim), t


# ---- value scales far apart -------------------------------------------------------------


@pytest.mark.parametrize("runs", ["ends", "mixed", "two_chunks", "far_chunks", "long"])
@pytest.mark.parametrize("span", [(-100, 0), (-60, 40), (-10, 90)], ids=str)
def test_attend_value_scales_far_apart(runs, span):
    """Value pages of scales up to 2^100 apart in one sequence: a position counts in
    the weights whatever its page's scale."""
    m = moe()
    c = ref.call(6, 2, 16, {**RUNS, **ATTEND}[runs], seed=65)
    c["vs"][...] = 2.0 ** c["rng"].choice([span[0], span[0] + 1, span[1]], c["vs"].shape)
    d = Dev(m, c)
    q = queries(c, 1.0)
    got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos)
    assert m.get_last_error() == 0
    check_attend(c, d, q, got)


@pytest.mark.parametrize("chunk,n_seq", [(1, 1), (1, 40), (140, 1), (17, 160)])
def test_attend_after_many_zero_values(chunk, n_seq):
    """16,384 positions of values that are all zeros, appended as such (scales of
    2^-100), whose scores rise once by less than what moves the exponent's base; then
    positions with values.  The sum of the weights stays in range.  (Several sequences
    read the same pages, so that no CTA's work is cut along the positions.)"""
    m = moe()
    n = 16384
    c = ref.call(1, 1, 128, [(0, n, chunk)], seed=67)
    c["k"][...] = ref.encode(np.ones(128))
    c["ks"][...] = 1.0
    for p in range(0, n, 128):
        pg = ref.page_of(c, 0, p)
        c["v"][pg], c["vs"][pg] = 0, 2.0 ** -100
    c["k"][ref.page_of(c, 0, 0)] = 0
    w = 7.5 * np.log(2.0) / np.sqrt(128)
    q = bf16(np.full((chunk, 1, 128), w)).cuda()
    want, room = ref.attend(c, q.double().cpu().numpy(), c["k"], c["v"], c["ks"], c["vs"])
    many = dict(c, seq=np.repeat(np.arange(n_seq, dtype=np.int32), chunk), pos=np.tile(c["pos"], n_seq),
                table=np.tile(c["table"], (n_seq, 1)))
    d = Dev(m, many)
    got = m.paged_attend(d.a, d.cache, q.repeat(n_seq, 1, 1), d.seq, d.pos)
    assert m.get_last_error() == 0
    got = got.double().cpu().numpy().reshape(n_seq, chunk, 1, 128)
    assert np.all(np.isfinite(got))
    assert np.max(np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** -10 * room)) <= 0


# ---- right behind what writes the inputs -------------------------------------------------


@pytest.mark.parametrize("runs", ["one", "ends", "mixed", "two_chunks", "many"])
def test_attend_right_behind_the_append(runs):
    """Appends and attentions without a pause, on rows, queries and tables that the
    kernels just ahead have written: the bits of calls that are waited for."""
    m = moe()
    c = ref.call(12, 2, 32, {**RUNS, **ATTEND}[runs], seed=66, pad=2)
    T = len(c["seq"])
    rows = [rows_for(c, "bf16")[0] for _ in range(6)]
    ws = m.paged_alloc_workspace(Dev(m, c).a, T)

    def run(wait):
        d = Dev(m, c)
        table, seq, pos = d.cache.page_table.clone(), d.seq.clone(), d.pos.clone()
        x = torch.empty_like(rows[0])
        outs = []
        torch.cuda.synchronize()
        for r in rows:
            x.copy_(r)
            d.cache.page_table.copy_(table)
            d.seq.copy_(seq)
            d.pos.copy_(pos)
            if wait:
                torch.cuda.synchronize()
            q = m.paged_append(d.a, d.cache, x, d.seq, d.pos)
            if wait:
                torch.cuda.synchronize()
            outs.append(m.paged_attend(d.a, d.cache, q, d.seq, d.pos, ws=ws))
            if wait:
                torch.cuda.synchronize()
            d.cache.page_table.fill_(-1)
            d.seq.fill_(-1)
        torch.cuda.synchronize()
        return outs

    want = run(True)
    for _ in range(3):
        for a, b in zip(run(False), want):
            assert torch.equal(a, b)
    assert m.get_last_error() == 0


# ---- tables with rows that a call does not use -----------------------------------------------


@pytest.mark.parametrize("rows", [1, 64, 300])
@pytest.mark.parametrize("n", [16, 48, 49, 100, 127, 128])
def test_attend_a_chunk_in_a_table_with_idle_rows(n, rows):
    """A chunk of one sequence, taken in tiles or token by token as the table's rows
    decide, its sequence the table's last."""
    m = moe()
    c = ref.call(6, 2, 32, [(0, 700, n)], seed=68, pad=2)
    c["table"] = np.concatenate([np.full((rows - 1, c["table"].shape[1]), 1 << 30, np.int32), c["table"]])
    c["seq"] = np.where(c["seq"] == 0, rows - 1, -1).astype(np.int32)
    d = Dev(m, c)
    q = queries(c)
    got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos)
    assert m.get_last_error() == 0
    check_attend(c, d, q, got)
    assert not got[n:].any()
