"""The paged 8-bit cache on the GPU against its plain 64-bit forms
(tests/paged_ref.py).

Bounds.  Stored numbers: y = x / scale is off by half a step of e4m3, 2^-4 |y|
and 2^-10 below the normal numbers, and by the fp32 rotation: sine and cosine to
2^-21 (the angle's own rounding, pi 2^-24, and the functions'), products of the
pair's magnitudes.  Queries: 2^-8 of themselves (bf16; below its normal numbers
2^-134, half of the smallest one's 2^-133) and the same.  ctx: 2^-8 of
itself (bf16) and 2^-10 of sum_j p_j |v_j|: probabilities rounded to no fewer
than 11 bits (2^-11), scores to ~2^-23 of their magnitude, twice over."""
import numpy as np
import pytest
import torch

from tests import paged_ref as ref
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


def moe():
    need_gpu()
    from paper_2506_23635_gb300 import moe as m
    return m


class Dev:
    """A call's tensors on the GPU."""

    def __init__(self, m, c):
        up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
        self.m, self.c = m, c
        self.a = m.sa_dims(768, c["hq"], c["hkv"], 128, c["base"])
        self.cache = m.PagedCache(up(c["k"]).view(torch.float8_e4m3fn),
                                  up(c["v"]).view(torch.float8_e4m3fn), up(c["ks"]), up(c["vs"]),
                                  up(c["table"]))
        self.seq, self.pos = up(c["seq"]), up(c["pos"])

    def host(self):
        k = self.cache
        return (k.k_pages.view(torch.uint8).cpu().numpy(), k.v_pages.view(torch.uint8).cpu().numpy(),
                k.k_scale.cpu().numpy(), k.v_scale.cpu().numpy())


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16()


def rows_for(c, dtype, width=1.5):
    x = c["rng"].normal(size=(len(c["seq"]), (c["hq"] + 2 * c["hkv"]) * 128)) * width
    t = bf16(x) if dtype == "bf16" else torch.from_numpy(x.astype(np.float32))
    return t.cuda(), t.double().numpy()


def check_append(c, before, q, after, qkv):
    """What a call has to have done to the cache, row by row."""
    want_q, room, pages = ref.append(c, qkv, *before)
    err = np.abs(q - want_q) - (2.0 ** -8 * np.abs(want_q) + 2.0 ** -21 * room + 2.0 ** -134)
    assert np.max(err, initial=0.0) <= 0, f"queries past their bound by {np.max(err):.3e}"
    k0, v0, ks0, vs0 = (x.copy() for x in before)
    k1, v1, ks1, vs1 = after
    for (w, pg, h), d in pages.items():
        b0, b1, s1 = (k0, k1, ks1) if w == "k" else (v0, v1, vs1)
        s = float(s1[pg, h])
        old = 0.0 if d["fresh"] else d["old"]
        near = [max(old, ref.scale_for(d["amax"] * f)) for f in (1, 1 - 2.0 ** -21, 1 + 2.0 ** -21)]
        assert s in [np.float32(x) for x in near], (w, pg, h, s, near)
        for off in range(c["page"]):
            got = ref.decode(b1[pg, h, off])
            if off in d["rows"]:
                x, mag = d["rows"][off]
                fine = np.isfinite(x)
                assert np.all(np.isnan(got[~fine]))
                y = np.where(fine, x, 0.0) / s
                lim = np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10) + 2.0 ** -21 * np.where(fine, mag, 0) / s
                bad = np.abs(np.where(fine, got, 0.0) - y) - lim
                assert np.all(bad <= 0), (w, pg, h, off, float(bad.max()))
            elif d["fresh"] or s == d["old"]:
                np.testing.assert_array_equal(b1[pg, h, off], b0[pg, h, off])
            else:
                y = ref.decode(b0[pg, h, off]) * (d["old"] / s)
                if np.log2(d["old"]) == np.round(np.log2(d["old"])):
                    np.testing.assert_array_equal(b1[pg, h, off] & 0x7f, ref.encode(y) & 0x7f)
                else:  # the multiplier is rounded
                    lim = np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10) + 2.0 ** -22 * np.abs(y)
                    assert np.all(np.abs(got - y) <= lim)
        (k0 if w == "k" else v0)[pg, h] = b1[pg, h]
        (ks0 if w == "k" else vs0)[pg, h] = s1[pg, h]
    for x, y, what in ((k0, k1, "k"), (v0, v1, "v"), (ks0, ks1, "ks"), (vs0, vs1, "vs")):
        np.testing.assert_array_equal(x, y, err_msg=f"{what}: what the call does not write")


def run_append(c, dtype="bf16", width=1.5, change=None, error=0):
    m = moe()
    d = Dev(m, c)
    before = d.host()
    x, xh = rows_for(c, dtype, width)
    if change:
        change(xh)
        x = torch.from_numpy(xh.astype(np.float32)).cuda().to(x.dtype)
        xh = x.double().cpu().numpy()
    q = m.paged_append(d.a, d.cache, x, d.seq, d.pos)
    assert m.get_last_error() == error
    check_append(c, before, q.double().cpu().numpy(), d.host(), xh)
    return d


def check_attend(c, d, q, got):
    want, room = ref.attend(c, q.double().cpu().numpy(), *d.host())
    g = got.double().cpu().numpy().reshape(want.shape)
    assert np.all(np.isfinite(g)), "non-finite output"
    err = np.abs(g - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** -10 * room)
    assert np.max(err, initial=0.0) <= 0, f"ctx past its bound by {np.max(err):.3e}"


def queries(c, width=1.5):
    return bf16(c["rng"].normal(size=(len(c["seq"]), c["hq"], 128)) * width).cuda()


def run_attend(c, width=1.5, error=0):
    m = moe()
    d = Dev(m, c)
    q = queries(c, width)
    got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos)
    assert m.get_last_error() == error
    check_attend(c, d, q, got)
    return d, q, got


HEADS = [(48, 8), (8, 1), (3, 1), (4, 4), (6, 2), (14, 2), (10, 2), (8, 2)]
RUNS = {
    "one": [(0, 0, 1)],
    "ends": [(i, p, 1) for i, p in enumerate([0, 1, 14, 15, 16, 17, 63, 64, 127, 128, 129, 300])],
    "chunk": [(0, 0, 40)],
    "mixed": [(0, 37, 150), (1, 5, 1), (2, 200, 1), (3, 0, 17), (4, 31, 2)],
    "gap": [(0, 3, 5), (0, 20, 4), (0, 9, 1)],  # pieces of one sequence, some in one page
}


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("runs", list(RUNS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append(page, runs, dtype):
    run_append(ref.call(6, 2, page, RUNS[runs], seed=page, pad=3), dtype)


@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_append_heads(heads):
    run_append(ref.call(*heads, 32, RUNS["mixed"], seed=heads[0]), "f32")


@pytest.mark.parametrize("page", [16, 64])
def test_append_in_any_order(page):
    """The tokens of a call mixed: a page's first token is not its lowest."""
    run_append(ref.call(6, 2, page, RUNS["mixed"] + [(0, 187, 30)], seed=4, pad=5, order="shuffled"))


@pytest.mark.parametrize("width", [1e-35, 1e-3, 0.05, 30.0, 1e30])
def test_append_scales(width):
    """Rows far smaller (the old scale stays) and far larger (the page's earlier
    rows become zeros) than what the pages hold, to the ends of fp32."""
    run_append(ref.call(6, 2, 32, RUNS["mixed"], seed=11), "f32", width)


def test_append_over_odd_scales():
    """Earlier scales that are no powers of two."""
    c = ref.call(6, 2, 32, RUNS["mixed"], seed=12)
    c["ks"] *= c["rng"].uniform(1.0, 2.0, c["ks"].shape).astype(np.float32)
    c["vs"] *= c["rng"].uniform(1.0, 2.0, c["vs"].shape).astype(np.float32)
    run_append(c, "f32", 3.0)


def test_append_nan_inf_and_zeros():
    def change(x):
        x[2, 130] = np.nan
        x[5, 6 * 128 + 3] = np.inf       # a key
        x[7, 9 * 128 + 7] = -np.inf      # a value
        x[20:26, 6 * 128:] = 0.0
    m = moe()
    c = ref.call(6, 2, 16, [(0, 0, 40)], seed=13)
    d = Dev(m, c)
    x, xh = rows_for(c, "f32")
    change(xh)
    x = torch.from_numpy(xh.astype(np.float32)).cuda()
    before = d.host()
    q = m.paged_append(d.a, d.cache, x, d.seq, d.pos).double().cpu().numpy()
    assert m.get_last_error() == 0
    assert np.isnan(q[2, 1, 2]) and np.isnan(q[2, 1, 66])
    q[2, 1, [2, 66]] = 0.0
    xq = xh.astype(np.float32).astype(np.float64)
    xq[2, [130, 130 + 64]] = 0.0
    q_at = ref.append(c, xq, *before)[0]
    q[2, 1, [2, 66]] = q_at[2, 1, [2, 66]]
    check_append(c, before, q, d.host(), xq)


def test_append_zero_pages():
    """All rows zero: the smallest scale, and numbers that are zero."""
    d = run_append(ref.call(4, 4, 16, [(0, 0, 16)], seed=14), "f32", 0.0)
    assert float(d.cache.k_scale[d.cache.page_table[0, 0]].max()) == 2.0 ** -100


def test_append_many_tokens():
    """More tokens than a block looks at together, over 1024, and in any order."""
    run_append(ref.call(3, 1, 64, [(0, 0, 700), (1, 61, 500), (2, 7, 1)], seed=15, pad=2))
    run_append(ref.call(3, 1, 16, [(0, 5, 600), (1, 3, 600)], seed=16, order="shuffled"))
    run_append(ref.call(2, 2, 16, [(i, i % 40, 1) for i in range(300)], seed=17))


def test_bad_tokens_and_pages():
    """Outside the table, and entries outside the pool: recorded, nothing
    written, nothing attended to; the other tokens as if they were not there."""
    m = moe()
    for what in ("seq", "pos", "neg", "page", "page_low"):
        c = ref.call(6, 2, 16, [(0, 0, 20), (1, 30, 1), (2, 17, 3)], seed=21)
        if what == "seq":
            c["seq"][3] = 3
        elif what == "pos":
            c["pos"][20] = c["table"].shape[1] * 16
        elif what == "neg":
            c["pos"][20] = -1
        else:
            c["table"][0, 1] = c["n_pages"] if what == "page" else -7
        d = run_append(c, error=6)
        q = queries(c)
        got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos)
        assert m.get_last_error() == 6, what
        check_attend(c, d, q, got)
    c = ref.call(6, 2, 16, [(0, 0, 10), (1, 30, 1)], seed=22)
    c["table"][0, 0] = 1 << 30  # nothing is left of the sequence
    d, _, got = run_attend(c, error=6)
    assert not got[:10].any()


def test_padding_is_no_error():
    m = moe()
    c = ref.call(6, 2, 16, [(0, 3, 4)], seed=23, pad=60)
    d = run_append(c)
    q = queries(c)
    ctx = torch.full((64, 768), float("nan"), dtype=torch.bfloat16, device="cuda")
    m.paged_attend(d.a, d.cache, q, d.seq, d.pos, ctx=ctx)
    assert m.get_last_error() == 0
    check_attend(c, d, q, ctx)
    assert not ctx[4:].any()
    c = ref.call(6, 2, 16, [(0, 3, 1)], seed=24)  # nothing but padding
    c["seq"][:] = -1
    run_append(c)
    run_attend(c)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("runs", list(RUNS))
def test_attend(page, runs):
    run_attend(ref.call(6, 2, page, RUNS[runs], seed=page + 1, pad=3))


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("runs", ["ends", "mixed"])
def test_attend_heads(heads, runs):
    run_attend(ref.call(*heads, 32, RUNS[runs], seed=heads[0] + 1))


ATTEND = {
    "long": [(0, 9000, 1), (1, 3, 1), (2, 2047, 1)],
    "many": [(i, (i * 37) % 260, 1) for i in range(200)],
    "two_chunks": [(0, 100, 300), (1, 0, 205)] + [(2 + i, 40 * i, 1) for i in range(24)],
    "full_tiles": [(0, 0, 384)],
    "late_chunk": [(0, 1900, 129)],
    "far_chunks": [(0, 7000, 40), (1, 100, 20), (2, 3000, 130)],  # units cut into parts
    "short_runs": [(i, 50 + i, 15) for i in range(10)],
    "chunks_of_24": [(i, 100 * i, 23 + i % 3) for i in range(12)],
    "chunks_of_16": [(i, 100 * i, 16) for i in range(12)],
}


@pytest.mark.parametrize("runs", list(ATTEND))
@pytest.mark.parametrize("heads", [(12, 2), (5, 5), (8, 1)], ids=str)
def test_attend_lengths(runs, heads):
    run_attend(ref.call(*heads, 64, ATTEND[runs], seed=31))


@pytest.mark.parametrize("runs", ["mixed", "two_chunks"])
def test_attend_any_order(runs):
    run_attend(ref.call(6, 2, 32, {**RUNS, **ATTEND}[runs], seed=32, pad=7, order="shuffled"))


@pytest.mark.parametrize("runs", ["ends", "two_chunks"])
def test_attend_odd_scales(runs):
    """Scales that are no powers of two and differ by 2^20 from page to page,
    and pages whose scale is zero."""
    c = ref.call(6, 2, 16, {**RUNS, **ATTEND}[runs], seed=33)
    for name in ("ks", "vs"):
        c[name] *= c["rng"].uniform(1.0, 2.0, c[name].shape).astype(np.float32)
    c["vs"] *= (2.0 ** c["rng"].integers(-14, 7, c["vs"].shape)).astype(np.float32)
    run_attend(c)
    c["vs"][c["rng"].random(c["vs"].shape) < 0.3] = 0.0
    c["ks"][c["rng"].random(c["ks"].shape) < 0.3] = 0.0
    run_attend(c)


@pytest.mark.parametrize("runs", ["ends", "long", "two_chunks"])
@pytest.mark.parametrize("width", [0.0, 0.01, 20.0])
def test_attend_score_range(runs, width):
    """Even weights, and scores of some hundreds, whose weights are all but one
    zero."""
    run_attend(ref.call(6, 2, 32, {**RUNS, **ATTEND}[runs], seed=34), width)


@pytest.mark.parametrize("step", [0.5, 3.0, 40.0])
@pytest.mark.parametrize("chunk", [1, 140])
def test_attend_rising_scores(step, chunk):
    """Keys whose scores rise along the sequence by `step` every 128 positions:
    the running maximum moves in every tile, or in few."""
    c = ref.call(6, 2, 64, [(0, 1300, chunk)], seed=35)
    n = 1300 + chunk
    direction = np.sign(c["rng"].normal(size=128))
    for p in range(n):
        pg = ref.page_of(c, 0, p)
        c["ks"][pg] = 2.0 ** -4
        c["k"][pg, :, p % 64] = ref.encode(direction * (p // 128) * step)
    m = moe()
    d = Dev(m, c)
    q = bf16(np.broadcast_to(direction * 16.0 / np.sqrt(128), (chunk, 6, 128))).cuda().contiguous()
    got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos)
    assert m.get_last_error() == 0
    check_attend(c, d, q, got)


@pytest.mark.parametrize("chunk", [1, 140])
def test_attend_one_high_score_first(chunk):
    """A first position that outweighs each later one 2^15 times and all of them
    together twice: small weights are not lost."""
    n = 16384
    c = ref.call(2, 1, 128, [(0, n - chunk, chunk)], seed=36)
    c["k"][...] = 0
    c["ks"][...] = 1.0
    pg = ref.page_of(c, 0, 0)
    c["k"][pg, :, 0] = ref.encode(np.full(128, 1.0))
    c["vs"][...] = 1.0
    c["v"][...] = ref.encode(np.ones(128))
    c["v"][pg, :, 0] = ref.encode(np.full(128, -1.0))
    m = moe()
    d = Dev(m, c)
    w = 15 * np.log(2.0) / np.sqrt(128)
    q = bf16(np.full((chunk, 2, 128), w)).cuda()
    got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos)
    assert m.get_last_error() == 0
    check_attend(c, d, q, got)


@pytest.mark.parametrize("runs", ["ends", "mixed", "two_chunks", "long"])
def test_attend_nan_where_nobody_looks(runs):
    """NaN in the rows past each sequence's end, in pages of nobody, and in
    scales of pages that no position needs."""
    c = ref.call(6, 2, 64, {**RUNS, **ATTEND}[runs], seed=37, extra_pages=4)
    live = np.zeros((c["n_pages"], 64), bool)
    for t in range(len(c["seq"])):
        for p in range(c["pos"][t] + 1):
            live[ref.page_of(c, c["seq"][t], p), p % 64] = True
    for x in ("k", "v"):
        c[x][np.broadcast_to(~live[:, None, :], c[x].shape[:3])] = 0x7f
    for x in ("ks", "vs"):
        c[x][~live.any(1)] = np.nan
    run_attend(c)


def test_attend_nan_stays_with_its_sequence():
    c = ref.call(6, 2, 16, [(0, 40, 1), (1, 50, 20), (2, 33, 1)], seed=38)
    m = moe()
    c["v"][ref.page_of(c, 1, 5), 1, 5, 7] = 0x7f
    d = Dev(m, c)
    q = queries(c)
    got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos).double().cpu().numpy().reshape(22, 6, 128)
    assert m.get_last_error() == 0
    nan = np.zeros((22, 6, 128), bool)
    nan[1:21, 3:, 7] = True
    assert np.array_equal(np.isnan(got), nan)


@pytest.mark.parametrize("first,n", [(0, 100), (300, 200), (2000, 60), (5, 20)])
def test_attend_nan_inside_a_chunk(first, n):
    """NaN in the values and in the keys of tokens inside a chunk: the tokens
    before them do not see them, those after do (in the values' dims, in all for
    a key); NaN ahead of the chunk reaches every token."""
    m = moe()
    for ahead in (False, True):
        c = ref.call(6, 2, 32, [(0, first, n), (1, 40, 1)], seed=45)
        at = lambda p: (ref.page_of(c, 0, p), p % 32)
        pv, pk = first + n // 3, first + n // 2
        pg, off = at(pv)
        c["v"][pg, 1, off, [7, 40, 127]] = [0x7f, 0xff, 0x7f]
        pg, off = at(pk)
        c["k"][pg, 0, off, 3] = 0xff
        if ahead and first:
            pg, off = at(first - 1)
            c["v"][pg, 0, off, 99] = 0x7f
        d = Dev(m, c)
        q = queries(c)
        got = m.paged_attend(d.a, d.cache, q, d.seq, d.pos).double().cpu().numpy().reshape(-1, 6, 128)
        assert m.get_last_error() == 0
        nan = np.zeros((n + 1, 6, 128), bool)
        nan[n // 3:n, 3:, [7, 40, 127]] = True
        nan[n // 2:n, :3] = True
        if ahead and first:
            nan[:n, :3, 99] = True
        np.testing.assert_array_equal(np.isnan(got), nan)
        # and the rest is as if they were not there
        for x in ("k", "v"):
            c[x][(c[x] & 0x7f) == 0x7f] = 0
        clean = Dev(m, c)
        want = m.paged_attend(d.a, clean.cache, q, d.seq, d.pos).double().cpu().numpy().reshape(got.shape)
        seen = ~nan
        seen[n // 3:n, 3:] = False  # (whose weights the zeros have changed)
        seen[:n, :3] &= not (ahead and first)
        np.testing.assert_array_equal(got[seen], want[seen])


def test_padding_beside_prompts_and_many_tokens():
    """Padding tokens in calls that are planned, and one of nothing else."""
    c = ref.call(6, 2, 32, [(0, 0, 150), (1, 77, 1)], seed=46, pad=200, order="given")
    run_attend(c)
    c = ref.call(4, 4, 16, [(i, 3 * i, 1) for i in range(140)], seed=47, pad=60, order="shuffled")
    run_append(c)
    run_attend(c)
    c = ref.call(6, 2, 32, [(0, 0, 1)], seed=48, pad=300)
    c["seq"][:] = -1
    run_append(c)
    run_attend(c)


def test_shared_pages_are_read():
    """Two sequences with the same first pages (a shared prompt)."""
    c = ref.call(6, 2, 16, [(0, 70, 1), (1, 90, 1)], seed=39)
    c["table"][1, :4] = c["table"][0, :4]
    run_attend(c)


def test_generation():
    """A prompt in two chunks, then tokens one by one beside another sequence:
    appended and attended to as a user would, each step against the plain forms."""
    m = moe()
    page = 32
    c = ref.call(6, 2, page, [(0, 0, 160), (1, 0, 90)], seed=40)
    d = Dev(m, c)
    steps = [[(0, 0, 70), (1, 0, 33)], [(0, 70, 61), (1, 33, 1)]]
    steps += [[(0, 131 + i, 1), (1, 34 + i, 1)] for i in range(8)]
    ws = m.paged_alloc_workspace(d.a, 256)
    for n, runs in enumerate(steps):
        s = dict(c, seq=np.concatenate([np.full(k, i, np.int32) for i, _, k in runs]),
                 pos=np.concatenate([np.arange(p, p + k, dtype=np.int32) for _, p, k in runs]))
        seq, pos = torch.from_numpy(s["seq"]).cuda(), torch.from_numpy(s["pos"]).cuda()
        before = d.host()
        x, xh = rows_for(s, "bf16" if n % 2 else "f32", 1.0 + 0.5 * n)
        q = m.paged_append(d.a, d.cache, x, seq, pos)
        got = m.paged_attend(d.a, d.cache, q, seq, pos, ws=ws)
        assert m.get_last_error() == 0
        check_append(s, before, q.double().cpu().numpy(), d.host(), xh)
        check_attend(s, d, q, got)


@pytest.mark.parametrize("runs", ["ends", "two_chunks"])
def test_same_bits_again_and_in_a_graph(runs):
    """The same call twice, on another stream, and captured and replayed beside
    a second graph that shares its workspace: the same bits."""
    m = moe()
    c = ref.call(12, 2, 32, {**RUNS, **ATTEND}[runs], seed=41)
    d = Dev(m, c)
    x, _ = rows_for(c, "bf16")
    ws = m.paged_alloc_workspace(d.a, len(c["seq"]))
    q = torch.empty((len(c["seq"]), 12, 128), dtype=torch.bfloat16, device="cuda")
    ctx = torch.empty((len(c["seq"]), 12 * 128), dtype=torch.bfloat16, device="cuda")

    def both(stream=None):
        m.paged_append(d.a, d.cache, x, d.seq, d.pos, q=q, stream=stream)
        m.paged_attend(d.a, d.cache, q, d.seq, d.pos, ctx=ctx, ws=ws, stream=stream)

    both()
    torch.cuda.synchronize()
    first = ctx.clone()
    both()
    assert torch.equal(ctx, first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ctx.zero_()
    torch.cuda.synchronize()
    both(side)
    side.synchronize()
    assert torch.equal(ctx, first)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            both()
    ws.random_(0, 256)
    for g in graphs + graphs:
        ctx.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(ctx, first)
    assert m.get_last_error() == 0


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes: the last pages."""
    m = moe()
    hkv, page = 8, 128
    n_pages = (1 << 32) // (hkv * page * 128) + 40
    c = ref.call(8, hkv, page, [(0, 200, 1), (1, 90, 30)], seed=42)
    big = [torch.zeros((n_pages, hkv, page, 128), dtype=torch.uint8, device="cuda") for _ in range(2)]
    shift = n_pages - c["n_pages"]
    d = Dev(m, c)
    for b, x in zip(big, (d.cache.k_pages, d.cache.v_pages)):
        b[shift:] = x.view(torch.uint8)
    scales = [torch.ones((n_pages, hkv), device="cuda") for _ in range(2)]
    for s, x in zip(scales, (d.cache.k_scale, d.cache.v_scale)):
        s[shift:] = x
    table = torch.where(d.cache.page_table >= 0, d.cache.page_table + shift, -1)
    far = m.PagedCache(*[b.view(torch.float8_e4m3fn) for b in big], *scales, table)
    x, _ = rows_for(c, "bf16")
    q0 = m.paged_append(d.a, d.cache, x, d.seq, d.pos)
    q1 = m.paged_append(d.a, far, x, d.seq, d.pos)
    assert torch.equal(q0, q1)
    assert torch.equal(big[0][shift:], d.cache.k_pages.view(torch.uint8))
    assert torch.equal(big[1][shift:], d.cache.v_pages.view(torch.uint8))
    assert torch.equal(scales[0][shift:], d.cache.k_scale)
    assert torch.equal(m.paged_attend(d.a, far, q1, d.seq, d.pos),
                       m.paged_attend(d.a, d.cache, q0, d.seq, d.pos))
    assert m.get_last_error() == 0
    assert not big[0][:shift].any() and not big[1][:shift].any()


def test_no_tokens():
    m = moe()
    d = Dev(m, ref.call(6, 2, 16, [(0, 0, 4)], seed=43))
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    q = m.paged_append(d.a, d.cache, torch.empty((0, 1280), device="cuda"), none, none)
    assert q.shape == (0, 6, 128)
    assert m.paged_attend(d.a, d.cache, q, none, none).shape == (0, 768)


def test_the_binding_refuses_other_devices_and_strides():
    m = moe()
    c = ref.call(6, 2, 16, [(0, 0, 4)], seed=44)
    d = Dev(m, c)
    q = queries(c)
    with pytest.raises(ValueError):
        m.paged_attend(d.a, d.cache, q, d.seq.cpu(), d.pos)
    with pytest.raises(ValueError):
        m.paged_attend(d.a, d.cache, q.transpose(0, 1).contiguous().transpose(0, 1), d.seq, d.pos)
    with pytest.raises(ValueError):
        m.paged_append(d.a, d.cache, torch.empty((4, 1280)), d.seq, d.pos)


@pytest.mark.parametrize("runs", ["ends", "mixed"])
def test_attend_queries_not_finite(runs):
    """NaN or an infinity in a query: its row is NaN, and no other."""
    m = moe()
    c = ref.call(6, 2, 32, RUNS[runs], seed=50, pad=2)
    d = Dev(m, c)
    q = queries(c)
    bad = q.clone()
    at = [(0, 1, 5, float("inf")), (3, 0, 127, float("nan")), (4, 5, 64, -float("inf"))]
    for t, h, i, x in at:
        bad[t, h, i] = x
    got = m.paged_attend(d.a, d.cache, bad, d.seq, d.pos).reshape(-1, 6, 128)
    assert m.get_last_error() == 0
    for t, h, _, _ in at:
        assert bool(got[t, h].isnan().all())
        got[t, h] = 0
    want, room = ref.attend(c, q.double().cpu().numpy(), *d.host())
    for t, h, _, _ in at:
        want[t, h] = 0
    err = np.abs(got.double().cpu().numpy() - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** -10 * room)
    assert np.max(err) <= 0


@pytest.mark.parametrize("n", [20, 300])
def test_append_of_the_same_position_twice(n):
    """The later token's row is stored, as if the earlier were padding."""
    m = moe()
    c = ref.call(6, 2, 32, [(0, 3, n), (1, 64, 2)], seed=51)
    twice = [(7, 2), (n - 1, 5), (n + 1, n)]  # token, and an earlier one
    caches = []
    x, _ = rows_for(c, "f32")
    for padded in (False, True):
        e = dict(c, seq=c["seq"].copy(), pos=c["pos"].copy())
        for t, u in twice:
            e["seq"][u], e["pos"][u] = (-1, 0) if padded else (c["seq"][t], c["pos"][t])
        d = Dev(m, e)
        m.paged_append(d.a, d.cache, x, d.seq, d.pos)
        assert m.get_last_error() == 0
        caches.append(d.host())
    for got, want in zip(*caches):
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("runs", ["ends", "two_chunks", "many"])
def test_two_calls_at_once(runs):
    """On two streams, each with a workspace of its own, over one cache."""
    m = moe()
    c = ref.call(12, 2, 32, {**RUNS, **ATTEND}[runs], seed=52)
    d = Dev(m, c)
    q = [queries(c), queries(c)]
    want = [m.paged_attend(d.a, d.cache, x, d.seq, d.pos) for x in q]
    streams = [torch.cuda.Stream() for _ in q]
    ws = [m.paged_alloc_workspace(d.a, len(c["seq"])) for _ in q]
    got = [torch.empty_like(x) for x in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            m.paged_attend(d.a, d.cache, q[i], d.seq, d.pos, ctx=got[i], ws=ws[i], stream=streams[i])
    torch.cuda.synchronize()
    assert m.get_last_error() == 0
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_long_chunks_in_either_order():
    """Chunks behind tens of thousands of positions: the same bits whichever of
    them comes first in the call."""
    m = moe()
    c = ref.call(3, 1, 128, [(0, 40000, 26), (1, 33000, 30), (2, 50, 1)], seed=53)
    d, q, got = run_attend(c)
    turn = np.concatenate([np.arange(26, 56), np.arange(26), [56]])
    index = torch.from_numpy(turn).cuda()
    again = m.paged_attend(d.a, d.cache, q[index].contiguous(), d.seq[index], d.pos[index])
    assert torch.equal(again[:56], got[index][:56])


def test_largest_call():
    """65536 tokens, most of them padding, in between and behind the others."""
    c = ref.call(2, 1, 16, [(0, 0, 300), (1, 40, 1), (2, 5, 35)], seed=54, pad=65536 - 336)
    order = np.concatenate([np.arange(336, 33000), np.arange(336), np.arange(33000, 65536)])
    c["seq"], c["pos"] = c["seq"][order], c["pos"][order]
    run_append(c)
    run_attend(c)


@pytest.mark.parametrize("page,runs,order", [
    (16, [(0, 5, 1000), (1, 0, 340)], "shuffled"),
    (16, [(0, 5, 2000), (1, 48, 620), (2, 9, 1)], "given"),
    (128, [(0, 70, 6000), (1, 0, 3000), (2, 128, 800)], "given"),
], ids=str)
def test_append_several_rows_a_block(page, runs, order):
    """Calls with blocks enough for each to take some of the heads' rows."""
    run_append(ref.call(8, 8, page, runs, seed=55, order=order, pad=3))
