"""Attention over the cache held in 8 bits against a plain form in 64 bits.

Tolerances, with u = 2^-8 / 2^-11 the half-step of a bf16 / fp16 output, per row:
  a score is a sum of products that the matrix units keep to 2^-24 of the largest at every one of up to 8 steps, of two or three terms: off by 16 * 2^-23 of
  `reach` (sum of |q_d k_d|); values of q below 2^-14 of the row's largest are held to 2^-22 of it: 2^-22 of `wide`; scaling, cap, bias and the base of the
  exponential round what is at most `high` a few times: 2^-22 * high; exp2 and log2 2^-22. Together d.
  lse: d + 4 * 2^-23 |lse|. weights: relatively 2 d + 8 * 2^-23 |lse| + 2^-20 for sums in fp32.
  out: u |out| for its own rounding; (2^-11 for a weight's three terms + 2 d + count * 2^-29 for what the matrix units cut of the sums, a step of 32
  tokens 2^-24) * size; and a weight is held to 2^-26 of the largest, for values of at most 448 scales: 2^-17 * count * top * vscale.
"""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache8_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def kvp():
    from paper_2508_13231_b200 import kvp
    return kvp


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def dev_bits(words):
    return cuda(words.view(np.int32))


def pack(bits):
    return np.packbits(np.pad(bits, (0, -len(bits) % 32)), bitorder="little").view(np.uint32)


def problem(kvp, b, t, heads, group, d, page, unit, lens, dtype=BF16, keep=1.0, qscale=2.0, vscale=1.0, kscale=1.0, seed=0, columns=None, junk=False):
    """A cache with NaN everywhere but at the sequences' tokens, and queries."""
    rng = np.random.default_rng(seed + 1000 * d + page)
    columns = columns or max(1, -(-max(max(lens), 1) // page))
    pages = b * columns + 2
    table = rng.permutation(pages)[: b * columns].reshape(b, columns).astype(np.int32)
    cache = torch.full((pages, heads, kvp.cache8_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    for i, n in enumerate(lens):
        n = min(max(n, 0), columns * page)
        if n:
            slots = table[i].astype(np.int64)[np.arange(n) // page] * page + np.arange(n) % page
            k = rng.standard_normal((n, heads, d)) * kscale + 0.3 * kscale
            v = rng.standard_normal((n, heads, d)) * vscale
            kvp.cache8_append(cache, cuda(k.astype(np.float32)), cuda(v.astype(np.float32)), cuda(slots))
    if junk:                                                   # pages that are none, in the middle and at the end of a row
        table[0, columns // 2], table[-1, -1] = -1, pages
    q = cuda((rng.standard_normal((b, t, heads * group, d)) * qscale).astype(np.float32)).to(dtype)
    units = None
    n = columns * page // unit
    if keep < 1.0:
        bits = rng.random((b, heads, n)) < keep
        if b > 1:
            bits[1] = False                                    # a sequence that may read nothing
        bits[0, 0, : n // 2] = False
        units = pack(bits.reshape(-1))
    return q, cache, table, np.array(lens, np.int32), units


def check(kvp, q, cache, table, lens, units, unit, scale=None, want_weights=True, slopes=None, **kw):
    d = q.shape[-1]
    scale = d ** -0.5 if scale is None else scale
    got = kvp.attend8(q, cache, cuda(table), cuda(lens), unit_tokens=unit, scale=scale, units=None if units is None else dev_bits(units),
                      want_lse=True, want_weights=want_weights, slopes=None if slopes is None else cuda(slopes.astype(np.float32)), **kw)
    want = plain.attend(q.double().cpu().numpy(), cache.cpu().numpy(), table, lens, unit, float(np.float32(scale)), units,
                        slopes=None if slopes is None else slopes.astype(np.float32).astype(np.float64), **kw)
    out, lse = (got[k].double().cpu().numpy() for k in ("out", "lse"))
    empty = want["count"] == 0
    assert np.array_equal(np.isneginf(lse), empty)
    assert not out[empty].any()
    score = 16 * 2.0 ** -23 * want["reach"] + 2.0 ** -22 * (want["wide"] + want["high"] + 1)
    exact = np.where(empty, 0, want["lse"])
    off = np.abs(np.where(empty, 0, lse) - exact)
    room = score + 4 * 2.0 ** -23 * np.abs(exact)
    assert np.all(off <= room), (off / room).max()
    half = 2.0 ** -8 if q.dtype == BF16 else 2.0 ** -11
    room = half * np.abs(want["out"]) + (2.0 ** -11 + 2 * score + want["count"] * 2.0 ** -29)[..., None] * want["size"] + \
        2.0 ** -17 * (want["count"] * want["top"] * want["vscale"])[..., None] + 2.0 ** -25
    bad = np.abs(out - want["out"]) / room
    assert np.all(bad <= 1), bad.max()
    if want_weights:
        weights = got["weights"].double().cpu().numpy()
        group = q.shape[2] // weights.shape[1]
        worst = score.reshape(*score.shape[:2], -1, group).max((1, 3))[..., None]
        lmost = np.abs(exact).reshape(*score.shape[:2], -1, group).max((1, 3))[..., None]
        room = want["weights"] * (2 * worst + 8 * 2.0 ** -23 * lmost + 2.0 ** -20) + 1e-37
        assert np.all(np.abs(weights - want["weights"]) <= room), (np.abs(weights - want["weights"]) / room).max()
    return got


@pytest.mark.parametrize("d", [128, 64, 256])
@pytest.mark.parametrize("lens", [[1], [16], [17], [300], [0], [15, 0, 33, 250, -3, 1000]])
def test_attend_lengths(kvp, d, lens):
    check(kvp, *problem(kvp, len(lens), 1, 2, 4, d, 16, 16, lens), 16)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("t,group,heads", [(1, 1, 1), (1, 3, 2), (1, 8, 2), (1, 12, 1), (2, 4, 3), (4, 3, 2), (5, 5, 1), (17, 2, 1), (9, 16, 1), (70, 3, 1)])
def test_attend_heads_and_queries(kvp, t, group, heads, dtype):
    # lengths below the number of queries: some queries see nothing
    for d in (64, 128, 256):
        check(kvp, *problem(kvp, 4, t, heads, group, d, 32, 32, [200, t, max(0, t - 1), 1], dtype=dtype), 32)


@pytest.mark.parametrize("page,unit", [(16, 1), (16, 2), (16, 4), (16, 8), (16, 16), (32, 32), (64, 16), (64, 64), (48, 48), (48, 16), (96, 48), (32, 1)])
@pytest.mark.parametrize("keep", [1.0, 0.4])
def test_attend_units(kvp, page, unit, keep):
    for group in (2, 5, 20):                                   # 4, 10 and 40 rows: segments of 8, 16 and 64
        q, cache, table, lens, units = problem(kvp, 3, 2, 3, group, 64, page, unit, [403, 120, 777], keep=keep)
        got = check(kvp, q, cache, table, lens, units, unit)
        if keep < 1:
            assert not got["out"][1].any() and not got["weights"][1].any()


@pytest.mark.parametrize("kw", [dict(cap=30.0), dict(cap=0.5), dict(window=1), dict(window=17, sink=3), dict(window=100, sink=200), dict(window=300), dict(window=2 ** 31),
                                dict(window=64, sink=16, cap=5.0), dict(sink=9)])
@pytest.mark.parametrize("bias", [False, True])
def test_attend_caps_biases_windows(kvp, kw, bias):
    for t, group, keep in ((1, 4, 1.0), (3, 2, 1.0), (40, 2, 1.0), (2, 3, 0.5)):
        p = problem(kvp, 4, t, 2, group, 128, 16, 16, [700, 33, 5, 0], keep=keep, qscale=4.0)
        slopes = np.exp2(-8 * np.arange(1, 2 * group + 1) / (2 * group)) if bias else None
        if bias and t == 3:
            slopes[0] = -0.01                                  # one that likes what is far
        check(kvp, *p, 16, slopes=slopes, **kw)


def test_attend_window_and_small_units(kvp):
    check(kvp, *problem(kvp, 2, 4, 2, 3, 64, 64, 1, [1500, 90], dtype=F16), 1, window=200, sink=20, slopes=np.exp2(-np.arange(1, 7.0)))


@pytest.mark.parametrize("qscale,kscale,vscale,scale", [(1e-3, 1.0, 1e-4, None), (1e4, 1e-4, 300.0, None), (30.0, 1.0, 1.0, None), (1.0, 1.0, 1e4, -0.1),
                                                        (1.0, 100.0, 1e-7, 0.0), (0.0, 1.0, 1.0, None), (1e30, 1e-4, 1.0, 1e-27), (1.0, 1e-20, 1e25, 1e19)])
def test_attend_magnitudes(kvp, qscale, kscale, vscale, scale):
    check(kvp, *problem(kvp, 2, 1, 2, 4, 128, 16, 16, [900, 130], qscale=qscale, kscale=kscale, vscale=vscale), 16, scale=scale)


def test_attend_values_whose_size_changes_along_the_sequence(kvp):
    """Scores and values that rise or fall by powers of ten along the sequence: the maximum and the largest scale move often."""
    d, page, n = 128, 16, 2000
    rng = np.random.default_rng(3)
    rise = np.linspace(-1, 1, n)[:, None, None]
    k = (rng.standard_normal((n, 2, d)) * 0.1 + rise).astype(np.float32)
    v = (rng.standard_normal((n, 2, d)) * 10.0 ** (2 * rise)).astype(np.float32)
    columns = n // page
    table = rng.permutation(columns).astype(np.int32)[None]
    cache = torch.full((columns, 2, kvp.cache8_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    slots = table[0].astype(np.int64)[np.arange(n) // page] * page + np.arange(n) % page
    kvp.cache8_append(cache, cuda(k), cuda(v), cuda(slots))
    for dtype in (F16, BF16):
        for sign in (1, -1):
            for rows in (8, 40):
                q = cuda(np.full((1, 1, rows, d), 0.7 * sign, np.float32)).to(dtype)
                check(kvp, q, cache, table, np.array([n], np.int32), None, 16)


def test_attend_queries_of_wide_range(kvp):
    """Queries whose values differ by many powers of two within a row; where fp16 does not hold them (2^20) the rows are not finite."""
    for dtype, powers in ((BF16, -torch.arange(128, device="cuda") % 21), (F16, -torch.arange(128, device="cuda") % 21), (BF16, -(torch.arange(128, device="cuda") % 21)),
                          (F16, -(torch.arange(128, device="cuda") % 21))):
        q, cache, table, lens, units = problem(kvp, 1, 1, 2, 4, 128, 16, 16, [500], dtype=dtype)
        q *= torch.exp2(powers).to(dtype)
        if bool(q.isfinite().all()):
            check(kvp, q, cache, table, lens, units, 16)
        else:
            assert bool(kvp.attend8(q, cache, cuda(table), cuda(lens))["out"].isnan().all())


def test_attend_a_large_batch(kvp):
    """More sequences than a warp goes through by itself; also with rows for more than one team of warps."""
    lens = [int(x) for x in np.random.default_rng(2).integers(0, 60, 300)]
    for group in (3, 33):
        check(kvp, *problem(kvp, 300, 1, 1, group, 64, 16, 16, lens), 16)


def test_attend_lists_longer_than_a_chunk(kvp):
    """So many units that a CTA's list of them comes in several pieces: a bitmap of ones reads what no bitmap reads, in the same order."""
    heads, d, page, tokens = 8, 64, 64, 64 * 9600
    pages = tokens // page
    cache = torch.zeros((pages, heads, kvp.cache8_page_bytes(d, page)), dtype=torch.uint8, device="cuda")
    torch.manual_seed(0)
    for at in range(0, tokens, 1 << 16):
        n = min(1 << 16, tokens - at)
        kvp.cache8_append(cache, torch.randn(n, heads, d, device="cuda"), torch.randn(n, heads, d, device="cuda"), torch.arange(at, at + n, device="cuda"))
    table = torch.randperm(pages, device="cuda").int()[None]
    lens = torch.tensor([tokens - 5], dtype=torch.int32, device="cuda")
    q = torch.randn(1, 2 * heads, d, device="cuda").to(BF16)
    for unit in (1, 16, 64):
        ones = torch.full((heads * tokens // unit // 32,), -1, dtype=torch.int32, device="cuda")
        a, b = (kvp.attend8(q, cache, table, lens, unit_tokens=unit, units=u, want_lse=True, want_weights=True) for u in (None, ones))
        assert all(torch.equal(a[k], b[k]) for k in a)
        assert abs(float(a["weights"].sum()) - 2 * heads) < 1e-3


@pytest.mark.parametrize("keep", [1.0, 0.1])
def test_attend_long_and_many(kvp, keep):
    check(kvp, *problem(kvp, 2, 1, 2, 2, 128, 32, 32, [20011, 40], keep=keep), 32)                       # many CTAs for one row
    lens = [int(x) for x in np.random.default_rng(1).integers(0, 150, 120)]
    check(kvp, *problem(kvp, 120, 1, 4, 2, 64, 16, 16, lens, keep=keep), 16)                             # many rows for one CTA
    check(kvp, *problem(kvp, 1, 1, 1, 2, 64, 16, 1, [17000], keep=keep), 1)                              # more units than are listed at once


def test_attend_a_chunk_of_a_prompt(kvp):
    for d, dtype in ((128, BF16), (64, F16), (256, BF16), (256, F16)):
        check(kvp, *problem(kvp, 2, 100, 1, 4, d, 16, 16, [1500, 100], dtype=dtype), 16, want_weights=d == 128)


def test_attend_skips_pages_that_are_none(kvp):
    for unit, keep in ((16, 1.0), (1, 1.0), (16, 0.5)):
        check(kvp, *problem(kvp, 3, 1, 2, 4, 128, 16, unit, [300, 100, 320], junk=True, columns=20, keep=keep), unit)


def test_attend_cuts_lengths_to_the_table(kvp):
    q, cache, table, lens, _ = problem(kvp, 2, 1, 2, 4, 128, 16, 16, [100, 64], columns=7)
    full = kvp.attend8(q, cache, cuda(table), cuda(np.array([64, 64], np.int32)))
    long = kvp.attend8(q, cache, cuda(table[:, :4]), cuda(np.array([2 ** 31 - 1, 64], np.int32)))
    assert torch.equal(full["out"], long["out"]) and full["lse"] is None and full["weights"] is None


def test_attend_strided_queries_and_shapes(kvp):
    q, cache, table, lens, _ = problem(kvp, 3, 2, 2, 4, 128, 16, 16, [100, 64, 7])
    want = kvp.attend8(q, cache, cuda(table), cuda(lens), want_lse=True, want_weights=True)
    wide = torch.full((3, 2, 20, 131), float("nan"), device="cuda").to(BF16)
    wide[:, :, 5:13, 3:] = q
    got = kvp.attend8(wide[:, :, 5:13, 3:], cache, cuda(table), cuda(lens), want_lse=True, want_weights=True)
    turned = kvp.attend8(q.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3), cache, cuda(table), cuda(lens), want_lse=True, want_weights=True)
    for other in (got, turned):
        assert all(torch.equal(want[k], other[k]) for k in want)
    rows = torch.full((2, want["weights"].numel()), -1.0, device="cuda")
    kvp.attend8(q, cache, cuda(table), cuda(lens), weights=rows[1])
    assert torch.equal(rows[1], want["weights"].view(-1)) and bool((rows[0] == -1).all())


def test_attend_with_values_that_are_not_finite_in_a_query(kvp):
    """NaN or infinity in one row's query stays in that row (and in the weights of its kv-head)."""
    q, cache, table, lens, _ = problem(kvp, 1, 1, 2, 4, 128, 16, 16, [200])
    want = kvp.attend8(q, cache, cuda(table), cuda(lens), want_weights=True)
    q[0, 0, 1, 5], q[0, 0, 2, 7] = float("nan"), float("inf")
    got = kvp.attend8(q, cache, cuda(table), cuda(lens), want_weights=True)
    rest = [0, 3, 4, 5, 6, 7]
    assert torch.equal(got["out"][0, 0, rest], want["out"][0, 0, rest]) and torch.equal(got["weights"][0, 1], want["weights"][0, 1])
    assert got["out"][0, 0, 1:3].isnan().all()


def test_attend_twice_on_streams_and_in_graphs(kvp):
    """Two calls under way at once, and graphs replayed with other lengths: each with the bits of a call of its own."""
    sets = [problem(kvp, 3, 1, 2, 4, 128, 16, 16, [900, 30, 411], keep=k, seed=s) for s, k in ((1, 1.0), (2, 0.5))]
    dev = [(q, c, cuda(t), cuda(n), None if u is None else dev_bits(u)) for q, c, t, n, u in sets]
    call = lambda i, **kw: kvp.attend8(dev[i][0], dev[i][1], dev[i][2], dev[i][3], units=dev[i][4], want_lse=True, want_weights=True, **kw)  # noqa: E731
    want = [call(i) for i in (0, 1)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[call(i, stream=streams[i]) for _ in range(20)] for i in (0, 1)]
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(want[i][k], r[k]) for r in got[i] for k in want[i])
    graphs, outs = [], []
    for i in (0, 1):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(i))
        graphs.append(g)
    short = torch.tensor([512, 17, 0], dtype=torch.int32, device="cuda")
    for new in (None, short):
        if new is not None:
            dev[0][3].copy_(new)
            want[0] = call(0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(want[i][k], outs[i][k]) for k in want[i])


def test_calls_refuse(kvp):
    q, cache, table, lens, _ = problem(kvp, 2, 1, 2, 4, 128, 16, 16, [100, 64])
    t, n = cuda(table), cuda(lens)
    for args, kw in (((q.float(), cache, t, n), {}), ((q[..., ::2], cache, t, n), {}), ((q[:, :, :3], cache, t, n), {}), ((q, cache, t[:1], n), {}),
                     ((q, cache, t.long(), n), {}), ((q, cache, t, n[:1]), {}), ((q, cache.cpu(), t, n), {}), ((q, cache[:, :, 1:], t, n), {}),
                     ((q[0, 0], cache, t, n), {}), ((q, cache, t, n), dict(units=torch.zeros(0, dtype=torch.int32, device="cuda"))),
                     ((q, cache, t, n), dict(weights=torch.zeros(3, device="cuda"))), ((q, cache, t, n), dict(unit_tokens=-1)), ((q, cache, t, n), dict(window=-1)),
                     ((q, cache, t, n), dict(slopes=torch.zeros(7, device="cuda"))), ((q, cache, t, n), dict(slopes=torch.zeros(8))),
                     ((q, torch.zeros(9, 2, 2560, dtype=torch.uint8, device="cuda"), t, n), {})):
        with pytest.raises((ValueError, TypeError)):
            kvp.attend8(*args, **kw)
    for kw in (dict(unit_tokens=32), dict(unit_tokens=3), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan"))):
        with pytest.raises(kvp.KvpError) as e:
            kvp.attend8(q, cache, t, n, **kw)
        assert e.value.code == kvp.ERR_ARG
