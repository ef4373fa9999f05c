"""Attention over the cache in 8 bits where values differ in size from block to block: what a row does not see, or gives no weight, does not change it.

Tolerance of out, per row, with u the half-step of its type, `score` as in test_gpu_attend8.py (how far a score may be off), size = sum of p |v| and
most = the largest product of a weight p and a scale of values over the tokens that the row sees: u |out| for its own rounding; (2^-11 for a weight's three
terms + 2 score + count * 2^-29 for what the matrix unit cuts of the sums) * size; a weight times a scale is held to 2^-26 of most, for values of at most 448
scales: 2^-17 * count * most.
"""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache8_plain as plain  # noqa: E402
from test_gpu_attend8 import BF16, F16, cuda, kvp  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def filled(kvp, k, v, page=16):  # noqa: F811
    """One sequence's cache, its pages out of order, NaN where no token is."""
    n, heads, d = k.shape
    columns = -(-n // page)
    table = np.random.default_rng(n).permutation(columns + 1)[:columns].astype(np.int32)[None]
    cache = torch.full((columns + 1, heads, kvp.cache8_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    slots = table[0].astype(np.int64)[np.arange(n) // page] * page + np.arange(n) % page
    kvp.cache8_append(cache, cuda(k.astype(np.float32)), cuda(v.astype(np.float32)), cuda(slots))
    return cache, table, np.array([n], np.int32)


def near(got, q, cache, table, lens, terms=2.0 ** -11, window=0, keep=None):
    """out of one sequence against 64 bits; keep: units of 16 tokens that are read"""
    b, t, hq, d = q.shape
    (keys, _), (vals, vscale) = plain.held(cache.cpu().numpy(), d)
    n, h = int(lens[0]), cache.shape[1]
    ids, page = np.arange(n), keys.shape[2]
    k, v, size = (x[table[0][ids // page], :, ids % page] for x in (keys, vals, vscale))
    out, x, scale = got["out"].double().cpu().numpy()[0], q.double().cpu().numpy()[0], float(np.float32(d ** -0.5))
    u = 2.0 ** -8 if q.dtype == BF16 else 2.0 ** -11
    for j in range(t):
        at = n - t + j
        see = ids <= at
        if window:
            see &= ids > at - window
        if keep is not None:
            see &= keep[ids // 16]
        for r in range(hq):
            a, w, s = k[see, r * h // hq], v[see, r * h // hq], size[see, r * h // hq]
            y = a @ x[j, r] * scale
            p = np.exp(y - y.max())
            p /= p.sum()
            score = 16 * 2.0 ** -23 * (np.abs(a) @ np.abs(x[j, r]) * scale).max() + 2.0 ** -22 * (np.abs(x[j, r]).max() * np.abs(a).sum(-1).max() * scale + np.abs(y).max() + 1)
            want = p @ w
            room = u * np.abs(want) + (terms + 2 * score + len(p) * 2.0 ** -29) * (p @ np.abs(w)) + 2.0 ** -17 * len(p) * (p * s).max() + 2.0 ** -25
            off = np.abs(out[j, r] - want)
            worst = float((off / room).max())
            assert worst <= 1, (j, r)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d,group,queries", [(128, 1, 20), (128, 4, 24), (64, 2, 40), (256, 3, 18), (128, 8, 18)])
@pytest.mark.parametrize("large", [2.0 ** 12, 2.0 ** 20, np.inf])
def test_a_later_token_with_large_values_leaves_earlier_queries_alone(kvp, d, group, queries, dtype, large):  # noqa: F811
    """The last query's token has values many times the others', also cut infinities: the queries before it, that do not see it, are as without it."""
    rng = np.random.default_rng(d + group)
    n = 320 + 1                                                # the last token has a block of its own
    k, v = rng.standard_normal((2, n, 1, d))
    v[-1] = large if np.isinf(large) else v[-1] * large
    cache, table, lens = filled(kvp, k, v)
    q = cuda(rng.standard_normal((1, queries, group, d)).astype(np.float32)).to(dtype)
    got = kvp.attend8(q, cache, cuda(table), cuda(lens), want_lse=True)
    before = dict(got, out=got["out"][:, :-1])
    near(before, q[:, :-1], cache, table, lens - 1)
    without = kvp.attend8(q[:, :-1], cache, cuda(table), cuda(lens - 1), want_lse=True)
    near(without, q[:, :-1], cache, table, lens - 1)
    if not np.isinf(large) and dtype == BF16:                  # fp16 does not hold 2^20 of the last row
        near(dict(out=got["out"][:, -1:]), q[:, -1:], cache, table, lens)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [1, 8, 12, 40])
def test_blocks_with_large_values_and_no_weight(kvp, dtype, rows):  # noqa: F811
    """A token that takes most of the weight, a long tail that takes the rest, and blocks of values 2^12 or 2^20 times the others' that no row gives weight: out holds the tail.
    The sequence is there many times, so that a CTA goes through all of it."""
    d, n, batch = 128, 6000, 1200
    rng = np.random.default_rng(rows)
    for large, where in ((2.0 ** 12, 0), (2.0 ** 20, 0), (2.0 ** 12, n - 16), (2.0 ** 20, 2992)):
        k = rng.standard_normal((n, 1, d)) * 0.05
        k[..., 0] = 0.0
        k[1000, 0, 0] = 100.0                                  # score 100 * 1.1 * scale = 9.7 over the tail's: e^9.7 tail tokens weigh as much
        k[where: where + 16, 0, 0] = -400.0                    # e^-39
        v = 1.0 + 0.1 * rng.standard_normal((n, 1, d))
        v[992: 1008] *= 2.0 ** -10                             # what has most weight is small
        v[where: where + 16] *= large
        cache, table, lens = filled(kvp, k, v)
        q = rng.standard_normal((1, 1, rows, d)) * 0.2
        q[..., 0] = 1.1
        q = cuda(q.astype(np.float32)).to(dtype)
        got = kvp.attend8(q.expand(batch, -1, -1, -1), cache, cuda(np.repeat(table, batch, 0)), cuda(np.repeat(lens, batch)))
        for i in (0, 7, batch // 2, batch - 1):
            near(dict(out=got["out"][i: i + 1]), q, cache, table, lens)


def test_what_windows_and_bitmaps_leave_out(kvp):  # noqa: F811
    """Large values behind a window, or in units that are not read, beside small ones that are."""
    d, n = 64, 700
    rng = np.random.default_rng(5)
    k, v = rng.standard_normal((2, n, 1, d))
    v[: 300] *= 2.0 ** 18
    cache, table, lens = filled(kvp, k, v)
    q = cuda(rng.standard_normal((1, 3, 4, d)).astype(np.float32)).to(BF16)
    # one query sees through the window the last token of the large ones' block, the others do not
    window = n - 3 + 1 - 303
    near(kvp.attend8(q, cache, cuda(table), cuda(lens), window=window), q, cache, table, lens, window=window)
    keep = np.arange(-(-n // 16)) >= 19
    units = cuda(np.packbits(np.pad(keep, (0, -len(keep) % 32)), bitorder="little").view(np.int32))
    near(kvp.attend8(q, cache, cuda(table), cuda(lens), unit_tokens=16, units=units), q, cache, table, lens, keep=keep)


def test_values_that_are_all_zero_or_tiny(kvp):  # noqa: F811
    """Rows whose heaviest tokens have values 0, or 2^-90 of the others': zeros add nothing, and what has a value is kept."""
    d, n = 128, 400
    rng = np.random.default_rng(6)
    for small in (0.0, 2.0 ** -90):
        for first in (0, 384):
            k, v = rng.standard_normal((2, n, 2, d)) * 0.3
            k[first: first + 16] = 0.0
            k[first: first + 16, :, 0] = 200.0                 # e^35 of the others
            v[first: first + 16] *= small
            cache, table, lens = filled(kvp, k, v)
            q = rng.standard_normal((1, 1, 8, d)) * 0.2
            q[..., 0] = 2.0
            q = cuda(q.astype(np.float32)).to(BF16)
            got = kvp.attend8(q, cache, cuda(table), cuda(lens))
            near(got, q, cache, table, lens)
            assert bool(got["out"].abs().amax() > 0)
    k = np.zeros((n, 2, d))
    cache, table, lens = filled(kvp, k, k)
    assert not kvp.attend8(q, cache, cuda(table), cuda(lens))["out"].any()


def test_parts_whose_values_differ_by_many_powers(kvp):  # noqa: F811
    """The heaviest tokens have values 0 and a CTA of their own, what has values of 2^50 or 2^90 is elsewhere: the parts are joined all the same."""
    d, n = 128, 3000
    rng = np.random.default_rng(7)
    for high in (1.0, 2.0 ** 50, 2.0 ** 90):
        for first, last in ((0, 640), (2000, 3000)):
            k, v = rng.standard_normal((2, n, 1, d)) * 0.3
            k[first: last, :, 0] = 60.0                        # e^10 of the others
            v[first: last] = 0.0
            v[1000: 1500] *= high
            cache, table, lens = filled(kvp, k, v)
            for rows in (4, 20):
                q = rng.standard_normal((1, 1, rows, d)) * 0.2
                q[..., 0] = 2.0
                q = cuda(q.astype(np.float32)).to(BF16)
                got = kvp.attend8(q, cache, cuda(table), cuda(lens), want_lse=True, want_weights=True)
                near(got, q, cache, table, lens)
                # 500 tokens of at most 1000 that weigh e^10.6 each: 1.2e-5 of the weight, of values that average 0.3 / sqrt(500) over them: 1.7e-7 = 2^-22.5 a dim, of 128 dims and more
                assert bool(got["out"].abs().amax() > high * 2.0 ** -24) and abs(float(got["weights"].sum()) - rows) < 1e-4 * rows


@pytest.mark.parametrize("d,rows", [(64, 8), (64, 16), (128, 6), (128, 12), (128, 33), (256, 8), (256, 20)])
def test_a_weight_keeps_fourteen_bits(kvp, d, rows):  # noqa: F811
    """A few tokens with values in dims of their own: out is the weights themselves, times numbers that 8 bits hold. A weight is three terms, each the nearest of four significant bits to
    what the ones before leave, 2^-5 of it at most: the third is off by 2^-14 of the weight, and the first remainder is rounded to fp16, 2^-16 of the weight. Together below 2^-13.
    fp16 outputs are rounded by 2^-11 themselves; weights that are as well would add as much again."""
    rng = np.random.default_rng(d + rows)
    for n in (2, 3, 5, 8):
        k, v = rng.standard_normal((n, 1, d)), np.zeros((n, 1, d))
        for i in range(n):
            v[i, 0, i::n] = 1.0
        cache, table, lens = filled(kvp, k, v)
        for _ in range(4):
            q = cuda((rng.standard_normal((1, 1, rows, d)) * 1.5).astype(np.float32)).to(F16)
            near(kvp.attend8(q, cache, cuda(table), cuda(lens)), q, cache, table, lens, terms=2.0 ** -13)


@pytest.mark.parametrize("rows", [1, 8, 12, 40])
@pytest.mark.parametrize("power", [0, -30, -13, 12, 25])
def test_lse_and_weights_beside_values_of_any_size(kvp, power, rows):  # noqa: F811
    """Values of size 2^x: scores are kept with an offset of x, whose rounding adds 2^-24 * (|x| + 4) in the exponent to base 2, once to the maximum and once to a score: 2^-23 * (|x| + 4)
    on top of what test_gpu_attend8.py allows. Scores are small, and one sequence has a single token, so that this is most of it."""
    d, n = 128, 900
    rng = np.random.default_rng(rows)
    k, v = rng.standard_normal((2, n, 2, d))
    q = cuda((rng.standard_normal((2, 1, 2 * rows, d)) * 1e-3).astype(np.float32)).to(BF16)
    cache, table, lens = filled(kvp, k, v * 2.0 ** power)
    table, lens = np.repeat(table, 2, 0), np.array([n, 1], np.int32)
    got = kvp.attend8(q, cache, cuda(table), cuda(lens), unit_tokens=16, want_lse=True, want_weights=True)
    want = plain.attend(q.double().cpu().numpy(), cache.cpu().numpy(), table, lens, 16, float(np.float32(d ** -0.5)))
    extra = 2.0 ** -23 * (abs(power) + 4)
    score = 16 * 2.0 ** -23 * want["reach"] + 2.0 ** -22 * (want["wide"] + want["high"] + 1) + extra
    off = np.abs(got["lse"].double().cpu().numpy() - want["lse"])
    assert np.all(off <= score + 4 * 2.0 ** -23 * np.abs(want["lse"])), off.max()
    off = np.abs(got["weights"].double().cpu().numpy() - want["weights"])
    assert np.all(off <= want["weights"] * (2 * score.max() + 8 * 2.0 ** -23 * np.abs(want["lse"]).max() + 2.0 ** -20)), off.max()


@pytest.mark.parametrize("rows", [4, 20])
@pytest.mark.parametrize("size,large", [(1.0, np.inf), (1e-12, np.inf), (1e20, 1e-15), (1.0, 2.0 ** 60), (2.0 ** -80, 2.0 ** 10)])
def test_weights_beside_values_of_another_size(kvp, size, large, rows):  # noqa: F811
    """A block whose values are 2^60 times or more as large (or small) as the others', with much more weight, or much less: units of small weight keep it, and lse is right.
    Tolerance as in test_gpu_attend8.py: weights 2 * score + 8 * 2^-23 |lse| + 2^-20 of themselves, lse score + 4 * 2^-23 |lse|; the offset of the scores adds 2^-23 * 99 to `score` at most, and
    beside values of 2^100 (what infinities count as) a weight below 2^-27 of the largest may be 0: 2^-27 a row and token, on either side."""
    d, n = 128, 700
    rng = np.random.default_rng(11)
    for where in (0, 304, 688):
        for weight in (110.0, -110.0):                         # scores of +-19 beside the others', e^19 = 2^28
            k, v = rng.standard_normal((2, n, 1, d)) * 0.3
            v = v * size
            k[where: where + 12, 0, 0] = weight
            v[where: where + 12] = large * np.sign(v[where: where + 12])
            cache, table, lens = filled(kvp, k, v)
            q = rng.standard_normal((1, 1, rows, d)) * 0.2
            q[..., 0] = 2.0
            q = cuda(q.astype(np.float32)).to(BF16)
            got = kvp.attend8(q, cache, cuda(table), cuda(lens), unit_tokens=16, want_lse=True, want_weights=True)
            want = plain.attend(q.double().cpu().numpy(), cache.cpu().numpy(), table, lens, 16, float(np.float32(d ** -0.5)))
            score = 16 * 2.0 ** -23 * want["reach"] + 2.0 ** -22 * (want["wide"] + want["high"] + 1) + 2.0 ** -23 * 99
            gone = 2.0 ** -27 if np.isinf(large) else 0.0
            off = np.abs(got["lse"].double().cpu().numpy() - want["lse"])
            assert np.all(off <= score + 4 * 2.0 ** -23 * np.abs(want["lse"]) + n * gone), off.max()
            off = np.abs(got["weights"].double().cpu().numpy() - want["weights"])
            room = want["weights"] * (2 * score.max() + 8 * 2.0 ** -23 * np.abs(want["lse"]).max() + 2.0 ** -20 + n * gone) + 16 * rows * gone
            assert np.all(off <= room), (off / np.maximum(room, 1e-300)).max()
            near(got, q, cache, table, lens)
