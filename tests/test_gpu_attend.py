"""The cache held in 4 bits, attention over it, bitmaps of recorded weights and eviction on the GPU, against plain forms in 64 bits.

Tolerances of attention, with u = 2^-8 / 2^-11 the half-step of a bf16 / fp16 output, per value:
  out: u |out| for the output's rounding, 2^-10 + 2^-13 of sum p (|zero| + scale q) for the two fp16 roundings (2^-11 each) that a weight times
  a scale goes through and for what the fp32 steps below move p, and what fp16 cannot hold below its smallest step: a weight is kept as p 8 / p_max times a scale
  over a power of two that is at most twice the largest scale, so each of the n tokens adds at most
  2 * 2^-25 (the two roundings) / 8 * p_max * 15 * 2 * scale <= 2^-23 p_max scale, doubled again for a maximum that lags.
  scores: a score is a sum of at most 40 fp32 sums and products of terms that add up to `reach`, each off by 2^-23 at most (the
  matrix units cut instead of rounding), so it is off by d = 40 * 2^-23 * reach; + 2^-22 for exp2 and log2 and 4 * 2^-23 of |lse| for the
  steps between the two bases. lse is off by that, weights relatively by twice that (score and lse) + 2^-20 for sums in fp32.
"""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def kvp():
    from paper_2508_13231_b200 import kvp
    return kvp


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def dev_bits(words):
    return cuda(words.view(np.int32))


def host_bits(t):
    return t.cpu().numpy().view(np.uint32)


# ---- writing and reading --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,page,heads,tokens,dtype", [(128, 16, 2, 1, BF16), (128, 32, 3, 37, F16), (64, 16, 1, 16, F32), (64, 48, 5, 101, BF16),
                                                       (256, 16, 2, 33, BF16), (256, 64, 1, 70, F32), (128, 16, 8, 130, F16)])
def test_append_and_read(kvp, d, page, heads, tokens, dtype):
    rng = np.random.default_rng(d + page + tokens)
    pages = tokens // page + 3
    x = rng.standard_normal((2, tokens, heads, d)) * np.exp2(rng.integers(-12, 8, (2, tokens, heads, 1)))
    if tokens > 30:
        x[0, 3] = 0.5                                         # all equal
        x[1, 5, 0, :5] = np.nan, np.inf, -np.inf, 1e30, 1e-30
        x[0, 7] *= 1e-9                                       # steps below the smallest of fp16
    k, v = (cuda(y.astype(np.float32)).to(dtype) for y in x)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    if tokens > 20:
        slots[4], slots[9], slots[11] = -1, pages * page, 2 ** 62
    cache = rng.integers(0, 256, (pages, heads, plain.page_bytes(d, page)), dtype=np.uint8)
    dev = cuda(cache)
    kvp.cache_append(dev, k, v, cuda(slots))
    kf, vf = k.float().cpu().numpy(), v.float().cpu().numpy()
    for i, slot in enumerate(slots):
        plain.put(cache, int(slot), kf[i], vf[i])
    assert np.array_equal(dev.cpu().numpy(), cache)           # also: nothing beside the slots is touched
    for out_type in (dtype, F32):
        for got, which in zip(kvp.cache_read(dev, cuda(slots), d, out_type), (0, 1)):
            want = np.stack([plain.read(cache, int(s), d)[which] for s in slots])
            assert torch.equal(got.cpu(), torch.from_numpy(want).to(out_type))


def test_append_strided_and_unaligned_rows(kvp):
    """Keys and values as slices of one fused projection, at an odd offset too; a whole prompt in pages out of order."""
    heads, d, page, tokens = 2, 64, 16, 50
    for shift in (0, 1, 8):
        fused = torch.randn(tokens, 6 * d + 16, device="cuda").to(BF16)
        k, v = fused[:, shift + 2 * d: shift + 4 * d].unflatten(1, (heads, d)), fused[:, shift + 4 * d: shift + 6 * d].unflatten(1, (heads, d))
        slots = torch.tensor([3, 0, 5, 1], device="cuda")[:, None] * page + torch.arange(page, device="cuda")
        slots = slots.view(-1)[:tokens].contiguous()
        a, b = (torch.zeros(6, heads, kvp.cache_page_bytes(d, page), dtype=torch.uint8, device="cuda") for _ in range(2))
        kvp.cache_append(a, k, v, slots)
        kvp.cache_append(b, k.contiguous(), v.contiguous(), slots)
        assert torch.equal(a, b)
        w = np.zeros(a.shape, np.uint8)
        for i, s in enumerate(slots.tolist()):
            plain.put(w, s, k[i].float().cpu().numpy(), v[i].float().cpu().numpy())
        assert np.array_equal(a.cpu().numpy(), w)


# ---- attention ------------------------------------------------------------------------------------------------------

def problem(kvp, b, t, heads, group, d, page, unit, lens, dtype=BF16, keep=1.0, qscale=2.0, vscale=1.0, kscale=1.0, seed=0, columns=None,
            junk=False):
    """A cache with garbage (also NaN scales) everywhere but at the sequences' tokens, and queries."""
    rng = np.random.default_rng(seed + 1000 * d + page)
    columns = columns or max(1, -(-max(max(lens), 1) // page))
    pages = b * columns + 2
    table = rng.permutation(pages)[: b * columns].reshape(b, columns).astype(np.int32)
    cache = torch.full((pages, heads, kvp.cache_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    for i, n in enumerate(lens):
        n = min(max(n, 0), columns * page)
        if n:
            slots = table[i].astype(np.int64)[np.arange(n) // page] * page + np.arange(n) % page
            k = rng.standard_normal((n, heads, d)) * kscale + 0.3
            v = rng.standard_normal((n, heads, d)) * vscale
            kvp.cache_append(cache, cuda(k.astype(np.float32)), cuda(v.astype(np.float32)), cuda(slots))
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
        units = plain.pack(bits.reshape(-1))
    return q, cache, table, np.array(lens, np.int32), units


def check(kvp, q, cache, table, lens, units, unit, scale=None, **kw):
    d = q.shape[-1]
    scale = d ** -0.5 if scale is None else scale
    got = kvp.attend(q, cache, cuda(table), cuda(lens), unit_tokens=unit, scale=scale, units=None if units is None else dev_bits(units),
                     want_lse=True, want_weights=True, **kw)
    want = plain.attend(q.double().cpu().numpy(), cache.cpu().numpy(), table, lens, unit, float(np.float32(scale)), units)
    out, lse, weights = (got[k].double().cpu().numpy() for k in ("out", "lse", "weights"))
    empty = want["count"] == 0
    assert np.array_equal(np.isneginf(lse), empty)
    assert not out[empty].any()
    score = 40 * 2.0 ** -23 * want["reach"] + 2.0 ** -22
    off = np.where(empty, 0, np.abs(np.where(empty, 0, lse) - np.where(empty, 0, want["lse"])))
    room = score + 4 * 2.0 ** -23 * np.abs(np.where(empty, 0, want["lse"]))
    assert np.all(off <= room), (off / room).max()
    half = 2.0 ** -8 if q.dtype == BF16 else 2.0 ** -11
    room = half * np.abs(want["out"]) + (2.0 ** -10 + 2.0 ** -13 + 2 * score[..., None]) * want["size"] + \
        2.0 ** -31 * (want["count"] * want["top"] * np.maximum(want["vscale"], 1))[..., None] + 2.0 ** -25
    bad = np.abs(out - want["out"]) / room
    assert np.all(bad <= 1), bad.max()
    group = q.shape[2] // weights.shape[1]
    worst = score.reshape(*score.shape[:2], -1, group).max((1, 3))[..., None]
    lmost = np.abs(np.where(empty, 0, want["lse"])).reshape(*score.shape[:2], -1, group).max((1, 3))[..., None]
    room = want["weights"] * (2 * worst + 8 * 2.0 ** -23 * lmost + 2.0 ** -20) + 1e-37
    assert np.all(np.abs(weights - want["weights"]) <= room), (np.abs(weights - want["weights"]) / room).max()
    return got


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens", [[1], [16], [17], [300], [0], [15, 0, 33, 250, -3, 1000]])
def test_attend_lengths(kvp, d, lens):
    check(kvp, *problem(kvp, len(lens), 1, 2, 4, d, 16, 16, lens), 16)


@pytest.mark.parametrize("t,group,heads", [(1, 1, 1), (1, 3, 2), (1, 8, 2), (1, 12, 1), (2, 4, 3), (4, 3, 2), (5, 5, 1), (17, 2, 1), (9, 16, 1)])
def test_attend_heads_and_queries(kvp, t, group, heads):
    # lengths below the number of queries: some queries see nothing
    check(kvp, *problem(kvp, 4, t, heads, group, 64 if t > 4 else 128, 32, 32, [200, t, max(0, t - 1), 1]), 32)


@pytest.mark.parametrize("page,unit", [(16, 1), (16, 2), (16, 4), (16, 8), (16, 16), (32, 32), (64, 16), (64, 64), (48, 48), (48, 16), (96, 48), (32, 1)])
@pytest.mark.parametrize("keep", [1.0, 0.4])
def test_attend_units(kvp, page, unit, keep):
    q, cache, table, lens, units = problem(kvp, 3, 2, 3, 2, 64, page, unit, [403, 120, 777], keep=keep)
    got = check(kvp, q, cache, table, lens, units, unit)
    if keep < 1:
        assert not got["out"][1].any() and not got["weights"][1].any()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attend_types(kvp, dtype):
    check(kvp, *problem(kvp, 2, 1, 2, 4, 128, 16, 16, [500, 333], dtype=dtype), 16)


@pytest.mark.parametrize("qscale,kscale,vscale,scale", [(1e-3, 1.0, 1e-4, None), (1e4, 1e-4, 300.0, None), (30.0, 1.0, 1.0, None), (1.0, 1.0, 1e4, -0.1),
                                                        (1.0, 100.0, 1e-7, 0.0), (0.0, 1.0, 1.0, None), (1e30, 1e-4, 1.0, 1e-27)])
def test_attend_magnitudes(kvp, qscale, kscale, vscale, scale):
    check(kvp, *problem(kvp, 2, 1, 2, 4, 128, 16, 16, [900, 130], qscale=qscale, kscale=kscale, vscale=vscale), 16, scale=scale)


def test_attend_values_whose_size_changes_along_the_sequence(kvp):
    """Scores and values that rise by powers of ten along the sequence: the maximum and the scales' power of two move often."""
    d, page, n = 128, 16, 2000
    rng = np.random.default_rng(3)
    rise = np.linspace(-1, 1, n)[:, None, None]
    k = (rng.standard_normal((n, 2, d)) * 0.1 + rise).astype(np.float32)
    v = (rng.standard_normal((n, 2, d)) * 10.0 ** (3 * rise)).astype(np.float32)
    columns = n // page
    table = rng.permutation(columns).astype(np.int32)[None]
    cache = torch.full((columns, 2, kvp.cache_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    slots = table[0].astype(np.int64)[np.arange(n) // page] * page + np.arange(n) % page
    kvp.cache_append(cache, cuda(k), cuda(v), cuda(slots))
    for sign in (1, -1):
        q = cuda(np.full((1, 1, 8, d), 0.7 * sign, np.float32)).to(F16)
        check(kvp, q, cache, table, np.array([n], np.int32), None, 16)


def test_attend_a_large_batch(kvp):
    """More sequences than a warp goes through by itself."""
    lens = [int(x) for x in np.random.default_rng(2).integers(0, 60, 300)]
    check(kvp, *problem(kvp, 300, 1, 1, 3, 64, 16, 16, lens), 16)


def test_attend_lists_longer_than_a_chunk(kvp):
    """So many tiles that a CTA's list of them comes in several pieces: a bitmap of ones reads what no bitmap reads, in the same order."""
    heads, d, page, tokens = 8, 64, 64, 64 * 9600                        # 307,200 tiles: more than 1024 for each of 296 CTAs
    pages = tokens // page
    cache = torch.empty((pages, heads, kvp.cache_page_bytes(d, page)), dtype=torch.uint8, device="cuda")
    torch.manual_seed(0)
    for at in range(0, tokens, 1 << 16):
        n = min(1 << 16, tokens - at)
        kvp.cache_append(cache, torch.randn(n, heads, d, device="cuda"), torch.randn(n, heads, d, device="cuda"), torch.arange(at, at + n, device="cuda"))
    table = torch.randperm(pages, device="cuda").int()[None]
    lens = torch.tensor([tokens - 5], dtype=torch.int32, device="cuda")
    q = torch.randn(1, 2 * heads, d, device="cuda").to(BF16)
    for unit in (1, 16, 64):
        ones = torch.full((heads * tokens // unit // 32,), -1, dtype=torch.int32, device="cuda")
        a, b = (kvp.attend(q, cache, table, lens, unit_tokens=unit, units=u, want_lse=True, want_weights=True) for u in (None, ones))
        assert all(torch.equal(a[k], b[k]) for k in a)
        assert abs(float(a["weights"].sum()) - 2 * heads) < 1e-3


def test_a_cache_beyond_four_gigabytes(kvp):
    """Tokens in the last pages of a cache of 4.9 GB, against the same tokens in a small one."""
    heads, d, page, tokens = 8, 256, 64, 150
    size = kvp.cache_page_bytes(d, page)
    pages = 30000
    big = torch.zeros((pages, heads, size), dtype=torch.uint8, device="cuda")
    small = torch.zeros((3, heads, size), dtype=torch.uint8, device="cuda")
    k, v = torch.randn(2, tokens, heads, d, device="cuda").to(BF16)
    slots = torch.arange(tokens, device="cuda")
    kvp.cache_append(small, k, v, slots)
    kvp.cache_append(big, k, v, slots + (pages - 3) * page)
    assert torch.equal(big[-3:], small) and not bool(big[:-3].any())
    for x, y in zip(kvp.cache_read(big, slots + (pages - 3) * page, d), kvp.cache_read(small, slots, d)):
        assert torch.equal(x, y)
    q = torch.randn(1, 2 * heads, d, device="cuda").to(BF16)
    lens = torch.tensor([tokens], dtype=torch.int32, device="cuda")
    table = torch.arange(3, dtype=torch.int32, device="cuda")[None]
    a, b = kvp.attend(q, small, table, lens, want_weights=True), kvp.attend(q, big, table + pages - 3, lens, want_weights=True)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["weights"], b["weights"])


@pytest.mark.parametrize("keep", [1.0, 0.1])
def test_attend_long_and_many(kvp, keep):
    check(kvp, *problem(kvp, 2, 1, 2, 2, 128, 32, 32, [20011, 40], keep=keep), 32)                       # many CTAs for one row
    lens = [int(x) for x in np.random.default_rng(1).integers(0, 150, 120)]
    check(kvp, *problem(kvp, 120, 1, 4, 2, 64, 16, 16, lens, keep=keep), 16)                             # many rows for one CTA
    check(kvp, *problem(kvp, 1, 1, 1, 2, 64, 16, 1, [17000], keep=keep), 1)                              # more tiles than are listed at once


def test_attend_skips_pages_that_are_none(kvp):
    for unit, keep in ((16, 1.0), (1, 1.0), (16, 0.5)):
        check(kvp, *problem(kvp, 3, 1, 2, 4, 128, 16, unit, [300, 100, 320], junk=True, columns=20, keep=keep), unit)


def test_attend_cuts_lengths_to_the_table(kvp):
    q, cache, table, lens, _ = problem(kvp, 2, 1, 2, 4, 128, 16, 16, [100, 64], columns=7)
    full = kvp.attend(q, cache, cuda(table), cuda(np.array([64, 64], np.int32)))
    long = kvp.attend(q, cache, cuda(table[:, :4]), cuda(np.array([2 ** 31 - 1, 64], np.int32)))
    assert torch.equal(full["out"], long["out"]) and full["lse"] is None and full["weights"] is None


def test_attend_strided_queries_and_shapes(kvp):
    q, cache, table, lens, _ = problem(kvp, 3, 2, 2, 4, 128, 16, 16, [100, 64, 7])
    want = kvp.attend(q, cache, cuda(table), cuda(lens), want_lse=True, want_weights=True)
    wide = torch.full((3, 2, 20, 131), float("nan"), device="cuda").to(BF16)
    wide[:, :, 5:13, 3:] = q
    got = kvp.attend(wide[:, :, 5:13, 3:], cache, cuda(table), cuda(lens), want_lse=True, want_weights=True)
    turned = kvp.attend(q.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3), cache, cuda(table), cuda(lens), want_lse=True, want_weights=True)
    for other in (got, turned):
        assert all(torch.equal(want[k], other[k]) for k in want)
    one = kvp.attend(q[:, 1], cache, cuda(table), cuda(lens), want_lse=True)
    assert one["out"].shape == (3, 8, 128) and one["lse"].shape == (3, 8)
    # weights written to a row of a recording
    rows = torch.full((2, want["weights"].numel()), -1.0, device="cuda")
    kvp.attend(q, cache, cuda(table), cuda(lens), weights=rows[1])
    assert torch.equal(rows[1], want["weights"].view(-1)) and bool((rows[0] == -1).all())


def test_attend_with_values_that_are_not_finite_in_a_query(kvp):
    """NaN or infinity in one row's query stays in that row (and in the weights of its kv-head)."""
    q, cache, table, lens, _ = problem(kvp, 1, 1, 2, 4, 128, 16, 16, [200])
    want = kvp.attend(q, cache, cuda(table), cuda(lens), want_weights=True)
    q[0, 0, 1, 5], q[0, 0, 2, 7] = float("nan"), float("inf")
    got = kvp.attend(q, cache, cuda(table), cuda(lens), want_weights=True)
    rest = [0, 3, 4, 5, 6, 7]
    assert torch.equal(got["out"][0, 0, rest], want["out"][0, 0, rest]) and torch.equal(got["weights"][0, 1], want["weights"][0, 1])
    assert got["out"][0, 0, 1].isnan().all()


def test_attend_twice_on_streams_and_in_graphs(kvp):
    """Two calls under way at once, and graphs replayed with other lengths: each with the bits of a call of its own."""
    sets = [problem(kvp, 3, 1, 2, 4, 128, 16, 16, [900, 30, 411], keep=k, seed=s) for s, k in ((1, 1.0), (2, 0.5))]
    dev = [(q, c, cuda(t), cuda(n), None if u is None else dev_bits(u)) for q, c, t, n, u in sets]
    call = lambda i, **kw: kvp.attend(dev[i][0], dev[i][1], dev[i][2], dev[i][3], units=dev[i][4], want_lse=True, want_weights=True, **kw)  # noqa: E731
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
                     ((q, cache, t, n), dict(weights=torch.zeros(3, device="cuda"))), ((q, cache, t, n), dict(unit_tokens=-1)),
                     ((q, cache.view(-1)[8: 8 + 3 * 5120].view(3, 2, 2560), t, n), {})):
        with pytest.raises((ValueError, TypeError)):
            kvp.attend(*args, **kw)
    for kw in (dict(unit_tokens=32), dict(unit_tokens=3), dict(scale=float("inf"))):
        with pytest.raises(kvp.KvpError) as e:
            kvp.attend(q, cache, t, n, **kw)
        assert e.value.code == kvp.ERR_ARG
    k = torch.zeros(4, 2, 128, device="cuda")
    s = torch.zeros(4, dtype=torch.int64, device="cuda")
    for args in ((cache, k, k.half(), s), (cache, k.double(), k.double(), s), (cache, k[:, :1], k[:, :1], s), (cache, k, k[:3], s), (cache, k, k, s[:3]),
                 (cache, k, k, s.int()), (cache, k[..., :96], k[..., :96], s), (cache, k, k.transpose(0, 2), s)):
        with pytest.raises(ValueError):
            kvp.cache_append(*args)
    with pytest.raises(ValueError):
        kvp.cache_read(cache, s, 96)
    with pytest.raises(ValueError):
        kvp.cache_read(cache, s, 128, torch.float64)


# ---- recorded weights -----------------------------------------------------------------------------------------------

def weights_of(rng, steps, groups, n, odd=True):
    w = (rng.random((steps, groups, n)) ** 8).astype(np.float32)
    if odd:
        w[rng.random(w.shape) < 0.2] = 0
        w[:, :, : n // 3] = np.round(w[:, :, : n // 3] * 8) / 8         # ties
        w[0, 0] = 0                                                     # a row without weight
        if steps > 1:
            w[1, 0] = 0.125                                             # all equal
            w[1, -1, 0] = np.nan
            w[1, -1, n // 2] = -1
            w[-1, -1, n - 1] = np.inf
    return w.reshape(steps, groups * n)


@pytest.mark.parametrize("groups,n,steps,topk", [(1, 1, 1, 1), (3, 7, 5, 2), (2, 32, 4, 32), (5, 100, 3, 9), (4, 256, 6, 25), (2, 1000, 5, 300),
                                                 (3, 2048, 4, 205), (2, 4096, 3, 205), (1, 8192, 2, 4000), (1, 8193, 2, 100), (2, 20000, 2, 2000), (1, 32768, 2, 33)])
def test_trace_weights(kvp, groups, n, steps, topk):
    w = weights_of(np.random.default_rng(n), steps, groups, n)
    got = kvp.trace_weights(cuda(w), groups, topk)
    assert np.array_equal(host_bits(got), plain.select(w, groups, topk))
    out = torch.full_like(got, -1)
    assert kvp.trace_weights(cuda(w), groups, topk, out=out).data_ptr() == out.data_ptr() and torch.equal(out, got)


@pytest.mark.parametrize("groups,n,steps,budget,sink,recent,decay", [
    (1, 1, 1, 1, 0, 0, 65536), (3, 7, 5, 4, 1, 1, 60000), (2, 32, 4, 32, 0, 0, 65536), (5, 100, 3, 9, 2, 3, 0), (4, 256, 6, 25, 1, 4, 65535),
    (2, 1000, 5, 300, 0, 8, 58982), (3, 2048, 4, 205, 1, 0, 65536), (2, 5000, 3, 0, 0, 0, 65536), (1, 8200, 3, 4000, 4, 4, 65000), (2, 32768, 2, 700, 1, 1, 65536)])
def test_evict(kvp, groups, n, steps, budget, sink, recent, decay):
    rng = np.random.default_rng(n + budget)
    w = weights_of(rng, steps, groups, n) * 8
    u = groups * n
    got = kvp.evict(cuda(w), groups, budget, sink=sink, recent=recent, decay_q=decay)
    rows, acc = plain.evict(w, groups, budget, sink, recent, decay)
    assert np.array_equal(host_bits(got["kept"]), rows) and np.array_equal(got["acc"].cpu().numpy(), acc)
    # a state from before, units already evicted, groups that are not full (one of them empty), sums at their limits
    start = (rng.random(u) ** 4 * 2 ** 30).astype(np.int64)
    start[rng.integers(0, u, 3)] = 2 ** 48 - 1, 2 ** 62, -5
    kept = plain.pack(rng.random(u) < 0.6)
    exist = rng.integers(0, n + 1, groups).astype(np.int32)
    exist[0] = -1 if groups > 1 else n
    exist[-1] = n + 5
    a = cuda(start)
    got = kvp.evict(cuda(w), groups, budget, sink=sink, recent=recent, decay_q=decay, acc=a, kept=dev_bits(kept), exist=cuda(exist))
    rows, acc = plain.evict(w, groups, budget, sink, recent, decay, start, kept, exist)
    assert np.array_equal(host_bits(got["kept"]), rows) and np.array_equal(got["acc"].cpu().numpy(), acc)
    assert np.array_equal(a.cpu().numpy(), start)
    again = kvp.evict(cuda(w), groups, budget, sink=sink, recent=recent, decay_q=decay, acc=a, kept=dev_bits(kept), exist=cuda(exist), acc_out=a)
    assert again["acc"].data_ptr() == a.data_ptr() and torch.equal(a, got["acc"]) and torch.equal(again["kept"], got["kept"])


def test_choices_in_graphs_and_on_streams(kvp):
    """Captured and replayed with other weights, on a stream of their own, in both forms of eviction (many steps of few groups, and one step)."""
    rng = np.random.default_rng(8)
    for groups, n, steps in ((2, 96, 40), (6, 2048, 1), (3, 4096, 12)):
        sets = [weights_of(rng, steps, groups, n) for _ in range(2)]
        w = cuda(sets[0])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        run = lambda **kw: (kvp.evict(w, groups, 30, sink=1, recent=2, decay_q=60000, **kw), kvp.trace_weights(w, groups, 20, **kw))  # noqa: E731
        first = run(stream=side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            caught = run()
        for i in (0, 1, 0):
            w.copy_(cuda(sets[i]))
            graph.replay()
            torch.cuda.synchronize()
            rows, acc = plain.evict(sets[i], groups, 30, 1, 2, 60000)
            assert np.array_equal(host_bits(caught[0]["kept"]), rows) and np.array_equal(caught[0]["acc"].cpu().numpy(), acc)
            assert np.array_equal(host_bits(caught[1]), plain.select(sets[i], groups, 20))
            if i == 0:
                assert torch.equal(first[0]["kept"], caught[0]["kept"]) and torch.equal(first[1], caught[1])


def test_choices_among_equal_weights(kvp):
    """Many units with the same sum, few above them: the lowest indices are chosen, in every size of row and both forms."""
    for n in (5, 200, 4096, 7000, 32768):
        for steps in (1, 3):
            w = np.full((steps, n), 0.25, np.float32)
            w[:, n // 2:: 97] = 0.5
            w[:, 1:: 131] = 0
            many = max(1, n // 3)
            assert np.array_equal(host_bits(kvp.trace_weights(cuda(w), 1, many)), plain.select(w, 1, many))
            rows, acc = plain.evict(w, 1, many, 0, 0, 65536)
            got = kvp.evict(cuda(w), 1, many)
            assert np.array_equal(host_bits(got["kept"]), rows) and np.array_equal(got["acc"].cpu().numpy(), acc)


def test_choices_over_a_long_drift(kvp):
    """Rows whose thresholds move slowly, jump, and come back, sums that share their upper bits, weights that differ in the last bit only."""
    rng = np.random.default_rng(12)
    n, steps = 1500, 60
    w = np.exp(rng.standard_normal(n)[None] + 0.1 * np.cumsum(rng.standard_normal((steps, n)), 0)).astype(np.float32)
    w[20] *= 1000
    w[30] = 1 + rng.integers(0, 40, n).astype(np.float32) * np.float32(2.0 ** -23)
    w[40:45] = 0
    w = np.minimum(w, 120).astype(np.float32)
    assert np.array_equal(host_bits(kvp.trace_weights(cuda(w), 1, 100)), plain.select(w, 1, 100))
    start = (2 ** 47 + rng.integers(0, 5000, n)).astype(np.int64)
    for acc, decay in ((None, 65536), (None, 60000), (start, 65536)):
        rows, sums = plain.evict(w, 1, 200, 1, 3, decay, acc)
        got = kvp.evict(cuda(w), 1, 200, sink=1, recent=3, decay_q=decay, acc=None if acc is None else cuda(acc))
        assert np.array_equal(host_bits(got["kept"]), rows) and np.array_equal(got["acc"].cpu().numpy(), sums)
        many = np.tile(w, (1, 3))                             # three groups alike: the other form for as many steps
        got = kvp.evict(cuda(many), 3, 200, sink=1, recent=3, decay_q=decay, acc=None if acc is None else cuda(np.tile(acc, 3)))
        bits = np.stack([plain.bit(r, np.arange(n)) for r in rows]).astype(bool)
        assert np.array_equal(host_bits(got["kept"]), plain.pack(np.tile(bits, (1, 3))))


def test_evict_step_by_step_is_the_whole_walk(kvp):
    w = weights_of(np.random.default_rng(4), 9, 4, 96)
    whole = kvp.evict(cuda(w), 4, 20, sink=1, recent=2, decay_q=60000)
    acc = None
    for s in range(9):
        r = kvp.evict(cuda(w[s]), 4, 20, sink=1, recent=2, decay_q=60000, acc=acc)
        acc = r["acc"]
        assert torch.equal(r["kept"][0], whole["kept"][s])
    assert torch.equal(acc, whole["acc"])


@pytest.mark.parametrize("groups,n,steps,decay", [(110, 4096, 9, 65536), (150, 3000, 7, 61000), (60, 8192, 4, 65536), (20, 16384, 4, 65536), (14, 30000, 3, 65000)])
def test_evict_many_groups(kvp, groups, n, steps, decay):
    """Enough units for the form that walks the steps of a group in one CTA."""
    w = weights_of(np.random.default_rng(n), steps, groups, n) * 4
    rows, acc = plain.evict(w, groups, n // 10, 1, 4, decay)
    got = kvp.evict(cuda(w), groups, n // 10, sink=1, recent=4, decay_q=decay)
    assert np.array_equal(host_bits(got["kept"]), rows) and np.array_equal(got["acc"].cpu().numpy(), acc)


@pytest.mark.parametrize("groups,n,steps", [(3, 96, 12), (3, 96, 5), (3, 96, 1), (2, 4096, 3), (1, 8192, 2), (2, 4096, 20)])
def test_policy_accumulated(kvp, groups, n, steps):
    w = weights_of(np.random.default_rng(6), steps, groups, n)
    access = kvp.trace_weights(cuda(w), groups, 10)
    prob = kvp.Problem(groups * n, 8192, steps, access, 80, 8 * 10 ** 12, 9 * 10 ** 11, 9 * 10 ** 11)
    for kw, budget in ((dict(), 80 // groups), (dict(budget=20, sink=1, recent=3, decay_q=62000), 20)):
        got = prob.policy_accumulated(cuda(w), groups, **kw)
        want, _ = plain.evict(w, groups, budget, kw.get("sink", 0), kw.get("recent", 0), kw.get("decay_q", 65536), before=True)
        assert np.array_equal(host_bits(got), want)
        ev = prob.eval(got)
        assert int(ev["bad_step"][0]) == -1


def test_policy_accumulated_where_everything_fits(kvp):
    w = cuda(weights_of(np.random.default_rng(6), 4, 3, 96))
    prob = kvp.Problem(3 * 96, 8192, 4, kvp.trace_weights(w, 3, 10), 3 * 96, 8 * 10 ** 12, 9 * 10 ** 11, 9 * 10 ** 11)
    assert bool((prob.policy_accumulated(w, 3) == -1).all())


def test_policy_accumulated_refuses(kvp):
    w = cuda(weights_of(np.random.default_rng(6), 4, 3, 96))
    prob = kvp.Problem(3 * 96, 8192, 4, kvp.trace_weights(w, 3, 10), 80, 8 * 10 ** 12, 9 * 10 ** 11, 9 * 10 ** 11)
    for kw, code in ((dict(groups=3, budget=27), kvp.ERR_CAPACITY), (dict(groups=3, budget=97), kvp.ERR_ARG), (dict(groups=5), kvp.ERR_ARG),
                     (dict(groups=0), kvp.ERR_ARG), (dict(groups=3, budget=5, sink=4, recent=2), kvp.ERR_ARG)):
        with pytest.raises(kvp.KvpError) as e:
            prob.policy_accumulated(w, **kw)
        assert e.value.code == code
    with pytest.raises(ValueError):
        prob.policy_accumulated(w[1:], 3)
    birth = torch.zeros(3 * 96, dtype=torch.int32, device="cuda")
    growing = kvp.Problem(3 * 96, 8192, 4, kvp.trace_weights(w, 3, 10), 80, 8 * 10 ** 12, 9 * 10 ** 11, 9 * 10 ** 11, birth=birth)
    with pytest.raises(kvp.KvpError) as e:
        growing.policy_accumulated(w, 3)
    assert e.value.code == kvp.ERR_ARG


def test_a_decode_loop_from_attention_to_the_bound(kvp):
    """As they are used together: tokens appended, attention over what eviction left, its weights recorded and accumulated, then
    the recording's bitmaps as a placement problem, scored and annealed."""
    heads, group, d, page, prompt, steps, budget = 2, 4, 64, 16, 200, 24, 8
    n = 14                                                     # columns of the table = units of 16 tokens
    rng = np.random.default_rng(9)
    cache = torch.full((n, heads, kvp.cache_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    table = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    x = rng.standard_normal((2, prompt + steps, heads, d)).astype(np.float32)
    k, v = cuda(x[0]).to(BF16), cuda(x[1]).to(BF16)
    slots = torch.arange(prompt + steps, device="cuda")
    kvp.cache_append(cache, k[:prompt], v[:prompt], slots[:prompt])
    record = torch.zeros(steps, heads * n, device="cuda")
    acc = torch.zeros(heads * n, dtype=torch.int64, device="cuda")
    kept, plain_acc, plain_kept = None, np.zeros(heads * n, np.int64), None
    for s in range(steps):
        here = prompt + s + 1
        kvp.cache_append(cache, k[here - 1: here], v[here - 1: here], slots[here - 1: here])
        q = cuda((2 * rng.standard_normal((1, 1, heads * group, d))).astype(np.float32)).to(BF16)
        lens = torch.tensor([here], dtype=torch.int32, device="cuda")
        check(kvp, q, cache, table.cpu().numpy(), lens.cpu().numpy(), plain_kept, page)
        kvp.attend(q, cache, table, lens, units=kept, weights=record[s])
        exist = torch.full((heads,), -(-here // page), dtype=torch.int32, device="cuda")
        r = kvp.evict(record[s], heads, budget, sink=1, recent=2, acc=acc, kept=kept, exist=exist, acc_out=acc)
        kept = r["kept"][0]
        rows, plain_acc = plain.evict(record[s: s + 1].cpu().numpy(), heads, budget, 1, 2, 65536, plain_acc, plain_kept, exist.cpu().numpy())
        plain_kept = rows[0]
        assert np.array_equal(host_bits(kept), plain_kept) and np.array_equal(acc.cpu().numpy(), plain_acc)
    access = kvp.trace_weights(record, heads, 4)
    assert np.array_equal(host_bits(access), plain.select(record.cpu().numpy(), heads, 4))
    prob = kvp.Problem(heads * n, kvp.cache_page_bytes(d, page), steps, access, heads * budget, 8 * 10 ** 12, 9 * 10 ** 11, 9 * 10 ** 11)
    look = prob.policy_accumulated(record, heads, sink=1, recent=2)
    ticks = int(prob.eval(look)["total_ticks"][0])
    best = prob.anneal(prob.make_params(chains=32, moves=4000, p0=1e-3, init_mode=kvp.INIT_USER, init_schedule=look))
    assert best["best_ticks"] <= ticks
