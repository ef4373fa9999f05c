"""Attention outputs where the values' sizes matter: small values, sizes that change along the sequence, fp16 outputs whose terms cancel.

How far an output may be off, with n tokens, p their weights, p_max the largest, S the largest scale of the values, v = zero + scale q, and
size = sum p (|zero| + scale q). Half a step of fp16 is 2^-11 of a value, or 2^-25 below 2^-14.
  the output's rounding: 2^-8 |out| bf16; 2^-11 |out| fp16, 2^-25 where that is subnormal
  bf16: a weight is rounded to fp16, and its product with a scale again: 2 * 2^-11 of size
  fp16: both are kept as two fp16 terms. What the first leaves is below 2^-11 of it and is rounded to 2^-11 of that, once for the weight, twice for the product:
        3 * 2^-22 of size, and the products of two remainders that are left out, 2^-22: together 2^-20
  fp32: sums over a warp's tiles, the warps and the parts, 64 steps at most where nothing else is said, each off by 2^-23 (the matrix units cut): 2^-17 of size
  scores: off by d = (40 * 2^-23 reach + 2^-22), which moves a weight by d and their sum by d: 2 d size. A query with one number other than
        0 has one product to sum, and 8 steps instead of 40
  below fp16's normal numbers: a weight enters as p / p_max * E with E at least 2^13 and is off by 2^-25; its product with a scale by up to 4 * 2^-25 more
        (a rounding each of the two terms, of what is left, and the weight's times a scale below 2), times q <= 15. Scales are taken times a power of two that makes the
        largest 1 .. 2 if it is below 2^-7 (2^15 at most); from 2 on the weights are taken as much lower. That is n p_max 15 * 2^-23 * 2^-13 * max(128 S, 2^-15)
        for the scales' part and n p_max 2^-38 max(1, S) max |zero| for the zeros'.
Nothing else: the room shrinks with the values.
"""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def kvp():
    from paper_2508_13231_b200 import kvp
    return kvp


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def off(kvp, k, v, q, scale, page=16, steps=40):
    """One sequence: k, v float32 [tokens][heads][d], q [1][T][heads * group][d] -> the largest error over the room for it."""
    n, heads, d = k.shape
    columns = -(-n // page)
    table = np.random.default_rng(n).permutation(columns).astype(np.int32)[None]
    cache = torch.full((columns, heads, kvp.cache_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    slots = table[0].astype(np.int64)[np.arange(n) // page] * page + np.arange(n) % page
    kvp.cache_append(cache, cuda(k.astype(np.float32)), cuda(v.astype(np.float32)), cuda(slots))
    lens = np.array([n], np.int32)
    got = kvp.attend(q, cache, cuda(table), cuda(lens), scale=scale)["out"].double().cpu().numpy()
    want = plain.attend(q.double().cpu().numpy(), cache.cpu().numpy(), table, lens, page, float(np.float32(scale)))
    assert np.isfinite(got).all()
    return (np.abs(got - want["out"]) / room_of(want, q.dtype, np.abs(v).max(), steps)).max()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("std", [1.0, 1e-3, 1e-4, 1e-6])
def test_small_values_under_dominant_tokens_in_every_part(kvp, std, dtype):
    """So many sequences that a warp takes more than a hundred tiles of each of its segments, with a token 12 above the rest among them. All
    sequences and heads are the same tokens, so that one of them is compared with the plain form and the others with the same."""
    n, d, heads, batch, page = 16384, 64, 8, 32, 64
    rng = np.random.default_rng(11)
    k = rng.standard_normal((n, 1, d)).astype(np.float32) * np.float32(0.3)
    k[3:: 16 * 101, 0, 5] = 12.0
    v = ((rng.standard_normal((n, 1, d)) + 2) * std).astype(np.float32)
    columns = n // page
    table = np.random.default_rng(n).permutation(columns).astype(np.int32)
    cache = torch.full((columns, heads, kvp.cache_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    slots = table.astype(np.int64)[np.arange(n) // page] * page + np.arange(n) % page
    kvp.cache_append(cache, cuda(k).expand(-1, heads, -1), cuda(v).expand(-1, heads, -1), cuda(slots))
    q = one_number(d, heads, 5, 1.0, dtype).expand(batch, -1, -1, -1)
    lens = np.full(batch, n, np.int32)
    got = kvp.attend(q, cache, cuda(table)[None].repeat(batch, 1), cuda(lens), scale=1.0)["out"].double().cpu().numpy()
    want = plain.attend(q[:1, :, :1].double().cpu().numpy(), cache[:, :1].contiguous().cpu().numpy(), table[None], lens[:1], page, 1.0)
    room = room_of(want, dtype, np.abs(v).max(), steps=8, sums=256)
    assert np.all(np.abs(got - want["out"]) <= room), (np.abs(got - want["out"]) / room).max()


def room_of(want, dtype, largest, steps=40, sums=64):
    """See the top of the file. largest: of the values, so that no zero is larger but for its rounding."""
    score = (steps * 2.0 ** -23 * want["reach"] + 2.0 ** -22)[..., None]
    half, low, rel = (2.0 ** -8, 0.0, 2.0 ** -10) if dtype == BF16 else (2.0 ** -11, 2.0 ** -25, 2.0 ** -20)
    many, most = (want["count"] * want["top"])[..., None], want["vscale"][..., None]
    return np.maximum(half * np.abs(want["out"]), low) + (rel + sums * 2.0 ** -23 + 2 * score) * want["size"] + \
        many * (15 * 2.0 ** -36 * np.maximum(128 * most, 2.0 ** -15) + 2.0 ** -38 * np.maximum(1, most) * largest * (1 + 2.0 ** -11)) + 1e-300


def one_number(d, heads, at, size, dtype):
    q = torch.zeros(1, 1, heads, d)
    q[..., at] = size
    return q.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("std", [1.0, 1e-2, 1e-3, 1e-4, 1e-5, 1e-6])
def test_small_values_under_one_dominant_token(kvp, std, dtype):
    """A token whose score is 11 above the rest over a long tail that holds most of the weight all the same."""
    n, d = 131001, 64
    rng = np.random.default_rng(7)
    k = rng.standard_normal((n, 1, d)).astype(np.float32)
    k[n // 3, 0, 5] = 11.0
    v = (rng.standard_normal((n, 1, d)) * std + 2 * std).astype(np.float32)
    assert off(kvp, k, v, one_number(d, 1, 5, 1.0, dtype), 1.0, steps=8) <= 1


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("sizes", [(1e-5, 1.0, 1e-5), (1.0, 1e-4), (1e-6, 1e-5, 1e-4, 1e-3, 1e-2, 0.1, 1.0, 10.0, 100.0, 1000.0), (0.0, 1e-4, 0.0), (0.0,),
                                   (300.0, 1e-3), (1e-7,), (3e4, 1e-2, 3e4)])
def test_sizes_that_change_along_the_sequence(kvp, sizes, d, dtype):
    rng = np.random.default_rng(len(sizes) + d)
    n = 1500
    step = np.array(sizes)[np.arange(n) * len(sizes) // n]
    k = rng.standard_normal((n, 2, d)).astype(np.float32)
    v = (rng.standard_normal((n, 2, d)) * step[:, None, None]).astype(np.float32)
    v[step == 0] = 0.75                                              # a scale of 0
    if dtype == F16:
        v = np.clip(v, -6e4, 6e4)
    q = torch.from_numpy(rng.standard_normal((1, 1, 8, d)).astype(np.float32)).to(dtype).cuda()
    assert off(kvp, k, v, q, d ** -0.5) <= 1


@pytest.mark.parametrize("n", [4, 8, 32, 100])
@pytest.mark.parametrize("std", [1.0, 1e-3])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_fp16_outputs_whose_terms_cancel(kvp, n, d, std):
    """Pairs of equal weights and opposite values: the output is far smaller than its terms, so what is rounded away of a weight times a
    scale shows; with one fp16 term for it these would be off by up to four times the room."""
    rng = np.random.default_rng(n)
    k = np.repeat(rng.standard_normal((n // 2, 1, d)), 2, 0).astype(np.float32)
    v = rng.standard_normal((n // 2, 1, d)) * std
    v = np.stack([v, -v], 1).reshape(n, 1, d).astype(np.float32)
    for at in (0, 17, d - 1):
        assert off(kvp, k, v, one_number(d, 1, at, 0.3, F16), 1.0, steps=8) <= 1


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_several_queries_and_a_bitmap_over_small_values(kvp, dtype):
    """The tail of a sequence is seen by some queries only, and units in between are not read: sizes there must not matter."""
    heads, group, d, page, n, t = 2, 4, 128, 16, 700, 3
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((n, heads, d)).astype(np.float32), (rng.standard_normal((n, heads, d)) * 1e-4).astype(np.float32)
    v[160:176] = 1e4 * rng.standard_normal((16, heads, d))           # not read
    columns = -(-n // page)
    table = rng.permutation(columns).astype(np.int32)[None]
    cache = torch.full((columns, heads, kvp.cache_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    slots = table[0].astype(np.int64)[np.arange(n) // page] * page + np.arange(n) % page
    kvp.cache_append(cache, cuda(k), cuda(v), cuda(slots))
    bits = rng.random((heads, columns)) < 0.7
    bits[:, 10] = False
    units = plain.pack(bits.reshape(-1))
    q = torch.from_numpy(rng.standard_normal((1, t, heads * group, d)).astype(np.float32)).to(dtype).cuda()
    lens = np.array([n], np.int32)
    got = kvp.attend(q, cache, cuda(table), cuda(lens), units=cuda(units.view(np.int32)))["out"].double().cpu().numpy()
    want = plain.attend(q.double().cpu().numpy(), cache.cpu().numpy(), table, lens, page, float(np.float32(d ** -0.5)), units)
    assert np.all(np.abs(got - want["out"]) <= room_of(want, dtype, 1e-3))
