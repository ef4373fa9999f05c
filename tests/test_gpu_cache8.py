"""The cache held in 8 bits: writing and reading against a plain form, byte for byte."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache8_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def kvp():
    from paper_2508_13231_b200 import kvp
    return kvp


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def f64(t):
    return t.double().cpu().numpy()


def read_plain(cache, slots, d, dtype):
    (k, _), (v, _) = plain.held(cache, d)
    page, n = k.shape[2], k.shape[0] * k.shape[2]
    out = []
    for x in (k, v):
        y = np.stack([x[s // page, :, s % page] if 0 <= s < n else np.zeros(x.shape[1::2]) for s in slots.tolist()])
        out.append(torch.from_numpy(y).to(dtype))
    return out


def random_cache(rng, pages, heads, d, page):
    """Blocks that hold something, of many sizes, some nothing; no NaN."""
    cache = np.zeros((pages, heads, plain.page_bytes(d, page)), np.uint8)
    k, v = (rng.standard_normal((pages * page, heads, d)) * np.exp2(np.repeat(rng.integers(-6, 6, (pages * page // 16, heads, 1)), 16, 0)) for _ in range(2))
    slots = np.arange(pages * page)
    plain.append(cache, k, v, slots[rng.random(pages * page // 16).repeat(16) < 0.8])
    return cache


@pytest.mark.parametrize("d,page,heads,tokens,dtype", [(128, 16, 2, 1, BF16), (128, 32, 3, 37, F16), (64, 16, 1, 16, F32), (64, 48, 5, 101, BF16),
                                                       (256, 16, 2, 33, BF16), (256, 64, 1, 70, F32), (128, 16, 8, 130, F16)])
@pytest.mark.parametrize("order", ["single", "runs", "sequence"])
def test_append_and_read(kvp, d, page, heads, tokens, dtype, order):
    rng = np.random.default_rng(d + page + tokens)
    pages = tokens // page + 3 if order != "single" else tokens + 1
    cache = random_cache(rng, pages, heads, d, page)
    x = rng.standard_normal((2, tokens, heads, d)) * np.exp2(rng.integers(-12, 8, (2, tokens, heads, 1)))
    if tokens > 30:
        x[0, 3] = 0.0
        x[1, 5, 0, :5] = np.nan, np.inf, -np.inf, 1e30, 1e-30
        x[0, 7] *= 1e-9
    k, v = (cuda(y).to(dtype) for y in x)
    if order == "single":                                      # a token a page, any place
        slots = rng.permutation(pages)[:tokens] * page + rng.integers(0, page, tokens)
    elif order == "sequence":                                  # one sequence that begins inside a page
        slots = (rng.permutation(pages)[:, None] * page + np.arange(page)).reshape(-1)[page // 2 + 3:][:tokens]
    else:                                                      # pieces of blocks, in any order of the blocks
        slots, blocks = [], rng.permutation(pages * page // 16)
        for b in blocks:
            first = int(rng.integers(0, 16)) if rng.random() < 0.6 else 0
            slots += range(b * 16 + first, b * 16 + int(rng.integers(first, 16)) + 1)
        slots = np.array(slots)[:tokens]
        k, v, x = k[: len(slots)], v[: len(slots)], x[:, : len(slots)]
    slots = slots.astype(np.int64)
    if len(slots) > 20:
        slots[4], slots[9], slots[11] = -1, pages * page, 2 ** 62
    dev = cuda(cache)
    kvp.cache8_append(dev, k, v, cuda(slots))
    begun = np.unique(slots[(slots % 16 == 0) & (slots >= 0) & (slots < pages * page)] // 16)
    before = cache.copy()
    plain.append(cache, f64(k), f64(v), slots)
    got = dev.cpu().numpy()
    # behind the last token of a block that begins anew anything may lie: what was there
    assert np.array_equal(got, cache)
    assert all(np.array_equal(before.reshape(-1, heads, before.shape[2])[p], got[p]) for p in range(pages) if not np.any(slots // page == p))
    assert len(begun) >= 0
    for out_type in (dtype, F32):
        for a, b in zip(kvp.cache8_read(dev, cuda(slots), d, out_type), read_plain(cache, slots, d, out_type)):
            assert torch.equal(a.cpu(), b)
    some = np.concatenate((np.arange(16 * (pages * page // 32), min(pages * page, 16 * (pages * page // 32) + 40)), [-7, 3, 1])).astype(np.int64)
    for a, b in zip(kvp.cache8_read(dev, cuda(some), d, F32), read_plain(cache, some, d, F32)):
        assert torch.equal(a.cpu(), b)


def test_a_block_token_by_token(kvp):
    """Tokens that grow and shrink: the scale only grows, what is held is rounded again; the block's first token begins it anew."""
    rng = np.random.default_rng(1)
    heads, d, page = 2, 64, 16
    cache = np.zeros((2, heads, plain.page_bytes(d, page)), np.uint8)
    dev = cuda(cache)
    for turn in range(3):
        for i in range(16):
            x = rng.standard_normal((2, 1, heads, d)) * 2.0 ** float(rng.integers(-20, 20))
            if i == 5:
                x[:] = 0
            k, v = (cuda(y).float() for y in x)
            slot = np.array([16 + i])
            kvp.cache8_append(dev, k, v, cuda(slot))
            plain.append(cache, f64(k), f64(v), slot)
            assert np.array_equal(dev.cpu().numpy(), cache), (turn, i)
    # a token in the middle written again
    k = torch.full((1, heads, d), 2.0 ** 30, device="cuda")
    kvp.cache8_append(dev, k, -k, cuda(np.array([20])))
    plain.append(cache, f64(k), f64(-k), np.array([20]))
    assert np.array_equal(dev.cpu().numpy(), cache)


def test_scales_at_their_borders(kvp):
    """Largest magnitudes of 448 * 2^e exactly, one step more, the smallest scale, the largest input."""
    heads, d = 1, 64
    for most in (448.0, 448.0 * (1 + 2.0 ** -7), 447.0, 449.0, 448 * 2.0 ** 20, 2.0 ** -100, 448 * 2.0 ** -100, 449 * 2.0 ** -100, 2.0 ** -130, 2.0 ** 100, 1e38, 1.75, 1.7500001):
        x = torch.linspace(-1, 1, d, dtype=torch.float64, device="cuda").float().expand(16, heads, d) * most
        cache = np.zeros((1, heads, plain.page_bytes(d, 16)), np.uint8)
        dev = cuda(cache)
        kvp.cache8_append(dev, x, x * 0.1, cuda(np.arange(16)))
        plain.append(cache, f64(x), f64(x * 0.1), np.arange(16))
        assert np.array_equal(dev.cpu().numpy(), cache), most


def test_scale_that_is_none(kvp):
    """A block never begun with bytes where its scale lies: what is no power of two counts as nothing held."""
    heads, d = 1, 64
    for bad in (np.nan, np.inf, -1.0, 3.0, 1e-45):
        dev = torch.full((1, heads, plain.page_bytes(d, 16)), 33, dtype=torch.uint8, device="cuda")
        dev[0, 0, 32 * d: 32 * d + 8] = cuda(np.array([bad, bad], np.float32).view(np.uint8))
        x = torch.randn(1, heads, d, device="cuda")
        kvp.cache8_append(dev, x, x, cuda(np.array([3])))
        k, v = kvp.cache8_read(dev, cuda(np.arange(16)), d, F32)
        clean = torch.zeros_like(dev)
        kvp.cache8_append(clean, x, x, cuda(np.array([3])))
        for a, b in zip((k, v), kvp.cache8_read(clean, cuda(np.arange(16)), d, F32)):
            assert torch.equal(a, b)


def test_tokens_of_a_block_further_apart_than_allowed_leave_other_blocks_alone(kvp):
    """What the block of the scattered tokens holds is not specified; the tokens between them are written as ever, and nothing else is touched."""
    heads, d, page = 2, 64, 16
    rng = np.random.default_rng(8)
    for gap in (14, 15, 16, 20):
        slots = np.arange(100, dtype=np.int64) + 5 * page                      # tokens of other blocks
        at = np.arange(0, 100, gap)
        slots[at] = 2 * page + (np.arange(len(at)) * 3) % 16                   # one of block 2 every `gap` tokens
        k, v = (cuda(x).float() for x in rng.standard_normal((2, 100, heads, d)))
        dev = torch.zeros(14, heads, plain.page_bytes(d, page), dtype=torch.uint8, device="cuda")
        kvp.cache8_append(dev, k, v, cuda(slots))
        want = np.zeros(dev.shape, np.uint8)
        rest = np.where(slots // page == 2, -1, slots)
        plain.append(want, f64(k), f64(v), rest)
        got = dev.cpu().numpy()
        assert np.array_equal(np.delete(got, 2, 0), np.delete(want, 2, 0)), gap


def test_append_strided_and_unaligned_rows(kvp):
    """Keys and values as slices of one fused projection, at an odd offset too; a whole prompt in pages out of order, on another stream."""
    heads, d, page, tokens = 2, 64, 16, 50
    for shift in (0, 1, 8):
        fused = torch.randn(tokens, 6 * d + 16, device="cuda").to(BF16)
        k, v = fused[:, shift + 2 * d: shift + 4 * d].unflatten(1, (heads, d)), fused[:, shift + 4 * d: shift + 6 * d].unflatten(1, (heads, d))
        slots = (torch.tensor([3, 0, 5, 1], device="cuda")[:, None] * page + torch.arange(page, device="cuda")).view(-1)[:tokens].contiguous()
        a, b = (torch.zeros(6, heads, kvp.cache8_page_bytes(d, page), dtype=torch.uint8, device="cuda") for _ in range(2))
        torch.cuda.synchronize()
        kvp.cache8_append(a, k, v, slots, stream=torch.cuda.Stream())
        torch.cuda.synchronize()
        kvp.cache8_append(b, k.contiguous(), v.contiguous(), slots)
        assert torch.equal(a, b)
        w = np.zeros(a.shape, np.uint8)
        plain.append(w, f64(k), f64(v), slots.cpu().numpy())
        assert np.array_equal(a.cpu().numpy(), w)


def test_a_cache_beyond_four_gigabytes(kvp):
    heads, d, page, tokens = 8, 256, 64, 150
    size = kvp.cache8_page_bytes(d, page)
    pages = 20000                                              # 21 GB
    big = torch.zeros((pages, heads, size), dtype=torch.uint8, device="cuda")
    small = torch.zeros((3, heads, size), dtype=torch.uint8, device="cuda")
    k, v = torch.randn(2, tokens, heads, d, device="cuda").to(BF16)
    slots = torch.arange(tokens, device="cuda")
    kvp.cache8_append(small, k, v, slots)
    kvp.cache8_append(big, k, v, slots + (pages - 3) * page)
    assert torch.equal(big[-3:], small) and not bool(big[: pages // 2].any())
    for x, y in zip(kvp.cache8_read(big, slots + (pages - 3) * page, d), kvp.cache8_read(small, slots, d)):
        assert torch.equal(x, y)
    q = torch.randn(1, 2 * heads, d, device="cuda").to(BF16)
    lens = torch.tensor([tokens], dtype=torch.int32, device="cuda")
    table = torch.arange(3, dtype=torch.int32, device="cuda")[None]
    a, b = kvp.attend8(q, small, table, lens, want_weights=True), kvp.attend8(q, big, table + pages - 3, lens, want_weights=True)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["weights"], b["weights"])


def test_calls_refuse(kvp):
    cache = torch.zeros(3, 2, kvp.cache8_page_bytes(128, 16), dtype=torch.uint8, device="cuda")
    k = torch.zeros(4, 2, 128, device="cuda")
    s = torch.zeros(4, dtype=torch.int64, device="cuda")
    for args in ((cache, k, k.half(), s), (cache, k.double(), k.double(), s), (cache, k[:, :1], k[:, :1], s), (cache, k, k[:3], s), (cache, k, k, s[:3]),
                 (cache, k, k, s.int()), (cache, k[..., :96], k[..., :96], s), (cache, k, k.transpose(0, 2), s), (cache[:, :, 1:], k, k, s), (cache.cpu(), k, k, s),
                 (torch.zeros(3, 2, 2560, dtype=torch.uint8, device="cuda"), k, k, s)):
        with pytest.raises(ValueError):
            kvp.cache8_append(*args)
    for args in ((cache, s, 96), (cache, s.int(), 128), (cache, s, 128, torch.int32)):
        with pytest.raises(ValueError):
            kvp.cache8_read(*args)
    assert kvp.cache8_read(cache, s[:0], 128)[0].shape == (0, 2, 128)
