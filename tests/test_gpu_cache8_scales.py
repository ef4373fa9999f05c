"""The cache held in 8 bits: blocks with bytes that are no scale, and tokens that are all zero; blocks that begin anew."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache8_plain as plain  # noqa: E402
from test_gpu_cache8 import F32, cuda, f64, kvp, random_cache  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,d", [(1, 64), (3, 128), (2, 256)])
def test_zeros_into_a_block_without_a_scale(kvp, heads, d):  # noqa: F811
    """Bytes where a block's scale lies that are no power of two count as nothing held, also when all that comes is 0 (or NaN, which is held as 0): the scale is 0 then, and so is what
    is read and attended to. The keys' scale and the values' by themselves."""
    for bad in (np.nan, np.inf, -1.0, -0.5, 3.0, 1e-45, -np.inf):
        for which in ((0,), (1,), (0, 1)):
            for fill in (0.0, float("nan")):
                dev = torch.full((1, heads, plain.page_bytes(d, 16)), 127, dtype=torch.uint8, device="cuda")       # e4m3 NaN
                scales = np.zeros(2, np.float32)
                scales[list(which)] = bad
                dev[0, :, 32 * d: 32 * d + 8] = cuda(scales.view(np.uint8))
                clean = torch.zeros_like(dev)
                x = torch.full((2, heads, d), fill, device="cuda")
                slots = cuda(np.array([3, 4]))
                for c in (dev, clean):
                    kvp.cache8_append(c, x, x, slots)
                assert torch.equal(dev[0, :, 32 * d: 32 * d + 8], clean[0, :, 32 * d: 32 * d + 8])
                some = slots if len(which) == 1 else cuda(np.arange(16))       # a side whose scale was 0 held nothing, so its other places may be anything
                for a, b in zip(kvp.cache8_read(dev, some, d, F32), kvp.cache8_read(clean, some, d, F32)):
                    assert torch.equal(a, b)
                y = torch.randn(1, heads, d, device="cuda")
                for c in (dev, clean):
                    kvp.cache8_append(c, y, y, cuda(np.array([9])))
                for a, b in zip(kvp.cache8_read(dev, cuda(np.arange(16)), d, F32), kvp.cache8_read(clean, cuda(np.arange(16)), d, F32)):
                    assert torch.equal(a, b)


@pytest.mark.parametrize("d,page,heads", [(64, 16, 2), (128, 32, 1), (256, 48, 1)])
def test_blocks_that_begin_anew_with_some_of_their_tokens(kvp, d, page, heads):  # noqa: F811
    """Runs that contain their block's first place, over blocks that held others: the scales are those of the new tokens alone, the bytes of the places behind them stay as they were
    (nothing reads them), and the other blocks are not touched."""
    rng = np.random.default_rng(d)
    pages = 6
    cache = random_cache(rng, pages, heads, d, page)
    blocks = rng.permutation(pages * page // 16)[:5]
    many = rng.integers(1, 16, 5)
    slots = np.concatenate([b * 16 + np.arange(n) for b, n in zip(blocks, many)]).astype(np.int64)
    k, v = (cuda(x).float() for x in rng.standard_normal((2, len(slots), heads, d)) * 2.0 ** -9)
    dev, before = cuda(cache), cache.copy()
    kvp.cache8_append(dev, k, v, cuda(slots))
    plain.append(cache, f64(k), f64(v), slots)
    got = dev.cpu().numpy()
    assert np.array_equal(got, cache)
    raw, old = (x.reshape(pages, heads, page // 16, -1).transpose(0, 2, 1, 3).reshape(pages * page // 16, heads, -1) for x in (got, before))
    keys, values = plain.places(d)
    for b, n in zip(blocks, many):
        for where in (keys, values):
            assert np.array_equal(raw[b][:, where[n:]], old[b][:, where[n:]])
        for x, field in ((k, 32 * d), (v, 32 * d + 4)):
            scale = np.ascontiguousarray(raw[b][:, field: field + 4]).view(np.float32)[:, 0]
            assert scale.tolist() == [plain.scale_of(float(np.abs(f64(x)[slots // 16 == b][:, j]).max())) for j in range(heads)]
    rest = np.setdiff1d(np.arange(len(raw)), blocks)
    assert np.array_equal(raw[rest], old[rest])
