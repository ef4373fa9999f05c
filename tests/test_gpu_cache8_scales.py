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
