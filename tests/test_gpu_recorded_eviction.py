"""The share of the attention weight that eviction leaves, in the recorded form of the sensitivity study: units that were evicted do not come back."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_evict_carry import Cache  # noqa: E402

pytestmark = pytest.mark.gpu


def test_weight_kept_by_eviction():
    from paper_2508_13231_b200 import figures
    from paper_2508_13231_b200 import workloads as wl
    cfg = wl.RECORDED["recorded_small"]
    h, steps, page = cfg["kv_heads"], cfg["steps"], cfg["unit_tokens"]
    weights, n = figures.record(cfg)
    w = weights.view(steps, h, n).cpu().numpy()
    for share in (0.5, 0.25):
        caches, left = [Cache(n) for _ in range(h)], 0.0
        for s in range(steps):
            if s:
                left += sum(float(w[s, g, u]) for g, c in enumerate(caches) for u in range(n) if u not in c.evicted)
            exist = -(-(cfg["prompt"] + s + 1) // page)
            for g, c in enumerate(caches):
                c.step(w[s, g], exist, max(4, int(share * n)), 1, 2, 65536)
        want = left / float(w[1:].astype(np.float64).sum())
        # float32 sums of 47 steps x 2 heads x 28 units on the other side: far below 2^-24 times their number, relative
        assert abs(figures.weight_kept(weights, cfg, n, share) - want) <= want * steps * h * n * 2.0 ** -24
