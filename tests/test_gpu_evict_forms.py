"""Eviction in each of its forms, against the plain form in whole numbers."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvp():
    from paper_2508_13231_b200 import kvp
    return kvp


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host_bits(t):
    return t.cpu().numpy().view(np.uint32)


@pytest.mark.parametrize("n", [4096, 4000])
def test_sums_are_not_added_to_while_a_row_is_still_chosen(kvp, n):
    """Many groups walk their steps in one CTA each, with the sums in shared memory: the weights of a step are added only when every lane of a
    warp has finished looking at the sums of the step before. Bands around the thresholds of sums without ties end in that branch at most steps."""
    groups, steps, budget = 300, 20, n // 10
    rng = np.random.default_rng(n)
    base = rng.random((1, groups, n)) ** 6
    w = (base * rng.uniform(0.5, 1.5, (steps, groups, n))).astype(np.float32).reshape(steps, groups * n)
    rows, acc = plain.evict(w, groups, budget, 1, 4, 65536)
    dev = cuda(w)
    for _ in range(5):
        got = kvp.evict(dev, groups, budget, sink=1, recent=4)
        assert np.array_equal(host_bits(got["kept"]), rows) and np.array_equal(got["acc"].cpu().numpy(), acc)
