"""Attention over the cache in 8 bits where many segments in a row have no tile that one of their rows sees: what their warps hand to each other stays in step."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_attend8 import BF16, F16, check, cuda, kvp, problem  # noqa: E402,F401

pytestmark = pytest.mark.gpu


class Part:
    """Stands for the module in check(): the rows `some` of a call that was made on a larger batch."""

    def __init__(self, got, some):
        self.got, self.some = got, some

    def attend8(self, *args, **kw):
        return {k: None if x is None else x[self.some] for k, x in self.got.items()}


@pytest.mark.parametrize("d,dtype,queries,group", [(128, BF16, 512, 4), (64, F16, 1024, 2), (256, BF16, 100, 3), (128, F16, 40, 1), (64, BF16, 24, 1)])
def test_segments_without_tiles_between_idle_rows(kvp, d, dtype, queries, group):  # noqa: F811
    """Sequences shorter than the queries of the call: only the last segments of each see a token, and a CTA goes through several that see none. Hundreds of
    idle rows of the batch between them make the way from one to the next long. Nothing is recorded, as only then such segments are passed over."""
    lens = [1 + (37 * i) % (queries - 1) for i in range(12)]
    q, cache, table, lens, units = problem(kvp, 12, queries, 2, group, d, 16, 16, lens, dtype=dtype)
    at = np.cumsum([401 if i % 3 == 0 else 2 for i in range(12)])
    some = cuda(at)
    batch = int(at[-1]) + 300
    many_q = torch.full((batch, *q.shape[1:]), 1.0, dtype=dtype, device="cuda")
    many_q[some] = q
    many_table, many_lens = np.zeros((batch, table.shape[1]), np.int32), np.zeros(batch, np.int32)
    many_table[at], many_lens[at] = table, lens
    got = kvp.attend8(many_q, cache, cuda(many_table), cuda(many_lens), want_lse=True)
    idle = torch.ones(batch, dtype=torch.bool, device="cuda")
    idle[some] = False
    assert not got["out"][idle].any() and bool(got["lse"][idle].isneginf().all())
    check(Part(got, some), q, cache, table, lens, units, 16, want_weights=False)


def test_segments_with_tiles_behind_empty_ones(kvp):  # noqa: F811
    """Empty segments, then one with tiles, over and over: an even and an odd number of empty ones before it."""
    for queries in (17, 33, 64, 65, 130):
        lens = [queries - 1, 1, 2, 0, 5, queries, 300, 3]
        check(kvp, *problem(kvp, len(lens), queries, 1, 8, 64, 16, 16, lens), 16, want_weights=False)
