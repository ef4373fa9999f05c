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
def test_sums_are_not_added_to_while_a_row_is_still_chosen(kvp, hooks, n):
    """Many groups walk their steps in one CTA each, with the sums in shared memory: the weights of a step are added only when every lane of a
    warp has finished looking at the sums of the step before. Bands around the thresholds of sums without ties end in that branch at most steps."""
    groups, steps, budget = 300, 20, n // 10
    rng = np.random.default_rng(n)
    base = rng.random((1, groups, n)) ** 6
    w = (base * rng.uniform(0.5, 1.5, (steps, groups, n))).astype(np.float32).reshape(steps, groups * n)
    rows, acc = plain.evict(w, groups, budget, 1, 4, 65536)
    dev = cuda(w)
    hooks(evict_form=1)
    for _ in range(5):
        got = kvp.evict(dev, groups, budget, sink=1, recent=4)
        assert np.array_equal(host_bits(got["kept"]), rows) and np.array_equal(got["acc"].cpu().numpy(), acc)


def drifting(rng, steps, groups, n):
    """Weights whose thresholds move slowly, jump, and come back; rows of equal weights, without weight, with NaN, negative and infinite ones."""
    w = np.exp(rng.standard_normal((groups, n))[None] + 0.1 * np.cumsum(rng.standard_normal((steps, groups, n)), 0))
    w[steps // 3] *= 1000
    w[steps // 2] = 1 + rng.integers(0, 40, (groups, n)) * 2.0 ** -23
    w[steps // 2 + 1: steps // 2 + 4] = 0
    w[steps // 2 + 4] = 0.125
    w[-2, -1, :: 7] = np.nan
    w[-2, -1, 1:: 11] = -3
    w[-1, 0, n // 2] = np.inf
    return w.astype(np.float32).reshape(steps, groups * n)


SIZES = [31, 200, 256, 257, 1500, 4064, 4095, 4096, 7000, 8192, 12000, 16384, 30000, 32768]


@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("form", [1, 2])
def test_both_forms_over_a_long_walk(kvp, hooks, form, n):
    groups, steps = 2 if n < 10000 else 1, 60
    rng = np.random.default_rng(n)
    w = drifting(rng, steps, groups, n)
    hooks(evict_form=form)
    near = (2 ** 47 + rng.integers(0, 5000, groups * n)).astype(np.int64)          # sums that share their upper bits
    full = np.where(rng.random(groups * n) < 0.5, 2 ** 48 - 1 - rng.integers(0, 2 ** 32, groups * n), 2 ** 40).astype(np.int64)   # reach the limit
    for budget, sink, recent, decay, acc in ((n // 10 + 2, 1, 1, 65536, None), (n // 3 + 4, 0, 4, 60000, None), (n // 8 + 1, 1, 0, 65536, near),
                                             (n // 2, 0, 0, 65536, full), (n // 2, 0, 0, 65535, full)):
        rows, sums = plain.evict(w, groups, budget, sink, recent, decay, acc)
        got = kvp.evict(cuda(w), groups, budget, sink=sink, recent=recent, decay_q=decay, acc=None if acc is None else cuda(acc))
        assert np.array_equal(got["acc"].cpu().numpy(), sums)
        assert np.array_equal(host_bits(got["kept"]), rows), (budget, decay)


@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("form", [1, 2])
def test_both_forms_on_equal_sums(kvp, hooks, form, n):
    """Ties across a whole row, with few units above them, and a state from before: evicted units, a group that is not full."""
    steps = 5
    w = np.full((steps, n), 0.25, np.float32)
    w[:, n // 2:: 97] = 0.5
    w[:, 1:: 131] = 0
    hooks(evict_form=form)
    rng = np.random.default_rng(n)
    kept = plain.pack(rng.random(n) < 0.6)
    exist = np.array([n - n // 5], np.int32)
    for budget in (0, 1, n // 3, n):
        for state in (dict(), dict(kept=kept, exist=exist)):
            rows, sums = plain.evict(w, 1, budget, 0, 0, 65536, **state)
            dev = {k: cuda(x.view(np.int32)) for k, x in state.items()}
            got = kvp.evict(cuda(w), 1, budget, **dev)
            assert np.array_equal(got["acc"].cpu().numpy(), sums) and np.array_equal(host_bits(got["kept"]), rows), (budget, bool(state))


@pytest.mark.parametrize("form", [1, 2])
def test_both_forms_as_a_policy(kvp, hooks, form):
    for n, groups in ((200, 3), (4096, 2), (12000, 1)):
        steps = 20
        w = drifting(np.random.default_rng(n), steps, groups, n)
        access = kvp.trace_weights(cuda(w), groups, 5)
        prob = kvp.Problem(groups * n, 8192, steps, access, groups * 40, 8 * 10 ** 12, 9 * 10 ** 11, 9 * 10 ** 11)
        hooks(evict_form=form)
        for decay in (65536, 62000):
            rows, _ = plain.evict(w, groups, 40, 1, 2, decay, before=True)
            assert np.array_equal(host_bits(prob.policy_accumulated(cuda(w), groups, sink=1, recent=2, decay_q=decay)), rows)


def test_a_policys_schedule_is_memory_of_its_own_stream(kvp):
    """A block that the current stream has just given back may still be read there; a schedule written on another stream must not lie in it."""
    groups, n, steps = 2, 2048, 600                                  # 307,200 bytes: a block of its own
    w = cuda(np.random.default_rng(0).random((steps, groups * n)).astype(np.float32))
    prob = kvp.Problem(groups * n, 8192, steps, kvp.trace_weights(w, groups, 5), 80, 8 * 10 ** 12, 9 * 10 ** 11, 9 * 10 ** 11)
    want = prob.policy_accumulated(w, groups)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    last = torch.empty_like(want)
    at = last.data_ptr()
    del last
    got = prob.policy_accumulated(w, groups, stream=side)
    assert got.data_ptr() != at
    side.synchronize()
    assert torch.equal(got, want)
