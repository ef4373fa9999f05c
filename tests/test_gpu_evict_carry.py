"""Eviction as a cache has it (carry): what a step leaves out stays out, units that come are candidates, and attention over the units kept sees the
token that opens a new one. The form it is compared with goes by sets of units, one at a time; nothing of it comes from the other plain forms."""
import ctypes
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache_plain as plain  # noqa: E402
from test_gpu_attend import check  # noqa: E402

pytestmark = pytest.mark.gpu
MOST = 2 ** 48 - 1


@pytest.fixture(scope="module")
def kvp():
    from paper_2508_13231_b200 import kvp
    return kvp


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def rows_of(t, groups, n):
    """A row (or rows) of kept as truth values [..., groups, n]."""
    words = t.cpu().numpy().view(np.uint32)
    return np.unpackbits(words.view(np.uint8), axis=-1, bitorder="little")[..., : groups * n].reshape(*words.shape[:-1], groups, n).astype(bool)


class Cache:
    """One group: the sums of its units, and the units that were evicted."""

    def __init__(self, n, acc=None, evicted=()):
        self.n, self.acc, self.evicted = n, [0] * n if acc is None else [min(max(int(x), 0), MOST) for x in acc], set(evicted)

    def step(self, weights, exist, budget, sink, recent, decay):
        for u, w in enumerate(weights):
            gain = 0 if not w > 0 else round(min(float(w), 128.0) * 2 ** 24)        # Python rounds ties to even
            self.acc[u] = min(self.acc[u] * decay // 65536 + gain, MOST)
        exist = min(max(exist, 0), self.n)
        always = {u for u in range(exist) if u < sink or u >= exist - recent}
        others = sorted((u for u in range(exist) if u not in always and u not in self.evicted), key=lambda u: (-self.acc[u], u))
        self.evicted = set(range(exist)) - always - set(others[: max(0, budget - len(always))])
        return [u not in self.evicted for u in range(self.n)]


@pytest.mark.parametrize("groups,n,steps,born,budget,sink,recent,decay", [
    (1, 8, 6, 1, 3, 0, 0, 65536), (3, 40, 30, 1, 12, 1, 0, 65536), (2, 65, 20, 3, 10, 0, 2, 60000), (2, 300, 25, 7, 40, 1, 0, 65536),
    (1, 1000, 12, 40, 100, 4, 8, 64881), (2, 4096, 6, 300, 700, 1, 0, 65536), (1, 4095, 5, 90, 3000, 0, 0, 65536), (1, 7000, 4, 10, 500, 1, 4, 65536),
    (1, 20000, 3, 1000, 2000, 0, 0, 50000), (3, 32, 5, 0, 9, 0, 0, 65536)])
def test_a_growing_cache(kvp, groups, n, steps, born, budget, sink, recent, decay):
    rng = np.random.default_rng(n + steps)
    exist = np.clip(n - born * (steps - 1 - np.arange(steps))[:, None] - rng.integers(0, 2, (1, groups)), 0, n).astype(np.int32)
    w = (rng.random((steps, groups, n)) ** 4).astype(np.float32)
    w[:, :, : n // 3] = np.round(w[:, :, : n // 3] * 4) / 4                 # ties
    for s in range(steps):
        for g in range(groups):
            w[s, g, exist[s, g]:] = 0                                       # what is not there receives nothing
            w[s, g, max(0, exist[s, g] - 2): exist[s, g]] *= 3              # the newest are often heavy
    acc = (rng.random((groups, n)) * 2 ** 24).astype(np.int64)
    kept = rng.random((groups, n)) < 0.8
    kept[np.arange(n)[None] >= exist[0][:, None]] = True
    for state in (False, True):
        caches = [Cache(n, acc[g] if state else None, np.flatnonzero(~kept[g]) if state else ()) for g in range(groups)]
        want = [[c.step(w[s, g], int(exist[s, g]), budget, sink, recent, decay) for g, c in enumerate(caches)] for s in range(steps)]
        kw = dict(acc=cuda(acc.reshape(-1)), kept=cuda(plain.pack(kept.reshape(-1)).view(np.int32))) if state else {}
        got = kvp.evict(cuda(w.reshape(steps, -1)), groups, budget, sink=sink, recent=recent, decay_q=decay, exist=cuda(exist), carry=True, **kw)
        assert np.array_equal(rows_of(got["kept"], groups, n), np.array(want))
        assert np.array_equal(got["acc"].cpu().numpy().reshape(groups, n), np.array([c.acc for c in caches]))
        # one step at a time, each with the row before
        row, sums = kw.get("kept"), kw.get("acc")
        for s in range(steps):
            one = kvp.evict(cuda(w[s].reshape(-1)), groups, budget, sink=sink, recent=recent, decay_q=decay, exist=cuda(exist[s]), carry=True, kept=row, acc=sums)
            row, sums = one["kept"][0].clone(), one["acc"]
            assert torch.equal(row, got["kept"][s])
        assert torch.equal(sums, got["acc"])


def test_new_units_are_candidates_without_recent(kvp):
    """Units of one token, the newest with most of the weight at every step, one and three new units a step, none protected."""
    n, budget = 48, 6
    for born in (1, 3):
        cache, kept, acc = Cache(n), None, None
        for s in range(12):
            here = 9 + born * s
            w = np.zeros(n, np.float32)
            w[:here] = 0.1 / here
            w[here - born] += 0.9                                # the first of the new ones
            r = kvp.evict(cuda(w), 1, budget, kept=kept, acc=acc, exist=torch.tensor([here], dtype=torch.int32, device="cuda"), carry=True)
            kept, acc = r["kept"][0].clone(), r["acc"]
            want = cache.step(w, here, budget, 0, 0, 65536)
            got = rows_of(kept, 1, n)[0]
            assert got.tolist() == want and got[here:].all() and got[:here].sum() == budget
            assert got[here - born] or s >= budget               # from then on as many older ones have received 0.9 and a little more


def test_evicted_units_stay_evicted(kvp):
    """A unit whose sum grows again after it was left out does not come back; without carry every step is a choice by itself."""
    w = np.zeros((3, 8), np.float32)
    w[0, :4], w[1, 4:], w[2, 6] = 1, 5, 5
    carried = rows_of(kvp.evict(cuda(w), 1, 4, carry=True)["kept"], 1, 8)[:, 0]
    single = rows_of(kvp.evict(cuda(w), 1, 4)["kept"], 1, 8)[:, 0]
    assert [np.flatnonzero(r).tolist() for r in carried] == [[0, 1, 2, 3]] * 3
    assert [np.flatnonzero(r).tolist() for r in single] == [[0, 1, 2, 3], [4, 5, 6, 7], [4, 5, 6, 7]]


@pytest.mark.parametrize("unit,born,recent", [(1, 1, 0), (1, 3, 0), (1, 3, 2), (16, 1, 1), (4, 3, 1)])
def test_a_serving_loop_sees_its_own_tokens(kvp, unit, born, recent):
    """Two sequences, `born` tokens a step: a query attends to its own token even where that opens a unit, and to all that was never evicted."""
    heads, group, d, page, budget, steps = 2, 2, 64, 16, 20 if unit == 1 else 4, 20
    starts = [60, 37]
    columns = 9
    n = columns * page // unit
    rng = np.random.default_rng(unit + born)
    cache = torch.full((2 * columns, heads, kvp.cache_page_bytes(d, page)), 255, dtype=torch.uint8, device="cuda")
    table = rng.permutation(2 * columns).reshape(2, columns).astype(np.int32)
    total = max(starts) + born * steps
    k, v = (torch.randn(2, total, heads, d, device="cuda") for _ in range(2))
    slot = lambda b, t: int(table[b, t // page]) * page + t % page  # noqa: E731
    for b in range(2):
        slots = torch.tensor([slot(b, t) for t in range(starts[b])], device="cuda")
        kvp.cache_append(cache, k[b, : starts[b]], v[b, : starts[b]], slots)
    caches = [Cache(n) for _ in range(2 * heads)]
    kept = torch.full((-(-2 * heads * n // 32),), -1, dtype=torch.int32, device="cuda")
    acc = torch.zeros(2 * heads * n, dtype=torch.int64, device="cuda")
    for s in range(steps):
        lens = np.array([x + born * (s + 1) for x in starts], np.int32)
        for b in range(2):
            at = range(int(lens[b]) - born, int(lens[b]))
            kvp.cache_append(cache, k[b, at.start: at.stop], v[b, at.start: at.stop], torch.tensor([slot(b, t) for t in at], device="cuda"))
        seen = np.array([[u not in c.evicted for u in range(n)] for c in caches])
        q = torch.randn(2, born, heads * group, d, device="cuda").half()
        got = check(kvp, q, cache, table, lens, plain.pack(seen.reshape(-1)), unit)
        loop = kvp.attend(q, cache, cuda(table), cuda(lens), unit_tokens=unit, units=kept, want_lse=True, want_weights=True)
        assert torch.equal(loop["out"], got["out"]) and torch.equal(loop["lse"], got["lse"]) and torch.equal(loop["weights"], got["weights"])
        w = loop["weights"].view(-1)
        exist = -(-lens // unit)
        assert bool((loop["weights"][torch.arange(2), :, torch.from_numpy(exist).long() - 1] > 0).all())    # the last token's unit
        r = kvp.evict(w, 2 * heads, budget, sink=1, recent=recent, acc=acc, acc_out=acc, kept=kept, exist=cuda(np.repeat(exist, heads).astype(np.int32)), carry=True)
        kept = r["kept"][0].clone()
        host = w.view(2 * heads, n).cpu().numpy()
        want = [c.step(host[i], int(exist[i // heads]), budget, 1, recent, 65536) for i, c in enumerate(caches)]
        assert np.array_equal(rows_of(kept, 2 * heads, n), np.array(want))


def test_carry_in_a_graph(kvp):
    """A captured step whose row is handed on between replays."""
    n, steps, budget = 64, 10, 9
    rng = np.random.default_rng(1)
    w = torch.zeros(n, device="cuda")
    kept = torch.full((2,), -1, dtype=torch.int32, device="cuda")
    acc = torch.zeros(n, dtype=torch.int64, device="cuda")
    exist = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = kvp.evict(w, 1, budget, kept=kept, acc=acc, acc_out=acc, exist=exist, carry=True)
        kept.copy_(r["kept"][0])
    acc.zero_()
    kept.fill_(-1)
    cache = Cache(n)
    for s in range(steps):
        row = rng.random(n).astype(np.float32)
        row[30 + 2 * s:] = 0
        w.copy_(cuda(row))
        exist.fill_(30 + 2 * s)
        graph.replay()
        assert rows_of(kept, 1, n)[0].tolist() == cache.step(row, 30 + 2 * s, budget, 0, 0, 65536)


def test_carry_refuses(kvp):
    w = torch.zeros(3, 32, device="cuda")
    for exist in (torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            kvp.evict(w, 1, 4, exist=exist, carry=True)
    with pytest.raises(ValueError):
        kvp.evict(w, 1, 4, exist=torch.zeros(3, dtype=torch.int32, device="cuda"))
    # a placement policy's units return
    prob = kvp.Problem(32, 8192, 3, torch.ones(3, 1, dtype=torch.int32, device="cuda"), 8, 8 * 10 ** 12, 9 * 10 ** 11, 9 * 10 ** 11)
    out = torch.full((3, 1), -1, dtype=torch.int32, device="cuda")
    for flags, code in ((2, kvp.ERR_ARG), (0, 0)):
        ep = kvp.EvictParams(1, 32, 3, 4, 0, 0, 65536, flags)
        rc = kvp._lib().kvp_policy_accumulated(prob._h, ctypes.byref(ep), ctypes.c_void_p(w.data_ptr()), ctypes.c_void_p(out.data_ptr()), None)
        torch.cuda.synchronize()
        assert rc == code and bool((out == (-1 if flags else 15)).all())
