"""Block tables and slot maps against a plain program that goes through the requests one by one. All numbers are equal."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache8_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvp():
    from paper_2508_13231_b200 import kvp
    return kvp


def pool(rng, batch, width, page, free, most=1.0, holes=0.0):
    """lens, table, ring, state of a pool in use."""
    lens = (rng.random(batch) ** 2 * most * width * page).astype(np.int32)
    lens[rng.random(batch) < 0.2] = 0
    used = -(-lens // page)
    pages = int(used.sum()) + free + 3
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((batch, width), -1, np.int32)
    at = 0
    for i, n in enumerate(used):
        table[i, :n] = order[at: at + n]
        at += n
    table[(rng.random(table.shape) < holes) & (table >= 0)] = pages + 7
    head = int(rng.integers(pages))
    ring = np.full(pages, -5, np.int32)
    ring[(head + np.arange(free)) % pages] = order[at: at + free]
    return lens, table, ring, np.array([head, free], np.int32)


def check(kvp, new, lens, table, ring, state, page, tokens, **kw):
    dev = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (new, lens, table, ring, state)]
    got = kvp.block_tables(*dev, page, tokens, **kw)
    want = plain.tables(new, lens, table, ring, state, page, tokens)
    got = dict(got, table=dev[2], ring=dev[3])
    assert set(got) == set(want)
    for k in want:
        assert np.array_equal(got[k].cpu().numpy(), want[k]), k
    return dev, want


@pytest.mark.parametrize("batch,width,page,tokens,new,free", [(1, 1, 16, 1, 1, 1), (1, 4, 16, 40, 33, 3), (7, 9, 16, 7, 1, 2), (33, 20, 32, 60, 2, 40),
                                                              (256, 64, 16, 256, 1, 30), (300, 40, 1, 4096, 20, 9000), (64, 128, 48, 4097, 100, 200),
                                                              (1500, 12, 16, 5000, 4, 900), (3000, 3, 16, 3000, 1, 5000), (40, 600, 64, 131072, 5000, 1700)])
@pytest.mark.parametrize("leave", [0.0, 0.2])
def test_tables(kvp, batch, width, page, tokens, new, free, leave):
    rng = np.random.default_rng(batch + tokens)
    lens, table, ring, state = pool(rng, batch, width, page, free, holes=0.05 if leave else 0.0)
    n = rng.integers(0, 2 * new + 1, batch).astype(np.int32) if new > 1 else np.ones(batch, np.int32)
    n[rng.random(batch) < leave] = -1
    check(kvp, n, lens, table, ring, state, page, tokens)


def test_tables_who_is_granted(kvp):
    """Too few pages, too few tokens, a row that is full; requests that ask for nothing of what is short are served all the same."""
    page, width = 16, 4
    lens = np.array([15, 16, 0, 64, 17, 1, 63, 0, -4, 999], np.int32)
    new = np.array([1, 1, 33, 1, 2, 0, 1, 2 ** 31 - 1, 1, -2], np.int32)
    table = np.arange(40, dtype=np.int32).reshape(10, 4)
    ring = np.arange(100, dtype=np.int32)
    for count in (0, 1, 3, 4, 5, 30):
        for tokens in (0, 1, 3, 36, 37, 60):
            check(kvp, new, lens, table, ring, np.array([90, count], np.int32), page, tokens)


def test_tables_everyone_leaves(kvp):
    rng = np.random.default_rng(5)
    lens, table, ring, state = pool(rng, 70, 100, 16, 10, holes=0.1)
    check(kvp, np.full(70, -1, np.int32), lens, table, ring, state, 16, 8)


def test_tables_in_place_over_many_steps(kvp):
    """A pool that lives in place, also in a graph that is replayed: no page is held twice or lost."""
    rng = np.random.default_rng(9)
    batch, width, page, pages = 24, 30, 16, 400
    lens, table = np.zeros(batch, np.int32), np.full((batch, width), -1, np.int32)
    ring, state = rng.permutation(pages).astype(np.int32), np.array([0, pages], np.int32)
    dev = [torch.from_numpy(x).cuda() for x in (np.zeros(batch, np.int32), lens, table, ring, state)]
    graph = torch.cuda.CUDAGraph()
    call = lambda: kvp.block_tables(*dev, page, 512, lens_out=dev[1], state_out=dev[4])  # noqa: E731
    call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = call()
    for step in range(40):
        new = np.where(rng.random(batch) < 0.3, rng.integers(0, 120, batch), 1).astype(np.int32)
        new[rng.random(batch) < 0.1] = -1
        want = plain.tables(new, lens, table, ring, state, page, 512)
        dev[0].copy_(torch.from_numpy(new))
        if step % 2:
            graph.replay()
            r = got
        else:
            r = call()
        for k in ("slots", "positions", "rows", "starts", "page_starts", "granted"):
            assert np.array_equal(r[k].cpu().numpy(), want[k]), (step, k)
        lens, table, ring, state = (want[k].astype(np.int32) for k in ("lens", "table", "ring", "state"))
        for x, k in ((dev[1], lens), (dev[2], table), (dev[3], ring), (dev[4], state)):
            assert np.array_equal(x.cpu().numpy(), k)
        used = [int(p) for i in range(batch) for p in table[i, : -(-lens[i] // page)]]
        free = [int(ring[(state[0] + i) % pages]) for i in range(state[1])]
        assert sorted(used + free) == list(range(pages))


def test_tables_refuse(kvp):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    ok = dict(new_tokens=i32(3), lens=i32(3), table=i32(3, 4), ring=i32(20), state=i32(2), page_tokens=16, tokens=5)
    kvp.block_tables(**ok)
    for kw in (dict(new_tokens=i32(2)), dict(lens=i32(4)), dict(table=i32(12)), dict(state=i32(3)), dict(lens=torch.zeros(3, device="cuda")), dict(ring=i32(20).cpu()),
               dict(table=i32(3, 8)[:, ::2]), dict(lens_out=i32(2)), dict(state_out=i32(1)), dict(tokens=-1)):
        with pytest.raises(ValueError):
            kvp.block_tables(**dict(ok, **kw))
    for kw, code in ((dict(page_tokens=0), kvp.ERR_ARG), (dict(ring=i32(0)), kvp.ERR_ARG), (dict(page_tokens=2 ** 29), kvp.ERR_RANGE)):
        with pytest.raises(kvp.KvpError) as e:
            kvp.block_tables(**dict(ok, **kw))
        assert e.value.code == code
