"""A decode loop as it is run: block tables, rotary positions, the cache held in 8 bits, attention and eviction, step by step and from one captured graph."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache8_plain as plain  # noqa: E402
from test_gpu_attend8 import check  # noqa: E402

pytestmark = pytest.mark.gpu
B, H, G, D, PAGE, WIDTH, PAGES, ROOM = 4, 2, 4, 64, 32, 12, 40, 300


class Loop:
    """The tensors of a loop; a step takes new tokens per request with their queries, keys and values (padded to `room`)."""

    def __init__(self, kvp):
        self.kvp = kvp
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.new, self.lens, self.table, self.state = i32(B), i32(B), torch.full((B, WIDTH), -1, dtype=torch.int32, device="cuda"), i32(2)
        self.ring = torch.randperm(PAGES, generator=torch.Generator().manual_seed(0)).int().cuda()
        self.state[1] = PAGES
        self.cache = torch.zeros(PAGES, H, kvp.cache8_page_bytes(D, PAGE), dtype=torch.uint8, device="cuda")
        self.frequencies = kvp.rope_frequencies(D // 2, scaling="parts", factor=2.0)[0].cuda()

    def step(self, q, k, v):
        kvp = self.kvp
        t = kvp.block_tables(self.new, self.lens, self.table, self.ring, self.state, PAGE, len(q), lens_out=self.lens, state_out=self.state)
        q, k = kvp.rope(q, k, t["positions"], self.frequencies, interleaved=True)
        kvp.cache8_append(self.cache, k, v, t["slots"])
        # the last new token of every request asks; a request without one asks with what lies there, its answer is not used
        last = (t["starts"][1:] - 1).clamp(min=0).long()
        r = kvp.attend8(q[last], self.cache, self.table, self.lens, unit_tokens=16, cap=20.0, want_lse=True, want_weights=True)
        return dict(r, q=q[last], **{x: t[x] for x in ("slots", "positions", "starts", "granted")})


def tokens(rng, room):
    return [torch.from_numpy(rng.standard_normal((room, h, D))).cuda().bfloat16() for h in (H * G, H, H)]


def follow(want, new):
    """The same step of the plain tables; -> slots"""
    r = plain.tables(new, want["lens"], want["table"], want["ring"], want["state"], PAGE, ROOM)
    want.update({k: r[k].astype(np.int32) for k in ("lens", "table", "ring", "state")})
    return r


def test_a_decode_loop():
    from paper_2508_13231_b200 import kvp
    rng = np.random.default_rng(0)
    loop = Loop(kvp)
    want = dict(lens=np.zeros(B, np.int32), table=loop.table.cpu().numpy(), ring=loop.ring.cpu().numpy(), state=loop.state.cpu().numpy())
    cache = np.zeros(loop.cache.shape, np.uint8)
    plan = [[33, 0, 100, 7], [1, 64, 1, 1], [1, 1, 1, 1], [-1, 1, 1, 0], [50, 1, 1, 1], [1, 1, -1, 1], [1, 1, 200, 1], [3, 1, 1, 900], [1, 1, 1, 1]]
    for new in plan:
        q, k, v = tokens(rng, ROOM)
        loop.new.copy_(torch.tensor(new, dtype=torch.int32))
        got = loop.step(q, k, v)
        t = follow(want, new)
        assert np.array_equal(got["slots"].cpu().numpy(), t["slots"]) and np.array_equal(got["granted"].cpu().numpy(), t["granted"])
        for x in ("lens", "table", "ring", "state"):
            assert np.array_equal(getattr(loop, x).cpu().numpy(), want[x]), x
        turned = kvp.rope(k, None, got["positions"], loop.frequencies, interleaved=True)[0]          # keys as they went into the cache
        near = plain.rope(k.double().cpu().numpy(), t["positions"], loop.frequencies.cpu().numpy(), True)
        assert np.all(np.abs(turned.double().cpu().numpy() - near) <= 2.0 ** -8 * np.abs(near) + 2.0 ** -20)
        plain.append(cache, turned.double().cpu().numpy(), v.double().cpu().numpy(), t["slots"])
        assert np.array_equal(loop.cache.cpu().numpy(), cache)
        again = check(kvp, got["q"][:, None], loop.cache, want["table"], want["lens"], None, 16, cap=20.0)
        assert torch.equal(again["out"][:, 0], got["out"]) and torch.equal(again["weights"], got["weights"])
        kept = kvp.evict(got["weights"].view(1, -1), B * H, WIDTH * 2 // 2, sink=1, recent=1, exist=((loop.lens + 15) // 16).repeat_interleave(H))
        assert kept["kept"].shape[0] == 1


def test_a_captured_step_replayed():
    """The same steps from a graph that is replayed, beside eager ones on another loop: the same bits."""
    from paper_2508_13231_b200 import kvp
    eager, graphed = Loop(kvp), Loop(kvp)
    rng = np.random.default_rng(1)
    q, k, v = tokens(rng, 64)
    warm = Loop(kvp)
    warm.step(q, k, v)                                         # what is set up at a first call is set up outside of the capture
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = graphed.step(q, k, v)
    for new in ([20, 3, 0, 41], [1, 1, 1, 1], [1, 1, -1, 1], [-1, 1, 30, 1], [1, 1, 1, 1]):
        x = tokens(rng, 64)
        for a, b in zip((q, k, v), x):
            a.copy_(b)
        n = torch.tensor(new, dtype=torch.int32)
        eager.new.copy_(n)
        graphed.new.copy_(n)
        want = eager.step(q, k, v)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[x], out[x]) for x in want)
        assert torch.equal(eager.cache, graphed.cache) and torch.equal(eager.table, graphed.table) and torch.equal(eager.lens, graphed.lens)


def test_lengths_that_a_kernel_just_before_makes():
    """A long kernel, block tables in place and attention right behind each other: every part of attention sees the new lengths, also those that come up early."""
    from paper_2508_13231_b200 import kvp
    rng = torch.Generator(device="cuda").manual_seed(3)
    batch, width, pages = 64, 40, 64 * 40
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = torch.zeros(pages, H, kvp.cache8_page_bytes(D, 16), dtype=torch.uint8, device="cuda")
    x = torch.randn(2, pages * 16, H, D, generator=rng, device="cuda").bfloat16()
    kvp.cache8_append(cache, x[0], x[1], torch.arange(pages * 16, device="cuda"))
    table, ring = torch.full((batch, width), -1, dtype=torch.int32, device="cuda"), torch.randperm(pages, generator=rng, device="cuda").int()
    lens, state, new = i32(batch), torch.tensor([0, pages], dtype=torch.int32, device="cuda"), i32(batch)
    q = torch.randn(batch, H * G, D, generator=rng, device="cuda").bfloat16()
    big, at, f = torch.randn(16384, 8, 128, device="cuda").bfloat16(), torch.arange(16384, dtype=torch.int32, device="cuda"), kvp.rope_frequencies(128)[0].cuda()
    for step in range(20):
        new.copy_(torch.randint(0, 60, (batch,), generator=rng, device="cuda"))
        new[torch.rand(batch, generator=rng, device="cuda") < 0.3] = -1                # these have no token then: their rows are zeros
        torch.cuda.synchronize()
        kvp.rope(big, None, at, f)
        kvp.block_tables(new, lens, table, ring, state, 16, 64 * 64, lens_out=lens, state_out=state)
        got = kvp.attend8(q, cache, table, lens, want_lse=True, want_weights=True)
        torch.cuda.synchronize()
        want = kvp.attend8(q, cache, table, lens, want_lse=True, want_weights=True)
        assert all(torch.equal(got[k], want[k]) for k in want), step
        assert bool(got["lse"][lens == 0].isneginf().all()) and not bool(got["out"][lens == 0].any())


def test_the_recorded_study_in_8_bits():
    from paper_2508_13231_b200 import figures
    out, kept = figures.recorded("recorded_small", quick=True, bits=8)
    assert set(out) == {"static", "reactive", "accumulated", "sa_guided"}
    assert all(ticks > 0 and 0 <= hits <= 1 for ticks, hits in out.values()) and out["sa_guided"][0] <= out["accumulated"][0]
    assert all(0 < s <= 1 + 1e-5 for s in kept.values())
