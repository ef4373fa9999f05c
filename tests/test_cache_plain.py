"""The layout of the cache held in 4 bits and the refusals of its calls, without a GPU."""
import ctypes as C
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache_plain as plain  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    from paper_2508_13231_b200 import build
    h = C.CDLL(build.build_library())
    h.kvp_cache_page_bytes.restype = C.c_uint64
    return h


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_tile_holds_every_number_once(lib, d):
    key, value, meta = plain.places(d)
    numbers = np.concatenate([key.reshape(-1), value.reshape(-1)])
    fields = np.concatenate([m.reshape(-1) for m in meta])
    taken = np.concatenate([np.sort(numbers) // 2, np.sort(np.concatenate([fields, fields + 1]))])
    assert np.array_equal(np.sort(numbers), np.arange(32 * d))
    assert np.array_equal(np.sort(np.concatenate([fields, fields + 1])), np.arange(16 * d, 20 * d))
    assert taken.max() + 1 == 20 * d == lib.kvp_cache_page_bytes(d, 16)
    assert lib.kvp_cache_page_bytes(d, 48) == 60 * d and lib.kvp_cache_page_bytes(d, 8) == 0
    assert lib.kvp_cache_page_bytes(96, 16) == 0


def test_quantising_keeps_values_within_half_a_step():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((50, 128)) * np.exp2(rng.integers(-6, 7, (50, 1)))).astype(np.float32)
    q, scale, zero = plain.quantised(x)
    back = zero.astype(np.float64)[..., None] + scale.astype(np.float64)[..., None] * q
    x = x.reshape(50, 4, 32).astype(np.float64)
    # half a step; the roundings of scale (times 15) and zero to fp16, half a step of fp16 each (2^-11, subnormal 2^-25)
    room = scale.astype(np.float64) * (0.5 + 15 * 2.0 ** -11) + np.abs(zero.astype(np.float64)) * 2.0 ** -11 + 16 * 2.0 ** -25
    assert np.all(np.abs(back - x) <= room[..., None] * (1 + 1e-6))
    same = np.full((1, 64), 0.7, np.float32)
    q, scale, zero = plain.quantised(same)
    assert not q.any() and abs(float(zero[0, 0]) - 0.7) <= 0.7 * 2 ** -11
    odd = np.zeros((1, 64), np.float32)
    odd[0, :3] = np.nan, np.inf, -np.inf
    q, scale, zero = plain.quantised(odd)
    assert np.isfinite(scale).all() and float(zero[0, 0]) == -65504.0


class Shape(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("pages", "kv_heads", "head_dim", "page_tokens", "reserved")]


class Attend(C.Structure):
    _fields_ = [("cache", Shape)] + [(n, C.c_uint32) for n in ("batch", "queries", "group", "table_pages", "unit_tokens", "dtype")] + \
               [("scale", C.c_float), ("reserved", C.c_uint32)] + [(n, C.c_int64) for n in ("b", "q", "h")]


class Evict(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("groups", "units_per_group", "steps", "budget", "sink", "recent", "decay_q", "reserved")]


ARG, RANGE = -1, -3


def attend_params(**change):
    v = dict(pages=4, kv_heads=2, head_dim=128, page_tokens=16, batch=1, queries=1, group=4, table_pages=4, unit_tokens=16, dtype=0,
             scale=0.1, reserved=0, b=1024, q=1024, h=128)
    v.update(change)
    cache = Shape(v.pop("pages"), v.pop("kv_heads"), v.pop("head_dim"), v.pop("page_tokens"), 0)
    return Attend(cache, **v)


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), ARG), (dict(queries=0), ARG), (dict(group=0), ARG), (dict(kv_heads=0), ARG), (dict(pages=0), ARG),
    (dict(table_pages=0), ARG), (dict(page_tokens=0), ARG), (dict(page_tokens=24), ARG), (dict(dtype=2), ARG), (dict(reserved=1), ARG),
    (dict(unit_tokens=0), ARG), (dict(unit_tokens=3), ARG), (dict(unit_tokens=32), ARG), (dict(page_tokens=48, unit_tokens=32), ARG),
    (dict(page_tokens=48, unit_tokens=24), ARG), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG),
    (dict(head_dim=96), RANGE), (dict(head_dim=0), RANGE), (dict(queries=1025), RANGE), (dict(queries=1024, group=5), RANGE),
    (dict(table_pages=1 << 27), RANGE), (dict(batch=1 << 24), RANGE), (dict(batch=1 << 23, kv_heads=2), RANGE)])
def test_attend_refuses(lib, change, code):
    n = C.c_uint64(7)
    assert lib.kvp_attend_workspace(C.byref(attend_params(**change)), 1, 1, C.byref(n)) == code and n.value == 7
    any_ = C.c_void_p(256)
    assert lib.kvp_attend(C.byref(attend_params(**change)), *[any_] * 8, any_, C.c_uint64(1 << 40), None) == code


def test_attend_refuses_nulls_and_small_workspaces(lib):
    p = attend_params()
    need, plain_need = C.c_uint64(), C.c_uint64()
    assert lib.kvp_attend_workspace(C.byref(p), 1, 1, C.byref(need)) == 0
    assert lib.kvp_attend_workspace(C.byref(p), 0, 0, C.byref(plain_need)) == 0 and plain_need.value < need.value
    assert lib.kvp_attend_workspace(None, 1, 1, C.byref(need)) == ARG and lib.kvp_attend_workspace(C.byref(p), 1, 1, None) == ARG
    some = [C.c_void_p(256)] * 9                    # q, cache, table, lens, units, out, lse, weights, workspace
    assert lib.kvp_attend(C.byref(p), *some, C.c_uint64(need.value - 1), None) == ARG
    for i in (0, 1, 2, 3, 5, 8):
        args = list(some)
        args[i] = None
        assert lib.kvp_attend(C.byref(p), *args, need, None) == ARG, i


def test_cache_calls_refuse(lib):
    some, st = C.c_void_p(256), C.c_int64(256)
    append = lambda c, dtype=0, tokens=4, cache=some, k=some: lib.kvp_cache_append(  # noqa: E731
        C.byref(c), cache, C.c_uint32(dtype), C.c_uint32(tokens), k, st, st, some, st, st, some, None)
    assert append(Shape(4, 2, 128, 16, 0), tokens=0) == 0                    # nothing to do
    assert append(Shape(4, 2, 96, 16, 0)) == RANGE
    for c in (Shape(0, 2, 128, 16, 0), Shape(4, 0, 128, 16, 0), Shape(4, 2, 128, 0, 0), Shape(4, 2, 128, 20, 0), Shape(4, 2, 128, 16, 1)):
        assert append(c) == ARG
    assert append(Shape(4, 2, 128, 16, 0), dtype=3) == ARG and append(Shape(4, 2, 128, 16, 0), k=None) == ARG
    assert lib.kvp_cache_read(C.byref(Shape(4, 2, 128, 16, 0)), None, 0, 4, some, some, some, None) == ARG
    assert lib.kvp_cache_read(None, some, 0, 4, some, some, some, None) == ARG


@pytest.mark.parametrize("change,code", [
    (dict(groups=0), ARG), (dict(units_per_group=0), ARG), (dict(steps=0), ARG), (dict(decay_q=65537), ARG), (dict(reserved=1), ARG),
    (dict(sink=5, recent=4), ARG), (dict(sink=0xFFFFFFFF, recent=2), ARG), (dict(budget=65), ARG),
    (dict(units_per_group=32769), RANGE), (dict(groups=1 << 26), RANGE)])
def test_evict_refuses(lib, change, code):
    v = dict(groups=2, units_per_group=64, steps=3, budget=8, sink=1, recent=2, decay_q=65536, reserved=0)
    v.update(change)
    some = [C.c_void_p(1 << 20), None, C.c_void_p(1 << 21), None, None, C.c_void_p(1 << 22)]
    assert lib.kvp_evict(C.byref(Evict(**v)), *some, None) == code
    assert lib.kvp_policy_accumulated(None, C.byref(Evict(**v)), some[0], some[5], None) == ARG


def test_evict_refuses_rows_that_overlap(lib):
    p = Evict(2, 64, 3, 8, 1, 2, 65536, 0)                                   # 16 bytes a row, three rows
    w, acc, out = C.c_void_p(1 << 20), C.c_void_p(1 << 21), 1 << 22
    for kept in (out, out + 32, out - 12):
        assert lib.kvp_evict(C.byref(p), w, None, acc, C.c_void_p(kept), None, C.c_void_p(out), None) == ARG
    for old in ((1 << 21) + 8, (1 << 21) - 8 * 127):                         # neither acc_out nor apart from it (128 units of 8 bytes)
        assert lib.kvp_evict(C.byref(p), w, C.c_void_p(old), acc, None, None, C.c_void_p(out), None) == ARG
    for i in (0, 2, 5):
        args = [w, None, acc, None, None, C.c_void_p(out)]
        args[i] = None
        assert lib.kvp_evict(C.byref(p), *args, None) == ARG


def test_trace_weights_refuses(lib):
    some = C.c_void_p(256)
    for g, n, s, k, code in ((0, 8, 1, 1, ARG), (1, 0, 1, 1, ARG), (1, 8, 0, 1, ARG), (1, 8, 1, 0, ARG), (1, 8, 1, 9, ARG),
                             (1, 32769, 1, 1, RANGE), (1 << 20, 4096, 1, 1, RANGE), (1 << 20, 8, 1 << 12, 1, RANGE)):
        assert lib.kvp_trace_weights(g, n, s, k, some, some, None) == code, (g, n, s, k)
    assert lib.kvp_trace_weights(1, 8, 1, 1, None, some, None) == ARG and lib.kvp_trace_weights(1, 8, 1, 1, some, None, None) == ARG


def test_plain_forms_agree_with_hand_worked_cases():
    w = np.array([[0.5, 0.25, 0.25, 0.0, np.nan, -1.0]], np.float32)
    assert plain.select(w, 1, 2)[0, 0] == 0b000011 and plain.select(w, 1, 6)[0, 0] == 0b000111 and plain.select(w, 2, 2)[0, 0] == 0b000011
    rows, acc = plain.evict(w, 1, 3, 1, 1, 65536)
    assert rows[0, 0] == 0b100011 and acc.tolist() == [1 << 23, 1 << 22, 1 << 22, 0, 0, 0]
    rows, acc = plain.evict(np.zeros((1, 6), np.float32), 1, 2, 0, 0, 32768, acc=[3, 8, 8, 9, 0, 0], kept=np.array([0b110111], np.uint32))
    assert rows[0, 0] == 0b000110 and acc.tolist() == [1, 4, 4, 4, 0, 0]


def test_calls_refuse_addresses_that_are_not_aligned(lib):
    """Checked on the host: the kernels move 16 bytes at a time."""
    some, st, off = C.c_void_p(256), C.c_int64(256), lambda n: C.c_void_p(256 + n)
    p, need = attend_params(), C.c_uint64(1 << 40)
    for i, by in ((0, 1), (1, 8), (2, 2), (3, 2), (4, 2), (5, 4), (6, 2), (7, 2), (8, 16)):     # q, cache, table, lens, units, out, lse, weights, workspace
        args = [some] * 9
        args[i] = off(by)
        assert lib.kvp_attend(C.byref(p), *args, need, None) == ARG, i
    shape = Shape(4, 2, 128, 16, 0)
    for dtype, by in ((0, 1), (1, 1), (2, 2)):
        for cache, k, v, slots in ((off(8), some, some, some), (some, off(by), some, some), (some, some, off(by), some), (some, some, some, off(4))):
            assert lib.kvp_cache_append(C.byref(shape), cache, C.c_uint32(dtype), C.c_uint32(4), k, st, st, v, st, st, slots, None) == ARG
    for cache, slots, k, v in ((off(8), some, some, some), (some, off(4), some, some), (some, some, off(8), some), (some, some, some, off(8))):
        assert lib.kvp_cache_read(C.byref(shape), cache, 0, 4, slots, k, v, None) == ARG
