"""The layout of the cache held in 8 bits, the frequencies of rotary positions and the refusals of the calls around them, without a GPU."""
import ctypes as C
import math
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache8_plain as plain  # noqa: E402

ARG, RANGE = -1, -3


@pytest.fixture(scope="module")
def lib():
    from paper_2508_13231_b200 import build
    h = C.CDLL(build.build_library())
    h.kvp_cache8_page_bytes.restype = C.c_uint64
    return h


class Shape(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("pages", "kv_heads", "head_dim", "page_tokens", "reserved")]


class Attend8(C.Structure):
    _fields_ = [("cache", Shape)] + [(n, C.c_uint32) for n in ("batch", "queries", "group", "table_pages", "unit_tokens", "dtype")] + \
               [("scale", C.c_float), ("cap", C.c_float)] + [(n, C.c_uint32) for n in ("window", "sink", "reserved")] + [(n, C.c_int64) for n in ("b", "q", "h")]


class Rope(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("tokens", "heads", "kv_heads", "head_dim", "rotary_dim", "dtype", "flags")] + [("scale", C.c_float), ("reserved", C.c_uint32)] + \
               [(n, C.c_int64) for n in ("qt", "qh", "qot", "qoh", "kt", "kh", "kot", "koh")]


class Tables(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("batch", "table_pages", "pages", "page_tokens", "tokens", "reserved")]


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_block_holds_every_value_once(lib, d):
    key, value = plain.places(d)
    assert np.array_equal(np.sort(np.concatenate([key.reshape(-1), value.reshape(-1)])), np.arange(32 * d))
    assert lib.kvp_cache8_page_bytes(d, 16) == 32 * d + 16 and lib.kvp_cache8_page_bytes(d, 48) == 3 * (32 * d + 16)
    assert lib.kvp_cache8_page_bytes(d, 8) == 0 and lib.kvp_cache8_page_bytes(96, 16) == 0


def test_plain_codes_are_e4m3():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(plain.values_of(codes.numpy()), want, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(5000) * np.exp2(rng.integers(-14, 8, 5000)), want[np.isfinite(want)], (plain.CODES[1:] + plain.CODES[:-1]) / 2, [0.0, -0.0, 448.0]])
    x = np.clip(x, -448, 448).astype(np.float32).astype(np.float64)
    assert np.array_equal(plain.code_of(x), torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_plain_blocks_keep_values_within_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 40, 2, 64)) * np.exp2(rng.integers(-8, 8, (2, 40, 2, 1)))
    cache = np.zeros((3, 2, plain.page_bytes(64, 16)), np.uint8)
    for a, b in ((0, 5), (5, 6), (6, 33), (33, 40)):                           # tokens come in several calls
        plain.append(cache, x[0, a:b], x[1, a:b], np.arange(a, b))
    for (held, scale), y in zip(plain.held(cache, 64), x):
        held, scale = (z.transpose(0, 2, 1, *range(3, z.ndim)).reshape(48, 2, *z.shape[3:])[:40] for z in (held, scale))
        # 2^-4 of a normal number, half of 2^-9 of a smaller one; rounded again when the scale grew, at most six times, below the normal numbers only
        assert np.all(np.abs(held - y) <= np.maximum(np.abs(y) * 2.0 ** -4, 0) + 6 * scale[..., None] * 2.0 ** -10)
        assert np.all(np.abs(y).max(-1) <= 448 * scale)


def test_plain_tables_agree_with_a_hand_worked_case():
    r = plain.tables([3, -1, 1, 2], [1, 5, 4, 0], np.array([[7, -1], [3, 9], [4, -1], [-1, -1]]), np.array([5, 8, 6] + [0] * 7), [1, 2], 4, 8)
    # request 0 stays in its page, 1 gives back 3 and 9, 2 takes page 8, 3 page 6
    assert r["slots"].tolist() == [29, 30, 31, 32, 24, 25, -1, -1] and r["positions"].tolist() == [1, 2, 3, 4, 0, 1, 0, 0]
    assert r["rows"].tolist() == [0, 0, 0, 2, 3, 3, -1, -1] and r["starts"].tolist() == [0, 3, 3, 4, 6] and r["page_starts"].tolist() == [0, 0, 0, 1, 2]
    assert r["granted"].tolist() == [1, 1, 1, 1] and r["lens"].tolist() == [4, 0, 5, 2] and r["state"].tolist() == [3, 2]
    assert r["ring"].tolist()[3:5] == [3, 9] and r["table"][2].tolist() == [4, 8]


# ---- frequencies ----------------------------------------------------------------------------------------------------

def test_rope_frequencies():
    """Against the formulas; pow and log of two libraries agree within a few steps of 2^-52."""
    from paper_2508_13231_b200 import kvp
    for r in (2, 64, 128, 18):
        j = np.arange(r // 2)
        base = 10000.0 ** (-2.0 * j / r)
        f, scale = kvp.rope_frequencies(r)
        assert scale == 1.0 and np.allclose(f.numpy(), base, rtol=1e-14, atol=0)
        f, scale = kvp.rope_frequencies(r, base=5e5, scaling="linear", factor=4)
        assert scale == 1.0 and np.allclose(f.numpy(), 5e5 ** (-2.0 * j / r) / 4, rtol=1e-14, atol=0)
        if r > 2:
            f, scale = kvp.rope_frequencies(r, scaling="base", factor=8)
            assert np.allclose(f.numpy(), (10000.0 * 8 ** (r / (r - 2))) ** (-2.0 * j / r), rtol=1e-13, atol=0)
            assert math.isclose(float(f[-1]), base[-1] / 8, rel_tol=1e-12) and float(f[0]) == 1.0
        f, scale = kvp.rope_frequencies(r, base=5e5, scaling="parts", factor=8, original_tokens=8192, low=1, high=4)
        plain_f = 5e5 ** (-2.0 * j / r)
        turns = 8192 * plain_f / (2 * np.pi)
        smooth = np.clip((turns - 1) / 3, 0, 1)
        assert scale == 1.0 and np.allclose(f.numpy(), (1 - smooth) * plain_f / 8 + smooth * plain_f, rtol=1e-13, atol=0)
    f, scale = kvp.rope_frequencies(128, scaling="ramp", factor=16, original_tokens=4096)
    j = np.arange(64)
    border = lambda turns: 64 * math.log(4096 / (turns * 2 * math.pi)) / math.log(10000)  # noqa: E731
    low, high = max(math.floor(border(32)), 0), min(math.ceil(border(1)), 63)
    ramp = np.clip((j - low) / (high - low), 0, 1)
    base = 10000.0 ** (-j / 64)
    assert np.allclose(f.numpy(), base / 16 * ramp + base * (1 - ramp), rtol=1e-13, atol=0) and scale == np.float32(0.1 * math.log(16) + 1)


def test_rope_frequencies_refuse():
    from paper_2508_13231_b200 import kvp
    for r, kw in ((3, {}), (0, {}), (-2, {}), (64, dict(scaling="cubic"))):
        with pytest.raises(ValueError):
            kvp.rope_frequencies(r, **kw)
    for kw in (dict(base=0.0), dict(base=float("nan")), dict(scaling="linear", factor=0.5), dict(scaling="parts", factor=2, low=4, high=4), dict(scaling="ramp", factor=2, original_tokens=0),
               dict(scaling="ramp", factor=float("inf"))):
        with pytest.raises(kvp.KvpError) as e:
            kvp.rope_frequencies(64, **kw)
        assert e.value.code == kvp.ERR_ARG
    with pytest.raises(kvp.KvpError):
        kvp.rope_frequencies(2, scaling="base", factor=2)
    with pytest.raises(ValueError):
        kvp.cache8_page_bytes(96, 16)


# ---- refusals --------------------------------------------------------------------------------------------------------

def attend_params(**change):
    v = dict(pages=4, kv_heads=2, head_dim=128, page_tokens=16, batch=1, queries=1, group=4, table_pages=4, unit_tokens=16, dtype=0,
             scale=0.1, cap=0.0, window=0, sink=0, reserved=0, b=1024, q=1024, h=128)
    v.update(change)
    cache = Shape(v.pop("pages"), v.pop("kv_heads"), v.pop("head_dim"), v.pop("page_tokens"), 0)
    return Attend8(cache, **v)


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), ARG), (dict(queries=0), ARG), (dict(group=0), ARG), (dict(kv_heads=0), ARG), (dict(pages=0), ARG),
    (dict(table_pages=0), ARG), (dict(page_tokens=0), ARG), (dict(page_tokens=24), ARG), (dict(dtype=2), ARG), (dict(reserved=1), ARG),
    (dict(unit_tokens=0), ARG), (dict(unit_tokens=3), ARG), (dict(unit_tokens=32), ARG), (dict(page_tokens=48, unit_tokens=32), ARG),
    (dict(page_tokens=48, unit_tokens=24), ARG), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(cap=-1.0), ARG),
    (dict(cap=float("inf")), ARG), (dict(cap=1e-44), ARG), (dict(cap=float("nan")), ARG), (dict(head_dim=96), RANGE), (dict(queries=1025), RANGE), (dict(queries=1024, group=5), RANGE),
    (dict(batch=1 << 24), RANGE), (dict(table_pages=1 << 26), RANGE), (dict(batch=1 << 16, table_pages=1 << 14), RANGE)])
def test_attend_refuses(lib, change, code):
    need, some = C.c_uint64(0), C.c_void_p(256)
    p = attend_params(**change)
    assert lib.kvp_attend8_workspace(C.byref(p), 1, 1, C.byref(need)) == code
    assert lib.kvp_attend8(C.byref(p), some, some, some, some, some, some, some, some, some, some, C.c_uint64(1 << 40), None) == code


def test_attend_refuses_pointers(lib):
    p, need, some, off = attend_params(), C.c_uint64(0), C.c_void_p(256), lambda n: C.c_void_p(256 + n)
    assert lib.kvp_attend8_workspace(C.byref(p), 1, 1, C.byref(need)) == 0 and need.value > 0
    assert lib.kvp_attend8_workspace(C.byref(p), 1, 1, None) == ARG and lib.kvp_attend8_workspace(None, 1, 1, C.byref(need)) == ARG
    good = [some] * 10                                                       # q, cache, table, lens, units, slopes, out, lse, weights, workspace
    assert lib.kvp_attend8(C.byref(p), *good, C.c_uint64(need.value - 1), None) == ARG
    for i in (0, 1, 2, 3, 6, 9):
        assert lib.kvp_attend8(C.byref(p), *good[:i], None, *good[i + 1:], C.c_uint64(1 << 40), None) == ARG, i
    for i, by in ((0, 1), (1, 8), (2, 2), (3, 2), (4, 2), (5, 2), (6, 4), (7, 2), (8, 2), (9, 16)):
        assert lib.kvp_attend8(C.byref(p), *good[:i], off(by), *good[i + 1:], C.c_uint64(1 << 40), None) == ARG, i


def test_append_and_read_refuse(lib):
    some, st, off = C.c_void_p(256), C.c_int64(256), lambda n: C.c_void_p(256 + n)
    for change, code in ((dict(pages=0), ARG), (dict(kv_heads=0), ARG), (dict(page_tokens=24), ARG), (dict(reserved=1), ARG), (dict(head_dim=96), RANGE), (dict(kv_heads=65536), RANGE)):
        shape = Shape(**dict(dict(pages=4, kv_heads=2, head_dim=128, page_tokens=16, reserved=0), **change))
        assert lib.kvp_cache8_append(C.byref(shape), some, 0, 4, some, st, st, some, st, st, some, None) == code
        assert lib.kvp_cache8_read(C.byref(shape), some, 0, 4, some, some, some, None) == code
    shape = Shape(4, 2, 128, 16, 0)
    assert lib.kvp_cache8_append(C.byref(shape), some, 3, 4, some, st, st, some, st, st, some, None) == ARG
    assert lib.kvp_cache8_append(C.byref(shape), None, 0, 0, None, st, st, None, st, st, None, None) == 0        # no tokens
    assert lib.kvp_cache8_append(C.byref(shape), some, 0, 1 << 31, some, st, st, some, st, st, some, None) == RANGE
    for dtype, by in ((0, 1), (1, 1), (2, 2)):
        for cache, k, v, slots in ((off(8), some, some, some), (some, off(by), some, some), (some, some, off(by), some), (some, some, some, off(4)), (None, some, some, some), (some, some, some, None)):
            assert lib.kvp_cache8_append(C.byref(shape), cache, C.c_uint32(dtype), C.c_uint32(4), k, st, st, v, st, st, slots, None) == ARG
    for cache, slots, k, v in ((off(8), some, some, some), (some, off(4), some, some), (some, some, off(8), some), (some, some, some, off(8))):
        assert lib.kvp_cache8_read(C.byref(shape), cache, 0, 4, slots, k, v, None) == ARG


def test_rope_refuses(lib):
    some, other, off = C.c_void_p(256), C.c_void_p(1 << 20), lambda n: C.c_void_p(256 + n)
    good = dict(tokens=4, heads=2, kv_heads=1, head_dim=64, rotary_dim=64, dtype=0, flags=0, scale=1.0, reserved=0, qt=128, qh=64, qot=128, qoh=64, kt=64, kh=64, kot=64, koh=64)
    call = lambda args=(some, other, some, other, some, some), **change: lib.kvp_rope(C.byref(Rope(**dict(good, **change))), *args, None)  # noqa: E731
    for change, code in ((dict(head_dim=0), ARG), (dict(rotary_dim=0), ARG), (dict(rotary_dim=63), ARG), (dict(rotary_dim=66), ARG), (dict(dtype=3), ARG), (dict(flags=4), ARG),
                         (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(reserved=1), ARG), (dict(heads=0, kv_heads=0), ARG),
                         (dict(tokens=1 << 31), RANGE), (dict(head_dim=65538), RANGE), (dict(heads=1 << 20), RANGE)):
        assert call(**change) == code, change
    assert call(args=(None,) * 6, tokens=0) == 0
    for i, by in ((0, 1), (1, 1), (2, 1), (3, 1), (4, 2), (5, 4)):
        args = [some, other, some, other, some, some]
        args[i] = off(by)
        assert call(args=args) == ARG, i
        args[i] = None
        assert call(args=args) == ARG, i
    assert call(args=(some, some, some, other, some, some), qot=256) == ARG and call(args=(some, other, some, some, some, some), koh=32) == ARG


def test_tables_refuse(lib):
    some, off = C.c_void_p(256), lambda n: C.c_void_p(256 + n)
    good = dict(batch=2, table_pages=4, pages=9, page_tokens=16, tokens=8, reserved=0)
    args = [some] * 13
    for change, code in ((dict(batch=0), ARG), (dict(table_pages=0), ARG), (dict(pages=0), ARG), (dict(page_tokens=0), ARG), (dict(reserved=1), ARG), (dict(table_pages=1 << 26), RANGE),
                         (dict(pages=1 << 30), RANGE), (dict(tokens=1 << 30), RANGE), (dict(batch=1 << 24), RANGE), (dict(page_tokens=1 << 30), RANGE)):
        assert lib.kvp_block_tables(C.byref(Tables(**dict(good, **change))), *args, None) == code, change
    for i in range(13):                                                      # new_tokens, lens, lens_out, table, ring, state, state_out, slots, positions, rows, starts, page_starts, granted
        for bad in (None, off(4 if i == 7 else 2)):
            assert lib.kvp_block_tables(C.byref(Tables(**good)), *args[:i], bad, *args[i + 1:], None) == ARG, i
