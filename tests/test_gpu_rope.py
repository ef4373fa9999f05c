"""Rotary positions against the formula in 64 bits.

Tolerance, with u the half-step of the output's type: a result is a sum of two fp32 products; sine and cosine are off by 2^-24 * (0.5 rounding of
the reduced angle, below 2^-2.6 turns of pi: 2^-25; 1.5 for two roundings of the function, the scale another 0.5): 3 * 2^-24 * scale, the products and the sum by 3
roundings of 2^-24 more; so 6 * 2^-24 * scale * (|a| + |b|) + u |result|, and half the smallest step of fp16 where results are that small.
"""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache8_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}


@pytest.fixture(scope="module")
def kvp():
    from paper_2508_13231_b200 import kvp
    return kvp


def near(got, x, positions, frequencies, interleaved, inverse, scale):
    dtype = got.dtype
    x, got = x.double().cpu().numpy(), got.double().cpu().numpy()
    want = plain.rope(x, positions, frequencies, interleaved, inverse, scale)
    r = 2 * len(frequencies)
    size = np.abs(x)
    both = size.copy()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    both[..., first] = both[..., second] = size[..., first] + size[..., second]
    room = 6 * 2.0 ** -24 * abs(scale) * both + HALF[dtype] * np.abs(want) + (2.0 ** -25 if dtype == F16 else 0)
    assert np.array_equal(got[..., r:], x[..., r:])
    bad = np.abs(got - want)[..., :r] / np.maximum(room[..., :r], 1e-300)
    assert np.all(np.abs(got - want)[..., :r] <= room[..., :r]), bad.max()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("tokens,heads,kv,dim,rotary,interleaved", [(1, 1, 1, 2, 2, False), (1, 32, 8, 128, 128, False), (5, 3, 1, 64, 32, True), (33, 4, 4, 96, 48, False),
                                                                    (33, 4, 2, 128, 64, True), (7, 2, 1, 80, 20, False), (7, 2, 1, 81, 30, True), (1000, 5, 5, 256, 256, False),
                                                                    (3000, 8, 2, 64, 64, True), (2, 1, 0, 32, 16, False)])
def test_rope(kvp, dtype, tokens, heads, kv, dim, rotary, interleaved):
    rng = np.random.default_rng(tokens + dim)
    q = torch.from_numpy(rng.standard_normal((tokens, heads, dim))).cuda().to(dtype)
    k = torch.from_numpy(rng.standard_normal((tokens, kv, dim))).cuda().to(dtype) if kv else None
    positions = rng.integers(0, 131072, tokens).astype(np.int32)
    positions[0] = 0
    f, _ = kvp.rope_frequencies(rotary)
    dev = torch.from_numpy(positions).cuda(), f.cuda()
    for inverse, scale in ((False, 1.0), (True, 1.0), (False, 1.2)):
        got = kvp.rope(q, k, *dev, interleaved=interleaved, inverse=inverse, scale=scale)
        for x, y in zip((q, k), got):
            if x is None:
                assert y is None
            else:
                near(y, x, positions, f.numpy(), interleaved, inverse, scale)


def test_rope_at_far_and_negative_positions(kvp):
    positions = np.array([2 ** 31 - 1, -2 ** 31, -1, 2 ** 24 + 1, 10 ** 9 + 7, -12345], np.int32)
    for f in (np.array([1.0, 0.1, 3e-5, 1e-9]), np.array([2.5, 0.0, -0.3, 6.2831853])):
        # 64-bit angles of the plain form are off by 2^-53 of up to 2^33: below 2^-20; the angles here are computed in 80 bits and reduced
        turns = (positions.astype(np.longdouble)[:, None] * f.astype(np.longdouble)[None]) / (2 * np.longdouble("3.14159265358979323846264338327950288"))
        angle = ((turns - np.rint(turns)) * 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(np.float64)
        x = np.random.default_rng(1).standard_normal((6, 2, 8))
        got, _ = kvp.rope(torch.from_numpy(x).float().cuda(), None, torch.from_numpy(positions).cuda(), torch.from_numpy(f).cuda())
        x = x.astype(np.float32).astype(np.float64)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        want = np.concatenate((x[..., :4] * c - x[..., 4:] * s, x[..., :4] * s + x[..., 4:] * c), -1)
        both = np.tile(np.abs(x[..., :4]) + np.abs(x[..., 4:]), 2)
        # frequencies are held as 64-bit fractions of a turn from a 53-bit product: 2^-52 of up to 2^31 * f / 2 pi turns, times 2 pi
        off = (np.abs(positions.astype(np.float64))[:, None] * np.abs(f)[None] * 2.0 ** -51)[:, None]
        room = (6 * 2.0 ** -24 + np.concatenate((off, off), -1)) * both + 2.0 ** -24 * np.abs(want)
        assert np.all(np.abs(got.double().cpu().numpy() - want) <= room)


def test_rope_strided_in_place_and_streams(kvp):
    """Queries and keys as slices of one projection, aligned and not, turned in place: the rest of it is left as it was."""
    tokens, heads, kv, d = 40, 4, 2, 64
    f = kvp.rope_frequencies(48)[0].cuda()
    at = torch.arange(1000, 1000 + tokens, dtype=torch.int32, device="cuda")
    for shift in (0, 1, 8):
        fused = torch.randn(tokens, (heads + 2 * kv) * d + 16, device="cuda").to(BF16)
        before = fused.clone()
        q, k = (fused[:, shift + a * d: shift + b * d].unflatten(1, (b - a, d)) for a, b in ((0, heads), (heads, heads + kv)))
        want = kvp.rope(q.contiguous(), k.contiguous(), at, f)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        out = kvp.rope(q, k, at, f, in_place=True, stream=s)
        torch.cuda.synchronize()
        assert out[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1])
        rest = torch.ones(fused.shape[1], dtype=torch.bool, device="cuda")
        rest[shift: shift + (heads + kv) * d] = False
        assert torch.equal(fused[:, rest], before[:, rest])
        turned = kvp.rope(before[:, shift: shift + heads * d].unflatten(1, (heads, d)).transpose(0, 1).contiguous().transpose(0, 1), None, at, f)
        assert torch.equal(turned[0], want[0]) and turned[1] is None


def test_rope_gradient(kvp):
    """inverse is the gradient: against the formula's, and against differences of the forward call."""
    rng = np.random.default_rng(4)
    for interleaved in (False, True):
        x, g = (torch.from_numpy(rng.standard_normal((9, 3, 32))).cuda() for _ in range(2))
        at = torch.arange(5, 14, dtype=torch.int32, device="cuda")
        f, scale = kvp.rope_frequencies(16, scaling="ramp", factor=4.0)
        f = f.cuda()
        got = kvp.rope(g.float(), None, at, f, interleaved=interleaved, inverse=True, scale=scale)[0]
        near(got, g.float(), at.cpu().numpy(), f.cpu().numpy(), interleaved, True, scale)
        fwd = lambda y: kvp.rope(y.float(), None, at, f, interleaved=interleaved, scale=scale)[0].double()  # noqa: E731
        for _ in range(20):
            d = torch.from_numpy(rng.standard_normal(x.shape)).cuda()
            slope = ((fwd(x + d) - fwd(x - d)) * g).sum() / 2         # exact up to roundings: the call is linear
            # roundings to fp32 of x +- d, of the results and of the gradient: 8 * 2^-24 of each term
            room = 8 * 2.0 ** -24 * scale * 2 * float(((x.abs() + d.abs()).sum((1, 2), keepdim=True) * g.abs()).sum())
            assert abs(float(slope - (got.double() * d).sum())) <= room


def test_rope_refuses(kvp):
    q, k = torch.zeros(4, 2, 32, device="cuda"), torch.zeros(4, 1, 32, device="cuda")
    at, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(16, dtype=torch.float64, device="cuda")
    for args in ((q.double(), k, at, f), (q, k.half(), at, f), (q, k, at[:3], f), (q, k, at.long(), f), (q, k, at, f.float()), (q, k[:3], at, f), (q, k[..., :16], at, f),
                 (q[0], k, at, f), (q.transpose(0, 2), None, at, f), (q, k.cpu(), at, f)):
        with pytest.raises(ValueError):
            kvp.rope(*args)
    for args, kw in (((q, k, at, torch.zeros(17, dtype=torch.float64, device="cuda")), {}), ((q, k, at, f[:0]), {}), ((q, k, at, f), dict(scale=float("nan")))):
        with pytest.raises(kvp.KvpError) as e:
            kvp.rope(*args, **kw)
        assert e.value.code == kvp.ERR_ARG
    assert kvp.rope(q[:0], k[:0], at[:0], f)[0].shape == (0, 2, 32)
