"""Frequencies of rotary positions where the borders of a ramp lie outside the pairs, without a GPU."""
import math

import numpy as np
import pytest


def ramped(r, base, factor, original, low, high):
    """From the definition: turns t = original * f / 2 pi; the dims where t is `high` and `low`, rounded outwards, linear between them."""
    half = r // 2
    dim = lambda turns: half * math.log(original / (turns * 2 * math.pi)) / math.log(base)  # noqa: E731
    first, last = max(math.floor(dim(high)), 0), math.ceil(dim(low))
    divided = np.clip((np.arange(half) - first) / (last - first), 0, 1)
    f = base ** (-np.arange(half) / half)
    return f / factor * divided + f * (1 - divided), f


@pytest.mark.parametrize("r,base,original,low,high", [(128, 1e4, 131072, 1, 32), (128, 1e4, 65536, 1, 32), (64, 1e3, 8192, 1, 32), (64, 1e4, 2 ** 20, 2, 64), (128, 1e4, 4096, 1, 32),
                                                      (96, 5e5, 8192, 1, 4), (32, 100.0, 10 ** 7, 0.5, 8)])
def test_ramp_whose_border_lies_behind_the_last_pair(r, base, original, low, high):
    from paper_2508_13231_b200 import kvp
    for factor in (1.0, 4.0, 16.0):
        want, f = ramped(r, base, factor, original, low, high)
        got, scale = kvp.rope_frequencies(r, base=base, scaling="ramp", factor=factor, original_tokens=original, low=low, high=high)
        assert np.allclose(got.numpy(), want, rtol=1e-13, atol=0) and math.isclose(scale, 0.1 * math.log(factor) + 1, rel_tol=1e-7)
        turns = original * f / (2 * math.pi)
        # `low` turns or fewer: divided; more than that, a whole dim further on: not in full
        assert np.allclose(got.numpy()[turns <= low], (f / factor)[turns <= low], rtol=1e-13)
        above = turns > low * base ** (2 / r)
        assert factor == 1.0 or np.all(got.numpy()[above] > (f / factor)[above] * (1 + 1e-9))


def test_ramp_without_a_lower_border_ends_at_the_last_pair():
    from paper_2508_13231_b200 import kvp
    got, _ = kvp.rope_frequencies(64, scaling="ramp", factor=8, original_tokens=8192, low=0.0, high=32)
    f = 1e4 ** (-np.arange(32) / 32)
    first = math.floor(32 * math.log(8192 / (64 * math.pi)) / math.log(1e4))
    divided = np.clip((np.arange(32) - first) / (31 - first), 0, 1)
    assert np.allclose(got.numpy(), f / 8 * divided + f * (1 - divided), rtol=1e-13, atol=0) and math.isclose(float(got[-1]), f[-1] / 8, rel_tol=1e-13)


@pytest.mark.parametrize("kw", [dict(scaling="ramp", base=1.0), dict(scaling="ramp", base=0.5), dict(scaling="base", base=1e300, factor=1e20), dict(scaling="base", base=2.0, factor=1e308),
                                dict(scaling="linear", base=1e-320)])
def test_frequencies_that_are_no_numbers_are_refused(kw):
    """A base of 1 has no borders between its pairs, one beyond 64 bits leaves frequencies of 0, one of almost 0 infinite ones: never NaN, infinity or 0 for a frequency."""
    from paper_2508_13231_b200 import kvp
    kw = dict(dict(factor=4.0, original_tokens=4096), **kw)
    with pytest.raises(kvp.KvpError) as e:
        kvp.rope_frequencies(4, **kw)
    assert e.value.code == kvp.ERR_ARG


def test_frequencies_of_bases_below_one():
    from paper_2508_13231_b200 import kvp
    got, _ = kvp.rope_frequencies(8, base=0.5)
    assert np.allclose(got.numpy(), 0.5 ** (-np.arange(4) / 4), rtol=1e-14, atol=0)
    got, _ = kvp.rope_frequencies(8, base=0.5, scaling="parts", factor=2.0, original_tokens=64)
    assert np.all(np.isfinite(got.numpy())) and np.all(got.numpy() > 0)
