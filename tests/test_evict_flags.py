"""The flags of kvp_evict_params, without a GPU."""
import ctypes as C

import pytest

ARG = -1


class Evict(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("groups", "units_per_group", "steps", "budget", "sink", "recent", "decay_q", "flags")]


@pytest.mark.parametrize("flags", [1, 3, 4, 6, 0x80000002])
def test_unknown_flags_are_refused(flags):
    from paper_2508_13231_b200 import build
    lib = C.CDLL(build.build_library())
    p = Evict(2, 64, 3, 8, 1, 2, 65536, flags)
    assert lib.kvp_evict(C.byref(p), C.c_void_p(1 << 20), None, C.c_void_p(1 << 21), None, None, C.c_void_p(1 << 22), None) == ARG


def test_the_binding_has_the_same_parameters():
    from paper_2508_13231_b200 import kvp
    assert [n for n, _ in kvp.EvictParams._fields_] == [n for n, _ in Evict._fields_] and C.sizeof(kvp.EvictParams) == 32


def test_choices_refuse_addresses_that_are_not_aligned():
    """Checked on the host, as the other calls between attention and the placement problem do."""
    from paper_2508_13231_b200 import build
    lib = C.CDLL(build.build_library())
    p = Evict(2, 64, 3, 8, 1, 2, 65536, 0)
    at = lambda n: C.c_void_p(n)  # noqa: E731
    good = [1 << 20, 1 << 21, 1 << 21, 1 << 22, 1 << 23, 1 << 24]                # weights, acc_in, acc_out, kept_in, exist, kept_out
    for i, by in enumerate((2, 4, 4, 2, 2, 2)):
        args = list(good)
        args[i] += by
        if i in (1, 2):
            args[3 - i] = 1 << 25                                                # apart, so that only the alignment is at fault
        assert lib.kvp_evict(C.byref(p), *[at(x) for x in args], None) == ARG, i
    some = at(1 << 20)
    assert lib.kvp_trace_weights(1, 8, 1, 1, at((1 << 20) + 2), some, None) == ARG
    assert lib.kvp_trace_weights(1, 8, 1, 1, some, at((1 << 20) + 2), None) == ARG
