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
