"""The ends of the ranges of the operators around the decode step, on the host (fake addresses: nothing is dereferenced)."""
import ctypes

import pytest

from paper_2609_35629_b200 import binding as sp
from paper_2609_35629_b200 import build as sp_build

A = 0x10000
BAD, SMALL = sp.SANTAPP_ERR_INVALID_ARG, sp.SANTAPP_ERR_WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module")
def lib():
    sp_build.build()
    return sp.load_library()


def geom(n=2, hq=28, hkv=4):
    return ctypes.byref(sp.Geometry(n, hq, hkv).c())


def ints(*v):
    return (ctypes.c_int32 * len(v))(*v)


# A workspace of one byte ends the call behind the checks of its options and ahead of any launch.
@pytest.mark.parametrize("scale,cap,want", [(0.0, 2.3e38, BAD), (0.0, 2.4e38, BAD), (0.0, 3.4e38, BAD), (2.4e38, 0.0, BAD), (3.4e38, 1e38, BAD), (1e-30, 1e9, BAD),
                                            (0.0, 1e-40, BAD), (0.0, 7e36, SMALL), (2.3e38, 0.0, SMALL), (1e-38, 0.0, SMALL), (1.0, 8e37, SMALL)])
def test_scales_and_caps_that_fp32_cannot_hold_are_refused(lib, scale, cap, want):
    o = sp.CAttnOpts(scale, cap, None, None)
    assert lib.santapp_prefix_decode_attn(geom(), A, A, 100, 100, None, A, A, A, A, 16, ctypes.byref(o), A, A, 1, None) == want
    if want == BAD:
        assert lib.santapp_prompt_attn(geom(), ints(5, 7), None, None, A, A, A, ctypes.byref(o), A, None) == want


def test_an_amplitude_beyond_fp32_is_refused(lib):
    r = sp.CRope(128, 0, 1e39, (ctypes.c_double * 64)(*([0.5] * 64)))
    assert lib.santapp_rope_append(geom(), ctypes.byref(r), A, 28 * 128, A, 512, A, 512, A, A, A, A, A, 16, None, None) == BAD
