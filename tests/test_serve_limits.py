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


def test_no_new_rows_launch_nothing_but_are_checked(lib):
    def call(lens, new, both=None, k=A, o=None):
        return lib.santapp_prompt_attn(geom(), lens, new, both, None, k, A, o, None, None)
    assert call(ints(5, 7), ints(0, 0)) == 0 and lib.santapp_last_launch_count() == 0
    assert call(ints(5, 7), ints(0, 1)) == BAD                       # (no queries)
    assert call(ints(5, 0), ints(0, 0)) == BAD
    assert call(ints(5, 7), ints(1, -1)) == BAD
    assert call(ints(5, 7), ints(0, 0), ints(6, 0)) == BAD
    assert call(ints(5, 7), ints(0, 0), k=None) == BAD
    assert call(ints(5, 7), ints(0, 0), o=ctypes.byref(sp.CAttnOpts(-1.0, 0.0, None, None))) == BAD


def test_the_binding_checks_calls_without_new_rows(lib):
    import torch
    g, x = sp.Geometry(2, 8, 2), torch.zeros(0, 8, 128, dtype=torch.bfloat16)
    k = torch.zeros(2, 12, 128, dtype=torch.bfloat16)
    for lens, new in (([5, 7], [0, 0]), ([5, 7], [1, -1]), ([5, 7], [1, -2]), ([-5, 4], [0, 0])):
        with pytest.raises(sp.SantappError) as e:
            sp.santapp_prompt_attn(g, lens, x, k, k, new_len=new)
        assert e.value.status == BAD


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


@pytest.mark.parametrize("new", [0x30000 + 4, 0x30000 - 4, 0x40000, 0x40000 + 4])
def test_append_refuses_lengths_that_overlap_what_it_reads(lib, new):
    r = sp.CRope(128, 0, 1.0, (ctypes.c_double * 64)(*([0.5] * 64)))
    assert lib.santapp_rope_append(geom(), ctypes.byref(r), A, 28 * 128, A, 512, A, 512, 0x40000, 0x30000, A, A, A, 16, new, None) == BAD
