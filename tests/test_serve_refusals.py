"""What the operators around the decode step refuse, on the host, before any launch (fake addresses: nothing is
dereferenced), and the rotary frequencies by their formulas."""
import ctypes
import math

import numpy as np
import pytest

from paper_2609_35629_b200 import binding as sp
from paper_2609_35629_b200 import build as sp_build

A = 0x10000
BAD, NO, SMALL = sp.SANTAPP_ERR_INVALID_ARG, sp.SANTAPP_ERR_UNSUPPORTED, sp.SANTAPP_ERR_WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module")
def lib():
    sp_build.build()
    return sp.load_library()


def geom(n=2, hq=28, hkv=4, **kw):
    return ctypes.byref(sp.Geometry(n, hq, hkv, **kw).c())


def rope(rot=128, inter=0, amp=1.0, freq=0.5):
    return sp.CRope(rot, inter, amp, (ctypes.c_double * 64)(*([freq] * 64)))


def ints(*v):
    return (ctypes.c_int32 * len(v))(*v)


@pytest.mark.parametrize("kw", [dict(q=None), dict(q=A + 8), dict(k=None), dict(v=A + 2), dict(qs=27 * 128), dict(ks=511), dict(vs=516),
                                dict(base=None), dict(len=None), dict(len=A + 2), dict(out=None), dict(kd=None), dict(vd=A + 4), dict(cap=0),
                                dict(cap=-4), dict(new=A + 1), dict(rope=None), dict(r=dict(rot=0)), dict(r=dict(rot=130)), dict(r=dict(inter=2)),
                                dict(r=dict(amp=math.nan)), dict(r=dict(freq=math.inf)), dict(out=A, q=A, qs=36 * 128)])
def test_append_refuses(lib, kw):
    r = rope(**kw.get("r", {}))
    p = dict(q=A, qs=28 * 128, k=A, ks=512, v=A, vs=512, base=A, len=A, out=2 * A, kd=A, vd=A, cap=16, new=None)
    p.update({k: v for k, v in kw.items() if k not in ("r", "rope")})
    rc = lib.santapp_rope_append(geom(), None if "rope" in kw else ctypes.byref(r), p["q"], p["qs"], p["k"], p["ks"], p["v"], p["vs"], p["base"],
                                 p["len"], p["out"], p["kd"], p["vd"], p["cap"], p["new"], None)
    assert rc == BAD


def test_append_does_not_support(lib):
    args = (A, 28 * 128, A, 512, A, 512, A, A, A, A, A, 16, None, None)
    assert lib.santapp_rope_append(geom(), ctypes.byref(rope(rot=24)), *args) == NO
    assert lib.santapp_rope_append(geom(head_dim=64), ctypes.byref(rope()), *args) == NO
    huge = args[:11] + (2 ** 30,) + args[12:]
    assert lib.santapp_rope_append(geom(), ctypes.byref(rope()), *huge) == NO


@pytest.mark.parametrize("kw,want", [(dict(n=0), BAD), (dict(n=-1), BAD), (dict(rows=9), BAD), (dict(rows=0, dst=A), BAD), (dict(pos=A + 2), BAD),
                                     (dict(dst=A + 1), BAD), (dict(n=2 ** 31, rows=2 ** 31), NO), (dict(rows=2 ** 31), NO)])
def test_prompt_rows_refuse(lib, kw, want):
    p = dict(n=10, rows=10, pos=None, dst=None)
    p.update(kw)
    assert lib.santapp_rope_prompt(geom(), ctypes.byref(rope()), p["n"], A, 28 * 128, A, 512, A, 512, p["pos"], p["dst"], A, A, A, p["rows"],
                                   None) == want


@pytest.mark.parametrize("kw,want", [(dict(src=None), BAD), (dict(src=A + 2), BAD), (dict(len=None), BAD), (dict(k=None), BAD), (dict(k=A + 8), BAD),
                                     (dict(v=A), BAD), (dict(cap=0), BAD), (dict(new=0x30000), BAD), (dict(new=0x30000 + 4), BAD),
                                     (dict(new=0x30000 - 4), BAD), (dict(new=0x40000 + 4), BAD), (dict(new=2), BAD), (dict(B=4097), NO),
                                     (dict(cap=2 ** 29), NO)])
def test_fork_refuses(lib, kw, want):
    p = dict(B=2, src=0x40000, len=0x30000, k=A, v=2 * A, cap=16, new=0x50000)
    p.update(kw)
    assert lib.santapp_suffix_fork(geom(p["B"]), p["src"], p["len"], p["k"], p["v"], p["cap"], p["new"], None) == want


@pytest.mark.parametrize("kw,want", [(dict(k=None), BAD), (dict(v=None), BAD), (dict(k=A + 8), BAD), (dict(N=-1), BAD), (dict(plane=99), BAD),
                                     (dict(tok=A + 2), BAD), (dict(q=None), BAD), (dict(out=A + 4), BAD), (dict(ws=None), BAD), (dict(size=64), SMALL),
                                     (dict(cap=-1), BAD), (dict(ks=None), BAD), (dict(o=dict(scale=-1.0)), BAD), (dict(o=dict(scale=math.nan)), BAD),
                                     (dict(o=dict(cap=-1.0)), BAD), (dict(o=dict(cap=math.inf)), BAD), (dict(o=dict(cap=1e-42)), BAD), (dict(o=dict(slopes=A + 1)), BAD),
                                     (dict(o=dict(status=A + 2)), BAD), (dict(N=2 ** 30, plane=2 ** 30), NO), (dict(plane=2 ** 31), NO),
                                     (dict(B=70000), NO), (dict(cap=2 ** 29), NO)])
def test_prefix_refuses(lib, kw, want):
    p = dict(B=2, k=A, v=A, N=100, plane=100, tok=None, q=A, ks=A, vs=A, len=A, cap=16, out=A, ws=A, size=1 << 40)
    p.update({k: v for k, v in kw.items() if k != "o"})
    o = sp.CAttnOpts(**kw.get("o", {}))
    assert lib.santapp_prefix_decode_attn(geom(p["B"]), p["k"], p["v"], p["N"], p["plane"], p["tok"], p["q"], p["ks"], p["vs"], p["len"], p["cap"],
                                          ctypes.byref(o), p["out"], p["ws"], p["size"], None) == want


def test_prefix_workspace(lib):
    size = lib.santapp_prefix_decode_workspace_bytes
    assert size(geom(), 0, 16) >= 16
    assert 2 * 7 * 4 * 128 * 4 <= size(geom(), 32768, 16) < 256 << 20
    assert size(geom(), -1, 16) == 0 and size(geom(), 2 ** 30, 0) == 0 and size(geom(head_dim=64), 100, 0) == 0


@pytest.mark.parametrize("kw,want", [(dict(q=None), BAD), (dict(k=A + 2), BAD), (dict(v=None), BAD), (dict(out=A + 8), BAD), (dict(lens=None), BAD),
                                     (dict(lens=ints(5, 0)), BAD), (dict(new=ints(6, 1)), BAD), (dict(new=ints(-1, 1)), BAD), (dict(both=ints(6, 1)), BAD),
                                     (dict(both=ints(0, -1)), BAD), (dict(lens=ints(2 ** 30, 5), new=ints(1, 1)), NO),
                                     (dict(lens=ints(2 ** 28, 5)), NO), (dict(o=dict(cap=math.nan)), BAD)])
def test_prompt_attention_refuses(lib, kw, want):
    p = dict(lens=ints(5, 7), new=None, both=None, q=A, k=A, v=A, out=A)
    p.update({k: v for k, v in kw.items() if k != "o"})
    o = sp.CAttnOpts(**kw.get("o", {}))
    assert lib.santapp_prompt_attn(geom(), p["lens"], p["new"], p["both"], p["q"], p["k"], p["v"], ctypes.byref(o), p["out"], None) == want


def test_the_binding_wants_cuda_tensors_of_the_right_shape(lib):
    import torch
    g, x = sp.Geometry(1, 8, 2), torch.zeros(1, 8, 128, dtype=torch.bfloat16)
    n = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(sp.SantappError) as e:
        sp.santapp_rope_append(g, sp.Rope(), x, x[:, :2], x[:, :2], n, n, x, x)
    assert e.value.status == BAD and "CUDA" in str(e.value)
    with pytest.raises(sp.SantappError):
        sp.santapp_prompt_attn(g, [1, 2], x, x, x)


# ---- frequencies ----
@pytest.mark.parametrize("rot,theta", [(128, 1e4), (64, 5e5), (16, 1e6)])
def test_frequencies(lib, rot, theta):
    want = theta ** (-np.arange(0, rot, 2) / rot)
    np.testing.assert_allclose(sp.Rope(rot, theta).inv_freq, want, rtol=1e-14)
    np.testing.assert_allclose(sp.Rope(rot, theta, factor=4.0).inv_freq, want / 4, rtol=1e-14)
    got = np.array(sp.Rope(rot, theta, factor=8.0, low=1.0, high=4.0, original_len=8192).inv_freq)
    turns = 8192 * want / (2 * math.pi)
    assert np.allclose(got[turns >= 4], want[turns >= 4], rtol=1e-14)
    assert np.allclose(got[turns <= 1], want[turns <= 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 4)
    keep = (turns[mid] - 1) / 3
    np.testing.assert_allclose(got[mid], want[mid] * (keep + (1 - keep) / 8), rtol=1e-12)


def test_frequencies_given(lib):
    assert sp.Rope(16, inv_freq=[1, 2, 3, 4, 5, 6, 7, 8]).inv_freq == [1, 2, 3, 4, 5, 6, 7, 8]
    with pytest.raises(sp.SantappError):
        sp.Rope(16, inv_freq=[1, 2])


@pytest.mark.parametrize("kw", [dict(theta=1.0), dict(theta=math.nan), dict(factor=0.5), dict(original_len=-1.0), dict(original_len=100.0, low=4.0, high=4.0)])
def test_frequencies_refuse(lib, kw):
    with pytest.raises(sp.SantappError) as e:
        sp.Rope(128, **{**dict(theta=1e4, factor=2.0), **kw})
    assert e.value.status == BAD
