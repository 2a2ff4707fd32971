"""santapp_prefix_decode_attn where scores are no numbers: what attends them is no number either, whatever part of the prompt they are in."""
import pytest
import torch

from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


def rand(*shape, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed + sum(shape))
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("B", [2, 6, 40])
@pytest.mark.parametrize("N", [100, 3000])
@pytest.mark.parametrize("suffix", ["empty", "none"])
def test_a_query_that_is_no_number_gives_none(B, N, suffix):
    hq, hkv = 12, 4
    geom, q, k, v = sp.Geometry(B, hq, hkv), rand(B, hq, D), rand(hkv, N, D, seed=1), rand(hkv, N, D, seed=2)
    ks, vs = rand(B, hkv, 8, D, seed=3), rand(B, hkv, 8, D, seed=4)
    rest = (ks, vs, torch.zeros(B, dtype=torch.int32, device="cuda")) if suffix == "empty" else (None, None, None)
    want = sp.santapp_prefix_decode_attn(geom, k, v, q, *rest)
    q[1, 5] = float("nan")
    got = sp.santapp_prefix_decode_attn(geom, k, v, q, *rest)
    assert bool(torch.isnan(got[1, 5]).all())
    got[1, 5] = want[1, 5]
    assert torch.equal(got, want)


@pytest.mark.parametrize("B,lens", [(2, [0, 5]), (40, None)])
@pytest.mark.parametrize("first,last", [(0, 128), (1024, 4096), (8000, 8192)])
def test_keys_that_are_no_numbers_are_not_left_out(B, lens, first, last):
    """A stretch of keys that fills one part of the prompt or several: whoever attends them gets no number, on that KV head alone."""
    hq, hkv, N = 8, 2, 8192
    geom, q, k, v = sp.Geometry(B, hq, hkv), rand(B, hq, D), rand(hkv, N, D, seed=1), rand(hkv, N, D, seed=2)
    ks, vs = rand(B, hkv, 8, D, seed=3), rand(B, hkv, 8, D, seed=4)
    n = torch.tensor(lens if lens else [b % 9 for b in range(B)], dtype=torch.int32, device="cuda")
    want = sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, n)
    k[1, first:last] = float("nan")
    got = sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, n)
    assert bool(torch.isnan(got[:, hq // 2:]).all())
    assert torch.equal(got[:, :hq // 2], want[:, :hq // 2])
