"""Calls at the edges of what the operators around the decode step take."""
import pytest
import torch

from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


def rand(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + sum(shape))
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def test_a_prompt_call_without_new_rows():
    geom, k, v = sp.Geometry(2, 8, 2), rand(2, 12, D), rand(2, 12, D, seed=1)
    none = torch.empty(0, 8, D, dtype=torch.bfloat16, device="cuda")
    assert sp.santapp_prompt_attn(geom, [5, 7], none, k, v, new_len=[0, 0]).shape == (0, 8, D)
    assert sp.santapp_last_launch_count() == 0
    for lens, new, kk in (([5, 7], [1, -1], k), ([5, 8], [0, 0], k), ([5, 7], [0, 0], k.float()), ([12, 0], [0, 0], k)):
        with pytest.raises(sp.SantappError) as e:
            sp.santapp_prompt_attn(geom, lens, none, kk, v, new_len=new)
        assert e.value.status == sp.SANTAPP_ERR_INVALID_ARG


def test_a_fork_on_a_given_stream():
    geom, k, v = sp.Geometry(2, 8, 2), rand(2, 2, 20, D), rand(2, 2, 20, D, seed=1)
    k0, v0 = k.clone(), v.clone()
    src, lens = torch.tensor([1, 0], dtype=torch.int32, device="cuda"), torch.tensor([20, 3], dtype=torch.int32, device="cuda")
    new = torch.zeros_like(lens)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    sp.santapp_suffix_fork(geom, src, lens, k, v, suffix_len_out=new, stream=s)
    s.synchronize()
    assert new.tolist() == [3, 20]
    assert torch.equal(k[1], k0[0]) and torch.equal(v[1], v0[0]) and torch.equal(k[0, :, :3], k0[1, :, :3]) and torch.equal(k[0, :, 3:], k0[0, :, 3:])


@pytest.mark.parametrize("new,both,hq,hkv", [(None, 0, 1, 1), (None, 0, 28, 4), (257, 0, 1, 1), (130, 0, 7, 1), (None, 300, 1, 1), (400, 461, 16, 2)])
def test_how_far_an_infinite_value_reaches(new, both, hq, hkv):
    """Queries that see row i have no finite output; those whose last visible row is more than 254 rows before it are as if it were finite."""
    n, i = 514, 511
    m = n if new is None else new
    geom, q, k, v = sp.Geometry(1, hq, hkv), rand(m, hq, D), rand(hkv, n, D, seed=1), rand(hkv, n, D, seed=2)
    opts = dict(new_len=None if new is None else [new], prefix_len=[both])
    want = sp.santapp_prompt_attn(geom, [n], q, k, v, **opts)
    v[:, i] = float("inf")
    got = sp.santapp_prompt_attn(geom, [n], q, k, v, **opts)
    last = torch.maximum(torch.arange(n - m, n, device="cuda"), torch.tensor(both - 1, device="cuda"))
    assert not bool(torch.isfinite(got[last >= i]).any())
    assert torch.equal(got[last < i - 254], want[last < i - 254])
