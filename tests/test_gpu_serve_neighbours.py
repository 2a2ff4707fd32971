"""What stands beside a sequence's rows, in the batch or behind them in memory, changes none of its bits."""
import pytest
import torch

from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


def rand(*shape, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed + sum(shape))
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("cap,bias", [(5.0, False), (0.0, True), (30.0, True)])
@pytest.mark.parametrize("what", [float("inf"), float("nan"), 1e4, -1e4])
@pytest.mark.parametrize("elem", ["bf16", "fp16"])
def test_other_sequences_reach_nothing_with_cap_and_bias(cap, bias, what, elem):
    """Not a bit of a sequence's rows depends on its neighbours' keys and values."""
    lens = [100, 130, 61]
    geom = sp.Geometry(3, 28, 4, elem_type=sp.SANTAPP_FP16 if elem == "fp16" else sp.SANTAPP_BF16)
    q, k, v = (rand(x, y, D, seed=z, dtype=geom.torch_dtype) for x, y, z in ((291, 28, 0), (4, 291, 1), (4, 291, 2)))
    slopes = torch.linspace(0.01, 0.4, 28, device="cuda") if bias else None
    want = sp.santapp_prompt_attn(geom, lens, q, k, v, cap=cap, slopes=slopes)
    for x in (k, v):
        x[:, :100], x[:, 230:] = what, what
    got = sp.santapp_prompt_attn(geom, lens, q, k, v, cap=cap, slopes=slopes)
    assert torch.equal(got[100:230], want[100:230])


@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_rows_behind_a_prefix_reach_nothing_with_a_cap(cap):
    B, N, plane = 5, 333, 1000
    geom, q = sp.Geometry(B, 12, 4), rand(B, 12, D)
    kp, vp = rand(4, plane, D, seed=1), rand(4, plane, D, seed=2)
    ks, vs = rand(B, 4, 10, D, seed=3), rand(B, 4, 10, D, seed=4)
    lens = torch.tensor([0, 3, 10, 7, 1], dtype=torch.int32, device="cuda")
    want = sp.santapp_prefix_decode_attn(geom, kp[:, :N].contiguous(), vp[:, :N].contiguous(), q, ks, vs, lens, cap=cap)
    for x in (kp, vp):
        x[:, N:] = float("inf")
    for b in range(B):
        ks[b, :, int(lens[b]):] = float("inf")
        vs[b, :, int(lens[b]):] = float("nan")
    assert torch.equal(sp.santapp_prefix_decode_attn(geom, kp[:, :N], vp[:, :N], q, ks, vs, lens, cap=cap), want)
