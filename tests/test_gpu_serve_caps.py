"""Caps of every size against the definition in 64 bits: a capped score keeps its accuracy, not the cap's."""
import math

import pytest
import torch

import serve_reference as ref
from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


def rand(*shape, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed + sum(shape))
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def capped(q, k, v, seen, scale, cap, weight_off):
    """One head, as ref.attend has it, but for the cap's own error: below 2^-19.9 of the capped score. With y = s / cap (its factor and its product
    rounded: 2^-23 of y, so at most that of tanh y): near zero a polynomial good to 2^-20.6, beyond it (1 - e) / (1 + e) with e = exp(-2 |y|) <= 0.37
    to 2^-21.6 of itself (2^-22 of the instruction, 2^-24 of its argument of at least 1.44), which moves it by 2 e / (1 - e^2) <= 0.86 of that; a
    quotient to 2^-22 and two products to 2^-24."""
    q, k, v = q.double(), k.double(), v.double()
    s = (q @ k.T) * scale
    raw = 136 * 2.0 ** -23 * (q.abs() @ k.abs().T) * scale
    s = cap * torch.tanh(s / cap)
    e = raw + 2.0 ** -19.9 * s.abs() + weight_off + 2.0 ** -18
    s = s.masked_fill(~seen, -math.inf)
    top = s.amax(1, keepdim=True)
    e = e + 2.0 ** -21 * (torch.where(seen, s, torch.zeros_like(s)).abs() + top.abs())
    p = torch.softmax(s, 1)
    o = p @ v
    pe = p * torch.where(seen, e, torch.zeros_like(e))
    return o, pe @ v.abs() + pe.sum(1, keepdim=True) * o.abs()


CAPS = [1e2, 1e4, 1e6, 1e9, 1e30, 1e36]


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("B,N,elem", [(3, 300, "bf16"), (3, 0, "fp16"), (40, 500, "fp16")])
def test_a_large_cap_leaves_the_suffix_its_scores(cap, B, N, elem):
    hq, hkv, room = 8, 2, 40
    geom = sp.Geometry(B, hq, hkv, elem_type=sp.SANTAPP_FP16 if elem == "fp16" else sp.SANTAPP_BF16)
    dt = geom.torch_dtype
    q, k, v = 3 * rand(B, hq, D, dtype=dt), rand(hkv, N, D, seed=1, dtype=dt), rand(hkv, N, D, seed=2, dtype=dt)
    ks, vs = rand(B, hkv, room, D, seed=3, dtype=dt), rand(B, hkv, room, D, seed=4, dtype=dt)
    lens = torch.full((B,), room, dtype=torch.int32, device="cuda")
    got = sp.santapp_prefix_decode_attn(geom, k if N else None, v if N else None, q, ks, vs, lens, cap=cap)
    for b in range(B):
        for h in range(hq):
            j = h // (hq // hkv)
            kk, vv = torch.cat([k[j], ks[b, j]]), torch.cat([v[j], vs[b, j]])
            want, tol = capped(q[b, h][None], kk, vv, torch.ones(1, len(kk), dtype=torch.bool, device="cuda"), 1 / math.sqrt(D), cap, 2.0 ** -16)
            ref.close_32(got[b, h], want[0], tol[0], f"sequence {b} head {h}")


@pytest.mark.parametrize("cap", [1e4, 1e6])
def test_small_scores_beside_scores_beyond_the_cap(cap):
    """Rows whose scores are small stand in one block with rows whose scores are several times the cap."""
    n, hq, hkv = 200, 4, 2
    geom = sp.Geometry(1, hq, hkv)
    q, k, v = 3 * rand(n, hq, D), rand(hkv, n, D, seed=1), rand(hkv, n, D, seed=2)
    q[::7] *= 4 * cap / 3
    got = sp.santapp_prompt_attn(geom, [n], q, k, v, cap=cap)
    seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    small = torch.arange(n, device="cuda") % 7 != 0
    for h in range(hq):
        want, tol = capped(q[:, h], k[h // 2], v[h // 2], seen, 1 / math.sqrt(D), cap, 2.0 ** -8 + 2.0 ** -17)
        ref.close_16(got[small, h], want[small], tol[small], f"head {h}")
    B = 8
    gq = 3 * rand(B, 8, D, seed=5)
    gq[::2] *= 4 * cap / 3
    one = sp.santapp_prefix_decode_attn(sp.Geometry(B, 8, hkv), k, v, gq, None, None, None, cap=cap)
    for b in range(1, B, 2):
        for h in range(8):
            want, tol = capped(gq[b, h][None], k[h // 4], v[h // 4], torch.ones(1, n, dtype=torch.bool, device="cuda"), 1 / math.sqrt(D), cap, 2.0 ** -16)
            ref.close_32(one[b, h], want[0], tol[0], f"sequence {b} head {h}")
