"""santapp_rope_append and santapp_rope_prompt against the rotation in 64 bits."""
import pytest
import torch

import serve_reference as ref
from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


def geometry(n, hq, hkv, elem):
    return sp.Geometry(n, hq, hkv, D, elem_type=sp.SANTAPP_FP16 if elem == "fp16" else sp.SANTAPP_BF16)


def qkv(n, hq, hkv, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, hq + 2 * hkv, D, generator=g, device="cuda").to(dtype)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


ROPES = [dict(rot_dim=128), dict(rot_dim=128, interleaved=True), dict(rot_dim=64, interleaved=True, theta=5e5), dict(rot_dim=96),
         dict(rot_dim=16), dict(rot_dim=32, interleaved=True, factor=4.0),
         dict(rot_dim=128, theta=5e5, factor=8.0, low=1.0, high=4.0, original_len=8192.0, amplitude=1.2)]


@pytest.mark.parametrize("kw", ROPES)
@pytest.mark.parametrize("elem", ["bf16", "fp16"])
@pytest.mark.parametrize("n,hq,hkv", [(1, 28, 4), (5, 8, 8), (67, 12, 4)])
def test_append_rotates_and_writes_one_row(kw, elem, n, hq, hkv):
    geom, rope, cap = geometry(n, hq, hkv, elem), sp.Rope(**kw), 9
    q, k, v = qkv(n, hq, hkv, geom.torch_dtype)
    lens = torch.tensor([(7 * b) % cap for b in range(n)], dtype=torch.int32, device="cuda")
    base = torch.tensor([(b * 104729) % 200000 for b in range(n)], dtype=torch.int32, device="cuda")
    ks = torch.randn(n, hkv, cap, D, device="cuda").to(geom.torch_dtype)
    vs = torch.randn(n, hkv, cap, D, device="cuda").to(geom.torch_dtype)
    k0, v0, out_len = ks.clone(), vs.clone(), torch.empty_like(lens)
    out = sp.santapp_rope_append(geom, rope, q, k, v, base, lens, ks, vs, suffix_len_out=out_len)
    pos = base.long() + lens.long()
    want, off = ref.rotate(rope, q, pos, kw.get("interleaved", False))
    ref.close_16(out, want, off, "q")
    want, off = ref.rotate(rope, k, pos, kw.get("interleaved", False))
    b = torch.arange(n, device="cuda")
    ref.close_16(ks[b, :, lens.long()], want, off, "k")
    assert torch.equal(vs[b, :, lens.long()], v)
    k0[b, :, lens.long()], v0[b, :, lens.long()] = ks[b, :, lens.long()], vs[b, :, lens.long()]
    assert torch.equal(ks, k0) and torch.equal(vs, v0), "other rows changed"
    assert torch.equal(out_len, lens + 1)
    rot = rope.c.rot_dim
    assert torch.equal(out[..., rot:], q[..., rot:]), "values past rot_dim are copied"


def test_append_for_a_very_large_batch():
    """Several tokens a block, the last block not full, lengths in place, some slots padded."""
    n, cap = 2501, 3
    geom, rope = geometry(n, 4, 2, "bf16"), sp.Rope(rot_dim=32)
    q, k, v = qkv(n, 4, 2, geom.torch_dtype, 2)
    lens = torch.arange(n, dtype=torch.int32, device="cuda") % 5 - 1
    base = torch.arange(n, dtype=torch.int32, device="cuda") * 7
    ks = torch.zeros(n, 2, cap, D, dtype=geom.torch_dtype, device="cuda")
    vs = torch.zeros_like(ks)
    n0 = lens.clone()
    out = sp.santapp_rope_append(geom, rope, q, k, v, base, lens, ks, vs, suffix_len_out=lens)
    live = (n0 >= 0) & (n0 < cap)
    assert torch.equal(lens, torch.where(live, n0 + 1, n0))
    b = live.nonzero()[:, 0]
    at = n0[b].long()
    want, off = ref.rotate(rope, q[b], base[b].long() + at, False)
    ref.close_16(out[b], want, off, "q")
    want, off = ref.rotate(rope, k[b], base[b].long() + at, False)
    ref.close_16(ks[b, :, at], want, off, "k")
    assert torch.equal(vs[b, :, at], v[b])
    written = torch.zeros(n, cap, dtype=torch.bool, device="cuda")
    written[b, at] = True
    assert not bool(ks.transpose(1, 2)[~written].any()) and not bool(vs.transpose(1, 2)[~written].any())


def test_append_in_place_and_lengths_in_place():
    geom, rope = geometry(6, 28, 4, "bf16"), sp.Rope()
    q, k, v = (x.contiguous() for x in qkv(6, 28, 4, geom.torch_dtype))
    lens = torch.tensor([0, 1, 2, 3, 0, 1], dtype=torch.int32, device="cuda")
    base = torch.full((6,), 100, dtype=torch.int32, device="cuda")
    ks, vs = torch.zeros(6, 4, 8, D, dtype=geom.torch_dtype, device="cuda"), torch.zeros(6, 4, 8, D, dtype=geom.torch_dtype, device="cuda")
    want = sp.santapp_rope_append(geom, rope, q, k, v, base, lens.clone(), ks.clone(), vs.clone())
    n0 = lens.clone()
    got = sp.santapp_rope_append(geom, rope, q, k, v, base, lens, ks, vs, q_out=q, suffix_len_out=lens)
    assert got.data_ptr() == q.data_ptr() and torch.equal(q, want) and torch.equal(lens, n0 + 1)


def test_append_leaves_full_and_padded_sequences_alone():
    geom, rope, cap = geometry(4, 8, 2, "bf16"), sp.Rope(), 4
    q, k, v = qkv(4, 8, 2, geom.torch_dtype)
    lens = torch.tensor([4, -1, 3, 2147483647], dtype=torch.int32, device="cuda")
    base = torch.full((4,), 2147483000, dtype=torch.int32, device="cuda")
    ks = torch.randn(4, 2, cap, D, device="cuda").to(geom.torch_dtype)
    vs, out = ks.clone(), torch.full((4, 8, D), 7.0, device="cuda").to(geom.torch_dtype)
    k0, out_len = ks.clone(), torch.empty_like(lens)
    sp.santapp_rope_append(geom, rope, q, k, v, base, lens, ks, vs, q_out=out, suffix_len_out=out_len)
    assert out_len.tolist() == [4, -1, 4, 2147483647]
    for b in (0, 1, 3):
        assert torch.equal(ks[b], k0[b]) and torch.equal(vs[b], k0[b]) and bool((out[b] == 7).all())
    assert torch.equal(ks[2, :, :3], k0[2, :, :3]) and not torch.equal(ks[2, :, 3], k0[2, :, 3])


@pytest.mark.parametrize("n", [1, 3, 590, 2368, 2371, 5001])
@pytest.mark.parametrize("kw,elem", [(ROPES[0], "bf16"), (ROPES[2], "fp16"), (ROPES[6], "bf16")])
def test_prompt_rows(n, kw, elem):
    geom, rope = geometry(1, 12, 4, elem), sp.Rope(**kw)
    q, k, v = qkv(n, 12, 4, geom.torch_dtype)
    kp = torch.zeros(4, n, D, dtype=geom.torch_dtype, device="cuda")
    vp = torch.zeros_like(kp)
    out = sp.santapp_rope_prompt(geom, rope, q, k, v, None, kp, vp)
    pos = torch.arange(n, device="cuda")
    want, off = ref.rotate(rope, q, pos, kw.get("interleaved", False))
    ref.close_16(out, want, off, "q")
    want, off = ref.rotate(rope, k, pos, kw.get("interleaved", False))
    ref.close_16(kp, want.transpose(0, 1), off.transpose(0, 1), "k")
    assert torch.equal(vp, v.transpose(0, 1))


def test_prompt_rows_go_where_they_are_sent():
    """Rows of a chunk into larger planes, in any order; a destination outside is not written; positions far out."""
    n, rows = 50, 200
    geom, rope = geometry(1, 28, 4, "bf16"), sp.Rope(theta=1e6)
    q, k, v = qkv(n, 28, 4, geom.torch_dtype)
    g = torch.Generator().manual_seed(3)
    dst = torch.randperm(rows, generator=g)[:n].to(torch.int32).cuda()
    dst[7], dst[9] = -1, rows
    pos = torch.randint(-5, 2 ** 31 - 1, (n,), generator=g).to(torch.int32).cuda()
    kp = torch.full((4, rows, D), 3.0, device="cuda").to(geom.torch_dtype)
    vp = kp.clone()
    out = sp.santapp_rope_prompt(geom, rope, q, k, v, pos, kp, vp, dst_row=dst)
    want, off = ref.rotate(rope, q, pos, False)
    ref.close_16(out, want, off, "q")
    want, off = ref.rotate(rope, k, pos, False)
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[7] = keep[9] = False
    at = dst[keep].long()
    ref.close_16(kp[:, at], want[keep].transpose(0, 1), off[keep].transpose(0, 1), "k")
    assert torch.equal(vp[:, at], v[keep].transpose(0, 1))
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert bool((kp[:, rest] == 3).all()) and bool((vp[:, rest] == 3).all())


def test_one_rotation_undoes_another():
    """Angles are odd in the position: a row turned by p and then by -p is itself, up to two roundings."""
    geom, rope, n = geometry(1, 8, 8, "bf16"), sp.Rope(theta=5e5), 33
    q, k, v = qkv(n, 8, 8, geom.torch_dtype)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 3989
    kp, vp = torch.empty(8, n, D, dtype=geom.torch_dtype, device="cuda"), torch.empty(8, n, D, dtype=geom.torch_dtype, device="cuda")
    there = sp.santapp_rope_prompt(geom, rope, q, k, v, pos, kp, vp)
    back = sp.santapp_rope_prompt(geom, rope, there, k, v, -pos, kp, vp)
    size = torch.sqrt(q.double()[..., :64] ** 2 + q.double()[..., 64:] ** 2).repeat(1, 1, 2)
    # roundings there move the pair by at most 2^-8 of its size, and as far when turned back; the last one is 2^-8 of the result
    assert bool(((back.double() - q.double()).abs() <= size * 2.02 * 2.0 ** -8 + 1e-6).all())
