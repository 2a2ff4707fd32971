"""santapp_suffix_fork against copies of whole slots taken before any is written."""
import pytest
import torch

from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


def run(src, lens, hkv, cap, elem="bf16", stream=None):
    n = len(src)
    geom = sp.Geometry(n, hkv, hkv, D, elem_type=sp.SANTAPP_FP16 if elem == "fp16" else sp.SANTAPP_BF16)
    g = torch.Generator(device="cuda").manual_seed(n * 31 + cap)
    k = torch.randn(n, hkv, cap, D, generator=g, device="cuda").to(geom.torch_dtype)
    v = torch.randn(n, hkv, cap, D, generator=g, device="cuda").to(geom.torch_dtype)
    k0, v0 = k.clone(), v.clone()
    s, t = torch.tensor(src, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    sp.santapp_suffix_fork(geom, s, t, k, v, suffix_len_out=out)
    want_len = []
    for b, a in enumerate(src):
        m = min(max(lens[a], 0), cap) if 0 <= a < n else 0
        want_len.append(m)
        assert torch.equal(k[b, :, :m], k0[a, :, :m] if m else k[b, :, :0]), (b, a)
        assert torch.equal(v[b, :, :m], v0[a, :, :m] if m else v[b, :, :0]), (b, a)
        assert torch.equal(k[b, :, m:], k0[b, :, m:]) and torch.equal(v[b, :, m:], v0[b, :, m:]), "rows behind the new length"
    assert out.tolist() == want_len
    assert t.tolist() == lens


@pytest.mark.parametrize("cap", [1, 15, 64, 257])
@pytest.mark.parametrize("src", [[0], [1, 0], [1, 2, 0], [0, 0, 0, 0], [3, 3, 1, 1, 7, -1, 5, 5], [2, 0, 4, 1, 3, 5, -5, 99]])
def test_chains_cycles_and_copies(src, cap):
    run(src, [(11 * b + 5) % (cap + 1) for b in range(len(src))], 4, cap)


@pytest.mark.parametrize("n,hkv,cap,elem", [(2, 8, 1024, "bf16"), (33, 1, 100, "fp16"), (257, 2, 7, "bf16"), (700, 1, 3, "bf16"), (1500, 1, 2, "fp16"), (4096, 1, 2, "bf16")])
def test_whole_batches(n, hkv, cap, elem):
    g = torch.Generator().manual_seed(n)
    src = torch.randint(-1, n + 1, (n,), generator=g).tolist()
    run(src, torch.randint(0, cap + 1, (n,), generator=g).tolist(), hkv, cap, elem)
    run(torch.randperm(n, generator=g).tolist(), [cap] * n, hkv, cap, elem)


def test_compaction_moves_the_live_slots_to_the_front():
    run([1, 4, 6, -1, -1, -1, -1], [5, 9, 1, 16, 3, 2, 8], 4, 16)


def test_lengths_are_clamped():
    run([1, 2, 0], [-3, 99, 2 ** 31 - 1], 2, 12)


def test_without_new_lengths():
    geom = sp.Geometry(2, 4, 4, D)
    k = torch.randn(2, 4, 8, D, device="cuda").to(torch.bfloat16)
    v, k0 = k.clone(), k.clone()
    src, n = torch.tensor([1, 1], dtype=torch.int32, device="cuda"), torch.tensor([8, 5], dtype=torch.int32, device="cuda")
    sp.santapp_suffix_fork(geom, src, n, k, v)
    assert torch.equal(k[0, :, :5], k0[1, :, :5]) and torch.equal(k[0, :, 5:], k0[0, :, 5:]) and torch.equal(k[1], k0[1])
