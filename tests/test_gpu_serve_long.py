"""One query over very many keys: a block of prompt attention walks all of them, a part of the shared prefix a share."""
import pytest
import torch

from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("rows", [1 << 20, (1 << 23) + 1])
def test_equal_keys_and_values_give_the_value(rows):
    """Sums of ones are exact up to 2^24. The last tile holds rows of the next sequence."""
    geom, lens = sp.Geometry(2, 1, 1), [rows + 1, 5]
    kv = torch.ones(1, sum(lens), D, dtype=torch.bfloat16, device="cuda")
    kv[:, rows + 1:] = float("nan")
    q = torch.randn(1, 1, D, device="cuda").to(torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = sp.santapp_prompt_attn(geom, lens, q, kv, kv, new_len=[1, 0], status=status)
    assert int(status) == 0 and bool((out == 1).all())
    out = sp.santapp_prefix_decode_attn(sp.Geometry(1, 1, 1), kv[:, :rows + 1], kv[:, :rows + 1], q, None, None, None, status=status)
    assert int(status) == 0 and bool((out == 1).all())


def test_a_mean_over_a_million_keys():
    """Keys of equal weight. A stream adds half of the n keys to its sums, 16 at a time; the tensor core cuts a sum to fp32 (less than 2^-23 of it
    each time), and the sum of weights, of whole numbers below 2^24, is exact. The prefix call cuts the keys into a part per SM of at most 56
    tiles: 28 for a stream, 16 products each (two terms of a weight), so cuts of 448 * 2^-23, and roundings of the merge below 2^-16: 2^-14 in
    all. Values are positive, so relative errors of the sums are those of the result."""
    n = 1 << 20
    k = torch.zeros(1, n, D, dtype=torch.bfloat16, device="cuda")
    v = torch.rand(1, n, D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    want = v.double().mean(1)[0]
    q = torch.randn(1, 1, D, device="cuda").to(torch.bfloat16)
    geom = sp.Geometry(1, 1, 1)
    out = sp.santapp_prompt_attn(geom, [n], q, k, v, new_len=[1])[0, 0]
    assert bool(((out.double() - want).abs() <= want * (2.0 ** -8 + n / 2 / 16 * 2.0 ** -23)).all())
    out = sp.santapp_prefix_decode_attn(geom, k, v, q, None, None, None)[0, 0]
    assert bool(((out.double() - want).abs() <= want * 2.0 ** -14).all())
