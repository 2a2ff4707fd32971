"""santapp_prompt_attn against softmax attention in 64 bits."""
import math

import pytest
import torch

import serve_reference as ref
from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


def inputs(lens, new, hq, hkv, elem, seed=0, q_scale=1.0):
    geom = sp.Geometry(len(lens), hq, hkv, D, elem_type=sp.SANTAPP_FP16 if elem == "fp16" else sp.SANTAPP_BF16)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = geom.torch_dtype
    q = (q_scale * torch.randn(sum(new), hq, D, generator=g, device="cuda")).to(dt)
    k = torch.randn(hkv, sum(lens), D, generator=g, device="cuda").to(dt)
    v = torch.randn(hkv, sum(lens), D, generator=g, device="cuda").to(dt)
    return geom, q, k, v


def slopes_of(hq):
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / hq) for i in range(hq)], dtype=torch.float32, device="cuda")


def check(lens, hq, hkv, elem, new=None, both=None, cap=0.0, bias=False, scale=0.0, q_scale=1.0):
    m, p = (lens if new is None else new), ([0] * len(lens) if both is None else both)
    geom, q, k, v = inputs(lens, m, hq, hkv, elem, sum(lens), q_scale)
    slopes = slopes_of(hq) if bias else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = sp.santapp_prompt_attn(geom, lens, q, k, v, new_len=new, prefix_len=both, scale=scale, cap=cap, slopes=slopes, status=status)
    want, tol = ref.prompt(q, k, v, lens, m, p, scale or 1 / math.sqrt(D), cap, slopes)
    assert int(status) == 0
    ref.close_16(out, want, tol)


@pytest.mark.parametrize("n", [1, 2, 17, 18, 19, 37, 64, 127, 128, 129, 255, 300, 513])
def test_lengths_of_one_prompt(n):
    check([n], 28, 4, "bf16")


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (16, 2), (12, 4), (5, 1), (6, 1)])
@pytest.mark.parametrize("elem", ["bf16", "fp16"])
def test_head_layouts(hq, hkv, elem):
    check([261, 3, 130], hq, hkv, elem)


@pytest.mark.parametrize("cap,bias", [(0.0, True), (5.0, False), (30.0, True)])
@pytest.mark.parametrize("elem", ["bf16", "fp16"])
def test_scores(cap, bias, elem):
    check([200, 1, 77, 400], 12, 4, elem, cap=cap, bias=bias, q_scale=3.0)


def test_scale():
    check([150], 4, 2, "bf16", scale=0.3)


@pytest.mark.parametrize("new", [[1, 1, 1], [0, 5, 130], [300, 0, 1], [0, 0, 77]])
def test_last_rows_alone(new):
    check([300, 129, 200], 28, 4, "bf16", new=new)


@pytest.mark.parametrize("both", [[0, 1], [100, 129], [300, 129], [299, 64]])
@pytest.mark.parametrize("new", [None, [40, 129]])
def test_bidirectional_beginning(both, new):
    check([300, 129], 16, 2, "bf16", new=new, both=both)
    check([300, 129], 8, 4, "fp16", new=new, both=both, bias=True)


def test_more_sequences_than_a_launch_takes():
    check([1 + (37 * i) % 50 for i in range(210)], 4, 2, "bf16")


def test_a_longer_prompt():
    check([2500], 14, 2, "bf16")


def test_other_sequences_reach_nothing():
    """Neighbours that hold infinities and NaN (and rows behind the last one) change no bit."""
    lens = [100, 130, 61]
    geom, q, k, v = inputs(lens, lens, 28, 4, "bf16")
    want = sp.santapp_prompt_attn(geom, lens, q, k, v)
    k2, v2 = k.clone(), v.clone()
    for x in (k2, v2):
        x[:, :100], x[:, 230:] = float("nan"), float("inf")
    got = sp.santapp_prompt_attn(geom, lens, q, k2, v2)
    assert torch.equal(got[100:230], want[100:230])


@pytest.mark.parametrize("elem", ["bf16", "fp16"])
@pytest.mark.parametrize("most", [3, 12, 60])
def test_large_logits_and_sharp_rows(elem, most):
    """Scores far apart, growing along the row, so the running maximum moves often and far (or a little and often)."""
    n = 700
    geom, q, k, v = inputs([n], [n], 8, 2, elem, 5)
    k = (k.float() * torch.linspace(0.1, most, n, device="cuda")[None, :, None]).to(k.dtype)
    out = sp.santapp_prompt_attn(geom, [n], q, k, v)
    want, tol = ref.prompt(q, k, v, [n], [n], [0], 1 / math.sqrt(D))
    ref.close_16(out, want, tol)


def test_values_at_the_type_s_edge():
    n = 200
    geom, q, k, v = inputs([n], [n], 4, 4, "fp16", 6)
    v = (v.float().clamp(-1, 1) * 60000).to(torch.float16)
    out = sp.santapp_prompt_attn(geom, [n], q, k, v)
    want, tol = ref.prompt(q, k, v, [n], [n], [0], 1 / math.sqrt(D))
    ref.close_16(out, want, tol)


def test_capped_scores_of_every_size():
    """Logits far inside the cap, about it and far beyond it: the three ways a tile's tanh is taken."""
    for scale in (0.01, 0.06, 0.09, 0.5, 4.0):
        check([300], 8, 2, "bf16", cap=2.0, scale=scale)
        check([300], 8, 2, "fp16", cap=2.0, scale=scale, bias=True)


def test_rows_that_see_infinities_and_zeros():
    """A key of zeros weighs like any other; an infinite value reaches exactly the queries behind it."""
    n = 260
    geom, q, k, v = inputs([n], [n], 4, 4, "bf16", 31)
    k[:, 5], q[7] = 0, 0
    v[:, 200] = float("inf")
    out = sp.santapp_prompt_attn(geom, [n], q, k, v)
    v2 = v.clone()
    v2[:, 200] = 0
    want, tol = ref.prompt(q, k, v2, [n], [n], [0], 1 / math.sqrt(D))
    ref.close_16(out[:128], want[:128], tol[:128])       # (queries 128 .. 199 share a tile of keys with row 200, as the header says)
    assert not bool(torch.isfinite(out[200:]).any())


def test_runs_are_alike_and_captured_ones_too():
    lens = [333, 80]
    geom, q, k, v = inputs(lens, lens, 28, 4, "bf16", 9)
    want = sp.santapp_prompt_attn(geom, lens, q, k, v)
    out = torch.empty_like(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            sp.santapp_prompt_attn(geom, lens, q, k, v, out=out)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.santapp_prompt_attn(geom, lens, q, k, v, out=out)
    q.copy_(torch.roll(q, 1, 0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, sp.santapp_prompt_attn(geom, lens, q, k, v))
