"""santapp_prefix_decode_attn against softmax attention in 64 bits, and against the dense call on repeated records."""
import math

import pytest
import torch

import serve_reference as ref
from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


def inputs(B, hq, hkv, N, cap, elem, seed=0, q_scale=1.5):
    geom = sp.Geometry(B, hq, hkv, D, elem_type=sp.SANTAPP_FP16 if elem == "fp16" else sp.SANTAPP_BF16)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = geom.torch_dtype

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    k, v = rand(hkv, N, D).to(dt), rand(hkv, N, D).to(dt)
    ks, vs = rand(B, hkv, cap, D).to(dt), rand(B, hkv, cap, D).to(dt)
    q = (q_scale * rand(B, hq, D)).to(dt)
    lens = torch.randint(0, cap + 1, (B,), generator=g, device="cuda").to(torch.int32)
    return geom, q, k, v, ks, vs, lens


def slopes_of(hq):
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / hq) / 8 for i in range(hq)], dtype=torch.float32, device="cuda")


def check(B, hq, hkv, N, cap, elem="bf16", cap_score=0.0, bias=False, packed=False, lens=None, scale=0.0):
    geom, q, k, v, ks, vs, n = inputs(B, hq, hkv, N, cap, elem, B * 1000 + N)
    if lens is not None:
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    seen = n.clamp(0, cap).tolist()
    # rows that nobody may see hold what must not be touched
    for b in range(B):
        ks[b, :, seen[b]:], vs[b, :, seen[b]:] = float("nan"), float("inf")
    token = None
    if packed:
        token = torch.stack([torch.randperm(N, device="cuda") for _ in range(hkv)]).to(torch.int32)
    slopes = slopes_of(hq) if bias else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = sp.santapp_prefix_decode_attn(geom, k if N else None, v if N else None, q, ks if cap else None, vs if cap else None, n if cap else None,
                                        scale=scale, cap=cap_score, slopes=slopes, prefix_token=token, status=status)
    want, tol = ref.prefix_decode(k if N else None, v, token, q, ks, vs, seen if cap else [0] * B, scale or 1 / math.sqrt(D), cap_score, slopes)
    assert int(status) == 0
    ref.close_32(out, want, tol)
    if not N:
        for b in range(B):
            if seen[b] == 0:
                assert bool((out[b] == 0).all())


@pytest.mark.parametrize("N", [1, 2, 127, 128, 129, 255, 257, 1000, 5000])
@pytest.mark.parametrize("B", [1, 3])
def test_prefix_lengths(N, B):
    check(B, 28, 4, N, 20)


@pytest.mark.parametrize("B", [18, 19, 36, 37, 40, 64])
def test_batches_beyond_one_row_tile(B):
    check(B, 7, 1, 700, 33)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (16, 2), (12, 4), (5, 1), (6, 1)])
@pytest.mark.parametrize("elem", ["bf16", "fp16"])
def test_head_layouts(hq, hkv, elem):
    check(4, hq, hkv, 1500, 50, elem)


@pytest.mark.parametrize("cap_score,bias,packed", [(0.0, True, False), (0.0, True, True), (20.0, False, False), (8.0, True, True)])
@pytest.mark.parametrize("B,elem", [(3, "bf16"), (40, "fp16")])
def test_scores(cap_score, bias, packed, B, elem):
    check(B, 8, 2, 1111, 40, elem, cap_score, bias, packed)


@pytest.mark.parametrize("cap", [1, 15, 16, 17, 300, 1024])
def test_suffix_lengths(cap):
    check(3, 12, 4, 300, cap, lens=[cap, cap // 2, 1])


def test_lengths_are_clamped_and_rows_may_be_empty():
    check(4, 28, 4, 200, 12, lens=[-3, 0, 99, 12])
    check(4, 28, 4, 0, 12, lens=[0, 5, -1, 12])
    check(2, 8, 2, 500, 0)
    check(2, 8, 2, 0, 0)


def test_a_large_batch():
    check(300, 8, 2, 260, 5)


def test_no_lengths_are_no_suffix():
    geom, q, k, v, ks, vs, lens = inputs(3, 8, 2, 300, 16, "bf16", 23)
    got = sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, None)
    assert torch.equal(got, sp.santapp_prefix_decode_attn(geom, k, v, q, None, None, None))


def test_a_first_call_may_be_captured():
    """Set-up that a kernel needs once (shared memory beyond the default) is no work on the stream."""
    B, N = 2, 200
    geom, q, k, v, ks, vs, lens = inputs(B, 12, 12, N, 8, "fp16", 29)
    slopes = slopes_of(12)
    out = torch.zeros(B, 12, D, device="cuda")
    ws = torch.empty(sp.santapp_prefix_decode_workspace_bytes(geom, N, 8), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens, cap=9.0, slopes=slopes, out=out, workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    want, tol = ref.prefix_decode(k, v, None, q, ks, vs, lens.tolist(), 1 / math.sqrt(D), 9.0, slopes)
    ref.close_32(out, want, tol)


def test_scale():
    check(2, 8, 2, 400, 8, scale=0.21)


def test_against_the_dense_call_on_repeated_records():
    B, N, cap = 3, 2000, 64
    geom, q, k, v, ks, vs, lens = inputs(B, 28, 4, N, cap, "bf16", 4)
    one = sp.Geometry(1, 28, 4)
    teams = sp.santapp_build_teams(one, [N], k, v)
    got = sp.santapp_prefix_decode_attn(geom, teams.k_packed, teams.v_packed, q, ks, vs, lens)
    many = sp.santapp_build_teams(geom, [N] * B, k.repeat(1, B, 1), v.repeat(1, B, 1))
    want = sp.santapp_dense_decode_attn(geom, many, q, ks, vs, lens)
    # both are fp32 evaluations of one sum: the dense call's own bar, once for each
    assert float((got - want).abs().max()) <= 2e-3 * float(v.abs().max())
    assert float((got - want).norm() / want.norm()) < 1e-4


def test_distance_over_team_records_is_that_of_token_order():
    B, N, cap = 2, 1500, 16
    geom, q, k, v, ks, vs, lens = inputs(B, 8, 2, N, cap, "bf16", 8)
    teams = sp.santapp_build_teams(sp.Geometry(1, 8, 2), [N], k, v)
    slopes = slopes_of(8)
    got = sp.santapp_prefix_decode_attn(geom, teams.k_packed, teams.v_packed, q, ks, vs, lens, slopes=slopes, prefix_token=teams.row_token)
    want, tol = ref.prefix_decode(k, v, None, q, ks, vs, lens.tolist(), 1 / math.sqrt(D), 0.0, slopes)
    ref.close_32(got, want, tol)


def test_rows_behind_the_prefix_reach_nothing():
    """A prompt that fills a part of its planes: what lies behind it holds NaN."""
    B, N, plane = 5, 333, 1000
    geom, q, k, v, ks, vs, lens = inputs(B, 12, 4, N, 10, "bf16", 12)
    kp = torch.full((4, plane, D), float("nan"), device="cuda").to(torch.bfloat16)
    vp = torch.full((4, plane, D), float("nan"), device="cuda").to(torch.bfloat16)
    kp[:, :N], vp[:, :N] = k, v
    got = sp.santapp_prefix_decode_attn(geom, kp[:, :N], vp[:, :N], q, ks, vs, lens)
    assert torch.equal(got, sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens))


@pytest.mark.parametrize("B,elem", [(2, "bf16"), (4, "fp16"), (40, "bf16"), (40, "fp16")])
@pytest.mark.parametrize("most", [3, 10, 50])
def test_large_logits_and_sharp_rows(B, elem, most):
    N = 3000
    geom, q, k, v, ks, vs, lens = inputs(B, 28, 4, N, 30, elem, 3)
    k = (k.float() * torch.linspace(0.1, most, N, device="cuda")[None, :, None]).to(k.dtype)
    out = sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens)
    want, tol = ref.prefix_decode(k, v, None, q, ks, vs, lens.tolist(), 1 / math.sqrt(D))
    ref.close_32(out, want, tol)


def test_capped_scores_of_every_size():
    for scale in (0.01, 0.06, 0.09, 0.5, 4.0):
        check(3, 8, 2, 700, 20, "bf16", 2.0, scale=scale)
        check(40, 8, 2, 700, 20, "fp16", 2.0, True, scale=scale)


def test_sequences_do_not_touch_one_another():
    """A query that is not a number spoils its own heads alone."""
    B, N = 6, 900
    geom, q, k, v, ks, vs, lens = inputs(B, 12, 4, N, 16, "bf16", 17)
    want = sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens)
    q[2, 5] = float("nan")
    got = sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens)
    assert bool(torch.isnan(got[2, 5]).all())
    got[2, 5] = want[2, 5]
    assert torch.equal(got, want)


def test_a_given_stream():
    B, N = 3, 600
    geom, q, k, v, ks, vs, lens = inputs(B, 8, 2, N, 16, "bf16", 19)
    want = sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens)
    s = torch.cuda.Stream()
    out, ws = torch.zeros_like(want), torch.empty(sp.santapp_prefix_decode_workspace_bytes(geom, N, 16), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens, out=out, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


def test_offsets_past_32_bits():
    """Planes and suffixes of more than 2^32 values (the rows used are few)."""
    B, hq, hkv, N, cap, plane = 3, 8, 8, 300, 20, 5_000_000
    geom, q, k, v, ks, vs, lens = inputs(B, hq, hkv, N, cap, "bf16", 2)
    kp = torch.empty(hkv, plane, D, dtype=torch.bfloat16, device="cuda")
    vp = torch.empty(hkv, plane, D, dtype=torch.bfloat16, device="cuda")
    kp[:, :N], vp[:, :N] = k, v
    want, tol = ref.prefix_decode(k, v, None, q, ks, vs, lens.tolist(), 1 / math.sqrt(D))
    ref.close_32(sp.santapp_prefix_decode_attn(geom, kp[:, :N], vp[:, :N], q, ks, vs, lens), want, tol)
    del kp, vp
    long = 1_500_000
    kl = torch.empty(B, hkv, long, D, dtype=torch.bfloat16, device="cuda")
    vl = torch.empty(B, hkv, long, D, dtype=torch.bfloat16, device="cuda")
    kl[:, :, :cap], vl[:, :, :cap] = ks, vs
    ref.close_32(sp.santapp_prefix_decode_attn(geom, k, v, q, kl, vl, lens), want, tol)
    src = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
    sp.santapp_suffix_fork(geom, src, lens, kl, vl)
    n = int(lens[0])
    assert torch.equal(kl[2, :, :n], ks[0, :, :n]) and torch.equal(vl[2, :, :n], vs[0, :, :n])


def test_streams_workspaces_and_graphs():
    B, N = 6, 4000
    geom, q, k, v, ks, vs, lens = inputs(B, 28, 4, N, 64, "bf16", 21)
    want = sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(want) for _ in streams]
    size = sp.santapp_prefix_decode_workspace_bytes(geom, N, 64)
    spaces = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in streams]      # (NaN wherever it is read first)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o, w in zip(streams, outs, spaces):
            with torch.cuda.stream(s):
                sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens, out=o, workspace=w)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graphs = []
    for o in outs:                                       # two graphs that share a workspace, one after the other
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens, out=o, workspace=spaces[0])
        graphs.append(g)
    q.copy_(torch.roll(q, 1, 0))
    lens.copy_(torch.roll(lens, 2, 0))
    for g in graphs * 2:
        g.replay()
    torch.cuda.synchronize()
    want = sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens)
    assert all(torch.equal(o, want) for o in outs)
