"""Buffers that the binding makes for a call on a given stream: they belong to that stream, so no work of the current stream is
beside them, neither what was under way when the call was made nor what comes after it."""
import pytest
import torch

from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128
HOLD = 200_000_000            # cycles: a stream is busy for about a tenth of a second, far longer than the calls below


def rand(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + sum(shape))
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def cases():
    """name -> (call(stream) -> tensor, bytes of the workspace it makes)"""
    B, hq, hkv, N, cap = 3, 8, 2, 900, 16
    geom, one = sp.Geometry(B, hq, hkv), sp.Geometry(1, hq, hkv)
    q, k, v = rand(B, hq, D), rand(hkv, N, D, seed=1), rand(hkv, N, D, seed=2)
    ks, vs = rand(B, hkv, cap, D, seed=3), rand(B, hkv, cap, D, seed=4)
    lens = torch.tensor([cap, 3, 0], dtype=torch.int32, device="cuda")
    at = torch.tensor([N, N, N], dtype=torch.int32, device="cuda")
    qp, kp, vp = rand(N, hq, D, seed=5), rand(N, hkv, D, seed=6), rand(N, hkv, D, seed=7)
    k_to, v_to = torch.zeros_like(k), torch.zeros_like(v)
    k_few, v_few, few_lens = rand(B, hkv, cap, D, seed=8), rand(B, hkv, cap, D, seed=11), torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    rope = sp.Rope()
    teams = sp.santapp_build_teams(sp.Geometry(B, hq, hkv, D, 64, 8), [300, 300, 300], k, v)
    tg = teams.geom
    lg = sp.LatentGeometry(2, 16, 16, 4)
    rows = rand(600, sp.LATENT_ROW, seed=9)
    latent = sp.santapp_latent_build_teams(lg, [400, 200], rows)
    ql = rand(2, 16, sp.LATENT_ROW, seed=10)
    torch.cuda.synchronize()
    return {
        "prefix_decode": (lambda s: sp.santapp_prefix_decode_attn(geom, k, v, q, ks, vs, lens, stream=s),
                          sp.santapp_prefix_decode_workspace_bytes(geom, N, cap)),
        "prompt": (lambda s: sp.santapp_prompt_attn(one, [N], qp, k, v, stream=s), 0),
        "rope_prompt": (lambda s: sp.santapp_rope_prompt(one, rope, qp, kp, vp, None, k_to, v_to, stream=s), 0),
        "rope_append": (lambda s: sp.santapp_rope_append(geom, rope, q, kp[:B], vp[:B], at, few_lens, k_few, v_few, stream=s), 0),
        "decode": (lambda s: sp.santapp_decode_attn(tg, teams, q, ks, vs, lens, 4, 11, 0, stream=s), sp.santapp_decode_workspace_bytes(tg, teams, 4)),
        "dense": (lambda s: sp.santapp_dense_decode_attn(tg, teams, q, ks, vs, lens, stream=s), sp.santapp_dense_workspace_bytes(tg, teams)),
        "dense_noalloc": (lambda s: sp.santapp_dense_decode_attn_noalloc(tg, teams, q, ks, vs, lens, stream=s), 0),
        "build": (lambda s: sp.santapp_build_teams(tg, [300, 300, 300], k, v, stream=s).k_packed, 0),
        "kmeans": (lambda s: sp.santapp_kmeans_fit(one, [N], [9], k, batch_size=128, max_iter=3, no_host_poll=True, stream=s)[0], 0),
        "latent_build": (lambda s: sp.santapp_latent_build_teams(lg, [400, 200], rows, stream=s).rows_packed, 0),
        "latent_decode": (lambda s: sp.santapp_latent_decode_attn(lg, latent, ql, None, None, 4, 11, 0, 0.07, stream=s),
                          sp.santapp_latent_decode_workspace_bytes(lg, latent, 4, 0)),
        "latent_dense": (lambda s: sp.santapp_latent_dense_decode_attn(lg, latent, ql, None, None, 0.07, stream=s),
                         sp.santapp_latent_dense_workspace_bytes(lg, latent)),
    }


NAMES = ["prefix_decode", "prompt", "rope_prompt", "rope_append", "decode", "dense", "dense_noalloc", "build", "kmeans", "latent_build", "latent_decode",
         "latent_dense"]


@pytest.mark.parametrize("name", NAMES)
def test_outputs_are_not_memory_that_the_current_stream_still_writes(name):
    call, _ = cases()[name]
    want = call(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    torch.cuda._sleep(HOLD)
    busy = [torch.empty(want.numel() * want.element_size(), dtype=torch.uint8, device="cuda") for _ in range(8)]
    for x in busy:
        x.fill_(7)                                       # runs when the current stream gets there
    del busy, x                                          # (that memory is free to be given again at once)
    got = call(s)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("name", ["prefix_decode", "decode", "dense", "latent_decode", "latent_dense"])
def test_a_workspace_is_not_given_on_while_the_stream_works_in_it(name):
    call, size = cases()[name]
    want = call(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(HOLD)
    got = call(s)
    mine = [torch.full((size,), 85, dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    assert all(bool((m == 85).all()) for m in mine)


def test_an_output_may_be_used_and_dropped_on_the_current_stream():
    """Once the current stream has waited for the call, what it does with the output is safe from the next call on the other stream."""
    call, _ = cases()["prefix_decode"]
    want = call(None)
    torch.cuda.synchronize()
    s, here = torch.cuda.Stream(), torch.cuda.current_stream()
    kept = []
    for _ in range(4):
        got = call(s)
        here.wait_stream(s)
        torch.cuda._sleep(HOLD // 10)
        kept.append(got.clone())
        del got
        with torch.cuda.stream(s):
            torch.full(tuple(want.shape), float("nan"), device="cuda")
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in kept)


def test_a_captured_call_on_a_stream_of_its_own():
    """A branch of a captured graph that makes its own buffers: they are the graph's, and stay so."""
    call, size = cases()["prefix_decode"]
    want = call(None)
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.wait_stream(torch.cuda.current_stream())
        got = [call(s) for _ in range(2)]
        torch.cuda.current_stream().wait_stream(s)
        both = got[0] + got[1]
    other = [torch.full((size,), 85, dtype=torch.uint8, device="cuda") for _ in range(3)]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want) and torch.equal(both, want + want)
    assert all(bool((x == 85).all()) for x in other)
