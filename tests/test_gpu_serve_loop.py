"""The operators as a serving loop runs them: a prompt's rows rotated and attended, several answers to it decoded beside
one another, forked and freed, each step against full attention in 64 bits."""
import math

import pytest
import torch

import serve_reference as ref
from paper_2609_35629_b200 import binding as sp

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("hq,hkv,N,chunk", [(28, 4, 300, 128), (8, 2, 129, 129)])
def test_answers_to_one_prompt(hq, hkv, N, chunk):
    dt, rope, cap = torch.bfloat16, sp.Rope(rot_dim=64, interleaved=True, theta=5e5), 8
    g = torch.Generator(device="cuda").manual_seed(7)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(dt)

    # the prompt, in chunks
    one = sp.Geometry(1, hq, hkv)
    kp, vp = torch.zeros(hkv, N, D, dtype=dt, device="cuda"), torch.zeros(hkv, N, D, dtype=dt, device="cuda")
    for first in range(0, N, chunk):
        n = min(chunk, N - first)
        x = rand(n, hq + 2 * hkv, D)
        at = torch.arange(first, first + n, dtype=torch.int32, device="cuda")
        q = sp.santapp_rope_prompt(one, rope, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], at, kp, vp, dst_row=at)
        keys = (kp[:, :first + n].contiguous(), vp[:, :first + n].contiguous())
        out = sp.santapp_prompt_attn(one, [first + n], q, *keys, new_len=[n])
        want, tol = ref.prompt(q, *keys, [first + n], [n], [0], 1 / math.sqrt(D))
        ref.close_16(out, want, tol, f"rows {first} on")

    # answers
    B = 5
    geom = sp.Geometry(B, hq, hkv)
    teams = sp.santapp_build_teams(one, [N], kp, vp)
    ks, vs = torch.zeros(B, hkv, cap, D, dtype=dt, device="cuda"), torch.zeros(B, hkv, cap, D, dtype=dt, device="cuda")
    lens, base = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), N, dtype=torch.int32, device="cuda")
    other = torch.empty_like(lens)
    kept = [([], []) for _ in range(B)]                 # rows of each answer as they were appended
    moves = {2: [0, 0, 2, 3, 2], 4: [1, 2, 0, -1, 4]}
    for step in range(7):
        x = rand(B, hq + 2 * hkv, D)
        q = sp.santapp_rope_append(geom, rope, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], base, lens, ks, vs, suffix_len_out=lens)
        for b, n in enumerate(lens.tolist()):
            kept[b][0].append(ks[b, :, n - 1].clone())
            kept[b][1].append(vs[b, :, n - 1].clone())
        out = sp.santapp_prefix_decode_attn(geom, teams.k_packed, teams.v_packed, q, ks, vs, lens)
        for b, n in enumerate(lens.tolist()):
            assert n == len(kept[b][0])
            want, tol = ref.prefix_decode(kp, vp, None, q[b:b + 1], torch.stack(kept[b][0], 1)[None], torch.stack(kept[b][1], 1)[None], [n],
                                          1 / math.sqrt(D))
            ref.close_32(out[b:b + 1], want, tol, f"step {step}, answer {b}")
        if step in moves:
            src = moves[step]
            sp.santapp_suffix_fork(geom, torch.tensor(src, dtype=torch.int32, device="cuda"), lens, ks, vs, suffix_len_out=other)
            lens, other = other, lens
            kept = [([], []) if a < 0 else (list(kept[a][0]), list(kept[a][1])) for a in src]


def test_a_captured_token_is_replayed():
    """Append, attend, lengths advanced in place: one graph, a token per replay."""
    B, hq, hkv, N, cap, dt = 3, 12, 4, 500, 6, torch.bfloat16
    geom, rope = sp.Geometry(B, hq, hkv), sp.Rope()
    g = torch.Generator(device="cuda").manual_seed(1)
    kp, vp = (torch.randn(hkv, N, D, generator=g, device="cuda").to(dt) for _ in range(2))
    x = torch.randn(B, hq + 2 * hkv, D, generator=g, device="cuda").to(dt)
    base = torch.full((B,), N, dtype=torch.int32, device="cuda")

    def state():
        return [torch.zeros(B, hkv, cap, D, dtype=dt, device="cuda"), torch.zeros(B, hkv, cap, D, dtype=dt, device="cuda"),
                torch.zeros(B, dtype=torch.int32, device="cuda"), torch.empty(B, hq, D, dtype=dt, device="cuda"),
                torch.empty(B, hq, D, device="cuda"),
                torch.empty(sp.santapp_prefix_decode_workspace_bytes(geom, N, cap), dtype=torch.uint8, device="cuda")]

    def token(s):
        ks, vs, lens, q, out, ws = s
        sp.santapp_rope_append(geom, rope, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], base, lens, ks, vs, q_out=q, suffix_len_out=lens)
        sp.santapp_prefix_decode_attn(geom, kp, vp, q, ks, vs, lens, out=out, workspace=ws)

    a, b = state(), state()
    token(a)                                            # (first calls outside the capture)
    a[2].zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token(a)
    for step in range(cap + 2):                         # two more than the suffix holds: nothing is written then
        x.copy_(torch.roll(x, 1, 0))
        graph.replay()
        token(b)
        torch.cuda.synchronize()
        assert torch.equal(a[4], b[4]) and torch.equal(a[2], b[2]) and a[2].tolist() == [min(step + 1, cap)] * B
