"""Operators around decode attention: what they compute, in plain form, and the calls that a user makes of them.

A case is a dict of plain values with a `kind`:

  rope_token    one new token per sequence: q and k rotated, k and v appended to the suffix
  rope_prompt   the rows of prompts: q and k rotated, k and v laid out as [n_kv_heads][rows][d]
  fork          the batch's slots after a selection: some continue another slot's answer, some are freed
  prefix        one decode step of a batch that shares one long prompt, each sequence with its own suffix
  prompt        attention of prompts (ragged, causal, a bidirectional beginning, or their last rows alone)

Rows follow the recipe of the library's workloads, drawn on the GPU: keys scattered around cluster centres
(sigma 0.3), four sink rows scaled by 4, queries that are noisy copies of rows they may see.
"""
import math
import random

import torch

own = False

D = 128                                    # head_dim of the K/V path


# ---- cases -----------------------------------------------------------------------------------------
def _rope(name, kind, n, q_heads, kv_heads, elem, rot, interleaved, scaled, lo, hi, cap=0):
    return dict(name=name, kind=kind, n=n, q_heads=q_heads, kv_heads=kv_heads, elem=elem, rot=rot,
                interleaved=interleaved, scaled=scaled, lo=lo, hi=hi, cap=cap, shape_seed=0)


def _fork(name, n, kv_heads, elem, cap, lo, hi, moved):
    return dict(name=name, kind="fork", n=n, q_heads=kv_heads, kv_heads=kv_heads, elem=elem, cap=cap, lo=lo, hi=hi,
                moved=moved, shape_seed=0)


def _prefix(name, n, q_heads, kv_heads, elem, prefix, lo, hi, cap, softcap=0.0, bias=False, packed=False):
    return dict(name=name, kind="prefix", n=n, q_heads=q_heads, kv_heads=kv_heads, elem=elem, prefix=prefix, lo=lo, hi=hi,
                cap=cap, softcap=softcap, bias=bias, packed=packed, shape_seed=0)


def _prompt(name, n, q_heads, kv_heads, elem, lo, hi, new=0, both=0, softcap=0.0, bias=False):
    return dict(name=name, kind="prompt", n=n, q_heads=q_heads, kv_heads=kv_heads, elem=elem, lo=lo, hi=hi, new=new,
                both=both, softcap=softcap, bias=bias, shape_seed=0)


def listed():
    return [
        # A single user's token: nothing but latency.
        _rope("rope_token_b1", "rope_token", 1, 28, 4, "bf16", 128, False, False, 32768, 32768, cap=256),
        # A serving batch's token, neighbouring pairs, half of the head, positions far past the trained length.
        _rope("rope_token_b64", "rope_token", 64, 32, 8, "fp16", 64, True, True, 8192, 131072, cap=1024),
        # The rows of one 32K prompt, after the projections of a layer.
        _rope("rope_prompt_32k", "rope_prompt", 1, 28, 4, "bf16", 128, False, True, 32768, 32768),
        # Four answers of which one is dropped for another: the smallest batch with something to move.
        _fork("fork_b4", 4, 4, "bf16", 256, 100, 100, 1),
        # A wide search: half of the slots continue another slot, answers of all lengths.
        _fork("fork_b32", 32, 4, "bf16", 1024, 1, 1024, 16),
        # Two answers to a short prompt: latency again.
        _prefix("prefix_b2_4k", 2, 28, 4, "bf16", 4096, 16, 16, 256),
        # Eight answers to one 32K prompt: the step is the reading of the prompt, once.
        _prefix("prefix_b8_32k", 8, 28, 4, "bf16", 32768, 1, 256, 256),
        # Five answers over an odd 128K prompt read from team records, in fp16, biased by distance.
        _prefix("prefix_b5_128k_bias", 5, 32, 8, "fp16", 131071, 1, 100, 256, bias=True, packed=True),
        # A full batch of answers to one 32K prompt, scores capped: tensor cores bound it, not memory.
        _prefix("prefix_b64_32k_cap", 64, 28, 4, "bf16", 32768, 1, 1024, 1024, softcap=50.0),
        # A ragged batch of short prompts, biased by distance.
        _prompt("prompt_ragged_bias", 12, 12, 4, "fp16", 1, 1024, bias=True),
        # The next thousand rows of two long prompts with a bidirectional beginning, scores capped.
        _prompt("prompt_chunk_cap", 2, 16, 2, "bf16", 4001, 8192, new=1024, both=512, softcap=30.0),
        # One 8K prompt.
        _prompt("prompt_8k", 1, 28, 4, "bf16", 8192, 8192),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the same calls at other sizes, head layouts, types and scores."""
    kind = rng.choice(["rope_token", "rope_prompt", "fork", "prefix", "prefix", "prompt", "prompt"])
    q_heads, kv_heads = rng.choice([(28, 4), (28, 4), (32, 8), (16, 2), (12, 4), (8, 8)])
    elem = rng.choice(["bf16", "bf16", "fp16"])
    softcap, bias = rng.choice([0.0, 0.0, 30.0, 50.0]), rng.choice([False, False, True])
    shape_seed = rng.randrange(1 << 20)
    if kind in ("rope_token", "rope_prompt"):
        rot, between, scaled = rng.choice([128, 128, 96, 64, 32, 16]), rng.choice([False, True]), rng.choice([False, True])
        if kind == "rope_token":
            hi = _log_int(rng, 1, 131072)
            case = _rope("", kind, _log_int(rng, 1, 256), q_heads, kv_heads, elem, rot, between, scaled, max(1, hi // 8), hi,
                         cap=rng.choice([16, 256, 1024]))
        else:
            n = rng.choice([1, 1, 3])
            hi = _log_int(rng, 1, 32768 // n)
            case = _rope("", kind, n, q_heads, kv_heads, elem, rot, between, scaled, max(1, hi // 4), hi)
    elif kind == "fork":
        n, cap = _log_int(rng, 2, 64), rng.choice([16, 256, 1024])
        case = _fork("", n, kv_heads, elem, cap, rng.randint(0, cap), cap, rng.randint(1, n // 2))
    elif kind == "prefix":
        n, cap = _log_int(rng, 1, 64), rng.choice([0, 16, 256, 1024])
        most = min(131072, (1 << 21) // n)
        case = _prefix("", n, q_heads, kv_heads, elem, _log_int(rng, 1, most), rng.randint(0, cap), cap, cap, softcap, bias,
                       rng.choice([False, True]))
    else:
        n = _log_int(rng, 1, 16)
        hi = _log_int(rng, 1, min(8192, 12288 // n))
        case = _prompt("", n, q_heads, kv_heads, elem, max(1, hi // rng.choice([1, 4, 64])), hi,
                       rng.choice([0, 0, 1 + hi // 8]), rng.choice([0, 0, hi // 4]), softcap, bias)
    del case["name"]
    case["shape_seed"] = shape_seed
    return case


# ---- shapes ----------------------------------------------------------------------------------------
def _lens(case, salt=0):
    rng = random.Random(case["shape_seed"] + salt)
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["n"])]


def _new_lens(case):
    return [min(n, case["new"]) if case["new"] else n for n in _lens(case)]


def _both_lens(case):
    return [min(n, case["both"]) for n in _lens(case)]


def _sources(case):
    """Slot that each slot continues: `moved` of them another one that stays, the rest themselves."""
    rng = random.Random(case["shape_seed"] + 1)
    slots = list(range(case["n"]))
    rng.shuffle(slots)
    src = list(range(case["n"]))
    for b in slots[:case["moved"]]:
        src[b] = rng.choice(slots[case["moved"]:])
    return src


def _dtype(case):
    return torch.float16 if case["elem"] == "fp16" else torch.bfloat16


# ---- inputs ----------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _slopes(case):
    h = case["q_heads"]
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / h) / 16 for i in range(h)], dtype=torch.float32, device="cuda")


def _keys(gen, case, n, dtype):
    """Clustered keys [n_kv_heads, n, D] and the clusters' centres."""
    centres = _normal(gen, case["kv_heads"], 256, D)
    which = torch.randint(256, (case["kv_heads"], n), generator=gen, device="cuda")
    k = torch.empty(case["kv_heads"], n, D, dtype=dtype, device="cuda")
    for j in range(case["kv_heads"]):
        k[j] = centres[j][which[j]] + 0.3 * _normal(gen, n, D)
    k[:, :4] *= 4.0
    return k, centres


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, n, hq, hkv, kind = _dtype(case), case["n"], case["q_heads"], case["kv_heads"], case["kind"]
    state = dict(case=dict(case), dtype=dtype)
    if kind in ("rope_token", "rope_prompt"):
        rows = n if kind == "rope_token" else sum(_lens(case))
        qkv = _normal(gen, rows, hq + 2 * hkv, D).to(dtype)          # the output of one fused projection
        state.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], q_out=torch.empty(rows, hq, D, dtype=dtype, device="cuda"))
        if kind == "rope_token":
            rng = random.Random(seed)
            state.update(base_pos=_i32(_lens(case)), suffix_len=_i32([rng.randint(0, case["cap"] - 1) for _ in range(n)]),
                         suffix_len_out=torch.empty(n, dtype=torch.int32, device="cuda"),
                         k_suffix=_normal(gen, n, hkv, case["cap"], D).to(dtype), v_suffix=_normal(gen, n, hkv, case["cap"], D).to(dtype))
        else:
            state.update(positions=torch.cat([torch.arange(m, dtype=torch.int32, device="cuda") for m in _lens(case)]),
                         k_prompt=torch.empty(hkv, rows, D, dtype=dtype, device="cuda"), v_prompt=torch.empty(hkv, rows, D, dtype=dtype, device="cuda"))
    elif kind == "fork":
        state.update(src=_i32(_sources(case)), suffix_len=_i32(_lens(case, 2)), suffix_len_out=torch.empty(n, dtype=torch.int32, device="cuda"),
                     k_suffix=_normal(gen, n, hkv, case["cap"], D).to(dtype), v_suffix=_normal(gen, n, hkv, case["cap"], D).to(dtype))
    elif kind == "prefix":
        N, cap = case["prefix"], case["cap"]
        k, centres = _keys(gen, case, N, dtype)
        v = _normal(gen, hkv, N, D).to(dtype)
        rows = torch.randint(N, (n, hkv, hq // hkv), generator=gen, device="cuda")
        q = torch.stack([k[j][rows[:, j]].float() for j in range(hkv)], 1)
        q = (q + 0.5 * _normal(gen, n, hkv, hq // hkv, D)).to(dtype).view(n, hq, D)
        which = torch.randint(256, (n, hkv, cap), generator=gen, device="cuda")
        k_suffix = torch.stack([centres[j][which[:, j]] for j in range(hkv)], 1) + 0.3 * _normal(gen, n, hkv, cap, D)
        token = None
        if case["packed"]:                                            # rows in the order of team records
            token = torch.stack([torch.randperm(N, generator=gen, device="cuda") for _ in range(hkv)])
            k = torch.stack([k[j][token[j]] for j in range(hkv)])
            token = token.to(torch.int32)
        state.update(q=q, k=k, v=v, token=token, suffix_len=_i32(_lens(case, 2)), k_suffix=k_suffix.to(dtype) if cap else None,
                     v_suffix=_normal(gen, n, hkv, cap, D).to(dtype) if cap else None,
                     out=torch.empty(n, hq, D, device="cuda"), slopes=_slopes(case) if case["bias"] else None)
    else:
        lens, new, both = _lens(case), _new_lens(case), _both_lens(case)
        k, _ = _keys(gen, case, sum(lens), dtype)
        v = _normal(gen, hkv, sum(lens), D).to(dtype)
        seq = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(new, device="cuda"))
        first = torch.tensor([sum(lens[:b]) for b in range(n)], device="cuda")
        pos = torch.cat([torch.arange(lens[b] - new[b], lens[b], device="cuda") for b in range(n)])
        past = (torch.rand(len(seq), hq // hkv, generator=gen, device="cuda") * (pos + 1)[:, None]).long() + first[seq][:, None]
        q = torch.stack([k[j][past].float() for j in range(hkv)], 1)
        q = 0.7 * (q + 0.5 * _normal(gen, len(seq), hkv, hq // hkv, D))
        state.update(q=q.to(dtype).view(len(seq), hq, D), k=k, v=v, lens=lens, new=new, both=both, seq=seq, pos=pos,
                     key_seq=torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(lens, device="cuda")),
                     key_pos=torch.cat([torch.arange(m, device="cuda") for m in lens]), both_of=torch.tensor(both, device="cuda"),
                     out=torch.empty(len(seq), hq, D, dtype=dtype, device="cuda"), slopes=_slopes(case) if case["bias"] else None)
    return state


# ---- rotary frequencies: by the formulas; the scaled ones keep short wavelengths and stretch long ones by 8
SCALE, LOW, HIGH, TRAINED, THETA = 8.0, 1.0, 4.0, 8192.0, 500000.0


def _frequencies(case):
    f = THETA ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])
    if case["scaled"]:
        keep = ((TRAINED * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / SCALE)
    return f


def _amplitude(case):
    return 0.1 * math.log(SCALE) + 1.0 if case["scaled"] else 1.0


# ---- plain forms -----------------------------------------------------------------------------------
def _rotated(case, x, positions):
    """x [n, heads, D] at the positions [n]: angles in 64 bits, the rotation in 32, one rounding."""
    angle = positions.double()[:, None] * _frequencies(case)[None, :]
    c = (angle.cos() * _amplitude(case)).float()[:, None, :]
    s = (angle.sin() * _amplitude(case)).float()[:, None, :]
    rot = case["rot"]
    y = x.float().clone()
    if case["interleaved"]:
        a, b = x[..., 0:rot:2].float(), x[..., 1:rot:2].float()
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :rot // 2].float(), x[..., rot // 2:rot].float()
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * s, b * c + a * s
    return y.to(x.dtype)


def _rope_token(s):
    at = s["suffix_len"].long()
    b = torch.arange(len(at), device="cuda")
    positions = s["base_pos"].long() + at
    s["q_out"].copy_(_rotated(s["case"], s["q"], positions))
    s["k_suffix"][b, :, at] = _rotated(s["case"], s["k"], positions)
    s["v_suffix"][b, :, at] = s["v"]
    s["suffix_len_out"].copy_(s["suffix_len"] + 1)
    return [s["q_out"], s["k_suffix"], s["v_suffix"], s["suffix_len_out"]]


def _rope_prompt(s):
    s["q_out"].copy_(_rotated(s["case"], s["q"], s["positions"]))
    s["k_prompt"].copy_(_rotated(s["case"], s["k"], s["positions"]).transpose(0, 1))
    s["v_prompt"].copy_(s["v"].transpose(0, 1))
    return [s["q_out"], s["k_prompt"], s["v_prompt"]]


def _forked(s):
    src = s["src"].long()
    new_len = s["suffix_len"][src]
    row = torch.arange(s["case"]["cap"], device="cuda")
    copied = (row[None, :] < new_len[:, None])[:, None, :, None]
    s["k_suffix"].copy_(torch.where(copied, s["k_suffix"][src], s["k_suffix"]))
    s["v_suffix"].copy_(torch.where(copied, s["v_suffix"][src], s["v_suffix"]))
    s["suffix_len_out"].copy_(new_len)
    return [s["k_suffix"], s["v_suffix"], s["suffix_len_out"]]


def _scored(x, softcap, slope, distance):
    """Logits from scaled products: the cap, then the bias."""
    if softcap:
        x = softcap * torch.tanh(x / softcap)
    if slope is not None:
        x = x - slope * distance
    return x


def _prefix_plain(s):
    case = s["case"]
    n, hq, hkv, N, cap = case["n"], case["q_heads"], case["kv_heads"], case["prefix"], case["cap"]
    g, scale = hq // hkv, 1.0 / math.sqrt(D)
    q = s["q"].float().view(n, hkv, g, D)
    length = s["suffix_len"].long()
    pos = N + length - 1                                              # the query's own row is the suffix's last
    x = torch.matmul(q.permute(1, 0, 2, 3).reshape(hkv, n * g, D), s["k"].float().transpose(1, 2)).view(hkv, n, g, N).transpose(0, 1) * scale
    slope = token = None
    if s["slopes"] is not None:
        slope = s["slopes"].view(1, hkv, g, 1)
        token = torch.arange(N, device="cuda")[None].expand(hkv, N) if s["token"] is None else s["token"].long()
        token = (pos[:, None, None, None] - token[None, :, None, :]).abs().float()
    x = _scored(x, case["softcap"], slope, token)
    if cap:
        row = torch.arange(cap, device="cuda")
        y = torch.matmul(q, s["k_suffix"].float().transpose(2, 3)) * scale
        y = _scored(y, case["softcap"], slope, (pos[:, None] - (N + row)[None, :]).abs().float()[:, None, None, :])
        x = torch.cat([x, torch.where((row[None] < length[:, None])[:, None, None, :], y, -math.inf)], 3)
    p = torch.exp(x - x.amax(3, keepdim=True))
    o = torch.matmul(p[..., :N].transpose(0, 1).reshape(hkv, n * g, N), s["v"].float()).view(hkv, n, g, D).transpose(0, 1)
    if cap:
        o = o + torch.matmul(p[..., N:], s["v_suffix"].float())
    s["out"].copy_((o / p.sum(3, keepdim=True)).reshape(n, hq, D))
    return s["out"]


def _prompt_plain(s):
    case = s["case"]
    hq, hkv, rows, keys = case["q_heads"], case["kv_heads"], s["q"].shape[0], s["k"].shape[1]
    g = hq // hkv
    q = s["q"].float().view(rows, hkv, g, D).permute(1, 2, 0, 3).reshape(hkv, g * rows, D)
    x = torch.matmul(q, s["k"].float().transpose(1, 2)).view(hkv, g, rows, keys) / math.sqrt(D)
    slope = distance = None
    if s["slopes"] is not None:
        slope, distance = s["slopes"].view(hkv, g, 1, 1), (s["pos"][:, None] - s["key_pos"][None, :]).abs().float()
    x = _scored(x, case["softcap"], slope, distance)
    seen = (s["key_pos"][None, :] <= s["pos"][:, None]) | (s["key_pos"][None, :] < s["both_of"][s["seq"]][:, None])
    seen &= s["key_seq"][None, :] == s["seq"][:, None]
    x = torch.where(seen, x, -math.inf)
    p = torch.exp(x - x.amax(3, keepdim=True))
    o = torch.matmul(p.view(hkv, g * rows, keys), s["v"].float()).view(hkv, g, rows, D) / p.sum(3, keepdim=True)
    s["out"].copy_(o.permute(2, 0, 1, 3).reshape(rows, hq, D).to(s["dtype"]))
    return s["out"]


# ---- the library's calls ---------------------------------------------------------------------------
def _kept(s):
    """What a user's program makes once and keeps: the geometry, the rotary table, the workspace."""
    from paper_2609_35629_b200 import binding as sp
    if "geom" not in s:
        case = s["case"]
        n = 1 if case["kind"] == "rope_prompt" else case["n"]
        s["geom"] = sp.Geometry(n, case["q_heads"], case["kv_heads"], D, elem_type=sp.SANTAPP_FP16 if case["elem"] == "fp16" else sp.SANTAPP_BF16)
        if "rot" in case:
            more = dict(factor=SCALE, low=LOW, high=HIGH, original_len=TRAINED, amplitude=_amplitude(case)) if case["scaled"] else {}
            s["rope"] = sp.Rope(case["rot"], THETA, interleaved=case["interleaved"], **more)
        if case["kind"] == "prefix":
            size = sp.santapp_prefix_decode_workspace_bytes(s["geom"], case["prefix"], case["cap"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return sp, s["geom"]


def _call(s):
    sp, geom = _kept(s)
    case, kind = s["case"], s["case"]["kind"]
    if kind == "rope_token":
        sp.santapp_rope_append(geom, s["rope"], s["q"], s["k"], s["v"], s["base_pos"], s["suffix_len"], s["k_suffix"],
                               s["v_suffix"], q_out=s["q_out"], suffix_len_out=s["suffix_len_out"])
        return [s["q_out"], s["k_suffix"], s["v_suffix"], s["suffix_len_out"]]
    if kind == "rope_prompt":
        sp.santapp_rope_prompt(geom, s["rope"], s["q"], s["k"], s["v"], s["positions"], s["k_prompt"], s["v_prompt"],
                               q_out=s["q_out"])
        return [s["q_out"], s["k_prompt"], s["v_prompt"]]
    if kind == "fork":
        sp.santapp_suffix_fork(geom, s["src"], s["suffix_len"], s["k_suffix"], s["v_suffix"],
                               suffix_len_out=s["suffix_len_out"])
        return [s["k_suffix"], s["v_suffix"], s["suffix_len_out"]]
    if kind == "prefix":
        return sp.santapp_prefix_decode_attn(geom, s["k"], s["v"], s["q"], s["k_suffix"], s["v_suffix"], s["suffix_len"],
                                             prefix_token=s["token"], cap=case["softcap"], slopes=s["slopes"], out=s["out"],
                                             workspace=s["workspace"])
    return sp.santapp_prompt_attn(geom, s["lens"], s["q"], s["k"], s["v"], new_len=s["new"], prefix_len=s["both"],
                                  cap=case["softcap"], slopes=s["slopes"], out=s["out"])


def run(state):
    if own:
        return _call(state)
    return {"rope_token": _rope_token, "rope_prompt": _rope_prompt, "fork": _forked, "prefix": _prefix_plain,
            "prompt": _prompt_plain}[state["case"]["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    n, hq, hkv, kind = case["n"], case["q_heads"], case["kv_heads"], case["kind"]
    if kind == "rope_token":
        return {"bytes": 2 * n * (hq + 2 * hkv) * D * 2 + 12 * n, "flops": 3 * n * (hq + hkv) * case["rot"]}
    if kind == "rope_prompt":
        rows = sum(_lens(case))
        return {"bytes": 2 * rows * (hq + 2 * hkv) * D * 2 + 4 * rows, "flops": 3 * rows * (hq + hkv) * case["rot"]}
    lens = _lens(case, 2)
    if kind == "fork":
        src = _sources(case)
        read = sum(lens[a] for a in {src[b] for b in range(n) if src[b] != b})
        written = sum(lens[src[b]] for b in range(n) if src[b] != b)
        return {"bytes": (read + written) * hkv * 2 * D * 2 + 12 * n, "flops": 0}
    if kind == "prefix":
        keys = case["prefix"] + sum(lens)
        return {"bytes": keys * hkv * 2 * D * 2 + n * hq * D * (2 + 4) + (4 * hkv * case["prefix"] if case["packed"] and case["bias"] else 0),
                "flops": 4 * D * hq * (n * case["prefix"] + sum(lens))}
    lens, new, both = _lens(case), _new_lens(case), _both_lens(case)
    pairs = 0
    for a, m, p in zip(lens, new, both):
        inside = max(0, p - (a - m))                                  # queries in the bidirectional beginning see all of it
        pairs += inside * p + sum(range(a - m + inside + 1, a + 1))
    return {"bytes": sum(lens) * hkv * 2 * D * 2 + sum(new) * hq * D * 2 * 2, "flops": 4 * D * hq * pairs}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _turned(case, x, positions):
    """Each pair as a complex number times amplitude * exp(i position frequency)."""
    rot = case["rot"]
    x = x.double()
    pairs = x[..., :rot].unflatten(-1, (rot // 2, 2)) if case["interleaved"] else x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    turn = torch.polar(torch.full((1,), _amplitude(case), dtype=torch.float64, device="cuda"), positions.double()[:, None] * _frequencies(case))
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None, :])
    y = y.flatten(-2) if case["interleaved"] else y.transpose(-1, -2).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _softmax_sum(logits, v):
    w = torch.softmax(logits, -1)
    return w @ v


def exact(case, seed):
    s = prepare(case, seed)
    n, hq, hkv, kind = case["n"], case["q_heads"], case["kv_heads"], case["kind"]
    if kind == "rope_token":
        k_suffix, v_suffix = s["k_suffix"].double(), s["v_suffix"].double()
        k = _turned(case, s["k"], s["base_pos"].double() + s["suffix_len"])
        for b, t in enumerate(s["suffix_len"].tolist()):
            k_suffix[b, :, t], v_suffix[b, :, t] = k[b], s["v"][b].double()
        return [_turned(case, s["q"], s["base_pos"].double() + s["suffix_len"]), k_suffix, v_suffix, s["suffix_len"] + 1]
    if kind == "rope_prompt":
        return [_turned(case, s["q"], s["positions"]), _turned(case, s["k"], s["positions"]).transpose(0, 1).contiguous(),
                s["v"].double().transpose(0, 1).contiguous()]
    if kind == "fork":
        k, v, lens = s["k_suffix"].double(), s["v_suffix"].double(), s["suffix_len"].tolist()
        k0, v0, src = k.clone(), v.clone(), _sources(case)
        for b, a in enumerate(src):
            k[b, :, :lens[a]], v[b, :, :lens[a]] = k0[a, :, :lens[a]], v0[a, :, :lens[a]]
        return [k, v, _i32([lens[a] for a in src])]
    g, g_scale, softcap = hq // hkv, D ** -0.5, case["softcap"]

    def logits(q, k, h, q_pos, k_pos):
        x = (q.double() @ k.double().T) * g_scale
        if softcap:
            x = torch.tanh(x / softcap) * softcap
        if case["bias"]:
            x = x - s["slopes"][h].double() * (q_pos.double()[:, None] - k_pos.double()[None, :]).abs()
        return x

    if kind == "prefix":
        N, out = case["prefix"], torch.empty(n, hq, D, dtype=torch.float64, device="cuda")
        for b, t in enumerate(s["suffix_len"].tolist()):
            q_pos = torch.tensor([N + t - 1], device="cuda")
            for h in range(hq):
                j = h // g
                k, v, k_pos = s["k"][j], s["v"][j], torch.arange(N, device="cuda") if s["token"] is None else s["token"][j]
                if t:
                    k, v = torch.cat([k, s["k_suffix"][b, j, :t]]), torch.cat([v, s["v_suffix"][b, j, :t]])
                    k_pos = torch.cat([k_pos, torch.arange(N, N + t, device="cuda")])
                out[b, h] = _softmax_sum(logits(s["q"][b, h][None], k, h, q_pos, k_pos), v.double())[0]
        return out
    out, row, key = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0, 0
    for a, m, p in zip(s["lens"], s["new"], s["both"]):
        q_pos, k_pos = torch.arange(a - m, a, device="cuda"), torch.arange(a, device="cuda")
        hidden = (k_pos[None, :] > q_pos[:, None]) & (k_pos >= p)[None, :]
        for h in range(hq):
            x = logits(s["q"][row:row + m, h], s["k"][h // g, key:key + a], h, q_pos, k_pos).masked_fill(hidden, -math.inf)
            out[row:row + m, h] = _softmax_sum(x, s["v"][h // g, key:key + a].double())
        row, key = row + m, key + a
    return out
