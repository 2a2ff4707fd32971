"""The operators around the decode step in 64 bits, from their definitions (include/santapp_serve.h), with the bound of
what the kernels' arithmetic may be off by."""
import math

import torch

D = 128


def rotate(rope, x, positions, interleaved):
    """x [n, heads, D] (any float type) at positions [n]; returns (y, bound of the fp32 error before rounding)."""
    w = torch.tensor(rope.inv_freq, dtype=torch.float64, device=x.device)
    rot, amp = 2 * len(w), rope.c.amplitude
    a = positions.double()[:, None] * w
    c, s = (amp * a.cos())[:, None], (amp * a.sin())[:, None]
    x = x.double()
    i = torch.arange(rot // 2, device=x.device)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    u, v = x[..., first], x[..., second]
    y, off = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = u * c - v * s, v * c + u * s
    # the angle in fp32 turns of at most 1/2: 2 pi 2^-25 rad; sine and cosine to 2 ulp (2^-23); three roundings (2^-24 each), the amplitude's
    # (2^-24): below 2^-22 + 2^-22 of |u| + |v|
    e = abs(amp) * 2.0 ** -21 * (u.abs() + v.abs())
    off[..., first], off[..., second] = e, e
    return y, off


def close_16(got, want, off, what=""):
    """got (16-bit) is the rounding of a value within `off` of `want`."""
    half = torch.finfo(got.dtype).eps / 2
    # (values below the smallest normal one are 2^-24 apart in fp16, and far smaller in bf16)
    tol = off + half * (want.abs() + off) + 2.0 ** -25
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol).nan_to_num(1e9).max()):.3g} of the tolerance"


def attend(q, k, v, seen, scale, cap=0.0, slope=None, distance=None, weight_off=2.0 ** -16):
    """One head: q [n, D], k and v [m, D], seen [n, m] bool. Returns (o, tolerance) in 64 bits, zeros for rows that see nothing.

    What the kernels may be off by, per weight, relative to it:
      products   16-bit factors are exact in fp32; 128 terms added by tensor cores, at most 136 * 2^-23 of sum |q_d k_d|
      fp32 steps scale, cap, bias and the maximum's subtraction: 2^-21 of the logits' size
      cap        tanh to 2^-20
      weight     weight_off: its rounding for the product with V
      sums       fp32, at most 2^-18 for the lengths here
    A relative error e_i of weight i moves o by at most sum p_i e_i (|v_i| + |o|)."""
    q, k, v = q.double(), k.double(), v.double()
    s = (q @ k.T) * scale
    e = 136 * 2.0 ** -23 * (q.abs() @ k.abs().T) * scale + weight_off + 2.0 ** -18
    if cap:
        s = cap * torch.tanh(s / cap)
        e = e + cap * 2.0 ** -20
    if slope is not None:
        s = s - float(slope) * distance.double()
    s = s.masked_fill(~seen, -math.inf)
    top = s.amax(1, keepdim=True) if s.shape[1] else torch.full((s.shape[0], 1), -math.inf, dtype=s.dtype, device=s.device)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = e + 2.0 ** -21 * (torch.where(seen, s, torch.zeros_like(s)).abs() + top.abs())
    p = torch.exp(s - top)
    total = p.sum(1, keepdim=True)
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    # 0 * what no row sees is nothing, whatever it holds
    v = torch.where(seen.any(0)[:, None], v, torch.zeros_like(v))
    pe = torch.where(seen, p * e, torch.zeros_like(p))
    o = p @ v
    return o, pe @ v.abs() + pe.sum(1, keepdim=True) * o.abs()


def prefix_decode(k, v, token, q, ks, vs, lens, scale, cap=0.0, slopes=None):
    """k, v [Hkv, N, D] (or None), token [Hkv, N] or None, q [B, Hq, D], ks, vs [B, Hkv, cap, D] or None, lens: visible rows."""
    B, hq, _ = q.shape
    dev = q.device
    hkv = ks.shape[1] if k is None else k.shape[0]
    N = 0 if k is None else k.shape[1]
    out = torch.zeros(B, hq, D, dtype=torch.float64, device=dev)
    tol = torch.zeros_like(out)
    for b in range(B):
        t = lens[b]
        for j in range(hkv):
            kk, vv = [], []
            pos = torch.arange(N, device=dev) if token is None or N == 0 else token[j].long()
            if N:
                kk.append(k[j]), vv.append(v[j])
            if t:
                kk.append(ks[b, j, :t]), vv.append(vs[b, j, :t])
                pos = torch.cat([pos, torch.arange(N, N + t, device=dev)])
            if not kk:
                continue
            kk, vv = torch.cat(kk), torch.cat(vv)
            dist = (N + t - 1 - pos).abs()[None]
            for h in range(j * hq // hkv, (j + 1) * hq // hkv):
                o, e = attend(q[b, h][None], kk, vv, torch.ones(1, len(kk), dtype=torch.bool, device=dev), scale, cap,
                              None if slopes is None else slopes[h], dist)
                out[b, h], tol[b, h] = o[0], e[0]
    return out, tol


def prompt(q, k, v, lens, new, both, scale, cap=0.0, slopes=None):
    """q [sum new, Hq, D], k, v [Hkv, sum lens, D]. Weights are rounded to the type of q."""
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    half = torch.finfo(q.dtype).eps / 2
    row = key = 0
    for n, m, p in zip(lens, new, both):
        qp, kp = torch.arange(n - m, n, device=q.device), torch.arange(n, device=q.device)
        seen = (kp[None] <= qp[:, None]) | (kp < p)[None]
        dist = (qp[:, None] - kp[None]).abs()
        for h in range(q.shape[1]):
            j = h // (q.shape[1] // k.shape[0])
            out[row:row + m, h], tol[row:row + m, h] = attend(q[row:row + m, h], k[j, key:key + n], v[j, key:key + n], seen, scale, cap,
                                                              None if slopes is None else slopes[h], dist, half + 2.0 ** -17)
        row, key = row + m, key + n
    return out, tol


def close_32(got, want, tol, what=""):
    err = (got.double() - want).abs()
    bad = ~(err <= tol + 2.0 ** -22 * want.abs())
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / (tol + 1e-30)).nan_to_num(1e9).max()):.3g} of the tolerance"
