"""Plain float64 definitions of the attention and KV-cache operators, for tests."""
import math

import torch

GROUP = 32
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def quantise(x, bits):
    """x [..., hd] -> (codes float64 [..., hd], scales float64 [..., hd / 32])."""
    Q = 127 if bits == 8 else 7
    g = x.detach().cpu().double().unflatten(-1, (-1, GROUP))
    a = g.abs().amax(-1)
    inv = torch.tensor(1.0 / Q, dtype=torch.float32).double()
    s = (a * inv).float().bfloat16().double()     # one fp32 product, one rounding to bfloat16
    s = torch.where(torch.isfinite(g).all(-1), s, float("nan"))
    q = g / s.unsqueeze(-1)
    q = torch.where(torch.isfinite(q), q, 0.0).round().clamp(-Q, Q)
    return q.flatten(-2), s


def stored(x, bits):
    """The values a cache holds for x, float64."""
    q, s = quantise(x, bits)
    return (q.unflatten(-1, (-1, GROUP)) * s.unsqueeze(-1)).flatten(-2)


def attention(q, k, v, visible, distance, scale, softcap=0.0, slopes=None, tol=None, floor=0.0):
    """q [Sq, H, hd], k and v [Sk, Hkv, hd], visible and distance [Sq, Sk] -> float64
    [Sq, H, hd].  Hidden keys are left out, not multiplied by zero.

    ``tol`` (a float64 tensor like the result) receives how far a kernel may be off:
    with u = eps / 2 of the dtype, w = sum_j p_j |v_j| and e the error of a score,
    u |out| for storing the output (half the smallest subnormal, tiny eps / 2, at
    the least), u w for rounding p (or p times a value's scale)
    to the dtype, and (2 e + (2 n + 16) 2^-24) w for p and the sums: a score's fp32
    dot product of hd terms, cap, bias and exponent argument are off by at most
    (hd + 16) 2^-24 (scale sum |q_c k_c| + |bias|) + 2^-20 softcap, an exponential
    by 2^-22, and the sums of n weights and of n products by n 2^-24 each.  ``floor``:
    what a weight loses at the most in the subnormals of fp16, relative to the largest
    weight (their sum is at least 1) times the largest value."""
    fi = torch.finfo(q.dtype)
    u = fi.eps / 2
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    Sq, H, hd = q.shape
    G = H // k.shape[1]
    out = torch.zeros(Sq, H, hd, dtype=torch.float64)
    for h in range(H):
        s = (q[:, h] @ k[:, h // G].t()) * scale
        if softcap > 0:
            s = softcap * torch.tanh(s / softcap)
        if slopes is not None:
            s = s - float(slopes[h]) * distance.double()
        s = torch.where(visible, s, -math.inf)
        vv = v[:, h // G]
        bad = ~torch.isfinite(vv).all(-1)
        p = torch.softmax(s, -1)
        p = torch.where(visible, p, 0.0)
        p = torch.where(visible.any(-1, keepdim=True), p, 0.0)
        o = p[:, ~bad] @ vv[~bad]
        for j in torch.nonzero(bad)[:, 0].tolist():   # a value row with Inf or NaN
            seen = visible[:, j]
            o[seen] += p[seen, j, None] * vv[j]
        out[:, h] = o
        if tol is not None:
            size = (q[:, h].abs() @ k[:, h // G].abs().t()) * abs(scale)
            if slopes is not None:
                size = size + float(slopes[h]) * distance.double()
            size = torch.where(visible & torch.isfinite(size), size, 0.0).amax(-1, keepdim=True)
            e = (hd + 16) * 2.0 ** -24 * size + 2.0 ** -20 * softcap
            w = torch.nan_to_num(p[:, ~bad]) @ vv[~bad].abs()
            n = k.shape[0]
            seen = visible.any(0) & ~bad
            largest = vv[seen].abs().max() if seen.any() else 0.0
            tol[:, h] = (u * o.abs() + u * fi.tiny + n * floor * largest
                         + (u + 2 * e + (2 * n + 16) * 2.0 ** -24) * w)
    return out


def prompt(q, k, v, causal=False, softcap=0.0, slopes=None, key_mask=None, q_doc=None, k_doc=None,
           prefix=None, q_offset=None, scale=None, tol=None):
    B, Sq, H, hd = q.shape
    Sk = k.shape[1]
    off = Sk - Sq if q_offset is None else q_offset
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    i, j = torch.arange(Sq)[:, None] + off, torch.arange(Sk)[None]
    out = torch.zeros(B, Sq, H, hd, dtype=torch.float64)
    for b in range(B):
        vis = torch.ones(Sq, Sk, dtype=torch.bool)
        if causal:
            vis = j <= i
            if prefix is not None:
                vis = vis | (j < int(prefix[b]))
        if key_mask is not None:
            vis = vis & (key_mask[b].cpu() != 0)[None]
        if q_doc is not None:
            vis = vis & (q_doc[b].cpu()[:, None] == k_doc[b].cpu()[None])
        # fp16 probabilities are held times 2^7: half a step of the subnormals is 2^-32
        out[b] = attention(q[b], k[b], v[b], vis, (i - j).abs(), scale, softcap, slopes,
                           None if tol is None else tol[b],
                           2.0 ** -32 if q.dtype == torch.float16 else 0.0)
    return out


def cached(q, k, v, lengths, bits, softcap=0.0, slopes=None, valid=None, scale=None, tol=None):
    """k and v [B, n, Hkv, hd] as written at positions 0 .. n - 1."""
    B, Sq, H, hd = q.shape
    n = k.shape[1]
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    ks, vs = stored(k, bits), stored(v, bits)
    out = torch.zeros(B, Sq, H, hd, dtype=torch.float64)
    for b in range(B):
        i, j = torch.arange(Sq)[:, None] + int(lengths[b]) - Sq, torch.arange(n)[None]
        vis = j <= i
        if valid is not None:
            vis = vis & (valid[b].cpu() != 0)[None]
        # 16-bit dtypes: a weight is p times a value's scale, in fp16 as 16 / b of itself with
        # b at most twice the largest scale s; half a step of the subnormals, 2^-25, stands for
        # 2^-25 b / 16 <= 2^-28 s, times a code of at most Q: 2^-28 of the largest value
        # (which may be Q s (1 - 2^-8) by the rounding of s)
        out[b] = attention(q[b], ks[b], vs[b], vis, (i - j).abs(), scale, softcap, slopes,
                           None if tol is None else tol[b],
                           0.0 if q.dtype == torch.float32 else 2.0 ** -28 * (1 + 2.0 ** -7))
    return out


def check(got, ref, tol, what=""):
    """got against ref within tol; Inf and NaN exactly where ref has them."""
    got = got.detach().cpu().double()
    same = (torch.isnan(got) & torch.isnan(ref)) | (got == ref)
    off = torch.where(same, 0.0, (got - ref).abs() - tol)
    bad = ~(off <= 0)
    worst = (torch.where(same, 0.0, (got - ref).abs()) / tol.clamp_min(1e-300)).nan_to_num(0).max()
    print(f"{what}: largest error {float(worst):.3f} of the tolerance", flush=True)
    assert not bad.any(), (what, int(bad.sum()), torch.nonzero(bad)[:4].tolist(), float(worst))
