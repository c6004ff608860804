"""Plain 64-bit statements of the paged K/V cache's operators, and the error bounds that their tests use."""
import math

import torch


def e4m3_round(y):
    """float64 y rounded to the nearest e4m3 value, ties to even (|y| <= 448)."""
    b = torch.frexp(y)[1].clamp(min=-5) - 1   # floor(log2 |y|), from 2^-6 on
    step = torch.exp2((b - 3).double())   # (torch.ldexp is a rounded power on the GPU)
    return torch.round(y / step) * step


def quantise(x):
    """(values that the 8-bit form holds for rows x [..., head_dim], exponents), in float64; finite x."""
    x = x.double()
    m, e = torch.frexp(x.abs().amax(-1))
    ex = torch.where(m == 0, torch.zeros_like(e), (e - 9 + (m > 0.875).to(e.dtype)).clamp(min=-126))
    s = torch.exp2(ex.double()).unsqueeze(-1)
    return e4m3_round(x / s) * s, ex


def entries(cache, which):
    """Every entry of a cache's K ("k") or V ("v") as float64 [n_blocks, n_kv_heads, block_tokens, head_dim]."""
    x = getattr(cache, which)
    if cache.dtype != "e4m3":
        return x.double()
    ex = getattr(cache, which + "_exp").double() - 127
    return x.view(torch.float8_e4m3fn).double() * torch.exp2(ex).unsqueeze(-1)


def positions(cache, which, seq, n):
    """Positions 0..n-1 of a sequence, float64 [n, n_kv_heads, head_dim]."""
    bt = cache.k.shape[2]
    p = torch.arange(n, device=cache.k.device)
    return entries(cache, which)[cache.block_table[seq].long()[p // bt], :, p % bt]


def attention(cache, q, q_start, kv_len):
    """(out, bound on an element's error) of the causal attention of each sequence's newest rows, float64.

    Bound, for P and out in the type of u = half a step: out is rounded once (u |out|), each weight once (u A with
    A = sum w |v|); a score is a sum of head_dim products in 32 bits, each addition off by at most 2^-23 of the partial
    sums (a tensor core may truncate), so off by d = head_dim 2^-23 sum |q k| / sqrt(head_dim), which moves a weight by
    (1 + 2 d) in numerator and denominator: 4 d A; sums of n weights and weighted V: 2 n 2^-23 A; base-2 exponentials
    and their argument: 2^-20 (1 + |s|) A.
    """
    rows, heads, dh = q.shape
    hk = cache.k.shape[1]
    u = torch.finfo(q.dtype).eps / 2
    out = torch.zeros(rows, heads, dh, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    for b, n in enumerate(kv_len):
        r0, r1 = q_start[b], q_start[b + 1]
        if r1 == r0:
            continue
        k, v = (positions(cache, w, b, n) for w in ("k", "v"))
        for h in range(heads):
            kk, vv = k[:, h // (heads // hk)], v[:, h // (heads // hk)]
            qq = q[r0:r1, h].double()
            s = qq @ kk.T / math.sqrt(dh)
            last = n - (r1 - r0) + torch.arange(r1 - r0, device=q.device)
            hide = torch.arange(n, device=q.device)[None, :] > last[:, None]
            s = s.masked_fill(hide, -math.inf)
            w = torch.nan_to_num(torch.softmax(s, -1), nan=0.0) if n else s
            vv = torch.where(hide.all(0)[:, None], torch.zeros_like(vv), vv)
            out[r0:r1, h] = w @ vv
            a = w @ vv.abs()
            size = (qq.abs() @ kk.abs().T / math.sqrt(dh)).masked_fill(hide, 0)
            most = size.amax(-1, keepdim=True) if n else torch.zeros(r1 - r0, 1, dtype=torch.float64, device=q.device)
            d = dh * 2.0 ** -23 * most
            p_u = 0.0 if q.dtype == torch.float32 else u
            tol[r0:r1, h] = u * out[r0:r1, h].abs() + (p_u + 4 * d + 2 * n * 2.0 ** -23 + 2.0 ** -20 * (1 + most)) * a
    return out, tol
