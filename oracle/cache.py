"""Plain fp64 oracle of the cache calls (obc_cache_append, obc_attend, obc_cache_read), row by row, on the CPU.

A cache is a dict: k, v [P,H,S,d] float64, table [B,M] integers or None (page b is sequence b).  8-bit rows are held as the values
their codes stand for.
"""
import math

import torch

BLOCK = 32


def e4m3_exponent(absmax: float) -> int:
    """Least e >= -117 with absmax <= 448 * 2^e."""
    e = -117
    if absmax > 0:
        e = max(e, math.frexp(absmax / 448.0)[1] - 2)
    while absmax > math.ldexp(448.0, e):
        e += 1
    return e


def e4m3_round(y: torch.Tensor) -> torch.Tensor:
    """float64 values of at most 448 to the nearest e4m3 number, ties to even; what is not finite becomes NaN."""
    mant, ex = torch.frexp(y)                             # y = mant 2^ex, mant in [1/2, 1)
    ex = torch.clamp(ex, min=-5)                          # normal from 2^-6 = 1/2 2^-5 on
    step = torch.ldexp(torch.ones_like(y), ex - 4)        # three bits behind the leading one
    r = torch.round(y / step) * step                      # torch.round: half to even
    return torch.where(torch.isfinite(y), r, torch.full_like(y, math.nan))


def e4m3(rows: torch.Tensor):
    """[..., d] float64 -> (values the codes stand for, biased exponents [..., d/32] int)."""
    blocks = rows.double().reshape(-1, BLOCK)
    out, es = torch.empty_like(blocks), []
    for i, x in enumerate(blocks):
        fine = x[torch.isfinite(x)].abs()
        e = e4m3_exponent(float(fine.max()) if fine.numel() else 0.0)
        out[i] = e4m3_round(x * 2.0 ** -e) * 2.0 ** e
        es.append(e + 127)
    return out.reshape(rows.shape), torch.tensor(es).reshape(*rows.shape[:-1], -1)


def place(cache, b: int, g: int, j: int):
    """(page, head, slot) of a row; None if its page is not in the pool."""
    if cache["table"] is None:
        return b, g, j
    S, P = cache["k"].shape[2], cache["k"].shape[0]
    page = int(cache["table"][b, j // S])
    return (page, g, j % S) if 0 <= page < P else None


def capacity(cache) -> int:
    return cache["k"].shape[2] * (1 if cache["table"] is None else cache["table"].shape[1])


def length(lens, b: int, g: int) -> int:
    return int(lens[b, g]) if lens.dim() == 2 else int(lens[b])


def turned(x, norm, eps, position, freq, scale, interleaved):
    """One head's row [d] float64: RMS norm, then the rotation."""
    if norm is not None:
        x = x / math.sqrt(float((x * x).mean()) + eps) * norm.double()
    if freq is None:
        return x
    y = x.clone()
    n = len(freq)
    for i in range(n):
        a = float(position) * float(freq[i])
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        y[p] = scale * (x[p] * math.cos(a) - x[q] * math.sin(a))
        y[q] = scale * (x[q] * math.cos(a) + x[p] * math.sin(a))
    return y


def append(cache, k, v, lens, q=None, new_lens=None, positions=None, inv_freq=None, rot_scale=1.0, interleaved=False, q_norm=None,
           k_norm=None, eps=1e-6):
    """Writes into cache["k"], cache["v"] (unrounded); returns q_out [B,Hq,T,d] float64 or None.  k, v, q [B,T,H,d]."""
    B, T, Hkv, _ = k.shape
    cap = capacity(cache)
    q_out = None
    if q is not None:
        q_out = torch.zeros(B, q.shape[2], T, q.shape[3], dtype=torch.float64)
    for b in range(B):
        for t in range(T):
            how = (None, 1.0, interleaved) if inv_freq is None else (inv_freq, rot_scale, interleaved)
            pos = None if positions is None else positions[b, t]
            if q is not None and (new_lens is None or t < min(int(new_lens[b]), T)):
                for h in range(q.shape[2]):
                    q_out[b, h, t] = turned(q[b, t, h].double(), q_norm, eps, pos, *how)
            for g in range(Hkv):
                n = T if new_lens is None else min(max(length(new_lens, b, g), 0), T)
                j = length(lens, b, g) - n + t
                at = place(cache, b, g, j) if t < n and 0 <= j < cap else None
                if at is not None:
                    cache["k"][at] = turned(k[b, t, g].double(), k_norm, eps, pos, *how)
                    cache["v"][at] = v[b, t, g].double()
    return q_out


def attend(q, cache, lens, new_lens=None, causal=True, scale=None):
    """q [B,Hq,T,d] -> (out [B,T,Hq,d], sum_j p_j |v_j| like it, largest sum_c |q_c k_c| * scale of a seen pair [B,T,Hq]) in float64."""
    B, Hq, T, d = q.shape
    Hkv = cache["k"].shape[1]
    scale = d ** -0.5 if scale is None else scale
    out, weight = (torch.zeros(B, T, Hq, d, dtype=torch.float64) for _ in range(2))
    size = torch.zeros(B, T, Hq, dtype=torch.float64)
    for b in range(B):
        n = T if new_lens is None else min(max(int(new_lens[b]), 0), T)
        for g in range(Hkv):
            x, cap = max(length(lens, b, g), 0), capacity(cache)
            at = [place(cache, b, g, j) for j in range(min(x, cap))]
            k = torch.stack([cache["k"][i] for i in at]) if at else torch.zeros(0, d, dtype=torch.float64)
            v = torch.stack([cache["v"][i] for i in at]) if at else k
            for t in range(n):
                seen = min(max(x - n + t + 1, 0) if causal else x, cap)      # (its own row is row x - n + t, within the cache or past it)
                if seen == 0:
                    continue
                for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                    row = q[b, h, t].double()
                    p = torch.softmax(k[:seen] @ row * scale, 0)
                    out[b, t, h], weight[b, t, h] = p @ v[:seen], p @ v[:seen].abs()
                    size[b, t, h] = float((k[:seen].abs() @ row.abs()).max()) * scale
    return out, weight, size


def read(cache, keep=None, n=None):
    """-> k, v [B,Hkv,n,d] float64."""
    B = cache["k"].shape[0] if cache["table"] is None else cache["table"].shape[0]
    H, d, cap = cache["k"].shape[1], cache["k"].shape[3], capacity(cache)
    n = keep.shape[2] if keep is not None else n
    out = torch.zeros(2, B, H, n, d, dtype=torch.float64)
    for b in range(B):
        for g in range(H):
            for j in range(n):
                row = int(keep[b, g, j]) if keep is not None else j
                if row >= 0:
                    at = place(cache, b, g, min(row, cap - 1))
                    out[0, b, g, j], out[1, b, g, j] = cache["k"][at], cache["v"][at]
    return out[0], out[1]
