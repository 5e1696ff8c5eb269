"""Small caches for the tests of obc_cache_append, obc_attend and obc_cache_read: device tensors and the oracle's view of them."""
import torch

from oracle import cache as oc

DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24, "e4m3": 2.0 ** -4}     # half a step, relative


def make(kind, B, Hkv, d, page, M, seed=0, filler=None, device="cuda", extra_pages=2):
    """(KvCache, oracle cache): pages dealt out in no order, `extra_pages` of nobody; page = rows per sequence and M = 0: no table.
    filler: value that every place holds (NaN: whoever reads what is not theirs is seen), else normal values."""
    from paper_2510_07651_amd import binding as obc

    g = torch.Generator().manual_seed(1000 + seed)
    P = B if M == 0 else B * M + extra_pages
    table = None if M == 0 else torch.randperm(P, generator=g)[:B * M].view(B, M).to(torch.int32)
    tensors, values, scales = [], [], []
    for _ in range(2):
        x = torch.randn(P, Hkv, page, d, generator=g) if filler is None else torch.full((P, Hkv, page, d), float(filler))
        if kind == "e4m3":
            codes, byte = quantise(x)
            tensors.append(codes)
            scales.append(byte)
            values.append(dequantise(codes, byte))
        else:
            tensors.append(x.to(DT[kind]))
            values.append(tensors[-1].double())
    dev = lambda t: None if t is None else t.to(device)  # noqa: E731
    s = scales if kind == "e4m3" else [None, None]
    cache = obc.KvCache(dev(tensors[0]), dev(tensors[1]), dev(table), dev(s[0]), dev(s[1]))
    return cache, {"k": values[0].clone(), "v": values[1].clone(), "table": table}


def quantise(x):
    """Quick form of the 8-bit rows, for inputs (the oracle's own is row by row)."""
    x = x.float()
    top = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).abs().unflatten(-1, (-1, oc.BLOCK)).amax(-1)
    e = torch.where(top > 0, torch.ceil(torch.log2(top.double() / 448 + 1e-300)), torch.full_like(top, -117).double()).clamp(-117, 120)
    codes = (x.double().unflatten(-1, (-1, oc.BLOCK)) / torch.exp2(e)[..., None]).flatten(-2).float().to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def dequantise(codes, byte):
    x = codes.cpu().to(torch.float32).double().unflatten(-1, (-1, oc.BLOCK))
    return (x * torch.exp2(byte.cpu().double() - 127)[..., None]).flatten(-2)


def held(cache):
    """k, v [P,Hkv,S,d] float64: what a KvCache holds now."""
    if cache.k_scale is None:
        return cache.k.double().cpu(), cache.v.double().cpu()
    return dequantise(cache.k, cache.k_scale), dequantise(cache.v, cache.v_scale)


def attend_tolerance(ref, weight, size, N, d, dtype):
    """Elementwise bound of |out - ref|.

    A logit is a sum of d products in fp32, each addition off by 2^-24 of what it has so far: (d + 2) 2^-24 sum |q k|; its product with
    log2(e) * scale, the subtraction of the maximum and the exponential's argument add 4 * 2^-24 of it.  A weight's relative error is that
    (times 2: the maximum's own logit) plus 2 ulp of the exponential; weights and sums over N tokens and up to 64 shares add (N + 72) 2^-24.
    bf16: the weights are rounded to bf16, half a step, and so is the result."""
    u = 2.0 ** -24
    rel = 2 * (d + 6) * u * size[..., None] + (2 * N + 80) * u
    if dtype == "bf16":
        rel = rel + HALF["bf16"]
    return rel * weight + HALF[dtype] * ref.abs() + 1e-30


def check_attend(got, want, N, d, dtype):
    ref, weight, size = want
    err = (got.double().cpu() - ref).abs()
    bound = attend_tolerance(ref, weight, size, N, d, dtype)
    assert bool((err <= bound).all()), (float((err / bound).max()), [int(i) for i in torch.nonzero(~(err <= bound))[0]])
    # (a lost token hides below the elementwise bound of bf16, not in the norm: roundings of both signs leave less than one half step)
    norm = float(ref.norm())
    if norm:
        assert float(err.norm()) <= (HALF["bf16"] if dtype == "bf16" else 2e-5) * norm + 1e-30


def rotation(pairs, theta=10000.0):
    return (theta ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))).float()


def close(got, ref, kind, slack):
    """|got - ref| <= half a step of the type + slack, elementwise."""
    err = (got.double().cpu() - ref).abs()
    bound = HALF[kind] * ref.abs() + slack
    assert bool((err <= bound).all()), (float((err / bound).max()), [int(i) for i in torch.nonzero(~(err <= bound))[0]])


def append_slack(x, norm, scale, eps=1e-6):
    """What fp32 arithmetic may add before the rounding, for rows x [...,d].

    Norm: the sum of d squares in lanes and exchanges, mean, root, quotient and two products: 20 * 2^-24 relative.  Rotation:
    cosine and sine off by 4 * 2^-24 (a turn's part rounded to fp32 times 2 pi, 2 ulp of the function), their scale and three
    roundings: 8 * 2^-24 of |x| + |y|, which is at most twice the row's largest value."""
    x = x.double()
    if norm is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * norm.double()
    top = x.abs().amax(-1, keepdim=True) * max(abs(scale), 1.0)
    return 2 * 28 * 2.0 ** -24 * top + 0 * x + 1e-37
