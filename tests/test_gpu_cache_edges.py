"""The cache calls where their definitions are easy to miss: values that are not finite, the cache's end, the ends of the number ranges."""
import math

import pytest
import torch

from oracle import cache as oc
from paper_2510_07651_amd import binding as obc

import cache_util as cu

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("bf16", "e4m3"), ("fp32", "fp32"), ("fp32", "e4m3")]


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _bits(x):
    return x.contiguous().view(torch.int16 if x.dtype is torch.bfloat16 else torch.int32)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("d,pairs", [(64, 8), (64, 16), (128, 16), (128, 32), (128, 56)])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "neighbours"])
def test_channels_that_are_not_turned_stay_as_they_are(dtype, kind, d, pairs, interleaved):
    """An infinity, a NaN and a negative zero, in channels that are turned and in others: nothing reaches a channel from 2 * pairs on, and of
    the turned ones only the other of the pair."""
    B, T, Hq, Hkv = 1, 9, 4, 2
    g = torch.Generator().manual_seed(d + pairs)
    rows = torch.randn(B, T, Hq + Hkv, d, generator=g)
    turned = 2 * pairs
    rows[:, :, :, turned::5] = -0.0
    at = {1: 3, 2: 3, 3: turned - 2, 4: pairs, 5: turned, 6: d - 1, 7: 0}
    for t, c in at.items():
        rows[:, t, :, c] = (math.inf, math.nan, -math.inf)[t % 3]
    rows[:, 8] = -0.0
    rows = rows.to(cu.DT[dtype])
    q, k = rows[:, :, :Hq], rows[:, :, Hq:]
    cache, _ = cu.make(kind, B, Hkv, d, 16, 1, seed=1)
    page = int(cache.page_table[0, 0])
    freq = cu.rotation(pairs)
    pos = torch.randint(1, 5000, (B, T), generator=g, dtype=torch.int32)
    got = obc.obc_cache_append(cache, k.cuda(), k.cuda(), _i32(T), q=q.cuda(), positions=pos.cuda(), inv_freq=freq.cuda(), interleaved=interleaved)
    torch.cuda.synchronize()
    assert torch.equal(_bits(got.transpose(1, 2)[..., turned:].cpu()), _bits(q[..., turned:]))
    if kind != "e4m3":
        assert torch.equal(_bits(cache.k[page, :, :T, turned:].cpu().transpose(0, 1)), _bits(k[0, ..., turned:]))
    held = cu.held(cache)[0][page]
    slack = cu.append_slack(torch.nan_to_num(rows.double(), nan=0.0, posinf=0.0, neginf=0.0), None, 1.0)
    for t in range(T):
        c = at.get(t, d)
        other = d if c >= turned else (c ^ 1 if interleaved else (c + pairs) % turned)
        fine = torch.tensor([i not in (c, other) for i in range(d)])
        for h in range(Hq + Hkv):
            want = oc.turned(rows[0, t, h].double(), None, 0, pos[0, t], freq, 1.0, interleaved)
            if h < Hq:
                cu.close(got[0, h, t].cpu()[fine], want[fine], dtype, slack[0, t, h][fine])
            elif kind != "e4m3":
                cu.close(held[h - Hq, t][fine], want[fine], kind, slack[0, t, h][fine])
            else:
                # blocks without a turned channel: the codes of these very values
                for i in range(0, d, 32):
                    if i >= turned:
                        codes, byte = oc.e4m3(rows[0, t, h, i:i + 32].double())
                        assert torch.equal(torch.nan_to_num(held[h - Hq, t, i:i + 32], nan=1e9), torch.nan_to_num(codes, nan=1e9))
                        assert int(cache.k_scale[page, h - Hq, t, i // 32]) == int(byte)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("d,T", [(64, 5), (128, 5), (128, 40)])
def test_chunks_that_reach_past_the_end(dtype, kind, d, T):
    """Rows for which the cache has no room are dropped; every other new token sees itself and what was there before it, those behind
    the end all of the cache.  Held to the same token alone, over a sequence that ends with it."""
    B, Hq, Hkv, page, M = 4, 4, 2, 16, 4
    cap = page * M
    cache, want = cu.make(kind, B, Hkv, d, page, M, seed=T)
    g = torch.Generator().manual_seed(T)
    rows = [torch.randn(B, T, h, d, generator=g).to(cu.DT[dtype]) for h in (Hq, Hkv, Hkv)]
    lens = [cap + 1, cap + T - 1, cap + T, 2 ** 31 - 1]
    q = obc.obc_cache_append(cache, rows[1].cuda(), rows[2].cuda(), _i32(*lens), q=rows[0].cuda())
    held = dict(zip("kv", cu.held(cache)), table=want["table"])
    for b in range(B):
        for t in range(T):
            j = lens[b] - T + t
            if j < cap and kind != "e4m3":                           # the token's own row lies where its limit says
                for h in range(Hkv):
                    assert torch.equal(held["k"][oc.place(held, b, h, j)], rows[1][b, t, h].double())
    for causal in (True, False):
        out = obc.obc_attend(q, cache, _i32(*lens), causal=causal)
        per_head = obc.obc_attend(q, cache, _i32(*([x] * Hkv for x in lens)), causal=causal)
        assert torch.equal(out, per_head)
        for t in range(T):
            ends = torch.tensor([min(x - T + t + 1, cap) if causal else cap for x in lens])
            ref = oc.attend(q[:, :, t:t + 1].cpu(), held, ends, causal=causal)
            cu.check_attend(out[:, t:t + 1], ref, cap, d, dtype)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("d,T,Hkv,N,step", [(128, 24, 1, 96, 32), (64, 24, 1, 96, 32), (128, 40, 1, 4000, 32), (128, 1, 64, 600, 128), (64, 7, 64, 600, 128),
                                            (128, 1, 64, 600, 32), (64, 8, 64, 600, 32)])
def test_values_near_the_end_of_the_range(dtype, kind, d, T, Hkv, N, step):
    """Weights are at most 1, so that N of the largest values of 1.5 * 2^e have a sum where N * 1.5 * 2^e has a place, also where logits grow from step to
    step by a little less than what a reference waits for.  All values are alike, and so are the outputs, to the roundings of the sums and of the
    result."""
    e = 127 - math.ceil(math.log2(N))
    cache, _ = cu.make(kind, 1, Hkv, d, 32, -(-N // 32), seed=3)
    rows, values = torch.zeros(1, N, Hkv, d), torch.full((1, N, Hkv, d), 1.5 * 2.0 ** e)
    rows[..., 0] = 5.0 * (torch.arange(N) // step).clamp(max=3)[:, None]     # (5 is 7.2 in log2)
    obc.obc_cache_append(cache, rows.to(cu.DT[dtype]).cuda(), values.to(cu.DT[dtype]).cuda(), _i32(N))
    q = torch.zeros(1, 4 * Hkv, T, d, dtype=cu.DT[dtype])
    q[..., 0] = 1.0
    out = obc.obc_attend(q.cuda(), cache, _i32(N), causal=False, scale=1.0).double().cpu() / 2.0 ** e
    rel = (2 * N + 80) * 2.0 ** -24 + cu.HALF[dtype]
    assert bool(((out - 1.5).abs() <= 1.5 * rel).all()), (float(out.min()), float(out.max()))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides_of_dimensions_of_size_1(dtype):
    """One token whose dimension was added behind the channels, one head behind a sequence: the same bits as from rows in order."""
    B, H, d = 3, 2, 64
    x = torch.randn(3, B, H, d, generator=torch.Generator().manual_seed(0)).to(cu.DT[dtype]).cuda()
    odd = [t[:, :, :, None].permute(0, 3, 1, 2) for t in x]            # [B,1,H,d], token stride 1
    assert odd[0].stride(1) == 1
    caches = [cu.make(dtype, B, H, d, 16, 2, seed=1)[0] for _ in range(2)]
    lens = _i32(5, 17, 32)
    outs = [obc.obc_cache_append(c, k, v, lens, q=q) for c, (q, k, v) in zip(caches, (odd, [t[:, None].contiguous() for t in x]))]
    assert torch.equal(*outs) and torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)
    single = x[0, :1, 0]                                               # [1,d] as one sequence of one head
    one = [cu.make(dtype, 1, 1, d, 16, 2, seed=1)[0] for _ in range(2)]
    for c, rows in zip(one, (single.as_strided((1, 1, 1, d), (7, 3, 5, 1)), single.view(1, 1, 1, d))):
        obc.obc_cache_append(c, rows, rows, _i32(9))
    assert torch.equal(one[0].k, one[1].k)
