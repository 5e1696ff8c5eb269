"""obc_cache_append and obc_cache_read against the oracle: norms, rotations, 8-bit rows, pages, ragged chunks."""
import math

import pytest
import torch

from oracle import cache as oc
from paper_2510_07651_amd import binding as obc

import cache_util as cu

pytestmark = pytest.mark.gpu


def _inputs(B, T, Hq, Hkv, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(B, T, (Hq + 2 * Hkv) * d, generator=g).to(cu.DT[dtype])
    return qkv, [Hq * d, Hkv * d, Hkv * d]


def _run(dtype, kind, B, T, Hq, Hkv, d, page, M, lens, new=None, pairs=0, interleaved=False, norm=False, scale=1.0, seed=0, layout="fused",
         positions=None):
    qkv, parts = _inputs(B, T, Hq, Hkv, d, dtype, seed)
    split = lambda t: [x.unflatten(-1, (-1, d)) for x in t.split(parts, -1)]  # noqa: E731
    q, k, v = split(qkv)
    dq, dk, dv = split(qkv.cuda())
    if layout == "heads first":
        dq, dk, dv = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (dq, dk, dv))
    elif layout == "apart":
        dq, dk, dv = (x.contiguous() for x in (dq, dk, dv))
    cache, want = cu.make(kind, B, Hkv, d, page, M, seed=seed)
    before = [x.clone() for x in cu.held(cache)]
    g = torch.Generator().manual_seed(seed + 5)
    qw, kw = ((1 + 0.3 * torch.randn(d, generator=g)).to(cu.DT[dtype]) if norm else None for _ in range(2))
    pos = torch.randint(0, 5000, (B, T), generator=g, dtype=torch.int32) if positions is None else positions
    freq = cu.rotation(pairs) if pairs else None
    on = lambda t: None if t is None else t.cuda()  # noqa: E731
    lens_t = torch.tensor(lens, dtype=torch.int32)
    new_t = None if new is None else torch.tensor(new, dtype=torch.int32)
    got_q = obc.obc_cache_append(cache, dk, dv, lens_t.cuda(), q=dq if Hq else None, new_lens=on(new_t),
                                 positions=pos.cuda() if pairs else None, inv_freq=on(freq), rot_scale=scale, interleaved=interleaved,
                                 q_norm=on(qw) if Hq else None, k_norm=on(kw))
    torch.cuda.synchronize()
    ref_q = oc.append(want, k, v, lens_t, q if Hq else None, new_t, pos if pairs else None, freq, scale, interleaved, qw if Hq else None, kw)
    if Hq:
        cu.close(got_q, ref_q, dtype, cu.append_slack(q.transpose(1, 2), qw, scale))
        if new is not None:
            for b in range(B):
                assert float(got_q[b, :, max(new[b], 0):].abs().sum()) == 0
    gk, gv = cu.held(cache)
    untouched = (want["k"] == before[0]) & (want["v"] == before[1])
    assert torch.equal(gk[untouched], before[0][untouched]) and torch.equal(gv[untouched], before[1][untouched])
    top = float((k.double().abs().max() if not norm else math.sqrt(d) * kw.double().abs().max()) * max(scale, 1.0))
    slack = 2 * 28 * 2.0 ** -24 * top if (norm or pairs) else 0.0
    if kind == "e4m3":
        # half a step of a normal code is relative; below 2^-6 of the block's power of two it is 2^-10 of that power.  (A largest value next to
        # 448 * 2^e may take the next power.)
        blocks = lambda x: x.unflatten(-1, (-1, 32))  # noqa: E731
        e = torch.ceil(torch.log2(blocks(want["k"]).abs().amax(-1, keepdim=True) / 448 + 1e-300)).clamp(min=-117)
        cu.close(blocks(gk), blocks(want["k"]), kind, slack + 2.0 ** -10 * torch.exp2(e + 1))
        if not (norm or pairs):
            assert torch.equal(gk[~untouched], oc.e4m3(want["k"])[0][~untouched])
        assert torch.equal(gv[~untouched], oc.e4m3(want["v"])[0][~untouched])
    else:
        cu.close(gk, want["k"], kind, slack)
        assert torch.equal(gv, want["v"])


@pytest.mark.parametrize("dtype,kind,d", [("bf16", "bf16", 128), ("bf16", "bf16", 64), ("fp32", "fp32", 128), ("fp32", "fp32", 64),
                                          ("bf16", "e4m3", 128), ("bf16", "e4m3", 64), ("fp32", "e4m3", 128), ("fp32", "e4m3", 64)])
@pytest.mark.parametrize("how", ["plain", "half", "neighbours", "part", "normed", "normed part"])
def test_append(dtype, kind, d, how):
    pairs = {"plain": 0, "half": d // 2, "neighbours": d // 2, "part": d // 4, "normed": 0, "normed part": 24}[how]
    _run(dtype, kind, B=2, T=5, Hq=6, Hkv=2, d=d, page=8, M=3, lens=[5, 22], pairs=pairs, interleaved=how in ("neighbours", "normed part"),
         norm="normed" in how, scale=1.25 if how == "part" else 1.0, seed=d + len(kind))


@pytest.mark.parametrize("layout", ["fused", "heads first", "apart"])
@pytest.mark.parametrize("B,T,Hq,Hkv,page,M,lens,new", [
    (1, 1, 32, 8, 40, 0, [40], None),                                # one token, the last place of an unpaged cache
    (1, 1, 1, 1, 1, 4, [1], None),                                   # one head, pages of one row
    (3, 4, 7, 7, 16, 2, [4, 9, 32], [4, 1, 0]),                      # ragged chunks, one of them empty
    (2, 3, 4, 2, 4, 2, [2, 11], None),                               # rows before row 0 and past the end are dropped
    (2, 3, 4, 2, 4, 2, [[3, 8], [5, 4]], [3, 9]),                    # lengths per head; more new rows than there are
    (2, 3, 4, 2, 4, 2, [0, -5], [-1, 2]),
], ids=["last place", "one row", "ragged", "outside", "per head", "negative"])
def test_append_places(layout, B, T, Hq, Hkv, page, M, lens, new):
    for dtype, kind in (("bf16", "bf16"), ("bf16", "e4m3"), ("fp32", "fp32")):
        _run(dtype, kind, B, T, Hq, Hkv, 128, page, M, lens, new, pairs=64, norm=True, layout=layout, seed=3)


def test_append_many_tokens():
    """More tokens than one row of heads' workgroups are started for."""
    _run("bf16", "bf16", B=2, T=700, Hq=2, Hkv=1, d=64, page=64, M=11, lens=[700, 703], pairs=32, norm=True, seed=11)


def test_append_of_kept_rows_with_a_length_per_head():
    """What a head-adaptive eviction keeps: lists of different lengths, padded with -1."""
    counts = [[3, 0], [6, 5]]
    _run("bf16", "e4m3", B=2, T=6, Hq=0, Hkv=2, d=128, page=4, M=2, lens=counts, new=counts, seed=4, layout="heads first")


@pytest.mark.parametrize("position", [0, 1, -7, 131071, 1000003, 2 ** 31 - 1])
def test_rotation_of_far_positions(position):
    """The angle is position * frequency to fp32's accuracy of the turned pair, wherever the position lies."""
    pos = torch.full((1, 2), position, dtype=torch.int32)
    _run("fp32", "fp32", B=1, T=2, Hq=2, Hkv=1, d=128, page=4, M=0, lens=[2], pairs=64, positions=pos, seed=6)


def test_codes_of_special_values():
    """Blocks of zeros, of tiny and huge values, next to 448 times a power of two, with infinities and NaN."""
    d = 128
    rows = torch.zeros(8, d)
    rows[1] = 2.0 ** -130
    rows[2] = 3e38
    rows[3] = 448.0 * torch.arange(d).remainder(2).mul(2).sub(1)
    rows[4] = torch.linspace(-450, 450, d)
    rows[5, ::5] = math.inf
    rows[5, 1::5] = math.nan
    rows[5, 2::5] = 3.0
    rows[6] = torch.exp(torch.linspace(-60, 60, d))
    rows[7, 3], rows[7, 40] = 1e-30, -math.inf
    for dtype in ("fp32", "bf16"):
        x = rows.to(cu.DT[dtype])[None, :, None]
        cache, _ = cu.make("e4m3", 1, 1, d, 8, 0)
        obc.obc_cache_append(cache, x.cuda(), x.cuda(), torch.tensor([8], dtype=torch.int32, device="cuda"))
        values, bytes_ = oc.e4m3(x[0, :, 0].double())
        assert torch.equal(cache.k_scale[0, 0].cpu().int(), bytes_.int())
        for got in (cu.held(cache)[0][0, 0], obc.obc_cache_read(cache, 8, dtype=torch.float32)[0][0, 0].double().cpu(),
                    obc.obc_cache_read(cache, 8)[0][0, 0].double().cpu()):
            assert torch.equal(torch.nan_to_num(got, nan=12345.0), torch.nan_to_num(values, nan=12345.0))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_codes_at_the_end_of_the_range(dtype):
    """Below 31/32 * 2^128 values keep to half a step; from there on the nearest code stands for 2^128."""
    inside, outside = 30 / 32 * 2.0 ** 128, 31 / 32 * 2.0 ** 128           # (both are fp32 and bf16 numbers)
    x = torch.zeros(1, 1, 1, 64)
    x[..., 0], x[..., 32], x[..., 33] = inside, outside, -outside
    cache, _ = cu.make("e4m3", 1, 1, 64, 8, 0)
    obc.obc_cache_append(cache, x.to(cu.DT[dtype]).cuda(), x.to(cu.DT[dtype]).cuda(), torch.tensor([1], dtype=torch.int32, device="cuda"))
    for out in (torch.float32, torch.bfloat16):
        got = obc.obc_cache_read(cache, 1, dtype=out)[0][0, 0, 0].cpu()
        assert got[0] == inside and got[32] == math.inf and got[33] == -math.inf and int((got == 0).sum()) == 61


@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("fp32", "fp32"), ("e4m3", "bf16"), ("e4m3", "fp32")])
@pytest.mark.parametrize("d", [64, 128])
def test_read(kind, dtype, d):
    """Listed rows (ends, -1, entries past the end, the same one twice) and the first rows, paged and not."""
    for M, page in ((3, 16), (0, 37)):
        cache, want = cu.make(kind, 2, 3, d, page, M, seed=d)
        cap = cache.capacity
        g = torch.Generator().manual_seed(1)
        keep = torch.randint(0, cap, (2, 3, 21), generator=g, dtype=torch.int32)
        keep[:, :, 0], keep[:, :, 1], keep[:, 1, 2], keep[1, :, 3], keep[:, :, 4] = 0, cap - 1, -1, cap + 5, keep[:, :, 5]
        for k, n in ((keep, None), (None, 1), (None, cap)):
            got = obc.obc_cache_read(cache, n, None if k is None else k.cuda(), dtype=cu.DT[dtype])
            for x, ref in zip(got, oc.read(want, k, n)):
                assert x.dtype is cu.DT[dtype] and torch.equal(x.double().cpu(), ref)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_read_many_rows(dtype):
    """Enough rows for a thread to take 16 codes; the numbers of rows and heads are no multiples of anything."""
    cache, _ = cu.make("e4m3", 3, 5, 64, 16, 560, seed=5)
    keep = torch.randint(-1, cache.capacity, (3, 5, 8801), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    got = obc.obc_cache_read(cache, keep_idx=keep.cuda(), dtype=cu.DT[dtype])
    table = cache.page_table.cpu().long()
    at = torch.gather(table[:, None].expand(3, 5, -1), 2, keep.clamp(min=0).long() // 16)
    for x, held in zip(got, cu.held(cache)):
        want = held[at, torch.arange(5)[:, None], keep.clamp(min=0).long() % 16] * (keep >= 0)[..., None]
        assert torch.equal(x.double().cpu(), want)


def test_rows_keep_their_values_when_stored_again():
    """e4m3 rows read back and stored again: the same values, whatever power of two the new block takes."""
    g = torch.Generator().manual_seed(9)
    rows = torch.randn(1, 300, 2, 128, generator=g) * torch.exp2(torch.randint(-20, 20, (1, 300, 2, 1), generator=g).float())
    cache, _ = cu.make("e4m3", 1, 2, 128, 64, 5)
    lens = torch.tensor([300], dtype=torch.int32, device="cuda")
    obc.obc_cache_append(cache, rows.cuda(), rows.cuda(), lens)
    first = obc.obc_cache_read(cache, 300)
    obc.obc_cache_append(cache, first[0].transpose(1, 2), first[1].transpose(1, 2), lens)
    for x, y in zip(first, obc.obc_cache_read(cache, 300)):
        assert torch.equal(x, y)


def test_pages_outside_the_pool():
    """Numbers outside the pool: writes are dropped, reads stay inside."""
    cache, _ = cu.make("bf16", 2, 2, 128, 4, 3, seed=2)
    cache.page_table[0, 1], cache.page_table[1, 0], cache.page_table[1, 2] = 10 ** 6, -3, 2 ** 31 - 1
    before = [x.clone() for x in (cache.k, cache.v)]
    rows = torch.randn(2, 4, 2, 128, device="cuda").bfloat16()
    obc.obc_cache_append(cache, rows, rows, torch.tensor([8, 4], dtype=torch.int32, device="cuda"))
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])
    k, _ = obc.obc_cache_read(cache, 12)
    P = cache.k.shape[0]
    assert torch.equal(k[0, :, 4:8], cache.k[P - 1]) and torch.equal(k[1, :, :4], cache.k[0]) and torch.equal(k[1, :, 8:], cache.k[P - 1])


def test_pool_beyond_32_bit_offsets():
    """A pool of more than 2^32 bytes and 2^31 elements: rows at its end."""
    cache = obc.KvCache.empty(33000, 8, 64, 128, page_table=torch.tensor([[32999, 1]], dtype=torch.int32, device="cuda"))  # 2.16e9 elements, 4.3 GB each
    rows = torch.randn(1, 64, 8, 128, device="cuda").bfloat16()
    lens = torch.tensor([64], dtype=torch.int32, device="cuda")
    obc.obc_cache_append(cache, rows, 2 * rows, lens)
    assert torch.equal(cache.k[32999], rows[0].transpose(0, 1)) and torch.equal(cache.v[32999], 2 * rows[0].transpose(0, 1))
    k, v = obc.obc_cache_read(cache, 64)
    assert torch.equal(k[0], cache.k[32999]) and torch.equal(v[0], cache.v[32999])
    q = torch.randn(1, 16, 3, 128, device="cuda").bfloat16()
    near = obc.KvCache(cache.k[32999:].contiguous(), cache.v[32999:].contiguous())
    assert torch.equal(obc.obc_attend(q, cache, lens), obc.obc_attend(q, near, lens))
