"""obc_attend against the oracle: types, head groups, lengths from nothing to several shares, pages, ragged chunks, what must not be read."""
import math

import pytest
import torch

from oracle import cache as oc
from paper_2510_07651_amd import binding as obc

import cache_util as cu

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("bf16", "e4m3"), ("fp32", "fp32"), ("fp32", "e4m3")]


def _poison(cache, want, lens, B, Hkv):
    """NaN in every place that no sequence's first `lens` rows lie in."""
    mine = torch.zeros(want["k"].shape[:3], dtype=torch.bool)
    for b in range(B):
        for g in range(Hkv):
            for j in range(min(max(oc.length(lens, b, g), 0), oc.capacity(want))):
                mine[oc.place(want, b, g, j)] = True
    for x in (cache.k, cache.v):
        bytes_ = x.view(torch.uint8)
        bytes_[~mine.cuda()] = 0x7f if x.dtype is torch.float8_e4m3fn else 0xff
    for x in (cache.k_scale, cache.v_scale):
        if x is not None:
            x[~mine.cuda()] = 0xff


def _run(dtype, kind, B, Hq, Hkv, T, d, page, M, lens, new=None, causal=True, scale=None, seed=0, sharp=2.0):
    cache, want = cu.make(kind, B, Hkv, d, page, M, seed=seed)
    lens = torch.tensor(lens, dtype=torch.int32)
    _poison(cache, want, lens, B, Hkv)
    g = torch.Generator().manual_seed(seed + 77)
    q = (sharp * torch.randn(B, Hq, T, d, generator=g)).to(cu.DT[dtype])
    news = None if new is None else torch.tensor(new, dtype=torch.int32)
    dev_q = q.cuda()
    if new is not None:
        for b in range(B):
            dev_q[b, :, max(new[b], 0):] = math.nan                  # padding
    out = torch.full((B, T, Hq, d), 7.0, dtype=cu.DT[dtype], device="cuda")
    need = obc.obc_attend_workspace_bytes(B, T, Hq, cache, q.dtype)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")  # (stale NaN: nobody reads a record that this call has not left)
    got = obc.obc_attend(dev_q, cache, lens.cuda(), None if news is None else news.cuda(), causal, scale, out=out, workspace=ws)
    torch.cuda.synchronize()
    assert got is out
    ref = oc.attend(q, want, lens, news, causal, scale)
    longest = int(max(lens.max(), 1))
    cu.check_attend(out, ref, longest, d, dtype)
    assert not bool(out[(ref[1] == 0).cuda()].any())
    return cache, dev_q, lens.cuda(), out


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 3, 40])
def test_attend(dtype, kind, d, T):
    for Hq, Hkv in ((4, 4), (8, 2), (7, 1)):
        _run(dtype, kind, 2, Hq, Hkv, T, d, 16, 6, [T, 93], seed=T + Hq)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("lens", [[1, 1], [31, 32], [33, 64], [65, 127], [128, 129], [200, 255], [256, 0]], ids=str)
def test_attend_lengths(dtype, kind, lens):
    """Around the sizes of tiles and shares, one token and a chunk, with every row in sight and causally."""
    for T, causal in ((1, True), (2, False), (17, False), (17, True)):
        _run(dtype, kind, 2, 8, 2, T, 128, 64, 4, lens, causal=causal, seed=lens[0])


@pytest.mark.parametrize("dtype,kind", TYPES)
def test_attend_rows_that_see_nothing(dtype, kind):
    """Empty sequences, chunks longer than what the cache holds, no new rows, lengths outside the cache."""
    _run(dtype, kind, 4, 4, 2, 5, 64, 16, 2, [0, 3, 32, 7], new=[5, 5, 0, 9])
    _run(dtype, kind, 2, 4, 2, 5, 128, 16, 2, [-4, 33], causal=True)
    _run(dtype, kind, 2, 4, 2, 70, 128, 16, 2, [20, 5], causal=True)
    _run(dtype, kind, 2, 4, 2, 5, 128, 16, 2, [0, 9], new=[3, -2], causal=False)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("T", [1, 33])
def test_attend_length_per_head(dtype, kind, T):
    """A head-adaptive eviction leaves every KV head its own rows; one of them may be empty but for the new ones."""
    _run(dtype, kind, 2, 12, 3, T, 128, 32, 8, [[T, 100, 256], [77, T + 1, 0]], seed=5)


@pytest.mark.parametrize("dtype,kind", TYPES)
def test_attend_without_a_table(dtype, kind):
    """The library's own [B,Hkv,N,d] caches, of a length that is no multiple of anything."""
    for T in (1, 50):
        _run(dtype, kind, 3, 4, 2, T, 128, 203, 0, [203, 51, 150], seed=8)
        _run(dtype, kind, 2, 6, 6, T, 64, 77, 0, [77, 64], new=[T, 1], seed=9)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("page", [1, 2, 8, 128])
def test_attend_page_sizes(dtype, kind, page):
    for T in (1, 20):
        _run(dtype, kind, 2, 4, 2, T, 64, page, max(1, 130 // page), [min(130, max(1, 130 // page) * page), 21], seed=page)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("G,T", [(1, 1), (2, 1), (3, 5), (8, 1), (8, 2), (16, 1), (17, 1), (32, 1), (33, 1), (5, 7), (16, 9), (64, 2)])
def test_attend_groups(dtype, kind, G, T):
    """Rows per KV head around the kernels' tiles."""
    _run(dtype, kind, 1, 2 * G, 2, T, 128, 32, 5, [149], seed=G)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("T,N", [(1, 3000), (1, 517), (9, 1300), (130, 700), (300, 300)])
def test_attend_several_shares(dtype, kind, T, N):
    _run(dtype, kind, 1, 4, 1, T, 128, 64, -(-N // 64), [N], seed=N)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("T", [1, 20, 140])
def test_attend_short_sequences_in_a_large_cache(dtype, kind, T):
    """Calls are cut up for what the cache could hold; most of the shares have nothing to do."""
    _run(dtype, kind, 2, 4, 1, T, 128, 64, 64, [T, 600], seed=T)


@pytest.mark.parametrize("dtype,kind", TYPES)
def test_attend_padding_beside_rows_that_see_much(dtype, kind):
    """Padded rows share a tile with rows that see several blocks, in one share and in several; their queries are NaN."""
    _run(dtype, kind, 2, 8, 2, 60, 128, 64, 16, [900, 333], new=[23, 59], seed=2)
    _run(dtype, kind, 2, 8, 2, 60, 64, 32, 4, [128, 100], new=[41, 1], seed=3)
    _run(dtype, kind, 2, 8, 2, 6, 128, 64, 16, [900, 333], new=[2, 5], seed=4)


@pytest.mark.parametrize("dtype,kind", TYPES)
def test_attend_scale_and_large_logits(dtype, kind):
    """A scale of the caller's; logits of hundreds, where one token takes everything."""
    _run(dtype, kind, 1, 4, 2, 3, 128, 16, 8, [100], scale=0.3)
    _run(dtype, kind, 1, 4, 2, 3, 128, 16, 8, [100], sharp=40.0)
    _run(dtype, kind, 1, 4, 2, 3, 128, 16, 8, [100], scale=1e-20)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("B,Hkv,G,T", [(3, 3, 2, 150), (5, 2, 1, 200), (3, 4, 2, 130), (1, 1, 8, 90), (24, 8, 1, 300)])
def test_attend_many_heads_and_tiles(kind, B, Hkv, G, T):
    """Heads that share dies evenly and not, more workgroups than run at once, tiles of all lengths."""
    _run("bf16", kind, B, G * Hkv, Hkv, T, 64, 32, 10, [min(320, T + 11 * b) for b in range(B)], seed=B)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 60])
def test_attend_powers_of_two_of_all_sizes(dtype, T):
    """8-bit values whose blocks' powers of two run from the least to large ones."""
    cache, want = cu.make("e4m3", 1, 2, 128, 16, 8, seed=6)
    e = torch.randint(10, 200, cache.v_scale.shape, generator=torch.Generator().manual_seed(1), dtype=torch.uint8)
    cache.v_scale.copy_(e)
    want["v"] = cu.held(cache)[1]
    lens = torch.tensor([100], dtype=torch.int32)
    q = torch.randn(1, 4, T, 128, generator=torch.Generator().manual_seed(2)).to(cu.DT[dtype])
    out = obc.obc_attend(q.cuda(), cache, lens.cuda())
    cu.check_attend(out, oc.attend(q, want, lens), 100, 128, dtype)


def test_attend_replays_with_other_lengths():
    """A chunk's call captured once, in several shares: lengths, queries and rows are read when it is replayed."""
    for dtype, kind in TYPES:
        cache, _ = cu.make(kind, 2, 2, 128, 64, 20, seed=3)
        q = torch.zeros(2, 8, 40, 128, dtype=cu.DT[dtype], device="cuda")
        lens, new = (torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2))
        out = torch.empty(2, 40, 8, 128, dtype=q.dtype, device="cuda")
        ws = torch.empty(obc.obc_attend_workspace_bytes(2, 40, 8, cache, q.dtype), dtype=torch.uint8, device="cuda")
        assert ws.numel() > 0
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            obc.obc_attend(q, cache, lens, new, out=out, workspace=ws)
        for i, (ls, ns) in enumerate((([1280, 700], [40, 40]), ([40, 0], [40, 3]), ([555, 1279], [1, 39]))):
            q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)))
            lens.copy_(torch.tensor(ls))
            new.copy_(torch.tensor(ns))
            ws.fill_(255)
            graph.replay()
            assert torch.equal(obc.obc_attend(q, cache, lens, new), out)
            torch.cuda.synchronize()


def test_attend_pages_outside_the_pool():
    """They are read as the nearest page inside."""
    cache, _ = cu.make("bf16", 1, 2, 128, 16, 4, seed=2)
    good = cache.page_table.clone()
    P = cache.k.shape[0]
    good[0, 1], good[0, 3] = P - 1, 0
    bad = good.clone()
    bad[0, 1], bad[0, 3] = 10 ** 6, -(2 ** 31)
    lens = torch.tensor([60], dtype=torch.int32, device="cuda")
    for T in (1, 40):
        q = torch.randn(1, 4, T, 128, device="cuda").bfloat16()
        outs = [obc.obc_attend(q, obc.KvCache(cache.k, cache.v, t), lens) for t in (good, bad)]
        assert torch.equal(*outs)


def test_attend_gives_the_same_bits_again():
    """Whatever the workspace holds, whatever ran before, and with outputs of its own."""
    for dtype, kind in TYPES:
        for T in (1, 45):
            cache, q, lens, out = _run(dtype, kind, 2, 8, 2, T, 128, 32, 12, [380, 200], seed=1)
            again = obc.obc_attend(q, cache, lens)
            assert torch.equal(again, out)
