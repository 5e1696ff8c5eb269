"""Ways through the cache kernels that only sizes choose: rows of a token in several trips, stores past the caches, vector loads of scale bytes, pages
smaller than a block at every head size, long sequences."""
import pytest
import torch

from oracle import cache as oc
from paper_2510_07651_amd import binding as obc

import cache_util as cu
from test_gpu_attend import TYPES, _run as attend_against_the_oracle

pytestmark = pytest.mark.gpu


def _same(x, y):
    for name in ("k", "v", "k_scale", "v_scale"):
        a, b = getattr(x, name), getattr(y, name)
        assert (a is None) == (b is None) and (a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))), name


def _in_pieces(T, most):
    return [(a, min(a + most, T)) for a in range(0, T, most)]


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("Hq,Hkv,d,pairs,interleaved", [(14, 2, 128, 64, False), (14, 2, 64, 16, True), (32, 8, 128, 48, True), (32, 8, 64, 32, False), (33, 3, 64, 32, True)])
def test_append_of_a_prompt(dtype, kind, Hq, Hkv, d, pairs, interleaved):
    """2 x 700 tokens in one call, whose 18, 39 and 48 rows per token take 16 lanes' groups two trips and more (and with 32/8 heads are stored past
    the caches): the bits of four calls of few tokens, and rows here and there against the oracle."""
    B, T, page, M = 2, 700, 64, 12
    g = torch.Generator().manual_seed(Hq + d)
    qkv = torch.randn(B, T, (Hq + 2 * Hkv) * d, generator=g).to(cu.DT[dtype])
    q, k, v = (x.unflatten(-1, (-1, d)) for x in qkv.cuda().split([Hq * d, Hkv * d, Hkv * d], -1))
    qw, kw = ((1 + 0.3 * torch.randn(d, generator=g)).to(cu.DT[dtype]).cuda() for _ in range(2))
    pos = torch.randint(0, 100000, (B, T), generator=g, dtype=torch.int32).cuda()
    freq = cu.rotation(pairs).cuda()
    lens, new = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([700, 730], [700, 655]))
    caches = [cu.make(kind, B, Hkv, d, page, M, seed=4)[0] for _ in range(2)]
    how = dict(inv_freq=freq, rot_scale=1.125, interleaved=interleaved, q_norm=qw, k_norm=kw)
    whole = obc.obc_cache_append(caches[0], k, v, lens, q=q, new_lens=new, positions=pos, **how)
    pieces = []
    for a, b in _in_pieces(T, 200):
        n = new.clamp(max=b) - new.clamp(max=a)
        pieces.append(obc.obc_cache_append(caches[1], k[:, a:b], v[:, a:b], lens - new + new.clamp(max=b), q=q[:, a:b], new_lens=n,
                                           positions=pos[:, a:b].contiguous(), **how))
    assert torch.equal(whole, torch.cat(pieces, 2))
    _same(*caches)
    held = dict(zip("kv", cu.held(caches[0])), table=caches[0].page_table.cpu())
    rows = qkv.unflatten(-1, (-1, d))
    slack = cu.append_slack(rows, torch.maximum(qw.abs(), kw.abs()).cpu(), 1.125)
    for b, t in ((0, 0), (0, 333), (0, 699), (1, 1), (1, 654)):
        row = int(lens[b] - new[b]) + t
        for h in range(Hq + Hkv):
            want = oc.turned(rows[b, t, h].double(), (qw if h < Hq else kw).cpu(), 1e-6, int(pos[b, t]), freq.cpu(), 1.125, interleaved)
            if h < Hq:
                cu.close(whole[b, h, t], want, dtype, slack[b, t, h])
            else:
                got = held["k"][oc.place(held, b, h - Hq, row)]
                # (half a step of a code that is not normal: 2^-10 of the block's power of two, which is below max / 224)
                extra = want.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True).expand(-1, 32).flatten() * 2.0 ** -10 / 224 if kind == "e4m3" else 0.0
                cu.close(got, want, kind, slack[b, t, h] + extra)
        for h in range(Hkv):
            want = rows[b, t, Hq + Hkv + h].double()
            assert torch.equal(held["v"][oc.place(held, b, h, row)], oc.e4m3(want)[0] if kind == "e4m3" else want)
    assert not bool(whole[1, :, 655:].any())


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("Hkv,d", [(8, 128), (7, 64)])
def test_store_of_many_rows(dtype, kind, Hkv, d):
    """3 x 2100 rows as an eviction leaves them, more than 8 MiB: what calls of 300 store, and the rows themselves."""
    B, T = 3, 2100
    g = torch.Generator().manual_seed(d)
    k, v = (torch.randn(B, Hkv, T, d, generator=g).to(cu.DT[dtype]).cuda() for _ in range(2))
    caches = [cu.make(kind, B, Hkv, d, 64, 34, seed=5)[0] for _ in range(2)]
    new = torch.tensor([[T - 17 * (b * Hkv + h) for h in range(Hkv)] for b in range(B)], dtype=torch.int32, device="cuda")
    obc.obc_cache_append(caches[0], k.transpose(1, 2), v.transpose(1, 2), new + 5, new_lens=new)
    for a, b in _in_pieces(T, 300):
        n = new.clamp(max=b) - new.clamp(max=a)
        obc.obc_cache_append(caches[1], k[:, :, a:b].transpose(1, 2), v[:, :, a:b].transpose(1, 2), new.clamp(max=b) + 5, new_lens=n)
    _same(*caches)
    if kind != "e4m3":
        got = obc.obc_cache_read(caches[0], T + 5)
        for b in range(B):
            for h in range(Hkv):
                n = int(new[b, h])
                assert torch.equal(got[0][b, h, 5:n + 5], k[b, h, :n]) and torch.equal(got[1][b, h, 5:n + 5], v[b, h, :n])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [204, 76, 96, 202])
def test_attend_over_8_bit_rows_without_a_table(dtype, d, rows):
    """Caches of 4 n and of 4 n + 2 rows: four tokens' scale bytes in one load where every head's rows start at a multiple of four."""
    for T, G in ((1, 2), (5, 4), (30, 3)):
        attend_against_the_oracle(dtype, "e4m3", 3, 3 * G, 3, T, d, rows, 0, [rows, rows - 9, max(T, rows // 2 + 1)], seed=rows + T)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("page", [1, 2, 4, 8])
def test_attend_over_small_pages(dtype, kind, page):
    for T in (1, 20, 50):
        attend_against_the_oracle(dtype, kind, 2, 4, 2, T, 128, page, 136 // page, [136, 67], seed=page)


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("T,lens", [(1, [20011, 9000]), (7, [4097, 12288]), (40, [16384, 5003])])
def test_attend_over_long_sequences(dtype, kind, T, lens):
    attend_against_the_oracle(dtype, kind, 2, 4, 1, T, 128, 64, 320, lens, seed=T)
