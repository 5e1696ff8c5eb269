"""The cache calls together, as a serving loop uses them: prefill in chunks, scoring, eviction, tokens; streams and captured steps."""
import pytest
import torch

from oracle import cache as oc
from paper_2510_07651_amd import binding as obc

import cache_util as cu

pytestmark = pytest.mark.gpu

HQ, HKV, D = 8, 2, 128


def _projection(B, T, seed, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, T, (HQ + 2 * HKV) * D, generator=g).to(dtype).cuda()
    return [t.unflatten(-1, (-1, D)) for t in x.split([HQ * D, HKV * D, HKV * D], -1)]


def _lens(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("adaptive", [False, True], ids=["one budget", "per head"])
def test_prefill_evict_decode(kind, adaptive):
    """Every attention of the loop is held to the oracle on what the cache holds at that moment."""
    B, page, M, budget = 2, 32, 16, 96
    cache, _ = cu.make(kind, B, HKV, D, page, M, seed=1)
    freq = cu.rotation(D // 2).cuda()

    def oracle_cache():
        k, v = cu.held(cache)
        return {"k": k, "v": v, "table": cache.page_table.cpu()}

    def step(lens, new, T, pos0, seed):
        q, k, v = _projection(B, T, seed)
        pos = (torch.tensor(pos0)[:, None] + torch.arange(T)[None]).int().cuda()
        qr = obc.obc_cache_append(cache, k, v, lens, q=q, new_lens=new, positions=pos, inv_freq=freq)
        out = obc.obc_attend(qr, cache, lens, new)
        ref = oc.attend(qr.cpu(), oracle_cache(), lens.cpu(), None if new is None else new.cpu())
        cu.check_attend(out, ref, int(lens.max()), D, "bf16")
        return qr

    # two prompts of 300 and 211 tokens, in chunks of 200
    step(_lens(200, 200), None, 200, [0, 0], 10)
    qr = step(_lens(300, 211), _lens(100, 11), 200, [200, 200], 11)
    window = torch.stack([qr[0, :, 92:100], qr[1, :, 3:11]]).contiguous()
    k, v = obc.obc_cache_read(cache, 300)
    scores = obc.obc_score(window, k, v, "joint", seq_lens=[300, 211])
    if adaptive:
        keep, counts = obc.obc_select_adaptive(scores, budget, 16, seq_lens=[300, 211])
        assert int(counts.sum()) == B * HKV * budget
    else:
        keep, counts = obc.obc_select(scores, budget, seq_lens=[300, 211]), _lens(budget, budget)
    kept = obc.obc_cache_read(cache, keep_idx=keep)
    for x, y in zip(kept, obc.obc_compact(k, v, keep)):
        assert torch.equal(x, y)                                     # the same rows as from the unpaged copy
    obc.obc_cache_append(cache, kept[0].transpose(1, 2), kept[1].transpose(1, 2), counts, new_lens=counts if adaptive else None)
    again = obc.obc_cache_read(cache, keep.shape[2])
    for b in range(B):
        for g in range(HKV):
            n = int(counts[b, g]) if adaptive else budget
            for x, y in zip(kept, again):
                assert torch.equal(x[b, g, :n], y[b, g, :n])
    # tokens: rows follow the kept ones, positions go on where the prompts ended
    lens = counts.clone()
    for i in range(3):
        lens += 1
        step(lens, None, 1, [300 + i, 211 + i], 20 + i)


def test_unpaged_cache_of_the_library():
    """The [B,Hkv,N,d] cache that obc_decode_step evicts from: append, attend, step."""
    N = 129
    k = torch.randn(1, HKV, N, D, device="cuda").bfloat16()
    v = torch.randn(1, HKV, N, D, device="cuda").bfloat16()
    scores = torch.rand(1, HKV, N, device="cuda")
    scores[..., N - 1] = 0
    cache = obc.KvCache(k, v)
    lens = _lens(N)
    for i in range(3):
        q, kn, vn = _projection(1, 1, 40 + i)
        qr = obc.obc_cache_append(cache, kn, vn, lens, q=q)
        assert torch.equal(k[:, :, N - 1], kn[:, 0]) and torch.equal(qr, q.transpose(1, 2))
        out = obc.obc_attend(qr, cache, lens)
        ref = oc.attend(qr.cpu(), {"k": k.double().cpu(), "v": v.double().cpu(), "table": None}, lens.cpu())
        cu.check_attend(out, ref, N, D, "bf16")
        obc.obc_decode_step(qr, k, v, scores, num_sinks=4, num_recent=16)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_captured_step_follows_the_lengths(kind):
    """A decoding step captured once: lengths, positions, pages and rows are device data, so replays go on where the last one ended."""
    B, steps = 2, 5
    caches = [cu.make(kind, B, HKV, D, 16, 8, seed=3)[0] for _ in range(2)]
    freq = cu.rotation(D // 2).cuda()
    rows = [_projection(B, 1, 60 + i) for i in range(steps)]
    start = _lens(30, 77)

    def tools(cache):
        return dict(lens=start.clone(), pos=start.view(B, 1).clone(), q=rows[0][0].contiguous(), k=rows[0][1].contiguous(),
                    v=rows[0][2].contiguous(), qr=torch.empty(B, HQ, 1, D, device="cuda", dtype=torch.bfloat16),
                    out=torch.empty(B, 1, HQ, D, device="cuda", dtype=torch.bfloat16),
                    ws=torch.empty(obc.obc_attend_workspace_bytes(B, 1, HQ, cache, torch.bfloat16), dtype=torch.uint8, device="cuda"))

    def step(cache, x):
        x["lens"].add_(1)
        x["pos"].add_(1)
        obc.obc_cache_append(cache, x["k"], x["v"], x["lens"], q=x["q"], q_out=x["qr"], positions=x["pos"], inv_freq=freq)
        obc.obc_attend(x["qr"], cache, x["lens"], out=x["out"], workspace=x["ws"])

    def feed(x, i):
        for name, t in zip(("q", "k", "v"), rows[i]):
            x[name].copy_(t)

    eager, captured = tools(caches[0]), tools(caches[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[1], captured)
    for i in range(steps):
        feed(eager, i)
        step(caches[0], eager)
        feed(captured, i)
        captured["ws"].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager["out"], captured["out"]) and torch.equal(eager["qr"], captured["qr"])
        for x, y in zip(cu.held(caches[0]), cu.held(caches[1])):
            assert torch.equal(x, y)


def test_calls_on_two_streams():
    """Each with its own workspace, on the stream that is current."""
    cache, _ = cu.make("bf16", 2, HKV, D, 32, 40, seed=4)
    lens = _lens(1200, 1000)
    qs = [torch.randn(2, HQ, 1, D, device="cuda").bfloat16() for _ in range(8)]
    want = [obc.obc_attend(q, cache, lens) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i, q in enumerate(qs):
        with torch.cuda.stream(streams[i % 2]):
            got.append(obc.obc_attend(q, cache, lens))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
