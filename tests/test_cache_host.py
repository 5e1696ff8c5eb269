"""What the cache calls refuse, before anything is launched (CPU): the C entry points with made-up pointers, the binding with tensors
that have no memory; and the oracle's own pins."""
import ctypes
import math

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from oracle import cache as oc
from paper_2510_07651_amd import binding as obc

FAKE, ODD = 4096, 4100            # never dereferenced


@pytest.fixture(scope="module")
def lib():
    return obc.load_library()


def _cache(**kw):
    x = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, page_table=FAKE, batch=2, num_pages=8, pages_per_seq=4, page_size=16, Hkv=2, d=128,
             dtype=obc.OBC_BF16)
    x.update(kw)
    return obc._CacheArg(**x)


BAD_CACHES = [
    (dict(k=None), obc.OBC_EINVAL), (dict(v=None), obc.OBC_EINVAL), (dict(k=ODD), obc.OBC_EINVAL), (dict(v=FAKE + 8), obc.OBC_EINVAL),
    (dict(page_table=FAKE + 2), obc.OBC_EINVAL), (dict(page_table=None), obc.OBC_EINVAL),
    (dict(page_table=None, batch=8, pages_per_seq=2), obc.OBC_EINVAL), (dict(num_pages=0), obc.OBC_EINVAL),
    (dict(pages_per_seq=0), obc.OBC_EINVAL), (dict(page_size=0), obc.OBC_EINVAL), (dict(page_size=-16), obc.OBC_EINVAL),
    (dict(batch=0), obc.OBC_EINVAL), (dict(Hkv=0), obc.OBC_EINVAL), (dict(page_size=24), obc.OBC_EUNSUPPORTED),
    (dict(d=96), obc.OBC_EUNSUPPORTED), (dict(d=0), obc.OBC_EINVAL), (dict(dtype=3), obc.OBC_EUNSUPPORTED), (dict(dtype=-1), obc.OBC_EUNSUPPORTED),
    (dict(k_scale=FAKE), obc.OBC_EINVAL), (dict(dtype=obc.OBC_E4M3), obc.OBC_EINVAL),
    (dict(dtype=obc.OBC_E4M3, k_scale=FAKE, v_scale=FAKE + 2), obc.OBC_EINVAL),
    (dict(page_size=1 << 20, pages_per_seq=1 << 11), obc.OBC_EUNSUPPORTED), (dict(batch=40000, Hkv=2), obc.OBC_EUNSUPPORTED),
]


def _rows(**kw):
    x = dict(data=FAKE, batch_stride=1024, token_stride=512, head_stride=128)
    x.update(kw)
    return obc._RowsArg(**x)


def _append(lib, cache=None, **kw):
    x = dict(q=None, k=_rows(), v=_rows(), q_out=None, lens=FAKE, per_head=0, new=None, new_per_head=0, pos=None, freq=None, pairs=0, rot_scale=1.0,
             inter=0, q_norm=None, k_norm=None, eps=1e-6, B=2, T=3, Hq=0, dtype=obc.OBC_BF16)
    x.update(kw)
    ref = lambda r: None if r is None else ctypes.byref(r)  # noqa: E731
    return lib.obc_cache_append(ref(x["q"]), ref(x["k"]), ref(x["v"]), None if cache == "none" else ref(cache or _cache()), x["q_out"], x["lens"],
                                x["per_head"], x["new"], x["new_per_head"], x["pos"], x["freq"], x["pairs"], x["rot_scale"], x["inter"],
                                x["q_norm"], x["k_norm"], x["eps"], x["B"], x["T"], x["Hq"], x["dtype"], None)


def _attend(lib, cache=None, **kw):
    x = dict(q=FAKE, out=FAKE, lens=FAKE, per_head=0, new=None, B=2, T=1, Hq=4, dtype=obc.OBC_BF16, causal=1, scale=0.1, ws=FAKE, ws_bytes=1 << 40)
    x.update(kw)
    return lib.obc_attend(x["q"], None if cache == "none" else ctypes.byref(cache or _cache()), x["out"], x["lens"], x["per_head"], x["new"], x["B"],
                          x["T"], x["Hq"], x["dtype"], x["causal"], x["scale"], x["ws"], x["ws_bytes"], None)


def _read(lib, cache=None, **kw):
    x = dict(keep=None, k_out=FAKE, v_out=FAKE, B=2, n=5, dtype=obc.OBC_BF16)
    x.update(kw)
    return lib.obc_cache_read(None if cache == "none" else ctypes.byref(cache or _cache()), x["keep"], x["k_out"], x["v_out"], x["B"], x["n"],
                              x["dtype"], None)


@pytest.mark.parametrize("change,status", BAD_CACHES, ids=[str(c) for c, _ in BAD_CACHES])
def test_caches_that_are_none(lib, change, status):
    for call in (_append, _attend, _read):
        assert call(lib, _cache(**change)) == status
    need = ctypes.c_size_t(0)
    assert lib.obc_attend_workspace_bytes(2, 1, 4, ctypes.byref(_cache(**change)), obc.OBC_BF16, ctypes.byref(need)) == status


def test_append_refusals(lib):
    q = dict(q=_rows(), q_out=FAKE, Hq=4)
    bad = [
        (dict(k=None), obc.OBC_EINVAL), (dict(v=None), obc.OBC_EINVAL), (dict(lens=None), obc.OBC_EINVAL), (dict(lens=FAKE + 2), obc.OBC_EINVAL),
        (dict(B=1), obc.OBC_EINVAL), (dict(T=0), obc.OBC_EINVAL), (dict(dtype=2), obc.OBC_EUNSUPPORTED), (dict(dtype=obc.OBC_F32), obc.OBC_EUNSUPPORTED),
        (dict(k=_rows(data=FAKE + 8)), obc.OBC_EINVAL), (dict(v=_rows(data=None)), obc.OBC_EINVAL), (dict(k=_rows(token_stride=130)), obc.OBC_EINVAL),
        (dict(k=_rows(batch_stride=-1024)), obc.OBC_EINVAL), (dict(v=_rows(head_stride=1 << 62)), obc.OBC_EINVAL),
        (dict(q_out=FAKE), obc.OBC_EINVAL), (dict(q_norm=FAKE), obc.OBC_EINVAL), (dict(Hq=4), obc.OBC_EINVAL),
        (dict(q, q_out=None), obc.OBC_EINVAL), (dict(q, q_out=FAKE + 8), obc.OBC_EINVAL), (dict(q, Hq=3), obc.OBC_EINVAL), (dict(q, Hq=0), obc.OBC_EINVAL),
        (dict(q, new=FAKE, new_per_head=1), obc.OBC_EINVAL), (dict(q, q=_rows(head_stride=4)), obc.OBC_EINVAL),
        (dict(pairs=-8), obc.OBC_EINVAL), (dict(pairs=72, pos=FAKE, freq=FAKE), obc.OBC_EINVAL), (dict(pairs=20, pos=FAKE, freq=FAKE), obc.OBC_EUNSUPPORTED),
        (dict(pairs=64, pos=FAKE), obc.OBC_EINVAL), (dict(pairs=64, freq=FAKE), obc.OBC_EINVAL),
        (dict(pairs=64, pos=FAKE, freq=FAKE, rot_scale=math.inf), obc.OBC_EINVAL), (dict(pairs=64, pos=FAKE + 1, freq=FAKE), obc.OBC_EINVAL),
        (dict(k_norm=FAKE + 4), obc.OBC_EINVAL), (dict(k_norm=FAKE, eps=-1.0), obc.OBC_EINVAL), (dict(k_norm=FAKE, eps=math.nan), obc.OBC_EINVAL),
        (dict(T=1 << 28), obc.OBC_EUNSUPPORTED),
    ]
    for change, status in bad:
        assert _append(lib, **change) == status, change
    assert _append(lib, "none") == obc.OBC_EINVAL
    assert _append(lib, _cache(dtype=obc.OBC_F32)) == obc.OBC_EUNSUPPORTED


@pytest.mark.parametrize("change", [dict(q=_rows(), q_out=FAKE, Hq=2), dict(pairs=64, pos=FAKE, freq=FAKE), dict(k_norm=FAKE)])
def test_append_refuses_more_tokens_than_a_grid_holds(lib, change):
    assert _append(lib, T=1 << 23, **change) == obc.OBC_EUNSUPPORTED          # 2 sequences: 2^24 workgroups of 2^8 threads
    assert _append(lib, T=1 << 26) == obc.OBC_EUNSUPPORTED


def test_attend_refusals(lib):
    bad = [
        (dict(q=None), obc.OBC_EINVAL), (dict(out=None), obc.OBC_EINVAL), (dict(lens=None), obc.OBC_EINVAL), (dict(q=FAKE + 8), obc.OBC_EINVAL),
        (dict(out=FAKE + 2), obc.OBC_EINVAL), (dict(lens=FAKE + 1), obc.OBC_EINVAL), (dict(new=FAKE + 2), obc.OBC_EINVAL), (dict(B=3), obc.OBC_EINVAL),
        (dict(T=0), obc.OBC_EINVAL), (dict(Hq=3), obc.OBC_EINVAL), (dict(Hq=0), obc.OBC_EINVAL), (dict(dtype=2), obc.OBC_EUNSUPPORTED),
        (dict(dtype=obc.OBC_F32), obc.OBC_EUNSUPPORTED), (dict(scale=0.0), obc.OBC_EINVAL), (dict(scale=-1.0), obc.OBC_EINVAL),
        (dict(scale=math.nan), obc.OBC_EINVAL), (dict(scale=math.inf), obc.OBC_EINVAL), (dict(scale=3e38), obc.OBC_EINVAL),
        (dict(T=1 << 25), obc.OBC_EUNSUPPORTED),
    ]
    for change, status in bad:
        assert _attend(lib, **change) == status, change
    assert _attend(lib, "none") == obc.OBC_EINVAL
    long = _cache(pages_per_seq=4096)
    need = ctypes.c_size_t(0)
    assert lib.obc_attend_workspace_bytes(2, 1, 4, ctypes.byref(long), obc.OBC_BF16, ctypes.byref(need)) == obc.OBC_OK
    assert need.value > 0 and need.value % 256 == 0
    for change in (dict(ws=None), dict(ws=FAKE + 16), dict(ws_bytes=need.value - 256)):
        assert _attend(lib, long, **change) == obc.OBC_EWORKSPACE, change
    assert lib.obc_attend_workspace_bytes(2, 1, 4, ctypes.byref(long), obc.OBC_BF16, None) == obc.OBC_EINVAL


def test_read_refusals(lib):
    bad = [(dict(k_out=None), obc.OBC_EINVAL), (dict(v_out=None), obc.OBC_EINVAL), (dict(k_out=FAKE + 8), obc.OBC_EINVAL), (dict(B=1), obc.OBC_EINVAL),
           (dict(n=0), obc.OBC_EINVAL), (dict(n=65), obc.OBC_EINVAL), (dict(n=(1 << 27) + 1, keep=FAKE), obc.OBC_EUNSUPPORTED), (dict(keep=FAKE + 2), obc.OBC_EINVAL), (dict(dtype=obc.OBC_F32), obc.OBC_EUNSUPPORTED),
           (dict(dtype=obc.OBC_E4M3), obc.OBC_EUNSUPPORTED)]
    for change, status in bad:
        assert _read(lib, **change) == status, change
    assert _read(lib, "none") == obc.OBC_EINVAL


def test_the_other_calls_take_no_8_bit_caches(lib):
    with pytest.raises(obc.ObcError) as e:
        obc.obc_score_workspace_bytes(1, 512, 16, 1, 1, 64, obc.OBC_E4M3, obc.OBC_JOINT)
    assert e.value.status == obc.OBC_EUNSUPPORTED


# ---- the binding ----

class _NoLaunch:
    """A library whose calls only note that they were reached."""

    def __init__(self):
        self.reached = []

    def __getattr__(self, name):
        def note(*args):
            if not name.endswith("_bytes"):
                self.reached.append(name)
            return obc.OBC_OK
        return note


@pytest.fixture
def stub(monkeypatch):
    x = _NoLaunch()
    monkeypatch.setattr(obc, "_lib", x)
    monkeypatch.setattr(obc, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with FakeTensorMode():
        yield x


BF16, FP32, I32, I64, U8, E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.uint8, torch.float8_e4m3fn
fake_pointers = pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")


def _t(shape, dtype=BF16, device="cuda"):
    return torch.empty(shape, dtype=dtype, device=device)


def _handle(kind=BF16, B=2, M=4, page=16, Hkv=2, d=128):
    return obc.KvCache.empty(B * M, Hkv, page, d, kind, page_table=_t((B, M), I32))


@fake_pointers
def test_handle_refusals(stub):
    k = _t((8, 2, 16, 128))
    good = obc.KvCache(k, k)
    assert (good.batch, good.capacity) == (8, 16) and obc.KvCache(k, k, _t((2, 4), I32)).capacity == 64
    assert _handle(E4M3).k_scale.shape == (8, 2, 16, 4)
    s = _t((8, 2, 16, 4), U8)
    k8 = _t((8, 2, 16, 128), E4M3)
    obc.KvCache(k8, k8, None, s, s)
    for args in [(k, _t((8, 2, 16, 64))), (k, _t((8, 2, 16, 128), FP32)), (k, _t((8, 2, 16, 128), device="cpu")), (_t((8, 2, 128)), _t((8, 2, 128))),
                 (_t((8, 2, 16, 96)), _t((8, 2, 16, 96))), (_t((0, 2, 16, 128)), _t((0, 2, 16, 128))), (k.transpose(1, 2), k.transpose(1, 2)),
                 (k, k, _t((2, 4), I64)), (k, k, _t((8,), I32)), (k, k, _t((2, 4), I32, "cpu")), (k, k, _t((2, 0), I32)), (k, k, _t((2, 8), I32)[:, ::2]),
                 (_t((8, 2, 24, 128)), _t((8, 2, 24, 128)), _t((2, 4), I32)), (k, k, None, s, s), (k8, k8), (k8, k8, None, s), (k8, k8, None, s, _t((8, 2, 16, 2), U8)),
                 (k8, k8, None, s, _t((8, 2, 16, 4), I32))]:
        with pytest.raises(ValueError):
            obc.KvCache(*args)
    with pytest.raises(TypeError):
        obc.KvCache(_t((8, 2, 16, 128), torch.float16), _t((8, 2, 16, 128), torch.float16))
    big = _t((1, 1, 1, 128)).expand(1, 1, 1, 128)
    with pytest.raises(ValueError):
        obc.KvCache(big, big, _t((1, (1 << 30) + 1), I32))


@fake_pointers
@pytest.mark.parametrize("change", [dict(k=(2, 3, 2, 64)), dict(k=(1, 3, 2, 128)), dict(k=(2, 3, 1, 128)), dict(k=(2, 3, 256)), dict(v=(2, 4, 2, 128)),
                                    dict(v=(2, 3, 4, 128)), dict(vd=FP32), dict(kd=FP32, vd=FP32, qd=FP32), dict(qd=FP32), dict(q=(2, 4, 4, 128)),
                                    dict(q=(2, 3, 3, 128)), dict(q=(2, 3, 0, 128)), dict(lens=(3,)), dict(lens=(2, 3)), dict(lens_d=I64), dict(new=(2, 2)),
                                    dict(new=(2,), new_d=I64), dict(out=(2, 3, 4, 128)), dict(out=(2, 4, 3, 128), out_d=FP32), dict(pos=(2, 3)),
                                    dict(freq=(64,)), dict(pos=(2, 4), freq=(64,)), dict(pos=(2, 3), freq=(64,), pos_d=I64),
                                    dict(pos=(2, 3), freq=(64,), freq_d=BF16), dict(pos=(2, 3), freq=(0,)), dict(q_norm=(64,)), dict(k_norm=(128,), norm_d=FP32),
                                    dict(channels_apart=True), dict(where="cpu")], ids=str)
def test_append_refuses_what_does_not_fit_together(change, stub):
    def call(k=(2, 3, 2, 128), v=(2, 3, 2, 128), q=(2, 3, 4, 128), kd=BF16, vd=BF16, qd=BF16, lens=(2,), lens_d=I32, new=None, new_d=I32, out=None,
             out_d=BF16, pos=None, pos_d=I32, freq=None, freq_d=FP32, q_norm=None, k_norm=None, norm_d=BF16, channels_apart=False, where="cuda",
             kind=BF16):
        on = lambda s, d: None if s is None else _t(s, d)  # noqa: E731
        kt = _t(k, kd, where)
        if channels_apart:
            kt = _t((2, 3, 128, 2)).transpose(2, 3)
        return obc.obc_cache_append(_handle(kind), kt, _t(v, vd), _t(lens, lens_d), q=on(q, qd), q_out=on(out, out_d), new_lens=on(new, new_d),
                                    positions=on(pos, pos_d), inv_freq=on(freq, freq_d), q_norm=on(q_norm, norm_d), k_norm=on(k_norm, norm_d))
    for good in (dict(), dict(q=None), dict(q=None, new=(2, 2)), dict(new=(2,), lens=(2, 2)), dict(pos=(2, 3), freq=(64,), q_norm=(128,), k_norm=(128,)),
                 dict(out=(2, 4, 3, 128)), dict(kind=E4M3), dict(kind=E4M3, kd=FP32, vd=FP32, qd=FP32)):
        call(**good)
    reached = len(stub.reached)
    assert reached == 8
    with pytest.raises((ValueError, TypeError)):
        call(**change)
    assert len(stub.reached) == reached


@fake_pointers
@pytest.mark.parametrize("change", [dict(q=(1, 4, 1, 128)), dict(q=(2, 4, 1, 64)), dict(q=(2, 3, 1, 128)), dict(q=(2, 4, 0, 128)), dict(q=(2, 4, 128)),
                                    dict(qd=FP32), dict(qd=torch.float16, kind=E4M3), dict(lens=(2, 3)), dict(lens_d=I64), dict(new=(2, 2)), dict(out=(2, 4, 1, 128)),
                                    dict(out=(2, 1, 4, 128), out_d=FP32), dict(turned=True), dict(ws="cpu"), dict(where="cpu")], ids=str)
def test_attend_refuses_what_does_not_fit_together(change, stub):
    def call(q=(2, 4, 1, 128), qd=BF16, lens=(2,), lens_d=I32, new=None, out=None, out_d=BF16, kind=BF16, turned=False, ws=None, where="cuda"):
        qt = _t(q, qd, where)
        if turned:
            qt = _t((2, 3, 4, 128)).transpose(1, 2)
        return obc.obc_attend(qt, _handle(kind), _t(lens, lens_d), None if new is None else _t(new, I32), out=None if out is None else _t(out, out_d),
                              workspace=None if ws is None else _t((1 << 20,), U8, ws))
    for good in (dict(), dict(lens=(2, 2), new=(2,)), dict(out=(2, 1, 4, 128)), dict(kind=E4M3), dict(kind=E4M3, qd=FP32), dict(ws="cuda")):
        call(**good)
    reached = len(stub.reached)
    assert reached == 6
    with pytest.raises((ValueError, TypeError)):
        call(**change)
    assert len(stub.reached) == reached


@fake_pointers
@pytest.mark.parametrize("change", [dict(n=0), dict(n=65), dict(n=None), dict(keep=(2, 2, 5), n=4), dict(keep=(2, 5), n=None), dict(keep=(2, 2, 5), keep_d=I64, n=None),
                                    dict(dtype=FP32), dict(dtype=E4M3, kind=E4M3), dict(out=(2, 2, 6, 128)), dict(out=(2, 2, 5, 128), out_d=FP32)], ids=str)
def test_read_refuses_what_does_not_fit_together(change, stub):
    def call(n=5, keep=None, keep_d=I32, dtype=None, kind=BF16, out=None, out_d=BF16):
        return obc.obc_cache_read(_handle(kind), n, None if keep is None else _t(keep, keep_d), dtype, None if out is None else _t(out, out_d))
    assert call()[0].dtype is BF16 and call(n=None, keep=(2, 2, 70))[1].shape == (2, 2, 70, 128) and call(kind=E4M3, dtype=FP32)[0].dtype is FP32
    assert call(out=(2, 2, 5, 128))[0].shape == (2, 2, 5, 128)
    reached = len(stub.reached)
    assert reached == 4
    with pytest.raises(ValueError):
        call(**change)
    assert len(stub.reached) == reached


@fake_pointers
def test_another_device_is_made_current(stub, monkeypatch):
    """The launch goes to the cache's GPU and to that one's current stream."""
    entered = []

    class Current:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            entered.append(self.index)

        def __exit__(self, *args):
            entered.append("left")
    cache = _handle()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "device", Current)
    obc.obc_cache_read(cache, 3)
    assert entered == [0, "left"] and stub.reached == ["obc_cache_read"]


# ---- the oracle's pins ----

def test_oracle_codes_are_torchs():
    """Its 8-bit rounding against torch's cast, over every pair of neighbouring codes and the middle between them."""
    codes = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float32).double()
    mid = (codes[1:] + codes[:-1]) / 2
    x = torch.cat([codes, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    x = torch.cat([x, -x])
    assert torch.equal(oc.e4m3_round(x), x.float().to(torch.float8_e4m3fn).to(torch.float32).double())
    for top, e in ((448.0, 0), (448.1, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.76, -7), (0.0, -117), (2.0 ** -130, -117), (3.4e38, 120)):
        assert oc.e4m3_exponent(top) == e


def test_oracle_attention_is_torchs():
    g = torch.Generator().manual_seed(0)
    q, k, v = torch.randn(1, 4, 5, 64, generator=g).double(), torch.randn(1, 2, 9, 64, generator=g).double(), torch.randn(1, 2, 9, 64, generator=g).double()
    mask = torch.ones(5, 9, dtype=torch.bool).tril(4)
    want = torch.nn.functional.scaled_dot_product_attention(q, k.repeat_interleave(2, 1), v.repeat_interleave(2, 1), attn_mask=mask)
    got, _, _ = oc.attend(q, {"k": k, "v": v, "table": None}, torch.tensor([9]))
    assert torch.allclose(got.transpose(1, 2), want, rtol=1e-12, atol=1e-13)
    # in pages: the same rows elsewhere
    pages = {x: torch.zeros(3, 2, 4, 64).double() for x in "kv"}
    table = torch.tensor([[2, 0, 1]])
    for j in range(9):
        for x, rows in (("k", k), ("v", v)):
            pages[x][int(table[0, j // 4]), :, j % 4] = rows[0, :, j]
    assert torch.equal(oc.attend(q, {**pages, "table": table}, torch.tensor([9]))[0], got)


def test_oracle_rotation_turns_and_keeps_norms():
    x = torch.arange(1.0, 9.0).double()
    freq = torch.tensor([1.0, 0.25])
    for interleaved, (p, q) in ((False, (0, 2)), (True, (0, 1))):
        y = oc.turned(x, None, 0, 3, freq, 1.0, interleaved)
        z = complex(x[p], x[q]) * complex(math.cos(3.0), math.sin(3.0))
        assert abs(complex(y[p], y[q]) - z) < 1e-12 and torch.equal(y[4:], x[4:]) and abs(float(y.norm() - x.norm())) < 1e-12
