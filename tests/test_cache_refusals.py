"""Calls of the cache that are taken or refused by their strides, their handles and the memory they would write (CPU): the C entry points with
made-up pointers.  What is taken reaches the launch, which fails where there is no GPU."""
import ctypes

import pytest
import torch

from paper_2510_07651_amd import binding as obc

BASE = 1 << 40                    # never dereferenced


@pytest.fixture(scope="module")
def lib():
    return obc.load_library()


@pytest.fixture(autouse=True)
def no_gpu():
    if torch.cuda.device_count() > 0:
        pytest.skip("made-up pointers are not given to a GPU")


def _cache(**kw):
    x = dict(k=BASE, v=BASE + (1 << 30), k_scale=None, v_scale=None, page_table=BASE + (3 << 30), batch=2, num_pages=8, pages_per_seq=4, page_size=16,
             Hkv=2, d=128, dtype=obc.OBC_BF16)
    x.update(kw)
    return obc._CacheArg(**x)


def _rows(at, batch, token, head):
    return obc._RowsArg(BASE + (4 << 30) + at, batch, token, head)


def _append(lib, k, v, q=None, q_out=None, B=2, T=3, Hq=4, cache=None):
    ref = lambda r: None if r is None else ctypes.byref(r)  # noqa: E731
    lens = BASE + (5 << 30)
    return lib.obc_cache_append(ref(q), ref(k), ref(v), ref(cache or _cache(batch=B)), q_out, lens, 0, None, 0, None, None, 0, 1.0, 0, None, None, 1e-6, B,
                                T, Hq if q is not None else 0, obc.OBC_BF16, None)


@pytest.mark.parametrize("B,T,Hkv,strides", [(1, 3, 2, (3, 256, 128)), (2, 1, 2, (256, 1, 128)), (2, 3, 1, (384, 128, 5)), (1, 1, 1, (1, 1, 1)), (1, 1, 2, (-7, 1 << 62, 128))])
def test_strides_of_dimensions_of_size_1_do_not_matter(lib, B, T, Hkv, strides):
    k = _rows(0, *strides)
    assert _append(lib, k, k, B=B, T=T, cache=_cache(batch=B, Hkv=Hkv)) == obc.OBC_ELAUNCH
    q = _rows(1 << 20, *strides)
    assert _append(lib, k, k, q, BASE + (6 << 30), B=B, T=T, Hq=Hkv, cache=_cache(batch=B, Hkv=Hkv)) == obc.OBC_ELAUNCH
    for i, n in enumerate((B, T, Hkv)):
        bad = [256 * 128, 256, 128]
        bad[i] += 1
        want = obc.OBC_EINVAL if n > 1 else obc.OBC_ELAUNCH
        assert _append(lib, _rows(0, *bad), k, B=B, T=T, cache=_cache(batch=B, Hkv=Hkv)) == want


MB = 1 << 20


def test_q_out_over_the_inputs_is_refused(lib):
    """[2,3,4,128] bf16 queries, 2 x 3 KB, against rows in every order: refused where one row is met, taken next to and between them."""
    B, T, Hq = 2, 3, 4
    row, size = 256, B * T * Hq * 256
    at = lambda x: BASE + (4 << 30) + x  # noqa: E731
    k = _rows(64 * MB, T * 256, 256, 128)
    for strides in ((T * Hq * 128, Hq * 128, 128), (T * Hq * 128, 128, T * 128), (MB, Hq * 128, 128), (512, MB, 128), (512, 128, MB), (0, 0, 128)):
        starts = [2 * (b * strides[0] + t * strides[1] + h * strides[2]) for b in range(B) for t in range(T) for h in range(Hq)]
        q = _rows(8 * MB, *strides)
        for start in sorted({s + shift for s in starts for shift in (-size, -size + 16, -16, 0, row - 16, row, MB, -MB)}):
            meets = any(start < s + row and start + size > s for s in starts)
            got = _append(lib, k, k, q, at(8 * MB + start), B, T, Hq)
            assert got == (obc.OBC_EINVAL if meets else obc.OBC_ELAUNCH), (strides, start)
    q = _rows(0, T * Hq * 128, Hq * 128, 128)
    for name in "kv":
        rows = dict(k=k, v=_rows(80 * MB, T * 256, 256, 128))
        for start, want in ((-size, obc.OBC_ELAUNCH), (-size + 16, obc.OBC_EINVAL), (0, obc.OBC_EINVAL), (B * T * 512 - 16, obc.OBC_EINVAL), (B * T * 512, obc.OBC_ELAUNCH)):
            assert _append(lib, rows["k"], rows["v"], q, rows[name].data + start, B, T, Hq) == want, (name, start)


def test_out_over_q_is_refused(lib):
    size, q = 2 * 4 * 128 * 2, BASE + (4 << 30)
    for start in (-size, -size + 16, -16, 0, 16, size - 16, size):
        got = lib.obc_attend(q, ctypes.byref(_cache()), q + start, BASE + (5 << 30), 0, None, 2, 1, 4, obc.OBC_BF16, 1, 0.1, None, 0, None)
        assert got == (obc.OBC_ELAUNCH if abs(start) == size else obc.OBC_EINVAL), start


def test_outputs_of_a_read_over_each_other_are_refused(lib):
    size, out = 2 * 2 * 5 * 128 * 2, BASE + (4 << 30)
    for start in (-size, -size + 16, 0, 16, size - 16, size):
        got = lib.obc_cache_read(ctypes.byref(_cache()), None, out, out + start, 2, 5, obc.OBC_BF16, None)
        assert got == (obc.OBC_ELAUNCH if abs(start) == size else obc.OBC_EINVAL), start
