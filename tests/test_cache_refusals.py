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
