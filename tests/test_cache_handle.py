"""A KvCache keeps the addresses of the tensors that it was made of: what it shows is what the calls work on (CPU)."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2510_07651_amd import binding as obc


@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_a_handles_tensors_are_not_exchanged():
    with FakeTensorMode():
        new = lambda *s, t=torch.bfloat16: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
        table = new(2, 4, t=torch.int32)
        cache = obc.KvCache(new(8, 2, 16, 128), new(8, 2, 16, 128), table)
        for name in ("k", "v", "k_scale", "v_scale", "page_table", "batch", "Hkv", "d", "dtype", "device", "capacity"):
            before = getattr(cache, name, None)
            with pytest.raises(AttributeError):
                setattr(cache, name, new(2, 8, t=torch.int32))
            assert getattr(cache, name, None) is before
        with pytest.raises(AttributeError):
            del cache.page_table
        assert cache.page_table is table and cache.capacity == 64
        cache.layer = 3                                                # a program's own notes are its own
        cache.layer = 4
        assert cache.layer == 4
        del cache.layer
