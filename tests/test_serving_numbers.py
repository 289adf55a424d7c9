"""Numbers that the library's 32-bit arguments cannot hold are refused, not cut off: a window of 2^32 + 5 is none of 5.  No GPU."""
import pytest
import torch

from paper_2506_23906_amd import binding as B


@pytest.mark.parametrize("number", [-1, 1 << 32, (1 << 32) + 5, 2.5])
def test_numbers_that_do_not_fit(libmmvseg_path, number):
    B.load()
    i, q = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cache = B.PagedCache.__new__(B.PagedCache)
    cache.k = cache.v = torch.zeros(2, 2, 8, 64, dtype=torch.bfloat16)
    cache._struct = B._CacheStruct(0, 0, B.MMV_TYPE_BF16, 8, 2, 64, 2, 1024, 512, 64, 1.0, 1.0)
    cache._ref = B.ctypes.addressof(cache._struct)
    with pytest.raises(B.MmvError, match="window"):
        B.mmv_paged_attention(q, cache, torch.zeros(4, 4, dtype=torch.int32), i, window=number)
    with pytest.raises(B.MmvError, match="page"):
        B.mmv_page_tables(i, i, i, torch.zeros(4, 4, dtype=torch.int32), number, 4)
