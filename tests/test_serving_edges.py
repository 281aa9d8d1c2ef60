"""CPU-only checks of the entry points behind the compressed rows at the edges of what they accept."""
import pytest
import torch

import paper_2605_07355_amd as ttf
from paper_2605_07355_amd import serving


def test_a_page_table_that_is_set_anew_is_the_one_used():
    k = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16)
    cache = ttf.TTFKVCache(k, k.clone(), torch.zeros((2, 4), dtype=torch.int32))
    for table in (torch.zeros((2, 9), dtype=torch.int32), torch.zeros((5, 6), dtype=torch.int32)[:, :3]):
        cache.page_table = table
        held = serving._KVCache.from_buffer_copy(cache._struct)
        assert cache.page_table is table and held.page_table == table.data_ptr()
        assert (held.table_width, held.table_stride) == (table.shape[1], table.stride(0)) and cache._batch == table.shape[0]
        assert (held.k, held.v, held.pages, held.page_size) == (cache.k.data_ptr(), cache.v.data_ptr(), 3, 16)
    for bad in (table.long(), table[0], table.t()):         # refused, and the one before stays
        with pytest.raises(ValueError):
            cache.page_table = bad
        assert cache.page_table is table and serving._KVCache.from_buffer_copy(cache._struct).page_table == table.data_ptr()
    for name in ("k", "v"):                                 # (their sizes and strides belong together)
        with pytest.raises(AttributeError):
            setattr(cache, name, k)
