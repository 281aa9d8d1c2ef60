"""CPU-only checks of the entry points behind the compressed rows at the edges of what they accept."""
import math

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


@pytest.mark.parametrize("R,base,length,factor", [
    (128, 1e4, 131072, 4.0),          # the last pair still turns twice
    (64, 1e4, 131072, 8.0),
    (128, 1e4, 4096, 16.0),           # the ramp ends between pairs
    (64, 1e6, 32768, 4.0),
    (16, 50.0, 100000, 4.0),          # all pairs turn more than 32 times: none is divided
])
def test_frequencies_divided_in_part_up_to_where_the_ramp_ends(R, base, length, factor):
    fast, slow = 32.0, 1.0

    def pair_that_turns(n):           # by bisection of the number of turns, which falls with the (broken) number of the pair
        lo, hi = -1000.0, 1000.0
        for _ in range(200):
            mid = (lo + hi) / 2
            lo, hi = (mid, hi) if length * base ** (-2 * mid / R) / (2 * math.pi) > n else (lo, mid)
        return lo

    low, high = max(0, math.floor(pair_that_turns(fast))), math.ceil(pair_that_turns(slow))
    got = ttf.ttf_rope_table(R, base, scaling="parts", factor=factor, original_length=length, fast=fast, slow=slow, device="cpu")
    f = [base ** (-2 * j / R) for j in range(R // 2)]
    g = [min(max((j - low) / (high - low), 0.0), 1.0) for j in range(R // 2)]
    want = torch.tensor([x * (1 - y) + x / factor * y for x, y in zip(f, g)], dtype=torch.float64)
    assert torch.allclose(got.inv_freq, want, rtol=1e-13, atol=0)
    if length * f[-1] / (2 * math.pi) > slow:              # a pair that turns more often than `slow` is not divided whole
        assert got.inv_freq[-1] > f[-1] / factor * (1 + 1e-9)


def test_a_workspace_is_enough_for_every_smaller_call():
    """Sizes do not fall where rows, sequences or max_rows grow."""
    counts = [1, 2, 3, 4, 5, 8, 9, 16, 17, 33, 64, 65, 500, 4096]
    for dtype in (torch.bfloat16, torch.float32):
        for heads, kv_heads, D in ((32, 8, 128), (16, 4, 256), (8, 8, 64), (7, 1, 72), (6, 2, 200), (64, 1, 64)):
            size = lambda rows, batch, n: ttf.ttf_attention_workspace_size(rows, batch, heads, kv_heads, D, dtype, max_rows=n)  # noqa: E731
            for rows in counts:
                by_max = [size(rows, rows, n) for n in counts]
                assert by_max == sorted(by_max), (dtype, heads, D, rows)
            for n in counts:
                by_rows = [size(rows, 4096, n) for rows in counts]
                assert by_rows == sorted(by_rows), (dtype, heads, D, n)
            # one sequence of all rows, and many that bring no more each
            for n in counts:
                assert size(n, 1, n) <= size(64 * n, 64, n)
