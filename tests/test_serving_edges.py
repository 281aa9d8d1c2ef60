"""CPU-only checks of the entry points behind the compressed rows at the edges of what they accept."""
import ctypes
import math

import pytest
import torch

import paper_2605_07355_amd as ttf
from paper_2605_07355_amd import serving
from test_serving_checks import A, INVALID, SMALL, UNSUPPORTED, _attention, _cache, _qk


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


# strides of 8 rows and 4 heads (2 key heads) of 64 entries; whether two heads share an entry
LAYOUTS = [(64, 64, True), (128, 64, True), (192, 64, True), (248, 64, True), (256, 64, False), (64, 504, True), (64, 512, False), (192, 128, True),
           (320, 192, False), (1024, 600, False), (1024, 1088, False), (1024, 1080, True)]


def _share(row, head, rows, heads, D):
    at = [i * row + j * head for i in range(rows) for j in range(heads)]
    return any(abs(a - b) < D for n, a in enumerate(at) for b in at[:n])


@pytest.mark.parametrize("row,head,shares", LAYOUTS)
def test_outputs_that_overlap_themselves_are_refused(row, head, shares):
    """Every call ends in a refusal before any HIP call: INVALID for the layout, or what stands behind it."""
    assert _share(row, head, 8, 4, 64) == shares
    lib, other = serving._library(), 2 * A
    # a misaligned norm weight and a workspace too small are found after the layouts
    qk = dict(q_out=other, qo_row=row, qo_head=head, q_weight=A + 2)
    want = INVALID if shares else UNSUPPORTED
    assert lib.ttf_qk_norm_rope(ctypes.byref(_qk(**qk)), None) == want
    assert lib.ttf_cache_append(ctypes.byref(_qk(**qk)), ctypes.byref(_cache()), None) == want
    p = _attention(out=other, o_row=row, o_head=head)
    assert lib.ttf_paged_attention(ctypes.byref(p), ctypes.byref(_cache()), A, 0, None) == (INVALID if shares else SMALL)
    two = _share(row, head, 8, 2, 64)
    assert lib.ttf_qk_norm_rope(ctypes.byref(_qk(k_out=other, ko_row=row, ko_head=head, q_weight=A + 2)), None) == (INVALID if two else UNSUPPORTED)
    # inputs are only read
    assert lib.ttf_qk_norm_rope(ctypes.byref(_qk(q_row=row, q_head=head, q_out=other, q_weight=A + 2)), None) == UNSUPPORTED


@pytest.mark.parametrize("slot,head", [(64, 64), (128, 64), (64, 960), (64, 1024), (192, 128), (320, 64)])
def test_append_refuses_a_cache_whose_heads_overlap(slot, head):
    lib, c = serving._library(), _cache(slot_stride=slot, head_stride=head)
    if _share(slot, head, 16, 2, 64):
        assert lib.ttf_cache_append(ctypes.byref(_qk()), ctypes.byref(c), None) == INVALID
    # reading such a cache is harmless
    assert lib.ttf_paged_attention(ctypes.byref(_attention()), ctypes.byref(c), A, 0, None) == SMALL


def test_layouts_that_overlap_are_found_far_apart_too():
    """Strides whose products with the sizes pass 63 bits."""
    lib, far = serving._library(), 1 << 40
    p = _attention(rows=1 << 24, heads=8, kv_heads=2, out=2 * A, o_row=far, o_head=far)
    assert lib.ttf_paged_attention(ctypes.byref(p), ctypes.byref(_cache()), A, 0, None) == INVALID
    p = _attention(rows=1 << 24, heads=8, kv_heads=2, out=2 * A, o_row=far, o_head=64)
    assert lib.ttf_paged_attention(ctypes.byref(p), ctypes.byref(_cache()), A, 0, None) == SMALL


def test_numbers_that_do_not_fit_their_fields_are_refused():
    """2^32 + 5 rows are not 5 rows."""
    for kw in (dict(rows=(1 << 32) + 5), dict(batch=1 << 32), dict(max_rows=1 << 31), dict(heads=(1 << 32) + 8), dict(head_dim=(1 << 32) + 64)):
        args = dict(rows=8, batch=2, heads=8, kv_heads=2, head_dim=64) | kw
        with pytest.raises(ValueError):
            ttf.ttf_attention_workspace_size(**args)
    with pytest.raises(TypeError):
        ttf.ttf_attention_workspace_size(8, 2, 8, 2, 64, torch.float16)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    k = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16)
    cache, offsets, cached = ttf.TTFKVCache(k, k.clone(), torch.zeros((2, 4), dtype=torch.int32)), torch.tensor([0, 2, 4]).int(), torch.tensor([0, 0]).int()
    for kw in (dict(window=1 << 31), dict(max_rows=1 << 40), dict(scale="0.125")):
        with pytest.raises(ValueError, match="field"):
            ttf.ttf_paged_attention(x, cache, offsets, cached, **kw)
    with pytest.raises(ttf.TTFError):                       # infinite in 32 bits
        ttf.ttf_paged_attention(x, cache, offsets, cached, scale=1e300)
