"""The operators behind the compressed rows at the edges of what they accept."""
import math

import pytest
import torch

from test_gpu_serving import BF, F32, _cache, _check_attention, _offsets, _problem, _run_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,heads_first", [(16, False), (16, True), (7, False)])
@pytest.mark.parametrize("D,dtype", [(8, BF), (16, BF), (24, BF), (8, F32), (24, F32)])
@pytest.mark.parametrize("rows", [[1, 2], [3, 40]])
def test_attention_of_short_heads(rows, D, dtype, page, heads_first):
    """Heads shorter than the 64 bytes that four lanes read side by side."""
    cached = [60, 11]
    q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, D, page, dtype, heads_first)
    out, lse = _run_attention(q, k, v, table, rows, cached, max_rows=max(rows))
    _check_attention(out, lse, q, ks, vs, rows, cached, True, 0, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [[3], [100, 1]])
@pytest.mark.parametrize("page", [1, 16])
def test_windows_behind_the_end_of_the_table(rows, page, dtype):
    """`cached` of up to 2^31 - 1, and windows that begin where the table has long ended: no entry is seen."""
    import paper_2605_07355_amd as ttf
    k, v = (t.cuda() for t in _cache(9, page, 2, 64, dtype, False, fill=1.0))
    table = torch.zeros((len(rows), 100), dtype=torch.int32, device="cuda")
    q = torch.ones((sum(rows), 4, 64), dtype=dtype, device="cuda")
    for cached in (2 ** 31 - 1, 2 ** 31 - 40, 10 ** 6):
        for window in (1, 33):
            lse = torch.zeros((sum(rows), 4), device="cuda")
            have = torch.full((len(rows),), cached, dtype=torch.int32, device="cuda")
            out = ttf.ttf_paged_attention(q, ttf.TTFKVCache(k, v, table), _offsets(rows).cuda(), have, window=window, lse=lse)
            assert bool((out == 0).all()) and bool((lse == -math.inf).all())
