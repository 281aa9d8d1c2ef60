"""The operators behind the compressed rows at the edges of what they accept."""
import pytest
import torch

from test_gpu_serving import BF, F32, _check_attention, _problem, _run_attention

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
